"""Attention over the 4-bit cache where each part of its arithmetic decides the result: the four planes in which a query meets
the keys, and the three bf16 terms in which a probability meets the values.

Planes.  Of each 32 channels of a query one is far larger than the others, whose keys are larger by as much, and the large
one's are zero: every group's part of a logit is of order one, and comes from one plane (powers of two) or two that follow each other
(channels of 8 bits).  All channels are sums of four planes without a remainder.  With powers of two the products of a plane are
multiples of half the group's unit, at most 31 * 12 of them, so their sum and the sum of the planes' parts are exact, and a logit
takes the roundings of the scale, the product with it and the bias (3u (|l| + |b|), u = 2^-24); else 128 products of at most
264u of their magnitudes, as in test_gpu_ncache.  The exponential: 4u (|l - max| + 6) for its argument, whose reference lies up to
6 above the largest logit, and 2^-21 for itself.  Sums as there: |out - ref| <= 2 (D + 6 L u) sum_j p_j |v_j|.

Terms.  All rows in use have the same values, so that the result is those values whatever the probabilities are: the
exponentials' errors, and the factors of a running maximum and of the joins, are in the sums of probabilities as they are in those of
products.  n <= 4 rows in use add n numbers each (masked ones add zeros, exactly): with 2u a step of the accumulator, n 2u for the first
term, 2^-7 of it for the others, 3u where terms meet, n u for the sum of probabilities, and, where rows are apart, 2u for each
of n changes of the reference, of n joins of waves and of n joins of chunks; 2u for the division: at most (4 * 2 + 3 + 4 + 3 * 8 + 2) u < 48 u.

The host's part emulates the same sums with a plane or a term left out: that has to exceed the bounds many times.
"""
import math

import numpy as np
import pytest
import torch

from oracle import ncache as on

U = 2.0 ** -24
SCALE = 1 / math.sqrt(128)
CODES = np.array(on.MAGNITUDES)


# ------------------------------------------------------------------------------------------------ planes
def e4m3(x):
    """Nearest e4m3 number, ties to even, for magnitudes well below 448."""
    step = np.exp2(np.maximum(np.floor(np.log2(np.abs(x) + 2.0 ** -40)), -6) - 3)
    return np.rint(x / step) * step


def planes(q):
    """[4][..., 128]: what each plane holds of queries q [..., 128]."""
    top = np.abs(q).reshape(*q.shape[:-1], 4, 32).max(-1)
    E = np.floor(np.log2(np.maximum(top, 2.0 ** -112))) + 1                 # top below 2^E
    unit = np.exp2(E).repeat(32, -1)
    r, out = q / unit, []
    for t in range(4):
        p = e4m3(r)
        out.append(p * unit * 2.0 ** (-5 * t))
        r = (r - p) * 32
    return np.stack(out)


def plane_case(g, P, G, R, whole):
    """Queries [P][G][128] (exact in bf16), keys [P][R][128] (exact in the cache) as float64."""
    q, k = np.zeros((P, G, 128)), np.zeros((P, R, 128))
    below = (1, 6, 11, 16) if whole else (1, 10, 15, 20)                     # channels lie 2^-below under the large one
    for p in range(P):
        for group, s in enumerate(g.permutation(below)):
            at, large, a = slice(32 * group, 32 * group + 32), 32 * group + g.integers(32), int(g.integers(-3, 4))
            q[p, :, at] = g.choice([-1.0, 1.0], (G, 32)) * 2.0 ** (a - s)
            if whole:
                q[p, :, at] *= 1 + g.integers(0, 128, (G, 32)) / 128
            q[p, :, large] = g.choice([-1.0, 1.0], G) * 2.0 ** a
            k[p, :, at] = g.choice([-1.0, 1.0], (R, 32)) * g.choice(CODES[1:], (R, 32)) * 2.0 ** (s - a - (1 if whole else 0))
            k[p, :, large] = 0
    return q, k


def plane_bound(q, k, v, b, x, whole):
    """Bound of a pair's outputs [G][128]: queries, rows in use, their bias and logits [G][rows]."""
    far = x.max(1, keepdims=True) - x
    d = U * (3 * (np.abs(x) + np.abs(b)) + 4 * (far + 6))
    if whole:
        d = d + 264 * U * SCALE * np.abs(q) @ np.abs(k).T
    D = np.where(far < 40, d, 0).max(1, keepdims=True) + 2.0 ** -21
    w = np.exp(-far)
    return 2 * (D + 6 * len(k) * U) * ((w / w.sum(1, keepdims=True)) @ np.abs(v)) + 1e-37


def attend64(x, v):
    w = np.exp(x - x.max(1, keepdims=True))
    return w @ v / w.sum(1, keepdims=True)


def bias_of(g, P, R):
    b = g.standard_normal((P, R)).astype(np.float32)
    b[g.random((P, R)) < 0.3] = -math.inf
    return b


@pytest.mark.parametrize("whole", [False, True])
def test_a_plane_left_out_would_show(whole):
    g = np.random.default_rng(1)
    q, k = plane_case(g, 4, 3, 300, whole)
    assert np.array_equal(q, torch.from_numpy(q).bfloat16().double().numpy())
    codes, scales = on.n_rows(k.reshape(-1, 128))
    assert np.array_equal(on.n_values(codes, scales), k.reshape(-1, 128))
    parts = planes(q)
    assert np.array_equal(parts.sum(0), q)
    for p in range(4):
        v = g.standard_normal((300, 128))
        x = SCALE * q[p] @ k[p].T
        want, tol = attend64(x, v), plane_bound(q[p], k[p], v, np.zeros(300), x, whole)
        for t in range(4):
            for instead in (0.0, 0.5, 2.0):                                  # left out, or its scale off by one
                other = SCALE * (q[p] + (instead - 1) * parts[t, p]) @ k[p].T
                # the last plane holds an eighth at most of a channel of 8 bits
                assert (np.abs(attend64(other, v) - want) / tol).max(1).min() > (5 if whole else 20), (p, t, instead)


@pytest.mark.gpu
@pytest.mark.parametrize("whole", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("G", [1, 3, 4, 7, 8, 9, 16])
@pytest.mark.parametrize("P,R", [(5, 300), (3, 64), (2, 6000)])
def test_every_plane(P, R, G, bias, whole):
    from tests.test_gpu_ncache import A, make_cache, np64
    g = np.random.default_rng(R + G)
    q, k = plane_case(g, P, G, R, whole)
    K, V = torch.from_numpy(k).float().cuda(), torch.from_numpy(g.standard_normal((P, R, 128))).float().cuda()
    c = make_cache(P, R)
    A().ncache_write(c, K, V)
    stored_k, stored_v = A().ncache_read(c, dtype=torch.float32)
    assert torch.equal(stored_k, K)
    b = bias_of(g, P, R) if bias else np.zeros((P, R), np.float32)
    print(f"planes P={P} R={R} G={G} bias={bias} whole={whole}", flush=True)
    out = np64(A().attend_ncache(torch.from_numpy(q).cuda().bfloat16(), c, torch.from_numpy(b).cuda() if bias else None))
    v = np64(stored_v)
    for p in range(P):
        use = b[p] > -math.inf
        x = SCALE * q[p] @ k[p, use].T + b[p, use]
        err, tol = np.abs(out[p] - attend64(x, v[p, use])), plane_bound(q[p], k[p, use], v[p, use], b[p, use], x, whole)
        assert (err <= tol).all(), (p, (err / tol).max())


# ------------------------------------------------------------------------------------------------ terms
ROWS = 4                   # in use
BOUND = 48 * U             # relative


def terms(p):
    """A float32's three bf16 terms: its upper half, and the upper halves of what is left."""
    out = []
    for _ in range(3):
        t = (p.view(np.uint32) & np.uint32(0xffff0000)).view(np.float32)
        out.append(t)
        p = p - t
    assert not p.any()
    return out


def test_a_term_left_out_would_show():
    g = np.random.default_rng(2)
    p = np.exp(g.standard_normal((1000, ROWS)) * 2 - 6).astype(np.float32)
    t, whole = [x.astype(np.float64).sum(1) for x in terms(p)], p.astype(np.float64).sum(1)
    loss = t[2] / whole
    assert np.median(loss) > 2 * BOUND and loss.max() > 4 * BOUND
    assert (t[1] / whole).min() > 10 * BOUND


def same_values(g, P):
    return g.choice([-1.0, 1.0], (P, 1, 128)) * g.choice(CODES[1:], (P, 1, 128)) * np.exp2(g.integers(-9, 9, (P, 1, 4)).repeat(32, 2))


@pytest.mark.gpu
@pytest.mark.parametrize("G", [1, 2, 4, 5, 8, 9, 16])
@pytest.mark.parametrize("where", ["one block", "one pair's blocks", "eight waves", "chunks", "tail", "blocks and tail"])
def test_every_term(where, G):
    """A softmax of rows with the same values gives those values."""
    from tests.test_gpu_ncache import A, i32, make_cache, np64
    g = np.random.default_rng(G)
    P, R = {"one block": (60, 64), "one pair's blocks": (300, 400), "eight waves": (60, 500), "chunks": (9, 30000), "tail": (40, 8),
            "blocks and tail": (60, 300)}[where]
    F = 40 if "tail" in where else 0
    bf = lambda x: torch.from_numpy(x).cuda().bfloat16()
    v, Q = same_values(g, P), g.standard_normal((P, G, 128))
    V, b, used_f = np.repeat(v, R, 1), np.full((P, R), -math.inf, np.float32), [0] * P
    V[:, ::3] = -V[:, ::3]                                                    # of rows not in use
    for p in range(P):
        n = 0 if where == "tail" else ROWS // 2 if F else ROWS
        used_f[p] = ROWS - n if F else 0
        at = g.choice(R, n, replace=False)
        V[p, at], b[p, at] = v[p], g.standard_normal(n)
    c = make_cache(P, R)
    A().ncache_write(c, bf(g.standard_normal((P, R, 128))), bf(V))
    K_f, V_f = (bf(g.standard_normal((P, F, 128))), bf(np.repeat(v, F, 1))) if F else (None, None)
    assert (A().attend_ncache_workspace_size(P, R, G, F) > 0) == (where == "chunks")
    print(f"terms {where} G={G}", flush=True)
    out = np64(A().attend_ncache(bf(Q), c, torch.from_numpy(b).cuda(), None, K_f, V_f, i32(used_f) if F else None))
    assert (np.abs(out / v - 1) <= BOUND).all(), np.abs(out / v - 1).max() / U
    if where == "one block":                                                  # rows by length instead of by bias
        length = g.integers(1, ROWS + 1, P)
        A().ncache_write(c, bf(g.standard_normal((P, R, 128))), bf(np.repeat(v, R, 1)))
        out = np64(A().attend_ncache(bf(Q), c, None, i32(length.tolist())))
        assert (np.abs(out / v - 1) <= BOUND).all(), np.abs(out / v - 1).max() / U
