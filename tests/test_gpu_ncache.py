"""The 4-bit cache on the GPU against its float64 oracle.

Codes, scale bytes and rows read back have to be equal: scales are powers of two, so every step is exact but the one
rounding, which is to nearest even on both sides.

Attention's tolerance, per output element, from its rounding steps (u = 2^-24, L the rows that take part):
  - a logit: a query channel may lose 2^-24 of the largest of its 32 channels, 128 exact products are summed in float32 (the
    accumulator may truncate: 2u an addition), as four parts that meet (3u), the scale and the bias:
    |dl| <= s (2 * 128 + 8) u sum_d |q_d k_d| + s u sum_d max|q| |k_d| + 2u |l|, and u |l - max| again where the exponential's
    argument is formed in base 2, with 2^-22 for the exponential itself;
  - a probability is off by that much relatively, so is the sum of them, each adds L rounding steps of u, and P V again,
    where a probability enters exactly, as three bf16 terms;
  - so |out - ref| <= 2 (D + 3 L' u) sum_j p_j |v_j|, D the largest |dl| + 2^-21, L' = 2 L for the accumulator's steps.
"""
import math

import numpy as np
import pytest
import torch

from oracle import ncache as on
from oracle import qcache as oq
from oracle import rotary as orot
import oracle

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def A():
    from paper_2609_36835_amd import arckv
    return arckv


def np64(x):
    return None if x is None else x.float().double().cpu().numpy()


def rows(g, *shape, outliers=False, dtype=torch.bfloat16):
    x = g.standard_normal(shape).astype(np.float32)
    if outliers:
        x[..., 60:64] *= 8
    return torch.from_numpy(x).cuda().to(dtype)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def make_cache(P, R):
    """Filled with what nothing may depend on (255 is a NaN scale)."""
    c = A().ncache(P, R)
    for t in c:
        t.fill_(255)
    return c


def mirror(c):
    return [t.cpu().numpy().copy() for t in c]


def write_mirror(m, K, V, start, count):
    K, V = np64(K), np64(V)
    for p in range(len(K)):
        n = max(0, min(count[p], len(K[p]), m[0].shape[1] - start[p]))
        for codes, scales, x in ((m[0], m[2], K), (m[1], m[3], V)):
            if n:
                codes[p, start[p]:start[p] + n], scales[p, start[p]:start[p] + n] = on.n_bytes(*on.n_rows(x[p, :n]))


def same(c, m):
    for name, want, got in zip(("K", "V", "K_scale", "V_scale"), m, c):
        bad = got.cpu().numpy() != want
        assert not bad.any(), (name, np.argwhere(bad)[:5])


# ------------------------------------------------------------------------------------------------ write and read
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("P,R,n", [(1, 1, 1), (2, 63, 63), (3, 64, 64), (2, 65, 17), (2, 200, 130), (1, 1000, 1000), (700, 3, 2)])
def test_write(dtype, P, R, n):
    print(f"write {dtype} P={P} R={R} n={n}", flush=True)
    g = np.random.default_rng(P + R)
    c = make_cache(P, R)
    m = mirror(c)
    K, V = rows(g, P, n, 128, outliers=True, dtype=dtype), rows(g, P, n, 128, dtype=dtype)
    A().ncache_write(c, K, V)
    write_mirror(m, K, V, [0] * P, [n] * P)
    same(c, m)


def test_write_ragged_in_steps():
    """Prompts of different lengths, then chunks and single tokens from where each pair stands (past the end, none at
    all, a rewind); nothing but the written rows changes."""
    g = np.random.default_rng(5)
    P, R = 6, 300
    c = make_cache(P, R)
    m = mirror(c)
    length = [0] * P
    steps = [(200, [0, 1, 63, 64, 65, 200]), (1, [1] * P), (1, [1, 0, 1, 1, 0, 1]), (70, [70, 64, 1, 2, 0, 70]),
             (2, [2] * P), (100, [100] * P), (1, [1] * P)]
    for step, (n, count) in enumerate(steps):
        if step == 4:
            length = [max(0, x - 5) for x in length]
        K, V = rows(g, P, n, 128, outliers=True) * (1.7 ** step), rows(g, P, n, 128) * (1.7 ** step)
        A().ncache_write(c, K, V, i32(length), i32(count))
        write_mirror(m, K, V, length, count)
        length = [min(a + b, R) for a, b in zip(length, count)]
        same(c, m)
    assert R in length
    A().ncache_write(c, K, V, i32([R + 7, R, R, R, R, 2 ** 31 - 1]), i32([1] * P))     # nowhere to write
    A().ncache_write(c, K, V, i32([3] * P), i32([0, -4, 0, 0, 0, -2 ** 31]))            # nothing to write
    same(c, m)
    A().ncache_write(c, K, V, i32([-7, 0, 0, 0, 0, -2 ** 31]), i32([1, 0, 0, 0, 0, 10 ** 9]))
    write_mirror(m, K, V, [0] * P, [1, 0, 0, 0, 0, 10 ** 9])
    same(c, m)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_write_rounding_borders_and_extremes(dtype):
    """Values on and next to the borders between codes at several scales, zeros of both signs, the smallest and the largest
    magnitudes."""
    m7 = np.array(on.MAGNITUDES, np.float32)
    mid = (m7[1:] + m7[:-1]) / 2
    vals = np.concatenate([mid, np.nextafter(mid, np.float32(0)), np.nextafter(mid, np.float32(9)), [6.0]])
    vals = np.concatenate([vals, -vals])
    big = float(torch.finfo(dtype).max)
    x = np.zeros((12, 128), np.float32)
    for r, e in enumerate((0, -100, 124, 20, -63)):
        x[r, 31] = 6 * 2.0 ** e
        x[r, 63] = -6 * 2.0 ** e
        x[r, :22], x[r, 32:54] = vals[:22] * 2.0 ** e, vals[22:] * 2.0 ** e
        x[r, 96:] = np.nextafter(np.float32(6), np.float32(7)) * 2.0 ** e     # the next scale
    x[5] = 1e-38                                         # far below the least scale
    x[6] = 1e-45
    x[7, ::2] = -0.0
    x[8, 5] = big
    x[8, 40], x[8, 41] = -big, 6 * 2.0 ** 124
    x[8, 70:75] = np.array([5.0, 5.5, 6.0, 6.5, 7.5]) * 2.0 ** 125 if dtype == torch.float32 else 0
    x[9] = np.random.default_rng(0).standard_normal(128) * 2.0 ** -101
    x[10] = np.random.default_rng(1).standard_normal(128) * 2.0 ** 120
    K = torch.from_numpy(x[None]).cuda().to(dtype)
    c = make_cache(1, 12)
    m = mirror(c)
    A().ncache_write(c, K, -K)
    write_mirror(m, K, -K, [0], [12])
    same(c, m)
    k, _ = A().ncache_read(c, dtype=torch.float32)
    assert k.isfinite().all() and k[0, 8, 5] == 6 * 2.0 ** 125


@pytest.mark.parametrize("bad", [math.nan, -math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_write_non_finite(bad, dtype):
    """A group with a non-finite number reads as NaN, its neighbours are untouched."""
    g = np.random.default_rng(8)
    K, V = rows(g, 2, 40, 128, dtype=dtype), rows(g, 2, 40, 128, dtype=dtype)
    K[1, 7, 33] = bad
    V[0, 39, 127] = bad
    c = make_cache(2, 40)
    m = mirror(c)
    A().ncache_write(c, K, V)
    write_mirror(m, K, V, [0, 0], [40, 40])
    same(c, m)
    for out in (torch.bfloat16, torch.float32):
        k, v = A().ncache_read(c, dtype=out)
        assert k[1, 7, 32:64].isnan().all() and v[0, 39, 96:].isnan().all()
        assert int(k.isnan().sum()) == int(v.isnan().sum()) == 32


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_read(out):
    g = np.random.default_rng(9)
    P, R = 5, 333
    c = make_cache(P, R)
    K, V = rows(g, P, R, 128, outliers=True), rows(g, P, R, 128) * 1e-3
    A().ncache_write(c, K, V)
    m = mirror(c)
    length = [0, 1, 64, 200, 10 ** 9]
    for first, n, ln in [(0, R, None), (0, R, length), (70, 1, length), (63, 100, length), (332, 1, None), (0, 1, [-5] * P)]:
        k, v = A().ncache_read(c, first, n, out, None if ln is None else i32(ln))
        for p in range(P):
            held = np.arange(first, first + n)[:, None] < (R if ln is None else ln[p])
            for got, codes, scales in ((k, m[0], m[2]), (v, m[1], m[3])):
                want = np.where(held, on.n_unpack(codes[p], scales[p])[first:first + n], 0)
                assert np.array_equal(np64(got[p]), want), (first, n, p)
    # a stored value written again reads as itself
    k, v = A().ncache_read(c, dtype=out)
    c2 = make_cache(P, R)
    A().ncache_write(c2, k, v)
    for a, b in zip(A().ncache_read(c2, dtype=out), (k, v)):
        assert torch.equal(a, b)


# ------------------------------------------------------------------------------------------------ attention
def check_attend(out, Q, cache, beta, length, K_f, V_f, length_f, scale=1 / math.sqrt(128)):
    m = [t.cpu().numpy() for t in cache]
    Q, beta, K_f, V_f, out = np64(Q), np64(beta), np64(K_f), np64(V_f), np64(out)
    P, R = m[0].shape[:2]
    worst = 0.0
    for p in range(P):
        n = R if length is None else min(max(int(length[p]), 0), R)
        f = 0 if K_f is None else K_f.shape[1] if length_f is None else min(max(int(length_f[p]), 0), K_f.shape[1])
        K, V = on.n_unpack(m[0][p, :n], m[2][p, :n]), on.n_unpack(m[1][p, :n], m[3][p, :n])
        b = np.zeros(n) if beta is None else beta[p, :n]
        keep = b > -math.inf
        K, V, b = K[keep], V[keep], b[keep]
        Kt, Vt = (K_f[p, :f], V_f[p, :f]) if f else (np.zeros((0, 128)), np.zeros((0, 128)))
        want, mass = oq.q_attend(Q[p], K, V, b, Kt, Vt, scale)
        K, b = np.concatenate([K, Kt]), np.concatenate([b, np.zeros(f)])
        if len(K) == 0:
            assert (out[p] == 0).all(), p
            continue
        X = scale * Q[p] @ K.T + b
        top = np.abs(Q[p]).reshape(len(Q[p]), 4, 32).max(2).repeat(32, 1)
        dl = scale * U * (264 * np.abs(Q[p]) @ np.abs(K).T + top @ np.abs(K).T) + 2 * U * np.abs(X) + U * np.abs(X - X.max(1, keepdims=True))
        # rows without weight do not count: exp(-40) of the largest is below every rounding step
        dl = np.where(X - X.max(1, keepdims=True) > -40, dl, 0)
        D = dl.max(1, keepdims=True) + 2.0 ** -21
        tol = 2 * (D + 6 * len(K) * U) * mass + 1e-37
        err = np.abs(out[p] - want)
        assert (err <= tol).all(), (p, (err / tol).max(), err.max())
        worst = max(worst, (err / tol).max())
    return worst


def filled(g, P, R, kscale=1.0):
    c = make_cache(P, R)
    A().ncache_write(c, rows(g, P, R, 128, outliers=True) * kscale, rows(g, P, R, 128))
    return c


SIZES = [(1, 1, 1, 0), (2, 1, 4, 1), (3, 63, 1, 0), (2, 64, 2, 31), (5, 65, 3, 32), (2, 128, 4, 33), (3, 200, 5, 7),
         (2, 1000, 8, 64), (2, 1025, 9, 0), (1, 4097, 16, 300), (8, 819, 4, 37), (1, 20000, 7, 0), (40, 130, 12, 1),
         (300, 700, 4, 40), (2, 33000, 4, 0), (800, 70, 1, 3),
         # about a workgroup's width: five blocks are one more than four waves take at once, 257 pairs one more than there are CUs
         (3, 256, 3, 0), (3, 257, 6, 0), (4, 256, 16, 1), (7, 512, 2, 33), (4, 513, 12, 64), (6, 1, 4, 190), (256, 330, 3, 0),
         (257, 330, 3, 0), (200, 2700, 4, 0), (200, 2700, 10, 1)]


@pytest.mark.parametrize("P,R,G,F", SIZES)
@pytest.mark.parametrize("bias", [False, True])
def test_attend_sizes(P, R, G, F, bias):
    print(f"attend P={P} R={R} G={G} F={F} bias={bias}", flush=True)
    g = np.random.default_rng(R + G)
    c = filled(g, P, R)
    Q = rows(g, P, G, 128)
    beta = None
    if bias:
        b = g.standard_normal((P, R)).astype(np.float32) * 3
        b[g.random((P, R)) < 0.2] = -math.inf
        beta = torch.from_numpy(b).cuda()
    K_f, V_f = (rows(g, P, F, 128, outliers=True), rows(g, P, F, 128)) if F else (None, None)
    out = A().attend_ncache(Q, c, beta, None, K_f, V_f)
    print("  of the tolerance:", check_attend(out, Q, c, beta, None, K_f, V_f, None), flush=True)
    # twice the same bits
    assert torch.equal(out, A().attend_ncache(Q, c, beta, None, K_f, V_f))


@pytest.mark.parametrize("G", [1, 4, 8, 16])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("P,R,F", [(12, 300, 50), (12, 5000, 70), (280, 1200, 33)])
def test_attend_ragged(G, bias, P, R, F):
    """Lengths from none to beyond the end of both parts; rows behind them hold NaN, in the tail too."""
    g = np.random.default_rng(G)
    length = ([0, 1, 63, 64, 65, R, R + 9, -3, 0, R // 2, 128, 200] * (P // 12 + 1))[:P]
    length_f = ([0, 1, 31, 32, 33, F, F + 1, -1, 5, 0, F, 2] * (P // 12 + 1))[:P]
    c = make_cache(P, R)
    A().ncache_write(c, rows(g, P, R, 128, outliers=True), rows(g, P, R, 128), None, i32(length))
    Q = rows(g, P, G, 128)
    beta = torch.from_numpy(g.standard_normal((P, R)).astype(np.float32)).cuda() if bias else None
    K_f, V_f = rows(g, P, F, 128), rows(g, P, F, 128)
    for p in range(P):
        K_f[p, max(0, length_f[p]):] = math.nan
        V_f[p, max(0, length_f[p]):] = math.nan
        if bias:
            beta[p, max(0, length[p]):] = math.nan
    print(f"attend ragged P={P} R={R} G={G} F={F} bias={bias}", flush=True)
    out = A().attend_ncache(Q, c, beta, i32(length), K_f, V_f, i32(length_f))
    assert (out[0] == 0).all()
    check_attend(out, Q, c, beta, length, K_f, V_f, length_f)


@pytest.mark.parametrize("G", [2, 6, 13])
def test_attend_masks(G):
    """Rows left out by a bias of -inf, whatever they hold; whole stretches, whole pairs; the type's lowest value is a bias."""
    g = np.random.default_rng(11)
    P, R, F = 6, 900, 20
    K, V = rows(g, P, R, 128, outliers=True), rows(g, P, R, 128)
    b = g.standard_normal((P, R)).astype(np.float32)
    b[0] = -math.inf
    b[1, :700] = -math.inf
    b[2, 64:] = -math.inf
    b[3, 3::7] = -math.inf
    b[4] = np.finfo(np.float32).min
    b[5, ::2] = np.finfo(np.float32).min
    hidden = torch.from_numpy(b == -math.inf).cuda()
    K[hidden] = math.nan
    V[hidden] = math.inf
    c = make_cache(P, R)
    A().ncache_write(c, K, V)
    Q, beta = rows(g, P, G, 128), torch.from_numpy(b).cuda()
    K_f, V_f = rows(g, P, F, 128), rows(g, P, F, 128)
    print(f"attend masks G={G}", flush=True)
    out = A().attend_ncache(Q, c, beta)
    assert (out[0] == 0).all() and out.isfinite().all()
    check_attend(out[:4], Q[:4], [t[:4] for t in c], beta[:4], None, None, None, None)
    check_attend(out[5:], Q[5:], [t[5:] for t in c], beta[5:], None, None, None, None)
    # all rows at the lowest value: logits drown in it, so the rows weigh the same
    want = np64(A().ncache_read(c)[1][4]).mean(0)
    assert np.abs(np64(out[4]) - want).max() <= 2 * (2.0 ** -21 + 12 * R * U) * np.abs(np64(V[4])).mean(0).max()
    out = A().attend_ncache(Q, c, beta, None, K_f, V_f, i32([0, 20, 20, 20, 20, 20]))
    assert (out[0] == 0).all()
    check_attend(out, Q, c, beta, None, K_f, V_f, [0, 20, 20, 20, 20, 20])


@pytest.mark.parametrize("G", [1, 7, 16])
def test_attend_non_finite(G):
    """A NaN key group makes the pair's rows NaN, a NaN value group its 32 channels; other pairs and query rows do not
    see it; a query row with a non-finite channel is NaN where there is a row to attend to."""
    g = np.random.default_rng(12)
    P, R = 5, 400
    K, V = rows(g, P, R, 128), rows(g, P, R, 128)
    K[1, 333, 40] = math.inf
    V[2, 77, 100] = math.nan
    c = make_cache(P, R)
    A().ncache_write(c, K, V)
    Q = rows(g, P, G, 128)
    Q[3, G - 1, 5] = math.inf
    Q[4, 0, 127] = math.nan
    print(f"attend non-finite G={G}", flush=True)
    out = A().attend_ncache(Q, c, None, i32([R, R, R, R, 0]))
    assert out[0].isfinite().all() and out[1].isnan().all()
    assert out[2, :, 96:].isnan().all() and out[2, :, :96].isfinite().all()
    assert out[3, G - 1].isnan().all() and out[3, :G - 1].isfinite().all()
    assert (out[4] == 0).all()
    K_f = rows(g, P, 5, 128)
    out = A().attend_ncache(Q, c, None, i32([R, R, R, R, 0]), K_f, K_f)
    assert out[3, G - 1].isnan().all() and out[4, 0].isnan().all() and out[4, 1:].isfinite().all() and out[0].isfinite().all()


@pytest.mark.parametrize("order", ["rising", "falling", "one"])
@pytest.mark.parametrize("G", [1, 8])
def test_attend_far_logits(order, G):
    """The largest logit last, first, or one row far above all others, with values of very different size: rows of small
    weight and large values count."""
    g = np.random.default_rng(13)
    P, R = 2, 3000
    K, V = rows(g, P, R, 128), rows(g, P, R, 128)
    b = np.linspace(-60, 60, R, dtype=np.float32)
    b = np.tile(b if order == "rising" else b[::-1] if order == "falling" else np.where(np.arange(R) == 1234, 80, 0), (P, 1))
    b = b.astype(np.float32)
    if order != "one":
        V = V * torch.from_numpy(np.exp(-b / 2)).cuda()[..., None]
        V = V.to(torch.bfloat16)
    c = make_cache(P, R)
    A().ncache_write(c, K, V)
    Q, beta = rows(g, P, G, 128), torch.from_numpy(b).cuda()
    print(f"attend {order} G={G}", flush=True)
    check_attend(A().attend_ncache(Q, c, beta), Q, c, beta, None, None, None, None)


@pytest.mark.parametrize("G", [3, 8, 16])
def test_attend_largest_values(G):
    """Rows of the largest magnitude, many of them of equal weight, or one behind others: a finite mean."""
    P, R = 3, 200
    big = 6 * 2.0 ** 125
    K, V = torch.zeros(P, R, 128, device="cuda"), torch.full((P, R, 128), 3.3e38, device="cuda")
    V[1, :, ::2] = -3.3e38
    V[2, :R - 1] = 1.0
    b = torch.zeros(P, R, device="cuda")
    b[2] = torch.linspace(-30, 30, R)
    c = make_cache(P, R)
    A().ncache_write(c, K, V)
    Q = torch.ones(P, G, 128, dtype=torch.bfloat16, device="cuda")
    out = np64(A().attend_ncache(Q, c, b))
    sign = np.where(np.arange(128) % 2 == 0, -1, 1)
    tol = 2 * (2.0 ** -21 + 12 * R * U) * big
    assert (np.abs(out[0] - big) <= tol).all() and (np.abs(out[1] - big * sign) <= tol).all()
    w = np.exp(np64(b[2]) - 30)
    assert (np.abs(out[2] - (w[-1] * big + w[:-1].sum()) / w.sum()) <= tol).all()


def test_attend_small_and_large_query_channels():
    """Query channels over the whole range beside a large one; keys are such that each part shows."""
    g = np.random.default_rng(14)
    P, R, G = 4, 500, 4
    K, V = rows(g, P, R, 128), rows(g, P, R, 128)
    q = g.standard_normal((P, G, 128)) * np.exp2(g.integers(-30, 1, (P, G, 128)))
    q[1] *= 2.0 ** 10
    q[2] *= 2.0 ** -20
    q[3, :, 1:] = 0
    K[1] *= 2.0 ** -9
    K[2] *= 2.0 ** 18
    Q = torch.from_numpy(q).float().cuda().bfloat16()
    c = make_cache(P, R)
    A().ncache_write(c, K, V)
    check_attend(A().attend_ncache(Q, c), Q, c, None, None, None, None, None)
    Q[:] = 0
    check_attend(A().attend_ncache(Q, c), Q, c, None, None, None, None, None)


def test_attend_scale():
    g = np.random.default_rng(15)
    c = filled(g, 2, 300)
    Q = rows(g, 2, 4, 128)
    for s in (0.5, 1e-3):
        check_attend(A().attend_ncache(Q, c, scale=s), Q, c, None, None, None, None, None, scale=s)


def test_attend_far_rows():
    """Offsets that pass 32 bits: pairs of 2^25 rows, keys of zero, so that all rows weigh the same but the one that a bias
    lifts, and the values are zero but for a few rows near both ends."""
    P, R, G = 3, 1 << 25, 2
    c = A().ncache(P, R)
    c.K.zero_()
    c.V.zero_()
    c.K_scale.fill_(127)
    c.V_scale.fill_(127)
    g = np.random.default_rng(16)
    V = rows(g, P, 3, 128)
    A().ncache_write(c, torch.zeros_like(V), V * 2.0 ** 20, i32([R - 3, 5, R - 3]), i32([3, 3, 3]))
    stored = np64(A().ncache_read(c, R - 3, 3)[1])
    first = np64(A().ncache_read(c, 5, 3)[1])
    Q = rows(g, P, G, 128)
    out = np64(A().attend_ncache(Q, c, None, i32([R, 9, R - 1])))
    want = [stored[0].sum(0) / R, first[1].sum(0) / 9, stored[2][:2].sum(0) / (R - 1)]
    mass = [np.abs(stored[0]).sum(0) / R, np.abs(first[1]).sum(0) / 9, np.abs(stored[2][:2]).sum(0) / (R - 1)]
    for p in range(P):
        # equal weights are exact; sums of ones are exact up to 2^24 in a partial, and partials join with L = 2^13 steps
        assert (np.abs(out[p] - want[p]) <= 2 ** 13 * 2 * U * mass[p] + 1e-30).all(), p
    read = A().ncache_read(c, R - 2, 2, torch.float32, i32([R, R, R - 1]))[1]
    assert (read[2, 1] == 0).all() and np.array_equal(np64(read[0]), stored[0][1:])


@pytest.mark.parametrize("P,R", [(3, 700), (3, 20000), (300, 900)])
def test_given_output_and_workspace(P, R):
    """Results do not depend on what a workspace held; a short one is refused."""
    g = np.random.default_rng(17)
    G = 4
    c = filled(g, P, R)
    Q = rows(g, P, G, 128)
    want = A().attend_ncache(Q, c)
    need = A().attend_ncache_workspace_size(P, R, G)
    out = torch.full((P, G, 128), math.nan, device="cuda")
    ws = torch.full((max(need, 256),), 255, dtype=torch.uint8, device="cuda")
    assert A().attend_ncache(Q, c, out=out, ws=ws) is out
    assert torch.equal(out, want)
    if need:
        with pytest.raises(A().ArckvError) as e:
            A().attend_ncache(Q, c, ws=ws[:need - 1])
        assert e.value.status == A().ERR_WORKSPACE


def test_binding_checks_tensors():
    c = A().ncache(2, 50)
    Q = torch.zeros(2, 4, 128, dtype=torch.bfloat16, device="cuda")
    x = torch.zeros(2, 3, 128, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(TypeError):
        A().attend_ncache(Q.float(), c)
    with pytest.raises(ValueError):
        A().attend_ncache(Q[:1], c)
    with pytest.raises(TypeError):
        A().attend_ncache(Q, c, length=torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        A().attend_ncache(Q, c, torch.zeros(2, 49, device="cuda"))
    with pytest.raises(ValueError):
        A().attend_ncache(Q, c, None, None, x, x[:, :2].contiguous())
    with pytest.raises(ValueError):
        A().ncache_write(c, x, x.transpose(0, 1).contiguous().transpose(0, 1))
    with pytest.raises(TypeError):
        A().ncache_write(c, x.half(), x.half())
    with pytest.raises(A().ArckvError):
        A().ncache_read(c, 49, 2)
    with pytest.raises(TypeError):
        A().ncache_read((c.K.view(torch.int8), *c[1:]))
    with pytest.raises(ValueError):
        A().ncache_read((c.K, c.V, c.K_scale[:, :49].contiguous(), c.V_scale))


# ------------------------------------------------------------------------------------------------ together
def chain(q, k, v, pos, freq, cache, length, beta, K_f, V_f, out=None, ws=None):
    """One decode step: the new token's queries and keys turned, its row appended, attention over what is then held."""
    S, H, kv = q.shape[0], q.shape[1], k.shape[1]
    qr, kr = A().rotary(q, freq, pos, k)
    P = S * kv
    A().ncache_write(cache, kr.view(P, 1, 128), v.reshape(P, 1, 128), length)
    held = length + 1
    return A().attend_ncache(qr.view(P, H // kv, 128), cache, beta, held, K_f, V_f, out=out, ws=ws)


def check_chain(out, q, k, v, pos, freq, before, cache, length):
    S, kv, R = q.shape[0], k.shape[1], cache[0].shape[1]
    m = [x.copy() for x in before]
    qr, kr = A().rotary(q, freq, pos, k)
    write_mirror(m, kr.view(S * kv, 1, 128), v.reshape(S * kv, 1, 128), length.tolist(), [1] * (S * kv))
    same(cache, m)
    check_attend(out, qr.view(S * kv, -1, 128), cache, None, (length + 1).tolist(), None, None, None)
    tol = 2.0 ** -8 * 1.01
    want = orot.rotary(np64(q), pos.tolist(), np64(freq))
    assert (np.abs(np64(qr) - want) <= tol * np.abs(want) + 1e-5).all()


def test_decode_steps_and_their_graph():
    """Prompt, eager steps, then the same step captured and replayed on new tokens, with eager work between."""
    g = np.random.default_rng(18)
    S, kv, H, R, T = 3, 2, 8, 400, 250
    freq = A().rotary_frequencies(128, 500000.0, "turns", 8.0, 8192.0, 1.0, 4.0)
    P = S * kv
    c = make_cache(P, R)
    prompt = rows(g, S * T, kv, 128, outliers=True)
    K = torch.empty(S, kv, T, 128, dtype=torch.bfloat16, device="cuda")
    for s in range(S):
        A().rotary(prompt[s * T:(s + 1) * T], freq, out=K[s].transpose(0, 1))
    A().ncache_write(c, K.view(P, T, 128), rows(g, P, T, 128))
    length = i32([T] * P)
    new = lambda: (rows(g, S, H, 128), rows(g, S, kv, 128, outliers=True), rows(g, S, kv, 128))
    for _ in range(3):
        q, k, v = new()
        before = mirror(c)
        pos = length[::kv].contiguous()
        out = chain(q, k, v, pos, freq, c, length, None, None, None)
        check_chain(out, q, k, v, pos, freq, before, c, length)
        length += 1
    q, k, v = new()
    pos = length[::kv].contiguous()
    out = torch.empty(P, H // kv, 128, device="cuda")
    ws = torch.empty(max(256, A().attend_ncache_workspace_size(P, R, H // kv)), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        chain(q, k, v, pos, freq, c, length, None, None, None, out, ws)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain(q, k, v, pos, freq, c, length, None, None, None, out, ws)
    for _ in range(4):
        for t, x in zip((q, k, v), new()):
            t.copy_(x)
        pos.copy_(length[::kv])
        before = mirror(c)
        graph.replay()
        check_chain(out, q, k, v, pos, freq, before, c, length)
        length += 1


def test_two_graphs_share_a_workspace():
    """Captured on one stream and replayed in turn: each call's result is its own."""
    g = np.random.default_rng(19)
    caches, Qs = [filled(g, 4, 20000), filled(g, 4, 20000)], [rows(g, 4, 4, 128), rows(g, 4, 4, 128)]
    ws = torch.empty(max(256, A().attend_ncache_workspace_size(4, 20000, 4)), dtype=torch.uint8, device="cuda")
    outs = [torch.empty(4, 4, 128, device="cuda") for _ in range(2)]
    want = [A().attend_ncache(q, c) for q, c in zip(Qs, caches)]
    graphs = []
    torch.cuda.synchronize()
    for i in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            A().attend_ncache(Qs[i], caches[i], out=outs[i], ws=ws)
        graphs.append(gr)
    for _ in range(3):
        for o in outs:
            o.fill_(math.nan)
        for gr in graphs:
            gr.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o, w)


def test_two_streams():
    g = np.random.default_rng(20)
    jobs = [(filled(g, 6, 9000), rows(g, 6, 4, 128)) for _ in range(2)]
    want = [A().attend_ncache(q, c) for c, q in jobs]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [None, None]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, (c, q) in enumerate(jobs):
            with torch.cuda.stream(streams[i]):
                got[i] = A().attend_ncache(q, c)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_compact_cache_in_4_bits():
    """A compaction's keys, biases and values written in 4 bits and attended to with a bf16 tail, against the oracle over
    the stored values."""
    from tests.gpu_common import make_inputs
    import synth
    wl = synth.custom("n4", kv_heads=2, T=600, q_heads_per_kv=4, n_pos=48, rho=0.2, dtype="bf16", rope=True)
    dev, _ = make_inputs(wl)
    anchors, C_k, beta, C_v, info = A().compact(dev["K"], dev["V"], dev["Q"], dev["W1"], dev["b1"], dev["w2"], dev["b2"], wl.rho)
    assert int(info.abs().sum()) == 0
    P, t = C_k.shape[:2]
    c = make_cache(P, t)
    m = mirror(c)
    A().ncache_write(c, C_k, C_v)
    for p in range(P):
        for i, x in ((0, C_k), (1, C_v)):
            m[i][p], m[2 + i][p] = on.n_bytes(*on.n_rows(x[p].double().cpu().numpy()))
    same(c, m)
    g = np.random.default_rng(21)
    Q, K_f, V_f = rows(g, P, 4, 128), rows(g, P, 19, 128), rows(g, P, 19, 128)
    out = A().attend_ncache(Q, c, beta, None, K_f, V_f)
    m = [x.cpu().numpy() for x in c]
    check_attend(out, Q, c, beta, None, K_f, V_f, None)


# ------------------------------------------------------------------------------------------------ large calls
@pytest.mark.parametrize("dtype,n", [(torch.bfloat16, 30001), (torch.float32, 15003)])
def test_large_write_is_many_small_ones(dtype, n):
    """A write whose source is read as a stream leaves the same bytes as one in pieces."""
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    P = 8
    K, V = (torch.randn(P, n, 128, device="cuda", generator=g).to(dtype) for _ in range(2))
    whole, pieces = make_cache(P, n + 5), make_cache(P, n + 5)
    A().ncache_write(whole, K, V, i32([3] * P))
    for a in range(0, n, 4000):
        b = min(a + 4000, n)
        A().ncache_write(pieces, K[:, a:b].contiguous(), V[:, a:b].contiguous(), i32([3 + a] * P))
    assert all(torch.equal(a, b) for a, b in zip(whole, pieces))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [450, 701, 1801])
def test_larger_ragged_writes(dtype, n):
    """Writes of 15 to 236 MB with a start and a count for each pair leave the same bytes as writes of a few pairs, and the others
    as they were."""
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    P, R = 64, 2000
    K, V = (torch.randn(P, n, 128, device="cuda", generator=g).to(dtype) for _ in range(2))
    start = torch.randint(0, R - 100, (P,), device="cuda", generator=g).int()
    count = torch.randint(0, n + 1, (P,), device="cuda", generator=g).int()
    count[:8] = i32([0, 1, 15, 16, 17, n, n + 3, -1])
    start[8:12] = i32([R - 1, R - 5, R, 0])
    whole, few = make_cache(P, R), make_cache(P, R)
    for t in (*whole, *few):
        t.fill_(0xab)
    A().ncache_write(whole, K, V, start, count)
    for a in range(0, P, 4):
        part = [t[a:a + 4] for t in few]
        A().ncache_write(tuple(part), K[a:a + 4], V[a:a + 4], start[a:a + 4].contiguous(), count[a:a + 4].contiguous())
    assert all(torch.equal(a, b) for a, b in zip(whole, few))
    for p in (0, 5, 9, 40):
        b = max(0, min(int(count[p]), n, R - int(start[p]))) + int(start[p])
        assert all((t[p, b:] == 0xab).all() and (t[p, :int(start[p])] == 0xab).all() for t in whole)


@pytest.mark.parametrize("G", [4, 8, 16])
def test_large_attend(G):
    """A call whose codes are read as streams, with bias, lengths and tail: some of its pairs against the oracle, all of them
    against calls of few pairs (other chunks, other order of sums)."""
    g = np.random.default_rng(G)
    P, R, F = 300, 3001, 40
    c = make_cache(P, R)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(G)
    randn = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    length = g.integers(1, R + 1, P).tolist()
    A().ncache_write(c, randn(P, R, 128).bfloat16(), randn(P, R, 128).bfloat16(), None, i32(length))
    Q, K_f, V_f = randn(P, G, 128).bfloat16(), randn(P, F, 128).bfloat16(), randn(P, F, 128).bfloat16()
    beta = randn(P, R)
    beta[:, ::5] = -math.inf
    print(f"large attend G={G}", flush=True)
    out = A().attend_ncache(Q, c, beta, i32(length), K_f, V_f)
    for p in (0, 17, 150, 299):
        check_attend(out[p:p + 1], Q[p:p + 1], [t[p:p + 1] for t in c], beta[p:p + 1], length[p:p + 1], K_f[p:p + 1], V_f[p:p + 1], None)
    for a in range(0, P, 25):
        part = slice(a, a + 25)
        few = A().attend_ncache(Q[part].contiguous(), tuple(t[part].contiguous() for t in c), beta[part].contiguous(), i32(length[part]),
                                K_f[part].contiguous(), V_f[part].contiguous())
        # each is within check_attend's bound of the formula: here 2 (2^-17 + 6 * 3041 * 2^-24) of a mean |v| below 1
        assert (few - out[part]).abs().max() <= 4 * (2.0 ** -17 + 6 * 3041 * U)


def test_many_pairs():
    """Pairs beyond one extent of a grid."""
    g = np.random.default_rng(22)
    P, R, G = 70000, 3, 1
    K, V, Q = (torch.randn(P, n, 128, device="cuda").bfloat16() for n in (R, R, G))
    c = make_cache(P, R)
    A().ncache_write(c, K, V)
    k, v = A().ncache_read(c, 1, 2)
    print("many pairs", flush=True)
    out = A().attend_ncache(Q, c, None, i32([2] * P))
    for p in (0, 1, 32767, 32768, 32769, 65535, 65536, P - 1):
        m = [t[p:p + 1] for t in c]
        same(m, [x[None] for x in (*(on.n_bytes(*on.n_rows(np64(K[p])))[:1]), on.n_bytes(*on.n_rows(np64(V[p])))[0],
                                   on.n_bytes(*on.n_rows(np64(K[p])))[1], on.n_bytes(*on.n_rows(np64(V[p])))[1])])
        assert np.array_equal(np64(k[p]), on.n_values(*on.n_rows(np64(K[p])))[1:])
        assert np.array_equal(np64(v[p]), on.n_values(*on.n_rows(np64(V[p])))[1:])
        check_attend(out[p:p + 1], Q[p:p + 1], m, None, [2], None, None, None)


@pytest.mark.parametrize("G", [2, 8, 16])
def test_attend_infinite_tail_values(G):
    """An infinite value of the tail makes its channel infinite, and nothing else."""
    g = np.random.default_rng(23)
    c = filled(g, 2, 200)
    Q, K_f, V_f = rows(g, 2, G, 128), rows(g, 2, 40, 128), rows(g, 2, 40, 128)
    V_f[0, 35, 7] = math.inf
    V_f[0, 3, 100] = -math.inf
    out = A().attend_ncache(Q, c, None, None, K_f, V_f)
    assert (out[0, :, 7] == math.inf).all() and (out[0, :, 100] == -math.inf).all()
    out[0, :, 7] = out[0, :, 100] = 0
    assert out.isfinite().all()


def test_binding_refuses_what_32_bits_do_not_hold():
    c = A().ncache(2, 50)
    for big in (1 << 31, 1 << 32, -(1 << 31) - 1):
        with pytest.raises(ValueError, match="first"):
            A().ncache_read(c, big, 4)
        with pytest.raises(ValueError, match="n:"):
            A().ncache_read(c, 0, big)
