"""The 8-bit cache on the GPU against its float64 oracle.

Codes, scales, bounds and rows read back have to be equal: scales are powers of two, so every step is exact but the one
rounding, which is to nearest even on both sides.  Block scores are exact sums rounded once to float32, and the blocks
are the top k of them.

Attention's tolerance, per output element, from its rounding steps (u = 2^-24, L the rows that take part):
  - a logit: 128 exact products summed in float32 (the accumulator may truncate: 2u an addition), the scale and the bias:
    |dl| <= s (2 * 128 + 4) u sum_d |q_d k_d| + 2u |l|, and u |l - max| again where the exponential's argument is
    formed in base 2, with 2^-22 for the exponential itself;
  - a probability is off by that much relatively, so is the sum of them, each adds L rounding steps of u, and P V again,
    where a probability enters as two fp16 terms: 2^-22 of it, or 2^-39 of its block's largest;
  - so |out - ref| <= 2 (D + 3 L' u) sum_j p_j |v_j|, D the largest |dl| + 2^-21, L' = 2 L for the accumulator's steps.
"""
import math

import numpy as np
import pytest
import torch

from oracle import qcache as oq
import oracle

pytestmark = pytest.mark.gpu
DT = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
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


def make_cache(P, R, fmt, garbage=True):
    """Arrays of a cache; `garbage`: filled with what nothing may depend on (0x7f is a NaN in e4m3)."""
    c = A().qcache(P, R, DT[fmt])
    for t in (c.K, c.V, c.K_bounds):
        t.view(torch.uint8).fill_(0x7f if garbage else 0)
    for t in (c.K_scale, c.V_scale):
        t.fill_(math.nan if garbage else 2.0 ** -100)
    return c


class Mirror:
    """The cache's state in float64, pair by pair."""

    def __init__(self, c, fmt):
        self.fmt = fmt
        self.K, self.V, self.Ks, self.Vs = (np64(t) for t in c[:4])
        self.B = np64(c.K_bounds)

    def write(self, K, V, start, count):
        for p in range(len(self.K)):
            for codes, scales, x, b in ((self.K, self.Ks, K, self.B), (self.V, self.Vs, V, None)):
                oq.q_write(codes[p], scales[p], np64(x[p])[:count[p]], start[p], self.fmt, None if b is None else b[p])

    def check(self, c):
        for name, want, got in zip(c._fields, (self.K, self.V, self.Ks, self.Vs, self.B), c):
            g = np64(got)
            bad = ~((g == want) | (np.isnan(g) & np.isnan(want)))
            assert not bad.any(), (name, np.argwhere(bad)[:5], g[bad][:5], want[bad][:5])


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------------------ write and read
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("P,R,n", [(1, 1, 1), (2, 63, 63), (3, 64, 64), (2, 65, 65), (2, 200, 130), (1, 1000, 1000)])
def test_write_whole(fmt, dtype, P, R, n):
    print(f"write {fmt} {dtype} P={P} R={R} n={n}", flush=True)
    g = np.random.default_rng(P + R)
    c = make_cache(P, R, fmt)
    m = Mirror(c, fmt)
    K, V = rows(g, P, n, 128, outliers=True, dtype=dtype), rows(g, P, n, 128, dtype=dtype)
    A().qcache_write(c, K, V)
    m.write(K, V, [0] * P, [n] * P)
    m.check(c)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_write_ragged_in_steps(fmt):
    """Prompts of different lengths, then chunks and single tokens from where each pair stands (across block borders, past
    the end, none at all, a rewind), the magnitudes growing so that open blocks are scaled anew."""
    g = np.random.default_rng(5)
    P, R = 6, 300
    c = make_cache(P, R, fmt)
    m = Mirror(c, fmt)
    length = [0] * P
    steps = [(200, [0, 1, 63, 64, 65, 200]), (1, [1] * P), (1, [1, 0, 1, 1, 0, 1]), (70, [70, 64, 1, 2, 0, 70]),
             (2, [2] * P), (100, [100] * P), (1, [1] * P)]
    for step, (n, count) in enumerate(steps):
        if step == 4:
            length = [max(0, x - 5) for x in length]     # rewind, into the middle of a block
        K = rows(g, P, n, 128, outliers=True) * (1.7 ** step)
        V = rows(g, P, n, 128) * (1.7 ** step)
        A().qcache_write(c, K, V, i32(length), i32(count))
        m.write(K, V, length, count)
        length = [min(a + b, R) for a, b in zip(length, count)]
        m.check(c)
    assert R in length
    before = [t.clone() for t in c]
    A().qcache_write(c, K, V, i32([R + 7, R, R, R, R, R]), i32([1] * P))      # nowhere to write
    A().qcache_write(c, K, V, i32([3] * P), i32([0, -4, 0, 0, 0, 0]))          # nothing to write
    for a, b in zip(before, c):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_write_rounding_borders_and_extremes(fmt):
    """Values on and next to the borders between codes, zeros, the smallest and largest magnitudes."""
    M = oq.LARGEST[fmt]
    y = np.arange(0, 128) if fmt == "int8" else torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    mid = ((y[1:] + y[:-1]) / 2).astype(np.float32)
    vals = np.concatenate([mid, np.nextafter(mid, np.float32(0)), np.nextafter(mid, np.float32(1e9)), -mid])
    x = np.zeros((5, 64, 128), np.float32)
    x[0].reshape(-1)[:len(vals)] = vals
    x[0, 63, 127] = M                                   # scale 1: the borders are where they are
    x[2] = 1e-38                                         # far below the least scale
    x[3, 5, 5] = np.float32(1.7e38)
    x[3, 6] = -3e30
    x[4] = np.random.default_rng(0).standard_normal((64, 128)) * 2.0 ** -98   # around the least scale
    x[4, 1, 1] = 0
    K = torch.from_numpy(x.reshape(1, 320, 128)).cuda()
    c = make_cache(1, 320, fmt)
    m = Mirror(c, fmt)
    A().qcache_write(c, K, -K)
    m.write(K, -K, [0], [320])
    m.check(c)
    assert c.K_scale[0, 0] == 1 and c.K_scale[0, 1] == c.K_scale[0, 2] == 2.0 ** -100


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_write_non_finite(fmt, bad):
    """A block with a non-finite number reads as NaN, its neighbours are untouched, and replacing its rows heals it."""
    g = np.random.default_rng(8)
    K, V = rows(g, 2, 192, 128), rows(g, 2, 192, 128)
    good = make_cache(2, 192, fmt)
    A().qcache_write(good, K, V)
    K[1, 70, 3] = bad
    V[0, 191, 127] = bad
    c = make_cache(2, 192, fmt)
    m = Mirror(c, fmt)
    A().qcache_write(c, K, V)
    m.write(K, V, [0, 0], [192, 192])
    m.check(c)
    k, v = A().qcache_read(c)
    assert k[1, 64:128].isnan().all() and v[0, 128:].isnan().all()
    assert not k[1, :64].isnan().any() and not k[0].isnan().any() and not v[1].isnan().any()
    one = rows(g, 2, 1, 128)
    A().qcache_write(c, one, one, i32([100, 100]))      # kept rows of the block are NaN: it stays so
    assert c.K_scale[1, 1].isnan() and not c.K_scale[0, 1].isnan()
    K2, V2 = rows(g, 2, 128, 128), rows(g, 2, 128, 128)
    A().qcache_write(c, K2, V2, i32([64, 64]))
    assert all(t.isfinite().all() for t in (c.K_scale, c.V_scale))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_read(fmt, out):
    g = np.random.default_rng(9)
    P, R = 5, 333
    c = make_cache(P, R, fmt)
    m = Mirror(c, fmt)
    K, V = rows(g, P, R, 128, outliers=True), rows(g, P, R, 128, dtype=torch.bfloat16) * 1e-3
    A().qcache_write(c, K, V)
    m.write(K, V, [0] * P, [R] * P)
    length = [0, 1, 64, 200, 10 ** 9]
    for first, n, ln in [(0, R, None), (0, R, length), (70, 1, length), (63, 100, length), (332, 1, None)]:
        k, v = A().qcache_read(c, first, n, out, None if ln is None else i32(ln))
        for p in range(P):
            held = np.arange(first, first + n)[:, None] < (R if ln is None else ln[p])
            for got, codes, scales in ((k, m.K, m.Ks), (v, m.V, m.Vs)):
                want = np.where(held, oq.q_values(codes[p], scales[p])[first:first + n], 0)
                assert np.array_equal(np64(got[p]), want), (first, n, p)
    # a stored value written again gives the same cache
    k, v = A().qcache_read(c, dtype=out)
    c2 = make_cache(P, R, fmt)
    A().qcache_write(c2, k, v)
    for a, b in zip(A().qcache_read(c2, dtype=out), (k, v)):
        assert torch.equal(a, b)


def test_write_without_bounds():
    g = np.random.default_rng(10)
    K = rows(g, 2, 100, 128)
    c = A().qcache(2, 100)
    A().qcache_write(c, K, K)
    d = A().qcache(2, 100, bounds=False)
    A().qcache_write(d, K, K)
    assert torch.equal(c.K.view(torch.uint8), d.K.view(torch.uint8)) and torch.equal(c.K_scale, d.K_scale)
    with pytest.raises(A().ArckvError):
        A().select_blocks(rows(g, 2, 4, 128), d, 1)


# ------------------------------------------------------------------------------------------------ attention
def attend_bound(Q, K, V, beta, K_f, s, mass_abs):
    keys = K if K_f is None else np.concatenate([K, K_f])
    b = np.zeros(len(keys))
    if beta is not None:
        b[:len(K)] = np.where(beta > -math.inf, beta, 0)
    sums, l = s * np.abs(Q) @ np.abs(keys).T, s * Q @ keys.T + b
    dl = (2 * 128 + 4) * U * sums + 2 * U * np.abs(l) + U * np.abs(l - l.max(axis=1, keepdims=True))
    return 2 * (dl.max() + 2.0 ** -21 + 6 * len(keys) * U) * mass_abs + 1e-30


def check_attend(out, Q, c, fmt, beta, length, K_f, V_f, length_f, blocks, s, pairs=None):
    """Every pair (or those listed) against the float64 attention over the stored values."""
    P, R, _ = c.K.shape
    worst = 0.0
    for p in range(P) if pairs is None else pairs:
        L = R if length is None else min(max(length[p], 0), R)
        at = np.arange(L)
        if blocks is not None:
            at = np.concatenate([np.arange(b * 64, min(b * 64 + 64, L)) for b in blocks[p].tolist()
                                 if 0 <= b * 64 < L] or [np.arange(0)]).astype(int)
        K, V = oq.q_values(np64(c.K[p]), np64(c.K_scale[p])), oq.q_values(np64(c.V[p]), np64(c.V_scale[p]))
        K, V = K[at], V[at]
        b = None if beta is None else np64(beta[p])[at]
        kf = vf = None
        if K_f is not None:
            F = K_f.shape[1] if length_f is None else min(max(length_f[p], 0), K_f.shape[1])
            kf, vf = np64(K_f[p, :F]), np64(V_f[p, :F])
        ref, mass_abs = oq.q_attend(np64(Q[p]), K, V, b, kf, vf, s)
        got = np64(out[p])
        if len(K) + (0 if kf is None else len(kf)) == 0:
            assert (got == 0).all()
            continue
        live = np.ones(len(K), bool) if b is None else b > -math.inf
        if not live.any() and (kf is None or len(kf) == 0):
            assert (got == 0).all()
            continue
        tol = attend_bound(np64(Q[p]), K[live], V[live], None if b is None else b[live], kf, s, mass_abs)
        err = np.abs(got - ref)
        assert (err <= tol).all(), (p, float((err / tol).max()), float(err.max()))
        worst = max(worst, float((err / tol).max()))
    print(f"    largest error / tolerance {worst:.3f}", flush=True)


def filled(g, P, R, fmt, length=None, scale=1.0):
    c = make_cache(P, R, fmt)
    K, V = rows(g, P, R, 128, outliers=True) * scale, rows(g, P, R, 128)
    A().qcache_write(c, K, V, None, None if length is None else i32([min(max(x, 0), R) for x in length]))
    return c


S = 1 / math.sqrt(128)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("P,G,R,F", [(256, 4, 1024, 0), (257, 4, 1024, 0), (4, 5, 1023, 1), (4, 5, 960, 33), (768, 1, 200, 70),
                                     (200, 8, 2100, 40), (32, 16, 9000, 0), (1000, 2, 300, 0)])
def test_attend_at_the_borders_of_the_splits(fmt, P, G, R, F):
    """One workgroup for a pair's 16 units and one more unit, the last pair of one launch, several chunks with a tail that
    shares a chunk with blocks, more pairs than workgroups that run at a time."""
    print(f"attend_qcache {fmt} P={P} G={G} R={R} F={F}", flush=True)
    g = np.random.default_rng(P + R)
    length = g.integers(0, R + 1, P).tolist()
    length_f = g.integers(0, F + 1, P).tolist()
    length[0], length[-1] = R, R
    c = filled(g, P, R, fmt, length)
    Q = rows(g, P, G, 128)
    K_f, V_f = (rows(g, P, F, 128), rows(g, P, F, 128)) if F else (None, None)
    beta = torch.from_numpy(g.uniform(-3, 3, (P, R)).astype(np.float32)).cuda() if P % 2 else None
    out = A().attend_qcache(Q, c, beta, i32(length), K_f, V_f, i32(length_f) if F else None)
    pairs = sorted({0, 1, P // 3, P // 2, P - 2, P - 1})
    check_attend(out, Q, c, fmt, beta, length, K_f, V_f, length_f if F else None, None, S, pairs=pairs)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("P,G,R,F", [(1, 1, 1, 0), (3, 4, 1, 1), (2, 1, 63, 0), (2, 8, 64, 0), (2, 2, 65, 31),
                                     (5, 4, 512, 0), (3, 4, 513, 257), (2, 16, 1000, 33), (2, 3, 1537, 0),
                                     (2, 13, 130, 256), (1, 4, 20000, 300), (70, 4, 700, 5)])
def test_attend(fmt, P, G, R, F):
    print(f"attend_qcache {fmt} P={P} G={G} R={R} F={F}", flush=True)
    g = np.random.default_rng(R + F)
    c = filled(g, P, R, fmt)
    Q = rows(g, P, G, 128)
    K_f, V_f = (rows(g, P, F, 128, outliers=True), rows(g, P, F, 128)) if F else (None, None)
    beta = torch.from_numpy(g.uniform(-3, 3, (P, R)).astype(np.float32)).cuda() if R % 2 else None
    out = A().attend_qcache(Q, c, beta, None, K_f, V_f)
    check_attend(out, Q, c, fmt, beta, None, K_f, V_f, None, None, S, pairs=range(0, P, max(1, P // 8)))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_attend_ragged_lengths_read_nothing_behind_them(fmt):
    """Lengths from none on; everything behind them is NaN (codes, scales, biases, tail)."""
    g = np.random.default_rng(21)
    length = [0, 1, 63, 64, 65, 511, 512, 513, 1100, 1300, -5, 10 ** 9]
    length_f = [0, 40, 0, 1, 32, 33, 300, 0, 255, 256, 0, 257]
    P, R, F, G = len(length), 1300, 300, 4
    c = filled(g, P, R, fmt, length)
    beta = torch.full((P, R), math.nan, device="cuda")
    Q, K_f, V_f = rows(g, P, G, 128), rows(g, P, F, 128), rows(g, P, F, 128)
    for p in range(P):
        L = min(max(length[p], 0), R)
        beta[p, :L] = torch.from_numpy(g.uniform(-3, 3, L).astype(np.float32)).cuda()
        K_f[p, length_f[p]:] = math.nan
        V_f[p, length_f[p]:] = math.inf
    out = A().attend_qcache(Q, c, beta, i32(length), K_f, V_f, i32(length_f))
    assert out.isfinite().all() and (out[0] == 0).all() and (out[10] == 0).all()
    check_attend(out, Q, c, fmt, beta, length, K_f, V_f, length_f, None, S)
    out = A().attend_qcache(Q, c, None, i32(length))
    assert (out[0] == 0).all()
    check_attend(out, Q, c, fmt, None, length, None, None, None, None, S)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_attend_masks(fmt):
    """Biases of -inf: single rows, whole blocks, whole pairs; what they hide may be NaN.  The type's lowest value and
    large biases are ordinary numbers."""
    g = np.random.default_rng(22)
    P, R, G = 4, 700, 4
    c = filled(g, P, R, fmt)
    Q = rows(g, P, G, 128)
    beta = torch.from_numpy(g.uniform(-30, 30, (P, R)).astype(np.float32)).cuda()
    beta[0, g.random(R) < 0.5] = -math.inf
    beta[1, 64:640] = -math.inf
    beta[2] = -math.inf
    beta[3, g.random(R) < 0.9] = torch.finfo(torch.float32).min
    hidden = beta == -math.inf
    if fmt == "e4m3":
        c.K.view(torch.uint8)[hidden] = 0x7f
        c.V.view(torch.uint8)[hidden] = 0xff
    c.V_scale[1, 3] = math.nan
    c.K_scale[1, 4] = math.inf
    out = A().attend_qcache(Q, c, beta)
    assert out.isfinite().all() and (out[2] == 0).all()
    c.V_scale[1, 3] = c.K_scale[1, 4] = 1.0
    for t in (c.K, c.V):
        t.view(torch.uint8)[hidden] = 0
    check_attend(out, Q, c, fmt, beta, None, None, None, None, None, S)
    # one pair's tail beside a block that is hidden whole
    K_f, V_f = rows(g, P, 3, 128), rows(g, P, 3, 128)
    out = A().attend_qcache(Q, c, beta, None, K_f, V_f)
    check_attend(out, Q, c, fmt, beta, None, K_f, V_f, None, None, S)
    # only the lowest value everywhere: a plain mean where the products vanish beside it
    low = torch.full((P, R), torch.finfo(torch.float32).min, device="cuda")
    out = A().attend_qcache(Q, c, low)
    want = np.stack([oq.q_values(np64(c.V[p]), np64(c.V_scale[p])).mean(axis=0) for p in range(P)])
    assert np.abs(np64(out) - want[:, None]).max() <= 4 * R * U * 8


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("R", [700, 5000])
def test_attend_large_and_small_magnitudes(fmt, R):
    """Values up to 2^112 and down to 2^-90, beside a tail of ordinary ones: sums neither overflow nor vanish."""
    g = np.random.default_rng(28)
    V = rows(g, 4, R, 128)
    V[0] *= 2.0 ** 110
    V[1] *= 2.0 ** -90
    V[2, :R // 2] *= 2.0 ** 100
    c = make_cache(4, R, fmt)
    A().qcache_write(c, rows(g, 4, R, 128), V)
    Q = rows(g, 4, 4, 128)
    out = A().attend_qcache(Q, c)
    assert out.isfinite().all()
    check_attend(out, Q, c, fmt, None, None, None, None, None, None, S)
    K_f, V_f = rows(g, 4, 40, 128), rows(g, 4, 40, 128)
    check_attend(A().attend_qcache(Q, c, None, None, K_f, V_f), Q, c, fmt, None, None, K_f, V_f, None, None, S)


def test_more_pairs_than_a_grid_row():
    """40,000 pairs: pairs lie over two extents of a launch's grid."""
    g = np.random.default_rng(29)
    P, R, G = 40000, 70, 2
    c = A().qcache(P, R, torch.int8)
    K, V = rows(g, 1, R, 128).expand(P, R, 128).clone(), rows(g, 1, R, 128).expand(P, R, 128).clone()
    K[32768:] *= 2
    V[39999] *= 4
    A().qcache_write(c, K, V)
    k, v = A().qcache_read(c)
    Q = rows(g, 1, G, 128).expand(P, G, 128).contiguous()
    blocks, scores = A().select_blocks(Q, c, 1)
    out = A().attend_qcache(Q, c)
    small = A().qcache(3, R, torch.int8)
    at = [0, 32768, 39999]
    A().qcache_write(small, K[at].contiguous(), V[at].contiguous())
    ks, vs = A().qcache_read(small)
    bs, ss = A().select_blocks(Q[at].contiguous(), small, 1)
    os = A().attend_qcache(Q[at].contiguous(), small)
    ranges = [slice(0, 32768), slice(32768, 39999), slice(39999, 40000)]
    tol = 2.0 ** -20      # other splits of the same sums
    for i, r in enumerate(ranges):
        for whole, one in ((k, ks), (v, vs), (scores, ss), (blocks, bs)):
            assert torch.equal(whole[r], one[i:i + 1].expand_as(whole[r]))
        assert (out[r] - os[i]).abs().max() <= tol * (1 + vs[i].float().abs().max())


def test_attend_small_probabilities_times_large_values():
    """A probability of e^-22 beside one of 1, its value 2^18 times the other's: what the fp16 terms keep of it shows."""
    c = make_cache(1, 64, "e4m3")
    K, V = torch.zeros(1, 64, 128, device="cuda"), torch.zeros(1, 64, 128, device="cuda")
    V[0, 0] = 2.0 ** -9
    V[0, 1] = 448
    A().qcache_write(c, K, V)
    assert c.V_scale[0, 0] == 1
    beta = torch.full((1, 64), -math.inf, device="cuda")
    beta[0, 0], beta[0, 1] = 0.0, -22.0
    Q = rows(np.random.default_rng(0), 1, 4, 128)
    out = np64(A().attend_qcache(Q, c, beta))
    want = (2.0 ** -9 + 448 * math.exp(-22)) / (1 + math.exp(-22))
    # the small one: 2^-39 of the largest probability lost, times 448; besides, float32's steps and the exponential
    assert np.abs(out - want).max() <= 2.0 ** -39 * 448 + want * 2.0 ** -20
    assert 448 * math.exp(-22) > 16 * (2.0 ** -39 * 448 + want * 2.0 ** -20)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_attend_nan_reaches_the_output_of_its_pair_alone(fmt):
    g = np.random.default_rng(23)
    c = filled(g, 3, 400, fmt)
    Q = rows(g, 3, 4, 128)
    want = A().attend_qcache(Q, c)
    c.V_scale[1, 2] = math.nan
    out = A().attend_qcache(Q, c)
    assert out[1].isnan().all() and torch.equal(out[0], want[0]) and torch.equal(out[2], want[2])


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_attend_listed_blocks(fmt):
    """Lists in any order, padded, with blocks that are not there or hold nothing, and one listed twice."""
    g = np.random.default_rng(24)
    P, R, G = 5, 1000, 4
    length = [1000, 1000, 100, 0, 640]
    c = filled(g, P, R, fmt, length)
    Q = rows(g, P, G, 128)
    lists = [[0, 3, 15, -1, -1, -1, -1, -1, -1], [15, 2, 9, 1, 4, 7, 0, 11, 12], [1, 5, 0, 99, -7, 2 ** 31 - 1, -2 ** 31, 3, 4],
             [0, 1, 2, 3, 4, 5, 6, 7, 8], [9, 10, -1, 3, 3, -1, -1, -1, 9]]
    blocks = i32(lists)
    for lst in (blocks, blocks[:, :1].contiguous(), blocks[:, :8].contiguous()):
        out = A().attend_qcache(Q, c, None, i32(length), blocks=lst)
        check_attend(out, Q, c, fmt, None, length, None, None, None, lst.cpu(), S)
    F = 70
    K_f, V_f = rows(g, P, F, 128), rows(g, P, F, 128)
    out = A().attend_qcache(Q, c, None, i32(length), K_f, V_f, None, blocks)
    check_attend(out, Q, c, fmt, None, length, K_f, V_f, None, blocks.cpu(), S)
    every = torch.arange(16, dtype=torch.int32, device="cuda").repeat(P, 1)
    assert torch.equal(A().attend_qcache(Q, c, None, i32(length), blocks=every), A().attend_qcache(Q, c, None, i32(length)))


def test_attend_infinite_tail_value():
    g = np.random.default_rng(25)
    c = filled(g, 2, 100, "e4m3")
    Q, K_f, V_f = rows(g, 2, 4, 128), rows(g, 2, 40, 128), rows(g, 2, 40, 128)
    V_f[1, 7, 5] = math.inf
    out = A().attend_qcache(Q, c, None, None, K_f, V_f)
    assert (out[1, :, 5] == math.inf).all() and out[1, :, :5].isfinite().all() and out[0].isfinite().all()


def test_attend_scale_argument():
    g = np.random.default_rng(26)
    c = filled(g, 2, 300, "int8")
    Q = rows(g, 2, 4, 128)
    check_attend(A().attend_qcache(Q, c, scale=0.3), Q, c, "int8", None, None, None, None, None, None, float(np.float32(0.3)))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_attend_of_a_compaction(fmt):
    """A prompt written in 8 bits, read back, compacted, the compact keys and values written in 8 bits, and a decode step
    over them and newer tokens: each step as the float64 attention over what the step before left."""
    import synth
    from tests import gpu_common as gc
    wl = synth.custom("q", kv_heads=2, T=900, q_heads_per_kv=4, n_pos=64, rho=0.2, dtype="bf16", rope=True)
    dev, host = gc.make_inputs(wl)
    g = np.random.default_rng(27)
    c = A().qcache(2, 900, DT[fmt])
    A().qcache_write(c, dev["K"], dev["V"])
    K, V = A().qcache_read(c)
    anchors, C_k, beta, C_v, info = A().compact(K, V, dev["Q"], dev["W1"], dev["b1"], dev["w2"], dev["b2"], 0.2)
    assert int(info.abs().sum()) == 0
    t = C_k.shape[1]
    cc = A().qcache(2, t, DT[fmt])
    A().qcache_write(cc, C_k, C_v)
    m = Mirror(make_cache(2, t, fmt), fmt)
    m.write(C_k, C_v, [0, 0], [t, t])
    m.check(cc)
    Q, K_f, V_f = rows(g, 2, 4, 128), rows(g, 2, 20, 128), rows(g, 2, 20, 128)
    out = A().attend_qcache(Q, cc, beta, None, K_f, V_f)
    check_attend(out, Q, cc, fmt, beta, None, K_f, V_f, None, None, S)


# ------------------------------------------------------------------------------------------------ block selection
def check_select(blocks, scores, Q, c, k, beta, length, s):
    P, n = scores.shape
    for p in range(P):
        L = c.K.shape[1] if length is None else min(max(length[p], 0), c.K.shape[1])
        want = oq.q_block_scores(np64(Q[p]), np64(c.K_bounds[p]), np64(c.K_scale[p]), L, s, None if beta is None else np64(beta[p]))
        got = np64(scores[p])
        fin = np.isfinite(want)
        assert np.array_equal(np.isfinite(got), fin) and np.array_equal(got[~fin], want[~fin])
        # half a step of float32; for the float64 sums' own roundings a little more; what is cut off the 128 channels
        reach = np.abs(np64(c.K_bounds[p])[fin]).max(axis=(1, 2)) * np64(c.K_scale[p])[fin]
        cut = 128 * 2.0 ** -32 * 2 * np.abs(np64(Q[p])).max() * reach * s
        assert (np.abs(got[fin] - want[fin]) <= np.abs(want[fin]) * (U + 2.0 ** -40) + cut).all()
        assert blocks[p].tolist() == sorted(oracle.select_topt(scores[p].cpu().numpy(), k).tolist())


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("P,G,R,k", [(1, 1, 1, 1), (2, 4, 64, 1), (3, 8, 65, 2), (2, 16, 5000, 7), (9, 3, 4095, 64),
                                     (2, 4, 70000, 100), (5, 4, 16384, 256), (3, 4, 16385, 200), (2, 8, 65536, 1024),
                                     (2, 4, 65537, 1), (2, 4, 131072, 64), (2, 2, 131073, 2049)])
def test_select_blocks(fmt, P, G, R, k):
    print(f"select_blocks {fmt} P={P} G={G} R={R} k={k}", flush=True)
    g = np.random.default_rng(R)
    c = filled(g, P, R, fmt)
    Q = rows(g, P, G, 128)
    beta = torch.from_numpy(g.uniform(-3, 3, (P, R)).astype(np.float32)).cuda()
    beta[torch.from_numpy(g.random((P, R)) < 0.3).cuda()] = -math.inf
    for b in (None, beta):
        blocks, scores = A().select_blocks(Q, c, k, b)
        check_select(blocks, scores, Q, c, k, b, None, float(S))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_select_blocks_wide_queries(fmt):
    """Channels that span 2^20 and more, of both signs, rows of zeros and of the smallest numbers: the sums stay exact for
    channels down to 2^-24 of the largest, so blocks that differ in their smallest channels alone keep their order."""
    g = np.random.default_rng(35)
    P, R, G = 3, 1500, 8
    c = filled(g, P, R, fmt)
    e = torch.from_numpy(g.uniform(-22, 0, (P, G, 128)).astype(np.float32)).cuda().exp2()
    Q = (rows(g, P, G, 128).sign() * e).to(torch.bfloat16)
    Q[1, 2:] = 0
    Q[2] *= 2.0 ** -120
    blocks, scores = A().select_blocks(Q, c, 6)
    check_select(blocks, scores, Q, c, 6, None, None, float(S))
    Q[0, 3, 7] = math.nan
    Q[1, 1, 9] = math.inf
    _, bad = A().select_blocks(Q, c, 6)
    assert bad[:2].isnan().all() and torch.equal(bad[2], scores[2])
    # blocks alike but for one code in a channel that the query weighs 2^-22 as much as the others
    K = rows(g, 1, 1, 128).repeat(1, 640, 1)
    K[0, 5 * 64:6 * 64, 3] += 0.25
    t = make_cache(1, 640, fmt)
    A().qcache_write(t, K, K)
    q = torch.ones(1, 1, 128, device="cuda")
    q[0, 0, 3] = 2.0 ** -22
    q = q.to(torch.bfloat16)
    blocks, scores = A().select_blocks(q, t, 1)
    check_select(blocks, scores, q, t, 1, None, None, float(S))


def test_select_blocks_ragged_masked_and_tied():
    g = np.random.default_rng(31)
    length = [0, 1, 64, 65, 1000, -3, 10 ** 9, 640]
    P, R, k = len(length), 1000, 5
    c = filled(g, P, R, "e4m3", length)
    Q = rows(g, P, 4, 128)
    beta = torch.full((P, R), math.nan, device="cuda")
    for p in range(P):
        beta[p, :min(max(length[p], 0), R)] = 0.5
    beta[4, 128:320] = -math.inf
    blocks, scores = A().select_blocks(Q, c, k, beta, i32(length), scale=0.25)
    check_select(blocks, scores, Q, c, k, beta, length, 0.25)
    assert blocks[0].tolist() == [0, 1, 2, 3, 4]
    # equal blocks: the lower ones; a NaN scale ranks last
    K = rows(g, 1, 64, 128).repeat(1, 10, 1)
    t = A().qcache(1, 640)
    A().qcache_write(t, K, K)
    t.K_scale[0, 1] = math.nan
    blocks, scores = A().select_blocks(Q[:1], t, 4)
    assert blocks.tolist() == [[0, 2, 3, 4]] and scores[0, 1].isnan()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_sparse_step(fmt):
    """Write token by token and in chunks, select, attend: what a decode step over a long context runs.  Attending to the
    selected blocks is near attention over all of them once a query prefers a few."""
    g = np.random.default_rng(33)
    P, R, G = 4, 2000, 4
    length = [2000, 1990, 777, 65]
    K, V = rows(g, P, R, 128), rows(g, P, R, 128)
    K[:, 300:310] = K[:, 300:301] * 3                  # what the queries look for
    Q = (K[:, 300:301] * torch.tensor([1.0, 0.9, 1.1, 1.0], device="cuda")[None, :, None]).to(torch.bfloat16).contiguous()
    c = make_cache(P, R, fmt)
    A().qcache_write(c, K, V, None, i32([x - 2 for x in length]))
    for i in (2, 1):
        at = [x - i for x in length]
        idx = torch.tensor(at, device="cuda")
        row = lambda x: x[torch.arange(P, device="cuda"), idx][:, None].contiguous()
        A().qcache_write(c, row(K), row(V), i32(at))
    blocks, scores = A().select_blocks(Q, c, 3, None, i32(length))
    check_select(blocks, scores, Q, c, 3, None, length, float(S))
    assert all(4 in b for b in blocks.tolist()[:3])
    out = A().attend_qcache(Q, c, None, i32(length), blocks=blocks)
    check_attend(out, Q, c, fmt, None, length, None, None, None, blocks.cpu(), S)


# ------------------------------------------------------------------------------------------------ streams, graphs, devices
def decode_step(c, Q, K, V, start, length, out, ws, k):
    A().qcache_write(c, K, V, start)
    blocks, scores = A().select_blocks(Q, c, k, None, length)
    A().attend_qcache(Q, c, None, length, blocks=blocks, out=out, ws=ws)
    return blocks, scores


def test_captured_and_replayed_with_eager_work_between():
    g = np.random.default_rng(41)
    P, R, G, k = 3, 1200, 4, 9
    lens = [1000, 64, 517]
    c = filled(g, P, R, "e4m3", lens)
    Q, K, V = rows(g, P, G, 128), rows(g, P, 1, 128), rows(g, P, 1, 128)
    start, length = i32(lens), i32([x + 1 for x in lens])
    ws = A()._workspace(A().attend_qcache_workspace_size(P, R, G, k), "cuda")
    out = torch.empty(P, G, 128, device="cuda")
    decode_step(c, Q, K, V, start, length, out, ws, k)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        decode_step(c, Q, K, V, start, length, out, ws, k)
    e = A().QCache(*(t.clone() for t in c))
    ws2 = ws.clone()
    for i in range(4):
        Q.copy_(rows(g, P, G, 128))
        K.copy_(rows(g, P, 1, 128))
        V.copy_(rows(g, P, 1, 128))
        graph.replay()
        torch.cuda.synchronize()
        want = torch.empty_like(out)
        off = (-ws2.data_ptr()) % 256
        decode_step(e, Q, K, V, start, length, want, ws2[off:] if off == 0 else None, k)
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
        for a, b in zip(c, e):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), i
        start += 1
        length += 1


def test_on_a_side_stream():
    g = np.random.default_rng(42)
    c = filled(g, 2, 900, "int8")
    Q = rows(g, 2, 4, 128)
    want = A().attend_qcache(Q, c)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out = A().attend_qcache(Q, c)
    s.synchronize()
    assert torch.equal(out, want)


def test_two_streams_at_once():
    """Calls on two streams with workspaces of their own (the binding's), each many chunks."""
    g = np.random.default_rng(45)
    cs = [filled(g, 8, 9000, "e4m3"), filled(g, 8, 9000, "int8")]
    Q = [rows(g, 8, 4, 128), rows(g, 8, 4, 128)]
    want = [(A().attend_qcache(q, c), A().select_blocks(q, c, 9)) for q, c in zip(Q, cs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append((A().attend_qcache(Q[i], cs[i]), A().select_blocks(Q[i], cs[i], 9)))
    torch.cuda.synchronize()
    for i in range(2):
        for out, (blocks, scores) in got[i]:
            assert torch.equal(out, want[i][0]) and torch.equal(blocks, want[i][1][0]) and torch.equal(scores, want[i][1][1])


def test_results_do_not_change_between_runs():
    g = np.random.default_rng(43)
    c = filled(g, 16, 3000, "e4m3")
    Q = rows(g, 16, 4, 128)
    first = A().attend_qcache(Q, c)
    for _ in range(3):
        assert torch.equal(A().attend_qcache(Q, c), first)


def test_offsets_past_32_bits():
    """A cache of more than 2^32 codes: the last pairs, written, read, selected from and attended to."""
    g = np.random.default_rng(44)
    P, R, G = 40, 1 << 20, 4
    c = A().qcache(P, R)
    K = rows(g, 1, 256, 128)
    n, at = 256, R - 256
    src = K.expand(P, n, 128).contiguous()
    start, full = i32([at] * P), i32([R] * P)
    for t in (c.K, c.V):
        t.view(torch.uint8).zero_()
    c.K_scale.fill_(1.0)
    c.V_scale.fill_(1.0)
    c.K_bounds.view(torch.uint8).zero_()
    src[P - 1] *= 2
    A().qcache_write(c, src, src, start)
    k, v = A().qcache_read(c, at, n, torch.bfloat16)
    small = A().qcache(2, n)
    A().qcache_write(small, src[P - 2:], src[P - 2:])
    ks, _ = A().qcache_read(small)
    assert torch.equal(k[P - 2:], ks) and torch.equal(v[P - 2:], ks)
    Q = K[:, :4].expand(P, G, 128).contiguous()
    blocks, _ = A().select_blocks(Q, c, 4, None, full)
    assert set(range(R // 64 - 4, R // 64)) == set(blocks[P - 1].tolist())
    out = A().attend_qcache(Q, c, None, full, blocks=blocks)
    every = torch.arange(4, dtype=torch.int32, device="cuda").repeat(2, 1)
    assert torch.equal(out[P - 2:], A().attend_qcache(Q[P - 2:].contiguous(), small, blocks=every))


@pytest.mark.parametrize("fmt,growth", [("int8", 1.02), ("int8", 1.1), ("e4m3", 1.1), ("e4m3", 1.4)])
def test_single_tokens_stay_within_a_step(fmt, growth):
    """Blocks written row by row, so that kept rows are rounded again whenever the scale grows: less than a step of the
    largest scale since in int8; in e4m3 2^-4 of the value from 2^-6 scale on, less than 2^-9 scale below."""
    g = np.random.default_rng(11)
    P, R = 3, 128
    x = rows(g, P, R, 128) * torch.tensor(growth).pow(torch.arange(R) % 64).cuda()[None, :, None]
    x = x.to(torch.bfloat16)
    c = make_cache(P, R, fmt)
    s = torch.zeros(P, R, 1, device="cuda", dtype=torch.float64)       # the largest scale since the row was written
    for i in range(R):
        A().qcache_write(c, x[:, i:i + 1].contiguous(), -x[:, i:i + 1].contiguous(), i32([i] * P))
        since = s[:, i // 64 * 64:i + 1]
        since.copy_(torch.maximum(since, c.K_scale[:, i // 64, None, None].double()))
    k, v = A().qcache_read(c, dtype=torch.float32)
    assert torch.equal(k, -v)
    err, x = (k.double() - x.double()).abs(), x.double().abs()
    half = s / 2 if fmt == "int8" else torch.maximum(x * 2.0 ** -4, s * 2.0 ** -10)
    if fmt == "int8":
        assert (err < s).all()
    else:
        assert torch.where(x >= 2.0 ** -6 * s, err <= 2.0 ** -4 * x, err < 2.0 ** -9 * s).all()
    assert (err > half).any()                            # more than a block written once is off by


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_block_scores_bound_the_logits_up_to_their_roundings(fmt):
    """No logit exceeds its block's score by more than half a step of float32 and what is cut off small channels: 2^-24 of
    s times the query's largest magnitude times the block's largest key.  Each can put the score below a logit."""
    g = np.random.default_rng(36)
    P, R, G = 4, 640, 4
    K = rows(g, P, R, 128)
    Q = rows(g, P, G, 128)
    K[1:3] = K[1:3].abs()
    K[1:3, :, 0] = 0
    Q[1, :, 1:] = 2.0 ** -33 * Q[1, :, 1:].abs().clamp(0.25, 2)         # beside channel 0, where the keys are 0
    Q[1:3, :, 0] = 1.0
    Q[2, :, 1:] = 2.0 ** -20 * Q[2, :, 1:].abs()
    K[3] = K[3, :1]                                                      # blocks of one key: the bound is its logit
    c = make_cache(P, R, fmt)
    A().qcache_write(c, K, K)
    _, scores = A().select_blocks(Q, c, 1)
    sc = np64(scores)
    over = np.zeros(P, bool)
    for p in range(P):
        k = oq.q_values(np64(c.K[p]), np64(c.K_scale[p]))
        logit = (S * np64(Q[p]) @ k.T).max(axis=0).reshape(-1, 64).max(axis=1)
        reach = np.abs(k).reshape(-1, 64 * 128).max(axis=1)
        slack = 1.001 * U * np.abs(sc[p]) + 2.0 ** -24 * S * np.abs(np64(Q[p])).max() * reach
        assert (logit <= sc[p] + slack).all(), p
        over[p] = (logit > sc[p]).any()
    assert over[1] and (sc[1] == 0).all()
