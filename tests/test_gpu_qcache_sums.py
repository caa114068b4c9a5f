"""Attention over the 8-bit cache where every row's share of the result shows.

Exact sums: keys, queries and biases are chosen so that a logit is the largest of its query's or at least 900 below it,
so a probability is 1 / n or 0; values are 0 and 1, stored without error.  The kernels' sums are then whole numbers, the
factors that join them 1 or 0, and what is left is one division: 2^-24 of the result, 2^-22 allowed.  A row that is lost,
read twice or read in another's place changes a sum by at least 1 of n <= 2^19.

Far logits: a block whose logits lie D below another's, its values larger by as much.  u = 2^-24; the logits are exact; an
exponential's argument is off by the steps of its subtraction, of its product and of log2 e, D u each, the exponential by 4u; 64
products are summed at 2u each (the accumulator may truncate), as are the probabilities, and each is halved into two
terms (4u); joining, scaling and dividing add 32u: (3 D + 320) u sum_j p_j |v_j|.
"""
import math

import numpy as np
import pytest
import torch

from oracle import qcache as oq
from tests.test_gpu_qcache import A, DT, U, np64

pytestmark = pytest.mark.gpu


def bits(g, *shape):
    return torch.from_numpy(g.integers(0, 2, shape, dtype=np.int8)).cuda().to(torch.bfloat16)


def lengths(g, P, most):
    x = g.integers(0, most + 1, P)
    x[0] = most
    x[P // 2] = min(most, 64)
    x[-1] = 0 if P > 2 else most
    return torch.from_numpy(x.astype(np.int32)).cuda()


def exact_sums(Q, K, V, weight, bias, K_f, V_f, weight_f):
    """[P][G][128] float32: the mean of the values of the largest logit, each row counted weight times."""
    chosen = Q.argmax(dim=2)                                        # the one channel of a query that is not zero
    size = Q.amax(dim=2).float()

    def logits(K, weight, bias):
        x = torch.gather(K.float(), 2, chosen[:, None, :].expand(-1, K.shape[1], -1)).transpose(1, 2) * size[:, :, None]
        if bias is not None:
            x = x + bias[:, None, :]
        return torch.where((weight > 0)[:, None, :], x, torch.full_like(x, -math.inf))
    x, w, v = logits(K, weight, bias), weight, V.float()
    if K_f is not None:
        x = torch.cat([x, logits(K_f, weight_f, None)], dim=2)
        w, v = torch.cat([w, weight_f], dim=1), torch.cat([v, V_f.float()], dim=1)
    top = x.amax(dim=2, keepdim=True)
    take = ((x == top) & (top > -math.inf)).float() * w[:, None, :]
    total, sums = take.sum(dim=2, keepdim=True), torch.matmul(take.contiguous(), v.contiguous())
    assert total.max() < 2 ** 19
    return torch.where(total > 0, sums / total.clamp(min=1), torch.zeros_like(sums))


# pairs, queries, rows, tail rows: one workgroup per pair and its last size; a unit a wave in many chunks; several units a
# wave in one, two and many chunks, blocks and tail in one chunk; more pairs than run at a time; caches that are streamed
SIZES = [(8, 4, 819, 37), (256, 3, 1024, 0), (257, 3, 1024, 0), (1, 5, 70000, 0), (2, 4, 20000, 300), (32, 16, 9000, 0),
         (300, 4, 2100, 40), (600, 2, 700, 257), (900, 1, 130, 0), (16, 8, 65537, 33), (1, 2, 262145, 70), (769, 7, 64, 1)]


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("form", ["plain", "bias", "listed", "listed with bias"])
@pytest.mark.parametrize("P,G,R,F", SIZES)
def test_every_row_once(fmt, form, P, G, R, F):
    print(f"attend_qcache {fmt} {form} P={P} G={G} R={R} F={F}", flush=True)
    g = np.random.default_rng(P * 7 + R)
    n = -(-R // 64)
    K, V = -bits(g, P, R, 128), bits(g, P, R, 128)
    c = A().qcache(P, R, DT[fmt])
    A().qcache_write(c, K, V)
    Q = torch.zeros(P, G, 128, device="cuda")
    for q in range(1, G):                                            # the first query: all rows alike
        Q[torch.arange(P, device="cuda"), q, torch.from_numpy(g.integers(0, 128, P)).cuda()] = 4096.0
    Q = Q.to(torch.bfloat16)
    length, length_f = lengths(g, P, R), lengths(g, P, F) if F else None
    at = torch.arange(R, device="cuda")
    weight = (at[None, :] < length[:, None]).float()
    bias = blocks = K_f = V_f = weight_f = None
    if "bias" in form:
        bias = torch.from_numpy(g.choice(np.array([0, 0, 0, -5000, -math.inf], np.float32), (P, R))).cuda()
        weight = torch.where(bias > -math.inf, weight, torch.zeros_like(weight))
    if "listed" in form:
        listed = torch.from_numpy(g.integers(-1, n + 1, (P, max(1, n // 3))).astype(np.int32)).cuda()   # some twice
        blocks = listed.contiguous()
        held = torch.zeros(P, n + 2, device="cuda")
        held.scatter_add_(1, listed.long() + 1, torch.ones_like(listed, dtype=torch.float32))
        weight = weight * held[:, 1:n + 1].repeat_interleave(64, dim=1)[:, :R]
    if F:
        K_f, V_f = -bits(g, P, F, 128), bits(g, P, F, 128)
        weight_f = (torch.arange(F, device="cuda")[None, :] < length_f[:, None]).float()
    out = A().attend_qcache(Q, c, bias, length, K_f, V_f, length_f, blocks, scale=1.0)
    want = exact_sums(Q, K, V, weight, bias, K_f, V_f, weight_f)
    bad = (out - want).abs() > 2.0 ** -22 * want
    assert not bad.any() and out.isfinite().all(), bad.nonzero()[:5].tolist()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("by", ["bias", "keys"])
@pytest.mark.parametrize("D", [20, 28, 30, 60])
@pytest.mark.parametrize("P", [3, 500])
def test_far_logits_with_large_values(fmt, by, D, P):
    """Two blocks that one wave takes in turn (500 pairs) or two waves do (3 pairs), in both orders: the one with the small
    probabilities decides the result."""
    print(f"attend_qcache {fmt} {by} D={D} P={P}", flush=True)
    g = np.random.default_rng(D)
    R, G = 512, 4
    K = torch.zeros(P, R, 128, device="cuda")
    bias = torch.full((P, R), -math.inf, device="cuda")
    V = torch.from_numpy(g.standard_normal((1, R, 128)).astype(np.float32)).cuda().repeat(P, 1, 1)
    K[:, :, 5] = -40.0                                               # 40 D below: nothing
    for p in range(2):
        near, far = (0, 256) if p == 0 else (256, 0)
        K[p::2, near:near + 64, 5] = 0.0
        K[p::2, far:far + 64, 5] = -1.0
        bias[p::2, near:near + 64] = 0.0
        bias[p::2, far:far + 64] = -float(D)
        V[p::2, far:far + 64] *= 2.0 ** (1.5 * D + 15)
    if by == "bias":
        K.zero_()
    else:
        bias = None
    Q = torch.zeros(P, G, 128, device="cuda", dtype=torch.bfloat16)
    Q[:, :, 5] = float(D)
    c = A().qcache(P, R, DT[fmt])
    A().qcache_write(c, K, V)
    out = np64(A().attend_qcache(Q, c, bias, scale=1.0))
    for p in sorted({0, 1, 2, P // 2, P - 1}):
        k, v = oq.q_values(np64(c.K[p]), np64(c.K_scale[p])), oq.q_values(np64(c.V[p]), np64(c.V_scale[p]))
        ref, mass = oq.q_attend(np64(Q[p]), k, v, None if bias is None else np64(bias[p]), None, None, 1.0)
        assert np.abs(ref).max() > 1e3                               # the far block's, not the near one's
        assert (np.abs(out[p] - ref) <= (3 * D + 320) * U * mass).all(), (p, float((np.abs(out[p] - ref) / mass).max()))
