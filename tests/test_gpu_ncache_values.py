"""Attention over the 4-bit cache at the ends of what its inputs may hold: queries that are not finite over the uncompressed
tail, and values whose mean is finite where a plain sum of them would not be."""
import math

import numpy as np
import pytest
import torch

from tests.test_gpu_ncache import A, U, check_attend, i32, make_cache, np64, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("held", ["tail only", "masked", "masked, many rows"])
@pytest.mark.parametrize("G", [1, 4, 7, 16])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_non_finite_query_over_the_tail(bad, G, held):
    """A query row with a non-finite channel is NaN where there is a row to attend to, also where that row is the tail's:
    whatever sign its keys have in that channel, zero among them.  Other query rows and pairs without a row do not see it."""
    g = np.random.default_rng(G)
    P, F = 4, 45
    R = 20000 if held == "masked, many rows" else 300
    c = make_cache(P, R)
    A().ncache_write(c, torch.ones(P, R, 128, device="cuda"), torch.ones(P, R, 128, device="cuda"))
    Q, K_f, V_f = rows(g, P, G, 128), rows(g, P, F, 128), rows(g, P, F, 128)
    K_f[0, :, 77], K_f[1, :, 77], K_f[2, :, 77], K_f[3, :, 77] = -1.5, 1.5, 0.0, -2.0
    Q[:, G - 1, 77] = bad
    beta = torch.full((P, R), -math.inf, device="cuda")
    length = i32([0] * P) if held == "tail only" else None
    print(f"bad={bad} G={G} {held}", flush=True)
    out = A().attend_ncache(Q, c, None if held == "tail only" else beta, length, K_f, V_f, i32([F, 1, 33, 0]))
    assert out[:3, G - 1].isnan().all()
    assert out[:3, :G - 1].isfinite().all()
    assert (out[3] == 0).all()
    if G > 1:
        check_attend(out[:3, :G - 1], Q[:3, :G - 1], [t[:3] for t in c], None, [0] * 3, K_f[:3], V_f[:3], [F, 1, 33])


BIG = 6 * 2.0 ** 125                                                 # the cache's largest value
MOST = float(torch.finfo(torch.bfloat16).max)


def near(out, want, n, big):
    """Within the attention's bound for n rows whose logits are exact, all values up to big."""
    out = np64(out)
    assert np.isfinite(out).all()
    assert (np.abs(out - want) <= 2 * (2.0 ** -21 + 12 * n * U) * big).all(), np.abs(out - want).max() / big


@pytest.mark.parametrize("G", [3, 8, 16])
@pytest.mark.parametrize("P,R,F", [(3, 400, 0), (3, 400, 70), (3, 4000, 40), (2, 30000, 0), (300, 700, 33), (200, 4000, 0)])
def test_many_rows_of_the_largest_values(P, R, F, G):
    """Rows of equal weight whose values are the largest that cache and tail hold: the mean is that value, however many."""
    c = make_cache(P, R)
    A().ncache_write(c, torch.zeros(P, R, 128, device="cuda"), torch.full((P, R, 128), 3.3e38, device="cuda"))
    Q = torch.ones(P, G, 128, dtype=torch.bfloat16, device="cuda")
    K_f, V_f = (torch.zeros(P, F, 128, device="cuda").bfloat16(), torch.full((P, F, 128), MOST, device="cuda").bfloat16()) if F else (None, None)
    print(f"largest P={P} R={R} F={F} G={G}", flush=True)
    want = (R * BIG + F * MOST) / (R + F)
    near(A().attend_ncache(Q, c, None, None, K_f, V_f), want, R + F, MOST)
    near(A().attend_ncache(Q, c, torch.zeros(P, R, device="cuda"), None, K_f, V_f), want, R + F, MOST)
    if F:
        near(A().attend_ncache(Q, c, None, i32([0] * P), K_f, V_f), MOST, F, MOST)


@pytest.mark.parametrize("G", [4, 16])
@pytest.mark.parametrize("step", [0.0, 0.5, 5.5, 6.0, 100.0])
def test_largest_values_behind_smaller_logits(step, G):
    """Values of one and logits of 0 first, then several rows of the largest values with logits a little or far above, in each
    of a wave's later blocks and in the tail."""
    P, R, F = 2, 3000, 40
    late = torch.zeros(P, R, dtype=torch.bool, device="cuda")
    late[:, 1500:] = torch.rand(P, 1500, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)) < 0.5
    V = torch.where(late[..., None], 3.3e38, 1.0).expand(P, R, 128).contiguous()
    b = torch.where(late, step, 0.0).float()
    c = make_cache(P, R)
    A().ncache_write(c, torch.zeros(P, R, 128, device="cuda"), V)
    Q = torch.zeros(P, G, 128, dtype=torch.bfloat16, device="cuda")
    Q[..., 0] = 1.0
    K_f, V_f = torch.zeros(P, F, 128, device="cuda").bfloat16(), torch.full((P, F, 128), MOST, device="cuda").bfloat16()
    K_f[..., 0] = step
    n, w = late.sum(1).double().cpu().numpy(), math.exp(-step)
    print(f"behind smaller logits step={step} G={G}", flush=True)
    out = A().attend_ncache(Q, c, b, scale=1.0)
    near(out, ((n * BIG + w * (R - n)) / (n + w * (R - n)))[:, None, None], R, MOST)
    out = A().attend_ncache(Q, c, b, None, K_f, V_f, scale=1.0)
    near(out, ((n * BIG + F * MOST + w * (R - n)) / (n + F + w * (R - n)))[:, None, None], R + F, MOST)


def test_small_values_at_many_rows():
    """What keeps large sums in range takes nothing from small values: rows of 2^-60, with random signs, many of them."""
    g = np.random.default_rng(3)
    P, R, G = 2, 5000, 4
    c = make_cache(P, R)
    A().ncache_write(c, rows(g, P, R, 128), rows(g, P, R, 128) * 2.0 ** -60)
    Q = rows(g, P, G, 128)
    K_f, V_f = rows(g, P, 40, 128), rows(g, P, 40, 128) * 2.0 ** -60
    check_attend(A().attend_ncache(Q, c, None, None, K_f, V_f) * 2.0 ** 60, Q, [c[0], c[1], c[2], c[3] + 60], None, None, K_f,
                 V_f * 2.0 ** 60, None)


@pytest.mark.parametrize("G", [1, 6, 16])
def test_logits_of_minus_infinity(G):
    """Rows whose logit is -inf, of an infinite key in the tail or of products beyond float32, count as left out; of +inf, the
    query is NaN."""
    g = np.random.default_rng(G)
    P, R, F = 3, 200, 50
    c = make_cache(P, R)
    K = rows(g, P, R, 128)
    K[0, ::3] = 0
    K[0, ::3, 9] = -2.0 ** 120
    K[1], K[1, :, 9] = 0, -2.0 ** 120
    A().ncache_write(c, K, rows(g, P, R, 128))
    Q, K_f, V_f = rows(g, P, G, 128), rows(g, P, F, 128), rows(g, P, F, 128)
    Q[:2] = 0
    Q[:2, :, 9] = 2.0 ** 20
    Q[2, :, 9] = 1.0
    K_f[:] = 0
    K_f[2, ::2, 9] = -math.inf
    print(f"logits of -inf G={G}", flush=True)
    out = A().attend_ncache(Q, c)
    beta = torch.zeros(P, R, device="cuda")
    beta[0, ::3] = -math.inf
    check_attend(out[:1], Q[:1], [t[:1] for t in c], beta[:1], None, None, None, None)
    assert (out[1] == 0).all() and out[2].isfinite().all()
    out = A().attend_ncache(Q, c, None, i32([0] * P), K_f, V_f)[2:]
    check_attend(out, Q[2:], [t[2:] for t in c], None, [0], K_f[2:, 1::2], V_f[2:, 1::2], None)
    K_f[2, 0, 9] = math.inf
    assert A().attend_ncache(Q, c, None, None, K_f, V_f)[2].isnan().all()
