"""Attention over the 4-bit cache where its codes are read as streams (above 96 MiB of them): pairs that eight waves take
whole, and those of four waves with and without bias.

Random rows: some pairs against the oracle, within test_gpu_ncache's bounds.

Every row of every pair: logits are 0 or at least 900 below it, so that n rows weigh the same and the others nothing; values are 0 and 1.
n equal probabilities are summed at u = 2^-24 each, their products at 2u for the first of three terms and 2^-7 of that
for the others, joins of at most eight waves, the exponentials that join them and the division add less than 100u: (4 n + 100) u.
A row that is lost, counted twice or takes another's place changes a channel's mean by about 1 / 2n; n <= 700, so the bound is a quarter
of that.
"""
import math

import pytest
import torch

from tests.test_gpu_ncache import A, U, check_attend, i32, make_cache

pytestmark = pytest.mark.gpu

SHAPES = [(256, 3300, 0), (256, 3200, 33), (200, 4000, 40), (300, 3001, 40)]
GS = [1, 4, 6, 8, 11, 16]


def lengths(P, R, F, gen):
    length = torch.randint(0, R + 1, (P,), device="cuda", generator=gen).int()
    length[:8] = i32([R, 0, 1, 63, 64, 65, R - 1, R // 2])
    return length, torch.randint(0, F + 1, (P,), device="cuda", generator=gen).int() if F else None


def streamed(P, R, F, G):
    assert P * R * 128 > 96 << 20
    assert P > 256 or A().attend_ncache_workspace_size(P, R, G, F) == 0      # one workgroup a pair
    gen = torch.Generator(device="cuda")
    gen.manual_seed(R + G)
    return gen


@pytest.mark.parametrize("plain", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("G", GS)
@pytest.mark.parametrize("P,R,F", SHAPES)
def test_streamed(P, R, F, G, bias, plain):
    """plain: all rows of all pairs, else lengths from none on; rows behind them hold what nothing may depend on."""
    gen = streamed(P, R, F, G)
    randn = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    length, length_f = (None, None) if plain else lengths(P, R, F, gen)
    c = make_cache(P, R)
    A().ncache_write(c, randn(P, R, 128).bfloat16(), randn(P, R, 128).bfloat16(), None, length)
    Q = randn(P, G, 128).bfloat16()
    K_f, V_f = (randn(P, F, 128).bfloat16(), randn(P, F, 128).bfloat16()) if F else (None, None)
    beta = None
    if bias:
        beta = randn(P, R)
        beta[:, ::5] = -math.inf
        beta[9] = -math.inf
    print(f"streamed P={P} R={R} F={F} G={G} bias={bias} plain={plain}", flush=True)
    out = A().attend_ncache(Q, c, beta, length, K_f, V_f, length_f)
    for p in (0, 1, 3, 9, P // 2, P - 1):
        cut = lambda t: None if t is None else t[p:p + 1]
        host = lambda t: None if t is None else t[p:p + 1].tolist()
        check_attend(cut(out), cut(Q), [cut(t) for t in c], cut(beta), host(length), cut(K_f), cut(V_f), host(length_f))
    assert torch.equal(out, A().attend_ncache(Q, c, beta, length, K_f, V_f, length_f))


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("G", GS)
@pytest.mark.parametrize("P,R,F", SHAPES)
def test_streamed_every_row(P, R, F, G, bias):
    gen = streamed(P, R, F, G)
    rand = lambda *s: torch.rand(*s, device="cuda", generator=gen)
    length, length_f = lengths(P, R, F, gen)
    at = 8 * torch.arange(G, device="cuda")                                  # the channel that a query looks at
    Q = torch.zeros(P, G, 128, dtype=torch.bfloat16, device="cuda")
    Q[:, torch.arange(G, device="cuda"), at] = 1.0

    def part(n, chance, held):
        """Keys, values and what each query counts of n rows."""
        use = rand(P, n, G) < chance
        K, V = torch.zeros(P, n, 128, device="cuda"), (rand(P, n, 128) < 0.5).float()
        K[:, :, at] = torch.where(use, 0.0, -1024.0)
        return K, V, use & (torch.arange(n, device="cuda")[None, :, None] < held[:, None, None])
    K, V, use = part(R, 600 / R, length)
    beta = None
    if bias:
        left_out = rand(P, R) < 0.2
        beta, use = torch.where(left_out, -math.inf, 0.0), use & ~left_out[..., None]
    c = make_cache(P, R)
    A().ncache_write(c, K, V, None, length)
    count = lambda use, V: torch.matmul(use.double().transpose(1, 2).contiguous(), V.double())
    total, n = count(use, V), use.sum(1)
    K_f = V_f = None
    if F:
        K_f, V_f, use_f = part(F, 0.3, length_f)
        total, n, K_f, V_f = total + count(use_f, V_f), n + use_f.sum(1), K_f.bfloat16(), V_f.bfloat16()
    # a query that looks at no row counts all that are held, alike
    some = n > 0
    assert int(n.max()) <= 700 and int(some.sum()) > P * G // 2
    print(f"streamed, every row P={P} R={R} F={F} G={G} bias={bias}", flush=True)
    out = A().attend_ncache(Q, c, beta, length, K_f, V_f, length_f, scale=1.0).double()
    want = total / n[..., None]
    bad = ((out - want).abs() > (4 * n[..., None] + 100) * U) & some[..., None]
    assert not bad.any(), (bad.nonzero()[:4], (out - want)[bad][:4])
