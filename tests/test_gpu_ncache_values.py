"""Attention over the 4-bit cache at the ends of what its inputs may hold: queries that are not finite over the uncompressed
tail."""
import math

import numpy as np
import pytest
import torch

from tests.test_gpu_ncache import A, check_attend, i32, make_cache, rows

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
