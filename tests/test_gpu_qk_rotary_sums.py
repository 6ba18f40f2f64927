"""Gradients of the norm's weights over long batches against sums in 64 bits, column by column."""
import pytest
import torch

import paper_1905_10395_amd as L
from test_gpu_qk_rotary import DEV, EPS, d, rnd, rotate

pytestmark = pytest.mark.gpu

# a lane adds up at most 8 rows here, a workgroup 64 teams, the join up to 682 workgroups as 16 stretches of 43, then those 16
ADDITIONS = 8 + 64 + 43 + 16


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", [64, 63, 200])
@pytest.mark.parametrize("interleaved", [False, True])
def test_weights_gradients_of_long_batches(dtype, D, interleaved):
    W, T, Hq, Hk = 3, 4000, 5, 2
    R = D // 2 * 2
    q, k = rnd(W, T, Hq, D, seed=1, dtype=dtype), rnd(W, T, Hk, D, seed=2, dtype=dtype)
    gq, gk = rnd(W, T, Hq, D, seed=3, dtype=dtype), rnd(W, T, Hk, D, seed=4, dtype=dtype)
    w = rnd(W, 2 * D, seed=5) * 0.3 + 1.0
    turns = L.rotary_turns(R, device=DEV)
    _, _, stats = L.qk_rotary(q, k, None, turns, w_q=w[:, :D], w_k=w[:, D:], interleaved=interleaved)
    dw = torch.full_like(w, 3.0)
    L.qk_rotary_grad(gq, gk, q, k, stats, None, turns, w_q=w[:, :D], w_k=w[:, D:], interleaved=interleaved, dw_q=dw[:, :D], dw_k=dw[:, D:])
    pos = torch.arange(T)[None].expand(W, T)
    for x, g, got, s in ((q, gq, dw[:, :D], stats[:, :, :Hq]), (k, gk, dw[:, D:], stats[:, :, Hq:])):
        dz, e = rotate(d(g), torch.zeros(g.shape, dtype=torch.float64), pos, d(turns), R, interleaved, 1.0, back=True)
        h = d(x) * d(s)[..., None]
        size = (dz * h).abs()
        # a term: the rotation's error, and a rounding of h and of the product each
        bound = (e * h.abs() + size * (ADDITIONS + 2) * EPS).sum((1, 2))
        assert bool(((d(got) - (dz * h).sum((1, 2))).abs() <= bound).all())
        # the bound is small beside any single row's term: one that is lost or counted twice shows
        assert float(bound.max()) < 0.05 * float(size.amax((1, 2)).min())
