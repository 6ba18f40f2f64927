"""Attention and its gradients where infinities and NaN lie among the data: what sees nothing stays zero, and what nothing sees has no effect."""
import math

import pytest
import torch

import paper_1905_10395_amd as L
from test_gpu_attention import BF16, F32, inputs, lengths

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")
# 32 rows or keys a workgroup, and 128; heads on 16 bytes, and off them
FEW = [(2, 100, 70, 6, 2, 64), (1, 100, 70, 1, 1, 45), (2, 75, 33, 4, 4, 128), (1, 130, 1, 2, 1, 3)]
MANY = [(24, 220, 150, 6, 6, 64), (24, 220, 150, 12, 6, 90), (24, 220, 150, 6, 6, 128), (24, 220, 150, 12, 6, 125), (24, 220, 150, 6, 6, 24)]


def poison(x, where):
    """NaN and both infinities in the marked rows [B, T] of x."""
    bad = torch.tensor([NAN, INF, -INF, NAN], dtype=x.dtype, device=x.device)[torch.arange(x.shape[3], device=x.device) % 4]
    return torch.where(where[:, :, None, None], bad, x)


@pytest.mark.parametrize("shape", FEW + MANY)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lens", [False, True])
def test_queries_that_see_no_key_have_no_effect(shape, dtype, lens):
    """Causal, more queries than keys: what stands at the first queries reaches neither results nor gradients."""
    B, Tq, Tk, Hq, Hk, D = shape
    q, k, v, do = inputs(B, Tq, Tk, Hq, Hk, D, dtype)
    nk = torch.full((B,), Tk)
    if lens:
        nk = torch.arange(B) * 7 % (Tk + 1)
    args = dict(causal=True, k_lens=lengths(nk.tolist()))
    out, lse = L.attention(q, k, v, **args)
    grads = L.attention_grad(do, q, k, v, out, lse, **args)
    blind = (torch.arange(Tq)[None] < (Tq - nk)[:, None]).to(q.device)
    q2, do2 = poison(q, blind), poison(do, blind)
    out2, lse2 = L.attention(q2, k, v, **args)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)
    assert bool((out2[blind] == 0).all()) and bool((lse2.transpose(1, 2)[blind] == -math.inf).all())
    got = L.attention_grad(do2, q2, k, v, poison(out2, blind), lse2, **args)
    for name, a, b in zip(("dq", "dk", "dv"), grads, got):
        assert torch.equal(a, b), name
    assert bool((got[0][blind] == 0).all())
