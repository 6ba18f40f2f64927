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


# by rows; by keys; keys split: B, Tq, Tk, H, D
ROUTES = [(24, 150, 150, 6, 64), (24, 150, 150, 6, 90), (24, 150, 150, 6, 128), (2, 40, 90, 6, 64), (2, 40, 90, 6, 45), (1, 20, 3000, 2, 64), (1, 20, 3000, 2, 101)]


def some_rows(B, Tq, Tk):
    """Lengths that leave each entry queries that see nothing and queries that see all keys of its length, and a key of each that is marked."""
    q_lens, k_lens = [1 + 5 * b % (Tq - 1) for b in range(B)], [Tk - b % 3 for b in range(B)]
    where = torch.zeros((B, Tk), dtype=torch.bool)
    for b in range(B):
        where[b, k_lens[b] // 2] = True
    blind = torch.arange(Tq)[None] >= torch.tensor(q_lens)[:, None]
    return lengths(q_lens), lengths(k_lens), where.to("cuda:0"), blind.to("cuda:0")


@pytest.mark.parametrize("B,Tq,Tk,H,D", ROUTES)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("which", ["v", "k"])
def test_queries_that_see_no_key_have_zeros(B, Tq, Tk, H, D, dtype, which):
    """Beside queries that see an infinity or NaN."""
    q, k, v, _ = inputs(B, Tq, Tk, H, H, D, dtype)
    q_lens, k_lens, where, blind = some_rows(B, Tq, Tk)
    args = dict(q_lens=q_lens, k_lens=k_lens)
    _, clean = L.attention(q, k, v, **args)
    out, lse = L.attention(q, *((k, poison(v, where)) if which == "v" else (poison(k, where), v)), **args)
    assert bool((out[blind] == 0).all()) and bool((lse.transpose(1, 2)[blind] == -math.inf).all())
    if which == "v":
        assert torch.equal(lse, clean)
        # 0, 3, ...: NaN; 1, 2: infinities, which may come out as NaN
        assert bool(out[~blind][:, :, ::4].isnan().all()) and not bool(out[~blind][:, :, 1::4].isfinite().any())


@pytest.mark.parametrize("B,Tq,Tk,H", [(24, 150, 150, 6), (2, 40, 90, 6), (1, 20, 3000, 2)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scores_of_minus_infinity(B, Tq, Tk, H, dtype):
    """A query whose scores are all minus infinity sees keys: 0 / 0, not the zeros of one that sees none."""
    q, k, v, _ = inputs(B, Tq, Tk, H, H, 32, dtype)
    k[0] = -INF
    out, lse = L.attention(q.abs() + 1, k, v)
    assert bool(out[0].isnan().all()) and not bool(lse[0].isfinite().any())
    assert bool(out[1:].isfinite().all()) and bool(lse[1:].isfinite().all())


@pytest.mark.parametrize("B,Tq,Tk,H,D", ROUTES)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("which", ["v", "k", "do"])
def test_gradients_of_queries_that_see_no_key_are_zeros(B, Tq, Tk, H, D, dtype, which):
    """Beside queries that see an infinity or NaN, or have one; as those of keys that nobody sees."""
    q, k, v, do = inputs(B, Tq, Tk, H, H, D, dtype)
    q_lens, k_lens, where, blind = some_rows(B, Tq, Tk)
    args = dict(q_lens=q_lens, k_lens=k_lens)
    k, v = (k, poison(v, where)) if which == "v" else (poison(k, where), v) if which == "k" else (k, v)
    out, lse = L.attention(q, k, v, **args)
    first = torch.arange(Tq, device=q.device)[None].expand(B, Tq) == 0
    dq, dk, dv = L.attention_grad(poison(do, first) if which == "do" else do, q, k, v, out, lse, **args)
    assert bool((dq[blind] == 0).all()) and not bool(dq[:, 0].isfinite().all())
    unseen = torch.arange(Tk, device=q.device)[None] >= k_lens[:, None]
    assert bool((dk[unseen] == 0).all()) and bool((dv[unseen] == 0).all())


@pytest.mark.parametrize("B,Tq,Tk,H,D", ROUTES)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("power", [-60, 106])
def test_values_of_any_size(B, Tq, Tk, H, D, dtype, power):
    """Powers of two in v are powers of two in the results, as long as 2^8 Tk max|v| is finite (3000 keys of up to 4 2^106 with p up to 2^8:
    below 2^128) and what fp32's third part of an element holds, 2^-24 of it, times a p of 2^-20, is a normal value."""
    q, k, v, _ = inputs(B, Tq, Tk, H, H, D, dtype)
    v = torch.where(v.abs() < 2.0 ** -10, torch.ones_like(v), v).clamp(-4.0, 4.0)
    out, lse = L.attention(q, k, v)
    got, glse = L.attention(q, k, v * 2.0 ** power)
    assert torch.equal(lse, glse) and torch.equal(got / 2.0 ** power, out)
