"""Attention and its gradients on the routes that small cases do not reach: workgroups of 128 rows or keys at every width of head, few rows of long
keys in several tiles and splits, many query heads to one key head, entries and keys beyond 2^31 elements; rotation captured in a graph."""
import pytest
import torch

import paper_1905_10395_amd as L
from test_gpu_attention import BF16, DEV, F32, Reference, both, d, inputs, lengths, rnd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [32, 64, 72, 90, 128])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
def test_many_rows_and_keys(D, dtype, causal):
    B, T = 24, 150
    lens = [(41 * b) % (T + 1) for b in range(B)]
    lens[7] = T
    both(*inputs(B, T, T, 6, 6, D, dtype), causal=causal, q_lens=lens, k_lens=lens)


@pytest.mark.parametrize("D", [64, 90, 128])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
def test_many_rows_of_shared_keys(D, dtype, causal):
    B, T = 24, 150
    lens = [(43 * b) % (T + 1) for b in range(B)]
    lens[2] = T
    both(*inputs(B, T, T, 12, 4, D, dtype), causal=causal, q_lens=lens, k_lens=lens)


@pytest.mark.parametrize("Tq,Tk,Hq,Hk,D,k_lens", [(50, 3000, 3, 1, 64, [2990]), (9, 2100, 8, 1, 128, [2100]), (40, 1100, 2, 2, 52, [1025])])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
def test_few_rows_of_long_keys(Tq, Tk, Hq, Hk, D, k_lens, dtype, causal):
    both(*inputs(1, Tq, Tk, Hq, Hk, D, dtype), causal=causal, k_lens=k_lens)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_many_heads_share_a_key_head(dtype):
    both(*inputs(2, 5, 80, 96, 2, 48, dtype), causal=True, k_lens=[80, 3])
    both(*inputs(1, 20, 33, 67, 1, 64, dtype))


@pytest.mark.parametrize("Tk", [0, 7, 5000])
def test_no_queries(Tk):
    q, k, v, do = inputs(2, 0, Tk, 4, 2, 64, BF16)
    out, lse = L.attention(q, k, v, causal=True)
    assert out.shape == q.shape and lse.shape == (2, 4, 0)
    dq, dk, dv = L.attention_grad(do, q, k, v, out, lse, causal=True)
    assert dq.shape == q.shape and not bool(dk.any()) and not bool(dv.any())


@pytest.mark.parametrize("B,Tq,Tk,D", [(24, 150, 150, 64), (24, 150, 150, 90), (2, 40, 90, 64), (2, 1, 5000, 64), (1, 3, 3000, 45), (1, 50, 3000, 128)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_nan_is_not_hidden(B, Tq, Tk, D, dtype):
    """A query with NaN, or one that sees a key with NaN, has NaN and says so; others have what they had."""
    H, t = 6, Tq // 2
    q, k, v, _ = inputs(B, Tq, Tk, H, H, D, dtype)
    want, wlse = L.attention(q, k, v)
    q[0, t, 1, D // 2] = float("nan")
    k[B - 1, Tk // 3, 2] = float("nan")
    out, lse = L.attention(q, k, v)
    bad = torch.zeros((B, Tq, H), dtype=torch.bool, device=DEV)
    bad[0, t, 1] = True
    bad[B - 1, :, 2] = True
    rest = ~bad.cpu()
    assert bool(out[bad].isnan().all()) and bool(lse.transpose(1, 2)[bad].isnan().all())
    # (rows of a wavefront are rescaled together, so other rows' sums may round elsewhere: values of up to 5 once to their type, twice)
    lim = 2e-5 if dtype is F32 else 5 * 2 ** -7
    assert float((d(out) - d(want))[rest].abs().max()) <= lim and float((d(lse) - d(wlse)).transpose(1, 2)[rest].abs().max()) <= 2e-5


def test_shared_keys_by_strides():
    """Keys of one entry for all entries and heads, by strides of zero."""
    q, k, v, do = inputs(3, 20, 70, 4, 4, 64, BF16)
    k0, v0 = (x[:1, :, :1].expand(3, 70, 4, 64) for x in (k, v))
    out, lse = L.attention(q, k0, v0)
    want, wlse = L.attention(q, k0.contiguous(), v0.contiguous())
    assert torch.equal(out, want) and torch.equal(lse, wlse)
    got = L.attention_grad(do, q, k0, v0, out, lse)
    for a, b in zip(got, L.attention_grad(do, q, k0.contiguous(), v0.contiguous(), out, lse)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("where", ["entries", "tokens"])
def test_beyond_31_bits(where):
    """A cache whose entries, or tokens, lie more than 2^31 elements apart."""
    far = 2 ** 31 + 4096
    D, n = 64, 3 if where == "entries" else 2
    big = torch.empty(far * (n - 1) + (1 << 16), dtype=BF16, device=DEV)
    B, T = (3, 40) if where == "entries" else (1, 2)
    strides = (far, D, D, 1) if where == "entries" else (far * n, far, D, 1)
    k, v = big.as_strided((B, T, 1, D), strides), big.as_strided((B, T, 1, D), strides, 1 << 14)
    k.copy_(rnd(B, T, 1, D, seed=1, dtype=BF16))
    v.copy_(rnd(B, T, 1, D, seed=2, dtype=BF16))
    q, do = rnd(B, 2, 3, D, seed=3, dtype=BF16), rnd(B, 2, 3, D, seed=4, dtype=BF16)
    out, lse = L.attention(q, k, v, causal=True)
    want, wlse = L.attention(q, k.contiguous(), v.contiguous(), causal=True)
    assert torch.equal(out, want) and torch.equal(lse, wlse)
    into = torch.empty_like(big).as_strided((B, T, 1, D), strides)
    _, dk, _ = L.attention_grad(do, q, k, v, out, lse, causal=True, dk=into)
    assert torch.equal(dk, L.attention_grad(do, q, k.contiguous(), v.contiguous(), out, lse, causal=True)[1])
    turned = L.qk_rotary(k, turns=L.rotary_turns(D, device=DEV), q_out=into)[0]
    assert torch.equal(turned, L.qk_rotary(k.contiguous(), turns=L.rotary_turns(D, device=DEV))[0])


def test_a_workspace_of_the_callers():
    q, k, v, do = inputs(2, 3, 5000, 4, 2, 64, BF16)
    lib = L.lib()
    n = lib.lsgd_attention_workspace_bytes(2, 3, 5000, 4, 2, 64, 1)
    ws = torch.full((n + 512,), 77, dtype=torch.uint8, device=DEV)
    out, lse = L.attention(q, k, v, causal=True, workspace=ws[:n])
    assert torch.equal(out, L.attention(q, k, v, causal=True)[0]) and bool((ws[n:] == 77).all())
    with pytest.raises(L.LsgdError, match="NOMEM"):
        L.attention(q, k, v, causal=True, workspace=ws[:n - 256])
    n = lib.lsgd_attention_grad_workspace_bytes(2, 3, 5000, 4, 2, 64, 1)
    ws = torch.full((n + 512,), 77, dtype=torch.uint8, device=DEV)
    grads = L.attention_grad(do, q, k, v, out, lse, causal=True, workspace=ws[:n])
    assert all(torch.equal(a, b) for a, b in zip(grads, L.attention_grad(do, q, k, v, out, lse, causal=True))) and bool((ws[n:] == 77).all())


def test_nothing_is_written_outside():
    """Results in the middle of larger buffers: what lies around stays."""
    for dtype, D in ((BF16, 64), (BF16, 37), (F32, 40), (F32, 33)):
        for B, T, H in ((2, 45, 2), (24, 150, 6)):
            q, k, v, do = inputs(B, T, T, H, H, D, dtype)
            hold = [torch.full((B, T + 2, H + 2, D + 8), 5.0, dtype=dtype, device=DEV) for _ in range(4)]
            inner = [h[:, 1:-1, 1:-1, :D] for h in hold]
            out, lse = L.attention(q, k, v, causal=True, out=inner[0])
            L.attention_grad(do, q, k, v, out, lse, causal=True, dq=inner[1], dk=inner[2], dv=inner[3])
            for h, i in zip(hold, inner):
                assert bool(torch.isfinite(i).all())
                i.fill_(5.0)
                assert bool((h == 5).all())


def test_rotation_captured_and_replayed():
    W, T, H, D = 2, 40, 3, 64
    x, g = rnd(W, T, H, D, seed=1, dtype=BF16), rnd(W, T, H, D, seed=2, dtype=BF16)
    pos, turns, dw = torch.arange(T, dtype=torch.int32, device=DEV)[None].clone(), L.rotary_turns(D, device=DEV), torch.zeros((W, D), device=DEV)
    L.qk_rotary(x, positions=pos, turns=turns)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, _, stats = L.qk_rotary(x, positions=pos, turns=turns)
        dx, _ = L.qk_rotary_grad(g, None, x, None, stats, pos, turns, dw_q=dw)
    for step in range(4):
        x.copy_(rnd(W, T, H, D, seed=10 + step, dtype=BF16))
        pos += 1000
        graph.replay()
        want, _, s = L.qk_rotary(x, positions=pos, turns=turns)
        dw2 = torch.zeros_like(dw)
        dx2, _ = L.qk_rotary_grad(g, None, x, None, s, pos, turns, dw_q=dw2)
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(dx, dx2) and torch.equal(dw, dw2)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [64, 63, 200])
def test_long_batches_rotated(dtype, D):
    """Workgroups with several tokens, and weights' sums over many of them."""
    W, T, Hq, Hk = 3, 4000, 5, 2
    q, k = rnd(W, T, Hq, D, seed=1, dtype=dtype), rnd(W, T, Hk, D, seed=2, dtype=dtype)
    gq, gk = rnd(W, T, Hq, D, seed=3, dtype=dtype), rnd(W, T, Hk, D, seed=4, dtype=dtype)
    w = rnd(W, 2 * D, seed=5) * 0.3 + 1.0
    turns = L.rotary_turns(D // 2 * 2, device=DEV)
    yq, yk, stats = L.qk_rotary(q, k, None, turns, w_q=w[:, :D], w_k=w[:, D:])
    dw = torch.zeros_like(w)
    dq, dk = L.qk_rotary_grad(gq, gk, q, k, stats, None, turns, w_q=w[:, :D], w_k=w[:, D:], dw_q=dw[:, :D], dw_k=dw[:, D:])
    # a stretch of tokens by itself gives the same rows
    pos = torch.arange(2500, 2600, dtype=torch.int32, device=DEV)[None]
    part = slice(2500, 2600)
    a, b, s = L.qk_rotary(q[:, part], k[:, part], pos, turns, w_q=w[:, :D], w_k=w[:, D:])
    assert torch.equal(a, yq[:, part]) and torch.equal(b, yk[:, part]) and torch.equal(s, stats[:, part])
    e, f = L.qk_rotary_grad(gq[:, part], gk[:, part], q[:, part], k[:, part], s.contiguous(), pos, turns, w_q=w[:, :D], w_k=w[:, D:])
    assert torch.equal(e, dq[:, part]) and torch.equal(f, dk[:, part])
    # and the weights' gradients are the sums of the stretches'
    total, size = torch.zeros_like(w, dtype=torch.float64), torch.zeros_like(w, dtype=torch.float64)
    for t in range(0, T, 500):
        part = slice(t, t + 500)
        one = torch.zeros_like(w)
        pos = torch.arange(t, t + 500, dtype=torch.int32, device=DEV)[None]
        L.qk_rotary_grad(gq[:, part], gk[:, part], q[:, part], k[:, part], stats[:, part].contiguous(), pos, turns, w_q=w[:, :D], w_k=w[:, D:],
                         dw_q=one[:, :D], dw_k=one[:, D:])
        total += one.double()
    # a lane adds up some 20 rows, a workgroup up to 64 teams, the join 700 workgroups as 16 stretches of 44, then 16: no value goes through
    # more than 150 additions, each of which rounds at 2^-24 of the magnitudes' sum, below 3 T H for terms of size 1; on both sides
    assert float((dw.double() - total).abs().max()) <= 2 * 150 * 2.0 ** -24 * 3 * T * Hq


def test_scores_of_any_scale():
    """The scale only shifts between its factors: powers of two of it and of q give the same bits."""
    q, k, v, do = inputs(2, 50, 60, 2, 2, 64, F32)
    out, lse = L.attention(q, k, v, scale=0.125)
    for s in (2.0 ** -40, 2.0 ** 30):
        o, l = L.attention(q * (0.125 / s), k, v, scale=s)
        assert torch.equal(o, out) and torch.equal(l, lse)
        ref = Reference(q * (0.125 / s), k, v, False, s, None, None)
        ref.check(o, l)
    assert float(d(out).abs().max()) > 0 and lengths([1]).numel() == 1
