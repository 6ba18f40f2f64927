"""Attention and its gradients against the formulas in 64 bits, at the sizes, lengths and layouts where they can go wrong."""
import math

import pytest
import torch

import paper_1905_10395_amd as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 2.0 ** -24
UNIT = {torch.float32: EPS, torch.bfloat16: 2.0 ** -8}
# p below the smallest normal value, 2^-126, has no relative accuracy: it is off by as much as that value (a key of some hundred below
# its row's others has p = 10^-39, and its dv is that times dout: 3.20e-39 in 64 bits, 3.38e-39 of fp32's steps of 1.4e-45 and an
# exponential that ends at 2^-126)
TINY = 2.0 ** -126
F32, BF16 = torch.float32, torch.bfloat16


def rnd(*shape, seed, dtype=F32, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype).to(DEV)


def d(t):
    return t.cpu().double()


def lengths(values):
    return None if values is None else torch.tensor(values, dtype=torch.int32, device=DEV)


def seen(B, Tq, Tk, causal, q_lens, k_lens):
    nq = torch.tensor([Tq] * B if q_lens is None else [min(max(n, 0), Tq) for n in q_lens])[:, None, None]
    nk = torch.tensor([Tk] * B if k_lens is None else [min(max(n, 0), Tk) for n in k_lens])[:, None, None]
    t, j = torch.arange(Tq)[:, None], torch.arange(Tk)[None]
    s = (t < nq) & (j < nk)
    return (s & (j <= t + nk - nq) if causal else s)[:, None]


class Reference:
    """Everything in 64 bits by head, and bounds on the kernels' errors from the roundings that a value goes through."""

    def __init__(self, q, k, v, causal, scale, q_lens, k_lens):
        B, Tq, Hq, D = q.shape
        Tk, self.Hk = k.shape[1], k.shape[2]
        self.dtype, self.scale, self.G = q.dtype, scale, Hq // self.Hk
        by_head = lambda x: d(x).transpose(1, 2).repeat_interleave(Hq // x.shape[2], 1)
        self.q, self.k, self.v = by_head(q), by_head(k), by_head(v)
        self.seen = seen(B, Tq, Tk, causal, q_lens, k_lens)
        hidden = ~self.seen
        # what lies where nothing is seen does not matter
        self.k, self.v = (x.masked_fill(~self.seen.any(2)[..., None], 0.0) for x in (self.k, self.v))
        self.q = self.q.masked_fill(~self.seen.any(3)[..., None], 0.0)
        s = scale * self.q @ self.k.transpose(2, 3)
        # a score: four roundings a product (fp32 in three parts) and D sums; its exponent: the difference to another of its row, rounded; exp2: 2 last bits
        es = scale * (self.q.abs() @ self.k.abs().transpose(2, 3)) * (D + 4) * EPS
        s = s.masked_fill(hidden, -math.inf)
        self.lse = torch.logsumexp(s, 3) if Tk else torch.full((B, Hq, Tq), -math.inf, dtype=torch.float64)
        lse = torch.where(self.lse == -math.inf, torch.zeros_like(self.lse), self.lse)[..., None]
        self.p = (s - lse).exp().masked_fill(hidden, 0.0)
        far = s.masked_fill(hidden, 0.0).abs().amax(3, keepdim=True) if Tk else torch.zeros_like(lse)
        self.far = far
        worst = es.masked_fill(hidden, 0.0).amax(3, keepdim=True) if Tk else torch.zeros_like(lse)
        self.rel = worst + (4 * far + 2 * lse.abs() + 12) * EPS
        self.Tk, self.Tq, self.D = Tk, Tq, D
        self.out = self.p @ self.v
        round_p = 0.0 if q.dtype is F32 else UNIT[BF16]
        self.out_bound = (self.p @ self.v.abs()) * (2 * self.rel + round_p * 1.01 + 2 * (Tk + 8) * EPS) + TINY * self.v.abs().sum(2, keepdim=True)
        self.lse_bound = (2 * self.rel[..., 0] + (Tk + 8) * EPS) + self.lse.abs() * 4 * EPS

    def check(self, out, lse):
        unit = UNIT[self.dtype] * 1.01
        got = d(out).transpose(1, 2)
        assert bool(((got - self.out).abs() <= self.out_bound + unit * self.out.abs()).all()), float((got - self.out).abs().max())
        empty = ~self.seen.any(3).expand(self.lse.shape)
        assert bool((got[empty] == 0).all())
        if lse is not None:
            assert bool((d(lse)[empty] == -math.inf).all())
            assert bool(((d(lse) - self.lse).abs() <= self.lse_bound)[~empty].all())

    def check_grad(self, dout, out, lse, dq, dk, dv):
        unit, half = UNIT[self.dtype] * 1.01, 0.0 if self.dtype is F32 else UNIT[BF16] * 1.01
        live = self.seen.any(3)[..., None]
        do = d(dout).transpose(1, 2).masked_fill(~live, 0.0)
        o = d(out).transpose(1, 2).masked_fill(~live, 0.0)
        lse = d(lse)[..., None]
        s = self.scale * self.q @ self.k.transpose(2, 3)
        p = (s - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)).exp().masked_fill(~self.seen, 0.0)
        ep = p * (self.rel + half) + TINY * self.seen
        delta, dp = (do * o).sum(3, keepdim=True), do @ self.v.transpose(2, 3)
        e = (do.abs() * o.abs()).sum(3, keepdim=True) * (self.D + 4) * EPS + (do.abs() @ self.v.abs().transpose(2, 3)) * (self.D + 4) * EPS
        ds = p * (dp - delta)
        eds = p * e + ds.abs() * (self.rel + half + 4 * EPS) + TINY * self.seen * (1.0 + (dp - delta).abs())
        shared = lambda x: x.unflatten(1, (self.Hk, self.G)).sum(2)
        B, H = self.q.shape[:2]
        t = lambda x: x.transpose(2, 3)
        for name, got, want, bound in (
                ("dv", dv, shared(t(p) @ do), shared(t(ep + p * (self.Tq * self.G + 8) * EPS) @ do.abs())),
                ("dq", dq, self.scale * ds @ self.k, self.scale * (eds + ds.abs() * (self.Tk + 8) * EPS) @ self.k.abs()),
                ("dk", dk, self.scale * shared(t(ds) @ self.q), self.scale * shared(t(eds + ds.abs() * (self.Tq * self.G + 8) * EPS) @ self.q.abs()))):
            got = d(got).transpose(1, 2)
            assert got.shape == want.shape
            assert bool(((got - want).abs() <= bound + unit * want.abs()).all()), (name, float((got - want).abs().max()))
            if name == "dq":
                assert bool((got[~self.seen.any(3).expand(got.shape[:3])] == 0).all())
            else:
                assert bool((got[~self.seen.any(2).expand(B, self.Hk, self.Tk)] == 0).all())


def both(q, k, v, dout, causal=False, scale=None, q_lens=None, k_lens=None):
    scale = q.shape[3] ** -0.5 if scale is None else scale
    args = dict(causal=causal, scale=scale, q_lens=lengths(q_lens), k_lens=lengths(k_lens))
    out, lse = L.attention(q, k, v, **args)
    ref = Reference(q, k, v, causal, scale, q_lens, k_lens)
    ref.check(out, lse)
    dq, dk, dv = L.attention_grad(dout, q, k, v, out, lse, **args)
    ref.check_grad(dout, out, lse, dq, dk, dv)
    return out, lse, dq, dk, dv


def inputs(B, Tq, Tk, Hq, Hk, D, dtype, std=1.0):
    return (rnd(B, Tq, Hq, D, seed=1, dtype=dtype, std=std), rnd(B, Tk, Hk, D, seed=2, dtype=dtype, std=std), rnd(B, Tk, Hk, D, seed=3, dtype=dtype),
            rnd(B, Tq, Hq, D, seed=4, dtype=dtype))


# B, Tq, Tk, Hq, Hk, D, q_lens, k_lens
SHAPES = [(1, 1, 1, 1, 1, 1, None, None), (2, 1, 7, 2, 1, 8, None, [7, 1]), (1, 5, 3, 3, 1, 20, None, None), (2, 31, 33, 2, 2, 32, [31, 0], [0, 33]),
          (3, 32, 64, 4, 2, 33, [1, 32, 17], [64, 63, 31]), (1, 65, 65, 6, 2, 40, None, None), (2, 100, 100, 4, 4, 64, [100, 61], [100, 61]),
          (1, 129, 127, 3, 1, 72, None, None), (2, 63, 200, 2, 1, 80, None, [129, 200]), (1, 128, 128, 2, 2, 96, None, None), (1, 70, 300, 5, 1, 100, [69], [257]),
          (2, 200, 130, 4, 2, 128, [200, 199], [130, 1]), (1, 33, 65, 2, 1, 125, None, None), (1, 3, 1, 8, 8, 128, None, None)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
def test_small(shape, dtype, causal):
    B, Tq, Tk, Hq, Hk, D, q_lens, k_lens = shape
    both(*inputs(B, Tq, Tk, Hq, Hk, D, dtype), causal=causal, q_lens=q_lens, k_lens=k_lens)


@pytest.mark.parametrize("D", [24, 50, 64, 96, 128])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
def test_many_entries_by_rows(D, dtype, causal):
    """Enough workgroups that each takes 128 rows; lengths of every kind."""
    B, T = 24, 150
    lens = [(37 * b) % (T + 1) for b in range(B)]
    lens[5] = T
    both(*inputs(B, T, T, 6, 6 if D < 64 else 3, D, dtype), causal=causal, q_lens=lens, k_lens=lens)


@pytest.mark.parametrize("B,Tq,Tk,Hq,Hk,D,k_lens", [(2, 1, 5000, 8, 2, 128, [5000, 1030]), (3, 2, 2500, 4, 2, 64, [0, 2500, 1]), (1, 1, 4099, 3, 3, 45, None),
                                                   (2, 4, 3000, 32, 2, 32, [2999, 3000])])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_new_tokens_to_a_long_cache(B, Tq, Tk, Hq, Hk, D, k_lens, dtype):
    both(*inputs(B, Tq, Tk, Hq, Hk, D, dtype), causal=True, k_lens=k_lens)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_many_queries_to_few_keys(dtype):
    """The gradients of the keys are sums over many rows, split over workgroups."""
    both(*inputs(1, 1500, 70, 4, 1, 64, dtype), k_lens=[65])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
def test_large_scores(dtype, causal):
    """Scores of some hundreds: one key takes nearly all; the running reference moves often."""
    q, k, v, do = inputs(1, 90, 260, 2, 1, 64, dtype, std=4.0)
    both(q, k, v, do, causal=causal, scale=1.0)
    k = k * torch.linspace(0.0, 3.0, 260, device=DEV)[None, :, None, None].to(dtype)
    both(q, k, v, do, causal=causal, scale=0.25)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_equal_scores(dtype):
    q, k, v, do = inputs(2, 40, 77, 2, 2, 64, dtype)
    out = both(q * 0, k, v, do)[0]
    assert float((d(out)[:, 0] - d(v).mean(1)).abs().max()) <= 2 ** -7


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [64, 45])
@pytest.mark.parametrize("many", [False, True])
def test_what_is_not_seen_does_not_matter(dtype, D, many):
    B, T = (20, 140) if many else (3, 70)
    H = 8 if many else 2
    lens = [(29 * b) % T for b in range(B)]
    q, k, v, do = inputs(B, T, T, H, H, D, dtype)
    clean = both(q, k, v, do, causal=True, q_lens=lens, k_lens=lens) if not many else None
    args = dict(causal=True, q_lens=lengths(lens), k_lens=lengths(lens))
    out, lse = L.attention(q, k, v, **args)
    grads = L.attention_grad(do, q, k, v, out, lse, **args)
    for b, n in enumerate(lens):
        for x in (q, k, v, do):
            x[b, n:] = float("nan")
            x[b, n:, :, ::3] = float("inf")
    out2, lse2 = L.attention(q, k, v, **args)
    out2[~torch.isfinite(out2)] = 5e3
    assert torch.equal(out, out2) and torch.equal(lse, lse2)
    for b, n in enumerate(lens):
        out2[b, n:] = float("nan")
    for a, b in zip(grads, L.attention_grad(do, q, k, v, out2, lse2, **args)):
        assert torch.equal(a, b)
    if clean:
        assert torch.equal(clean[0], out)


def test_lengths_out_of_range_are_the_ends():
    q, k, v, do = inputs(3, 20, 30, 2, 1, 32, F32)
    a = L.attention(q, k, v, causal=True, q_lens=lengths([-5, 99, 20]), k_lens=lengths([10, 31, -2 ** 31]))
    b = L.attention(q, k, v, causal=True, q_lens=lengths([0, 20, 20]), k_lens=lengths([10, 30, 0]))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [64, 36])
def test_views(dtype, D):
    """Parts of one projection from an odd place on, heads outermost, gradients into one buffer."""
    B, T, Hq, Hk = 2, 75, 4, 2
    flat = rnd(B * T * (Hq + 2 * Hk) * D + 3, seed=1, dtype=dtype)[3:].view(B, T, Hq + 2 * Hk, D)
    q, k, v = flat[:, :, :Hq], flat[:, :, Hq:Hq + Hk], flat[:, :, Hq + Hk:]
    do = rnd(B, Hq, T, D, seed=2, dtype=dtype).transpose(1, 2)
    args = dict(causal=True)
    out, lse = L.attention(q.contiguous(), k.contiguous(), v.contiguous(), **args)
    grads = L.attention_grad(do.contiguous(), q.contiguous(), k.contiguous(), v.contiguous(), out, lse, **args)
    placed = torch.zeros((B, Hq, T, D), dtype=dtype, device=DEV).transpose(1, 2)
    out2, lse2 = L.attention(q, k, v, out=placed, **args)
    assert out2 is placed and torch.equal(out, placed) and torch.equal(lse, lse2)
    into = torch.full_like(flat, 9.0)
    got = L.attention_grad(do, q, k, v, placed, lse2, dq=into[:, :, :Hq], dk=into[:, :, Hq:Hq + Hk], dv=into[:, :, Hq + Hk:], **args)
    for a, b in zip(grads, got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_queries_in_several_calls(dtype):
    """A text in two halves against the cache gives what one call gives, to the roundings of sums in another order."""
    q, k, v, _ = inputs(2, 120, 120, 4, 2, 64, dtype)
    whole = L.attention(q, k, v, causal=True)[0]
    a = L.attention(q[:, :50], k[:, :50], v[:, :50], causal=True)[0]
    b = L.attention(q[:, 50:], k, v, causal=True)[0]
    one = L.attention(q[:, 119:], k, v, causal=True, with_lse=False)
    assert one[1] is None
    lim = 2e-6 if dtype is F32 else 2 ** -8 * 6                       # values up to 3, rounded twice each
    assert float((d(torch.cat([a, b], 1)) - d(whole)).abs().max()) <= lim
    assert float((d(one[0]) - d(whole[:, 119:])).abs().max()) <= lim


def test_gradient_is_the_slope():
    B, Tq, Tk, Hq, Hk, D = 1, 5, 9, 2, 1, 6
    q, k, v, do = inputs(B, Tq, Tk, Hq, Hk, D, F32)
    out, lse = L.attention(q, k, v, causal=True)
    grads = L.attention_grad(do, q, k, v, out, lse, causal=True)
    scale = D ** -0.5
    f = lambda a: float((Reference(*a, True, scale, None, None).out * d(do).transpose(1, 2)).sum())
    step = 1e-5
    for which, g in enumerate(grads):
        for i in range(0, g.numel(), 3):
            side = []
            for sign in (1, -1):
                a = [d(q), d(k), d(v)]
                a[which].view(-1)[i] += sign * step
                side.append(f(a))
            assert abs((side[0] - side[1]) / (2 * step) - float(g.reshape(-1)[i])) < 2e-5


def test_nothing_to_do():
    q, k, v, do = inputs(2, 5, 4, 2, 1, 16, F32)
    out, lse = L.attention(q, k[:, :0], v[:, :0])
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    dq, dk, dv = L.attention_grad(do, q, k[:, :0], v[:, :0], out, lse)
    assert bool((dq == 0).all()) and dk.shape == (2, 0, 1, 16)
    out, lse = L.attention(q[:, :0], k, v)
    assert out.shape == (2, 0, 2, 16) and lse.shape == (2, 2, 0)
    dq, dk, dv = L.attention_grad(do[:, :0], q[:, :0], k, v, out, lse)
    assert bool((dk == 0).all()) and bool((dv == 0).all())


@pytest.mark.parametrize("Tq,Tk", [(1, 3000), (200, 200)])
def test_equal_calls_give_equal_bits_on_any_stream(Tq, Tk):
    q, k, v, do = inputs(2, Tq, Tk, 4, 2, 64, BF16)
    out, lse = L.attention(q, k, v, causal=True)
    grads = L.attention_grad(do, q, k, v, out, lse, causal=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out2, lse2 = L.attention(q, k, v, causal=True, stream=side)
    grads2 = L.attention_grad(do, q, k, v, out2, lse2, causal=True, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, out2) and torch.equal(lse, lse2) and all(torch.equal(a, b) for a, b in zip(grads, grads2))


def test_captured_and_replayed():
    """Decoding and a training step in graphs, replayed with new contents and lengths, eager work in between."""
    q, k, v, do = inputs(2, 1, 2200, 4, 2, 64, BF16)
    tq, tk, tv, tdo = inputs(2, 130, 130, 4, 2, 64, BF16)
    lens = lengths([2200, 900])
    L.attention(q, k, v, k_lens=lens)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = L.attention(q, k, v, k_lens=lens)
        tout, tlse = L.attention(tq, tk, tv, causal=True)
        grads = L.attention_grad(tdo, tq, tk, tv, tout, tlse, causal=True)
    for step in range(4):
        q.copy_(rnd(*q.shape, seed=20 + step, dtype=BF16))
        tq.copy_(rnd(*tq.shape, seed=40 + step, dtype=BF16))
        lens.copy_(lengths([100 + 500 * step, 2200 - step]))
        graph.replay()
        want = L.attention(q, k, v, k_lens=lens)
        twant = L.attention(tq, tk, tv, causal=True)
        gwant = L.attention_grad(tdo, tq, tk, tv, *twant, causal=True)
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and torch.equal(tout, twant[0])
        assert all(torch.equal(a, b) for a, b in zip(grads, gwant))
