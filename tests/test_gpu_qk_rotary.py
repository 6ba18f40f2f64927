"""Norm and rotation of queries and keys, and the gradients, against the formulas in 64 bits."""
import math

import pytest
import torch

import paper_1905_10395_amd as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 2.0 ** -24
UNIT = {torch.float32: EPS, torch.bfloat16: 2.0 ** -8}
NORM_EPS = 1e-5
# cos and sin of an angle: the fraction of a turn rounded to fp32 (2 pi 2^-26, 1.6 EPS), sincospi (4 last bits, 8 EPS), times the magnitude
ANGLE = 11


def rnd(*shape, seed, dtype=torch.float32, std=1.0, mean=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std + mean).to(dtype).to(DEV)


def weights(W, D, seed, lead=0):
    x = rnd(W, lead + 2 * D + 3, seed=seed, std=0.3, mean=1.0)
    return x[:, lead:lead + D], x[:, lead + D:lead + 2 * D]


def d(t):
    return None if t is None else t.cpu().double()


def pairs(x, R, interleaved):
    return (x[..., 0:R:2], x[..., 1:R:2]) if interleaved else (x[..., :R // 2], x[..., R // 2:R])


def join(a, b, x, R, interleaved):
    z = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([z, x[..., R:]], -1)


def rotate(x, bound, pos, turns, R, interleaved, magnitude, back=False):
    """x [W, T, H, D] turned, and a bound on the fp32 result's error given one on x's."""
    a, b = pairs(x, R, interleaved)
    ea, eb = pairs(bound, R, interleaved)
    angle = 2 * math.pi * (pos.double()[..., None] * turns)[:, :, None]
    c, s = magnitude * torch.cos(angle), magnitude * torch.sin(angle) * (-1 if back else 1)
    y = join(a * c - b * s, a * s + b * c, x, R, interleaved)
    m = abs(magnitude)
    e = m * (ea + eb + (a.abs() + b.abs()) * (ANGLE + 3) * EPS)
    return y, join(e, e, bound, R, interleaved)


def reference(x, w, pos, turns, norm, interleaved, magnitude=1.0):
    D, R = x.shape[3], 2 * turns.numel()
    x = d(x)
    w = (torch.ones((x.shape[0], D), dtype=torch.float64) if w is None else d(w))[:, None, None]
    q = (x.pow(2).mean(3) + NORM_EPS).rsqrt() if norm else torch.ones(x.shape[:3], dtype=torch.float64)
    z = x * q[..., None] * w
    y, e = rotate(z, z.abs() * ((D / 2 + 24) * EPS if norm else 2 * EPS), pos, d(turns), R, interleaved, magnitude)
    return y, e, q


def positions(W, T, seed, far):
    g = torch.Generator().manual_seed(seed)
    return (torch.randint(-5, far, (W, 1), generator=g) + torch.arange(T)).to(torch.int32)


# W, T, Hq, Hk, D, R
SHAPES = [(1, 1, 1, 0, 1, 0), (1, 1, 1, 1, 2, 2), (2, 3, 2, 1, 7, 4), (2, 5, 3, 1, 16, 16), (3, 9, 4, 2, 64, 64), (2, 33, 6, 2, 72, 36), (1, 17, 2, 2, 80, 80), (2, 7, 5, 5, 101, 50),
          (1, 70, 8, 2, 128, 128), (2, 11, 3, 1, 128, 64), (1, 5, 2, 1, 255, 254), (1, 4, 2, 1, 256, 256), (1, 3, 2, 1, 256, 0), (1, 300, 3, 1, 20, 12),
          (4, 65, 2, 1, 96, 24), (1, 3, 40, 8, 254, 252)]


@pytest.mark.parametrize("W,T,Hq,Hk,D,R", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [True, False])
def test_forward_and_gradient(W, T, Hq, Hk, D, R, dtype, interleaved, norm):
    q = rnd(W, T, Hq, D, seed=1, dtype=dtype, std=2.0)
    k = rnd(W, T, Hk, D, seed=2, dtype=dtype, std=2.0) if Hk else None
    wq, wk = weights(W, D, 3, lead=D % 3)
    pos = positions(W, T, 4, 100000)
    turns = L.rotary_turns(R, device=DEV)
    m = 1.25
    got = L.qk_rotary(q, k, pos.to(DEV), turns, w_q=wq, w_k=wk if Hk else None, norm=norm, eps=NORM_EPS, interleaved=interleaved, magnitude=m)
    unit = UNIT[dtype]
    factors = []
    for x, w, y in ((q, wq, got[0]), (k, wk, got[1])):
        if x is None:
            assert y is None
            continue
        want, e, f = reference(x, w, pos, turns, norm, interleaved, m)
        assert bool(((d(y) - want).abs() <= e + unit * 1.01 * want.abs()).all())
        factors.append(f)
    if norm:
        f = torch.cat(factors, 2)
        assert bool(((d(got[2]) - f).abs() <= f * (D / 2 + 24) * EPS).all())
    else:
        assert got[2] is None

    gq = rnd(W, T, Hq, D, seed=5, dtype=dtype)
    gk = rnd(W, T, Hk, D, seed=6, dtype=dtype) if Hk else None
    x_grad = torch.full((W, 2 * D + 1), 7.0, device=DEV)
    dwq, dwk = x_grad[:, :D], x_grad[:, D:2 * D] if Hk else None
    before = x_grad.clone()
    dq, dk = L.qk_rotary_grad(gq, gk, q, k, got[2], pos.to(DEV), turns, w_q=wq, w_k=wk if Hk else None, norm=norm, interleaved=interleaved, magnitude=m,
                              dw_q=dwq, dw_k=dwk, accumulate=interleaved)
    for x, w, g, dx, dw, first in ((q, wq, gq, dq, dwq, 0), (k, wk, gk, dk, dwk, Hq)):
        if x is None:
            assert dx is None
            continue
        dz, e = rotate(d(g), torch.zeros(g.shape, dtype=torch.float64), pos, d(turns), R, interleaved, m, back=True)
        ww, f = d(w)[:, None, None], d(got[2])[:, :, first:first + x.shape[2], None] if norm else 1.0
        h, t = d(x) * f, dz * ww
        et = e * ww.abs() + t.abs() * EPS
        if norm:
            mean = (t * h).mean(3, keepdim=True)
            em = (et * h.abs() + (t * h).abs() * (D + 4) * EPS).mean(3, keepdim=True)
            want = f * (t - h * mean)
            bound = f * (et + t.abs() * 4 * EPS + h.abs() * em + (h * mean).abs() * 6 * EPS)
        else:
            want, bound = t, et
        assert bool(((d(dx) - want).abs() <= bound + unit * 1.01 * want.abs()).all())
        base = 7.0 if interleaved else 0.0
        n = T * x.shape[2]
        assert bool(((d(dw) - base - (dz * h).sum((1, 2))).abs() <= (e * h.abs() + (dz * h).abs() * (n + 8) * EPS).sum((1, 2)) + base * (2 * EPS)
                     + EPS * (dz * h).sum((1, 2)).abs()).all())
    assert torch.equal(x_grad[:, (2 if Hk else 1) * D:], before[:, (2 if Hk else 1) * D:])


def test_gradient_is_the_slope():
    """Against differences of the 64-bit formula."""
    W, T, H, D, R = 1, 3, 2, 12, 8
    x, w, g = rnd(W, T, H, D, seed=1), weights(W, D, 2)[0], rnd(W, T, H, D, seed=3)
    pos, turns = positions(W, T, 4, 1000), L.rotary_turns(R, device=DEV)
    _, _, stats = L.qk_rotary(x, positions=pos.to(DEV), turns=turns, w_q=w, eps=NORM_EPS)
    dw = torch.zeros((W, D), device=DEV)
    dx, _ = L.qk_rotary_grad(g, None, x, None, stats, pos.to(DEV), turns, w_q=w, dw_q=dw)
    f = lambda x, w: float((reference(x, w, pos, turns, True, False)[0] * d(g)).sum())
    step = 1e-5
    for i in range(0, x.numel(), 5):
        a, b = d(x), d(x)
        a.view(-1)[i] += step
        b.view(-1)[i] -= step
        assert abs((f(a, d(w)) - f(b, d(w))) / (2 * step) - float(dx.view(-1)[i])) < 1e-5 * 10       # third derivatives of size 10 x step^2, and fp32
    for i in range(D):
        a, b = d(w).clone(), d(w).clone()
        a[0, i] += step
        b[0, i] -= step
        assert abs((f(d(x), a) - f(d(x), b)) / (2 * step) - float(dw[0, i])) < 1e-5 * 10


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D,R", [(64, 64), (72, 36), (33, 20)])
def test_views_and_places(dtype, D, R):
    """Queries and keys as columns of one projection that begins at an odd place, heads outermost, results in place and into a cache."""
    W, T, Hq, Hk = 2, 13, 4, 2
    flat = rnd(W * T * (Hq + 2 * Hk) * D + 1, seed=1, dtype=dtype)[1:].view(W, T, Hq + 2 * Hk, D)
    q, k, v = flat[:, :, :Hq], flat[:, :, Hq:Hq + Hk], flat[:, :, Hq + Hk:]
    pos, turns = positions(W, T, 2, 5000).to(DEV), L.rotary_turns(R, device=DEV)
    wq, wk = weights(W, D, 3)
    kept = v.clone()
    want = L.qk_rotary(q.contiguous(), k.contiguous(), pos, turns, w_q=wq, w_k=wk)
    headed = q.transpose(1, 2).contiguous().transpose(1, 2)
    cache = torch.full((W, T + 9, Hk, D), 3.0, dtype=dtype, device=DEV)
    a, b, s = L.qk_rotary(headed, k, pos, turns, w_q=wq, w_k=wk, q_out=headed, k_out=cache[:, 4:4 + T])
    assert a is headed and torch.equal(a, want[0]) and torch.equal(cache[:, 4:4 + T], want[1]) and torch.equal(s, want[2])
    assert bool((cache[:, :4] == 3).all()) and bool((cache[:, 4 + T:] == 3).all())
    gq, gk = rnd(W, T, Hq, D, seed=7, dtype=dtype), rnd(W, T, Hk, D, seed=8, dtype=dtype)
    dq, dk = L.qk_rotary_grad(gq, gk, q.contiguous(), k.contiguous(), s, pos, turns, w_q=wq, w_k=wk)
    out = torch.zeros_like(flat)
    L.qk_rotary_grad(gq, gk, q, k, s, pos, turns, w_q=wq, w_k=wk, dq=out[:, :, :Hq], dk=out[:, :, Hq:Hq + Hk])
    assert torch.equal(out[:, :, :Hq], dq) and torch.equal(out[:, :, Hq:Hq + Hk], dk) and bool((out[:, :, Hq + Hk:] == 0).all())
    L.qk_rotary_grad(gq, gk, q, k, s, pos, turns, w_q=wq, w_k=wk, dq=gq, dk=k)
    assert torch.equal(gq, dq) and torch.equal(k, dk)
    L.qk_rotary(q, None, pos, turns, w_q=wq, q_out=q)
    assert torch.equal(q, want[0]) and torch.equal(v, kept)


def test_positions_and_weights_shared_by_workers():
    W, T, H, D = 3, 6, 2, 16
    x, turns = rnd(W, T, H, D, seed=1), L.rotary_turns(D, device=DEV)
    w, pos = weights(W, D, 2)[0], positions(1, T, 3, 900).to(DEV)
    a = L.qk_rotary(x, positions=pos, turns=turns, w_q=w[:1])[0]
    assert torch.equal(a, L.qk_rotary(x, positions=pos.expand(W, T).contiguous(), turns=turns, w_q=w[:1].expand(W, D).contiguous())[0])
    b = L.qk_rotary(x, turns=turns)[0]
    assert torch.equal(b, L.qk_rotary(x, positions=torch.arange(T, dtype=torch.int32, device=DEV)[None], turns=turns)[0])


def test_norm_alone_and_rotation_alone():
    W, T, H, D = 2, 5, 3, 40
    x = rnd(W, T, H, D, seed=1)
    assert torch.equal(L.qk_rotary(x, turns=L.rotary_turns(D, device=DEV), positions=torch.zeros((1, T), dtype=torch.int32, device=DEV), norm=False)[0], x)
    g = rnd(W, T, H, D, seed=2)
    turns, pos = L.rotary_turns(D, device=DEV), positions(W, T, 3, 50)
    dx, none = L.qk_rotary_grad(g, positions=pos.to(DEV), turns=turns, norm=False)            # neither q nor stats
    want, e = rotate(d(g), torch.zeros(g.shape, dtype=torch.float64), pos, d(turns), D, False, 1.0, back=True)
    assert none is None and bool(((d(dx) - want).abs() <= e + EPS * want.abs()).all())


def test_stretched_turns():
    t = L.rotary_turns(64, base=500.0, device="cpu")
    assert torch.equal(L.rotary_turns(64, base=500.0, stretch=4.0, device="cpu"), t / 4)
    s = L.rotary_turns(64, base=500.0, stretch=4.0, keep=(2048, 1.0, 32.0), device="cpu")
    n = t * 2048
    assert torch.equal(s[n >= 32], t[n >= 32]) and torch.equal(s[n <= 1], t[n <= 1] / 4)
    assert bool((s[:-1] > s[1:]).all()) and bool((s <= t).all()) and bool((s >= t / 4).all())


def test_rows_do_not_reach_into_each_other():
    W, T, H, D = 1, 6, 3, 64
    x, turns = rnd(W, T, H, D, seed=1), L.rotary_turns(D, device=DEV)
    clean = L.qk_rotary(x, turns=turns)[0]
    x[0, 2, 1, 5], x[0, 4, 0, 7] = float("nan"), float("inf")
    x[0, 1, 2] = 0.0
    y = L.qk_rotary(x, turns=turns)[0]
    same = torch.ones((T, H), dtype=torch.bool)
    same[2, 1] = same[4, 0] = same[1, 2] = False
    assert torch.equal(y[0][same], clean[0][same]) and bool((y[0, 1, 2] == 0).all()) and bool(torch.isnan(y[0, 2, 1]).all())


def test_nothing_to_do():
    turns = L.rotary_turns(16, device=DEV)
    q, k, s = L.qk_rotary(torch.empty((2, 0, 3, 16), device=DEV), torch.empty((2, 0, 1, 16), device=DEV), turns=turns)
    assert q.shape == (2, 0, 3, 16) and k.shape == (2, 0, 1, 16) and s.shape == (2, 0, 4)
    dw = torch.full((2, 16), 5.0, device=DEV)
    L.qk_rotary_grad(q, k, q, k, s, turns=turns, dw_q=dw, accumulate=True)
    assert bool((dw == 5).all())
    L.qk_rotary_grad(q, k, q, k, s, turns=turns, dw_q=dw)
    assert bool((dw == 0).all())


def test_equal_calls_give_equal_bits_on_any_stream():
    W, T, H, D = 2, 700, 4, 64
    x, g, turns = rnd(W, T, H, D, seed=1, dtype=torch.bfloat16), rnd(W, T, H, D, seed=2, dtype=torch.bfloat16), L.rotary_turns(D, device=DEV)
    dw = [torch.zeros((W, D), device=DEV) for _ in range(2)]
    y, _, s = L.qk_rotary(x, turns=turns)
    dx, _ = L.qk_rotary_grad(g, None, x, None, s, turns=turns, dw_q=dw[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y2, _, s2 = L.qk_rotary(x, turns=turns, stream=side)
    dx2, _ = L.qk_rotary_grad(g, None, x, None, s2, turns=turns, dw_q=dw[1], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, y2) and torch.equal(dx, dx2) and torch.equal(dw[0], dw[1])
