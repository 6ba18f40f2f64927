"""Token-model operators on routes that small sizes do not reach: teams that norm several tokens one after the other, blocks without
a norm behind them, wide sorts and large tables, and all of them in captured graphs.  References in 64 bits on the GPU."""
import pytest
import torch

import paper_1905_10395_amd as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 2.0 ** -24
UNIT = {torch.float32: EPS, torch.bfloat16: 2.0 ** -8}
BOTH = [torch.float32, torch.bfloat16]
NORM_EPS = 1e-5
SCALE = 0.5
BOOL = [False, True]


def rnd(*shape, seed, dtype=torch.float32, std=1.0, mean=0.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.empty(shape, device=DEV).normal_(mean, std, generator=g).to(dtype)


def within(got, ref, bound, what=""):
    bad = (got.double() - ref).abs() > bound
    assert not bool(bad.any()), (what, int(bad.sum()), float(((got.double() - ref).abs() / bound.clamp(min=1e-300)).max()))


def slack(D, u=None):
    """Relative error of a product with a norm's factor (a sum of D squares) and, with u, a sigmoid of u."""
    return (D / 2 + 24 + (0 if u is None else 2 * u.abs())) * EPS


def check_forward(r, y, u, wp, wn, post):
    """block_norm against the formulas; returns what the gradient needs."""
    got_r, got_n, stats = L.block_norm(r, y, gate=u, w_post=wp, w_pre=wn, scale=SCALE, eps=NORM_EPS, post_norm=post)
    D, unit = r.shape[2], UNIT[r.dtype]
    y64, u64 = y.double(), None if u is None else u.double()
    qp = (y64.pow(2).mean(2) + NORM_EPS).rsqrt() if post else torch.ones(y.shape[:2], dtype=torch.float64, device=DEV)
    b = SCALE * y64 * qp[..., None] * wp.double()[:, None]
    if u is not None:
        b = b * torch.sigmoid(u64)
    R = r.double() + b
    br = b.abs() * slack(D, u64) + R.abs() * 2 * EPS
    qn = (R.pow(2).mean(2) + NORM_EPS).rsqrt()
    N = R * qn[..., None] * wn.double()[:, None]
    dq = br.norm(dim=2) / R.norm(dim=2)                                # q moves at most by the row's error over its 2-norm
    within(got_r, R, br + unit * R.abs() * 1.01, "r_out")
    within(got_n, N, br * (qn[..., None] * wn.double()[:, None]).abs() + N.abs() * (slack(D) + dq[..., None] + unit * 1.01), "n")
    if post:
        within(stats[0], qp, qp * slack(D), "q_post")
    within(stats[1], qn, qn * (slack(D) + dq), "q_pre")


def check_backward(dn, dR, r, y, u, wp, wn, post, weights=True):
    W, T, D = r.shape
    q = torch.stack([(t.double().pow(2).mean(2) + NORM_EPS).rsqrt() for t in (y, r)]).float()
    grads = torch.full((W, 2 * D + 4), 9.0, device=DEV)
    dwp, dwn = (grads[:, 1:1 + D], grads[:, 2 + D:2 + 2 * D]) if weights else (None, None)
    args = dict(gate=u, w_post=wp, w_pre=wn, scale=SCALE, post_norm=post, dw_post=dwp, dw_pre=dwn)
    dr, dy, du = L.block_norm_grad(dn, dR, r, q, y, **args)
    unit, f64 = UNIT[r.dtype], torch.float64
    wp, wn = wp.double()[:, None], wn.double()[:, None]
    eps = slack(D) + D / 2 * EPS
    qn = q[1].double()[..., None]
    h, t = r.double() * qn, dn.double() * wn
    ref = qn * (t - h * (t * h).mean(2, keepdim=True))
    br = eps * qn * (t.abs() + h.abs() * (t * h).abs().mean(2, keepdim=True))
    if dR is not None:
        ref = ref + dR.double()
        br = br + dR.double().abs() * 4 * EPS
    within(dr, ref, br + unit * ref.abs() * 1.01, "dr")
    if weights:
        dh = dn.double() * h
        within(dwn, dh.sum(1), dh.abs().sum(1) * (T + 17) * EPS, "dw_pre")
    qp = q[0].double()[..., None] if post else torch.ones((W, T, 1), dtype=f64, device=DEV)
    z = y.double() * qp
    su, a = 8 * EPS, torch.ones((), dtype=f64, device=DEV)
    if u is not None:
        u64 = u.double()
        a, su = torch.sigmoid(u64), (8 + 2 * u64.abs()) * EPS
        dg = SCALE * ref * z * wp * a * torch.sigmoid(-u64)
        # exp(-u): 2 |u| + 2 roundings, a(1-a) 6 |u| + 14 in all, the other factors 6
        within(du, dg, SCALE * br * (z * wp).abs() * a * torch.sigmoid(-u64) + dg.abs() * ((6 * u64.abs() + 20) * EPS + unit * 1.01), "dgate")
    e = SCALE * ref * a
    be = SCALE * br * a + e.abs() * su
    if weights:
        within(dwp, (e * z).sum(1), (be * z.abs()).sum(1) + (e * z).abs().sum(1) * (T + 17) * EPS, "dw_post")
        assert bool((grads[:, 0] == 9).all()) and bool((grads[:, 1 + D] == 9).all()) and bool((grads[:, 2 + 2 * D:] == 9).all())
    t, bt = e * wp, be * wp.abs()
    if post:
        ref = qp * (t - z * (t * z).mean(2, keepdim=True))
        b = qp * (bt + z.abs() * (bt * z.abs()).mean(2, keepdim=True)) + eps * qp * (t.abs() + z.abs() * (t * z).abs().mean(2, keepdim=True))
    else:
        ref, b = t, bt + t.abs() * 4 * EPS
    within(dy, ref, b + unit * ref.abs() * 1.01, "dy")
    return dr, dy, du, grads


def tensors(W, T, D, dtype, gate, back):
    """r, y, u and, backward, dn, dR; weights as columns of wider rows."""
    x = rnd(W, 2 * D + 3, seed=9, std=0.3, mean=1.0)
    act = [rnd(W, T, D, seed=k, dtype=dtype, std=s) for k, s in ((1, 1.0), (2, 3.0), (3, 2.0), (4, 1.0), (5, 1.0))[:5 if back else 3]]
    if not gate:
        act[2] = None
    return act, x[:, 1:1 + D], x[:, 1 + D:1 + 2 * D]


# So many workers that a team takes two to five tokens: of 8 to 64 lanes, of a workgroup, with two pieces a lane; aligned and not.
@pytest.mark.parametrize("W,T,D", [(16384, 70, 8), (16384, 35, 65), (16384, 11, 264), (32768, 3, 520), (32768, 2, 1001), (8192, 3, 2056),
                                   (4096, 2, 8200), (512, 20, 8195)])
@pytest.mark.parametrize("dtype", BOTH)
def test_forward_teams_take_several_tokens(W, T, D, dtype):
    (r, y, u), wp, wn = tensors(W, T, D, dtype, D % 2 == 0, False)
    check_forward(r, y, u, wp, wn, True)


@pytest.mark.parametrize("W,T,D", [(256, 700, 8), (64, 600, 64), (512, 70, 65), (256, 90, 201), (512, 33, 264), (512, 37, 520), (512, 37, 1001),
                                   (256, 9, 2056), (128, 9, 8200), (128, 9, 8195)])
@pytest.mark.parametrize("dtype", BOTH)
def test_backward_teams_take_several_tokens(W, T, D, dtype):
    (r, y, u, dn, dR), wp, wn = tensors(W, T, D, dtype, D % 2 == 0, True)
    first = check_backward(dn, dR, r, y, u, wp, wn, True)
    again = check_backward(dn, dR, r, y, u, wp, wn, True)
    assert all(a is b is None or torch.equal(a, b) for a, b in zip(first, again))


# The usual block of a token model has no norm behind it.
@pytest.mark.parametrize("W,T,D", [(2, 3, 7), (3, 37, 64), (2, 9, 203), (2, 33, 520), (1, 5, 2056), (1, 3, 8195)])
@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("gate", BOOL)
def test_blocks_without_a_norm_behind(W, T, D, dtype, gate):
    (r, y, u, dn, dR), wp, wn = tensors(W, T, D, dtype, gate, True)
    check_forward(r, y, u, wp, wn, False)
    full = check_backward(dn, dR, r, y, u, wp, wn, False)
    bare = check_backward(dn, dR, r, y, u, wp, wn, False, weights=False)
    assert all(a is b is None or torch.equal(a, b) for a, b in zip(full[:3], bare[:3]))


@pytest.mark.parametrize("post", BOOL)
@pytest.mark.parametrize("W,T,D", [(3, 37, 64), (2, 9, 203), (1, 3, 8195)])
def test_backward_with_nothing_past_the_next_block(W, T, D, post):
    (r, y, u, dn, _), wp, wn = tensors(W, T, D, torch.bfloat16, True, True)
    check_backward(dn, None, r, y, u, wp, wn, post)


def draw_tokens(W, T, V, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    u = torch.rand((W, T), device=DEV, generator=g, dtype=torch.float64)
    tok = (torch.exp(u * torch.log(torch.tensor(V + 1.0, dtype=torch.float64))) - 1).long().clamp(0, V - 1)
    tok[:, ::11] = torch.randint(0, V, tok[:, ::11].shape, device=DEV, generator=g)           # rare ones among them
    return tok.masked_fill(torch.rand((W, T), device=DEV, generator=g) < 0.05, -1).to(torch.int32)


# One launch with two tokens a thread, with room for all zeros of large tables and with more than 2^22 rows; eight tokens a thread
# in a tile of the long sort; three digits.
@pytest.mark.parametrize("W,T,V,D", [(1, 1025, 700, 40), (2, 2048, 131, 101), (2, 1100, (1 << 20) + 9, 17), (1, 100, (1 << 22) + 5, 1), (1, 131072 + 77, 257, 8),
                                     (1, 8200, (1 << 20) + 3, 3), (2, 140001, (1 << 20) + 3, 4)])
@pytest.mark.parametrize("accumulate", BOOL)
def test_embedding_gradient(W, T, V, D, accumulate):
    tok = draw_tokens(W, T, V, seed=T)
    dout = rnd(W, T, D, seed=2, dtype=torch.bfloat16)
    rows = rnd(W, V * D + 7, seed=3)
    before, dtable = rows.clone(), rows[:, 2:2 + V * D].unflatten(1, (V, D))
    ref = before[:, 2:2 + V * D].unflatten(1, (V, D)).double() if accumulate else torch.zeros((W, V, D), dtype=torch.float64, device=DEV)
    mag, n = ref.abs(), torch.zeros((W, V, 1), dtype=torch.float64, device=DEV)
    for w in range(W):
        ok = tok[w] >= 0
        at, d = tok[w, ok].long(), dout[w, ok].double() * 1.75
        ref[w].index_add_(0, at, d)
        mag[w].index_add_(0, at, d.abs())
        n[w].index_add_(0, at, torch.ones((len(at), 1), dtype=torch.float64, device=DEV))
    L.embed_grad(dout, tok, dtable, scale=1.75, accumulate=accumulate)
    within(dtable, ref, mag * (n + 3) * EPS)                           # n sums in some order, the product, the sum with what was there
    none = (n == 0).expand_as(ref)
    assert torch.equal(dtable[none], ref[none].float())
    assert torch.equal(rows[:, :2], before[:, :2]) and torch.equal(rows[:, 2 + V * D:], before[:, 2 + V * D:])


@pytest.mark.parametrize("T", [1, 300, 9000])
def test_in_a_captured_graph(T):
    """Lookup, norms and their gradients: every replay, with other work between, gives the bits of the same calls made one by one."""
    W, V, D = 2, 301, 72
    tok, table = draw_tokens(W, T, V, seed=1), rnd(W, V, D, seed=2)
    wp, wn = rnd(W, D, seed=3), rnd(W, D, seed=4)
    dtable, dw = torch.zeros((W, V, D), device=DEV), torch.zeros((2, W, D), device=DEV)

    def step():
        r0 = L.embed_lookup(table, tok, scale=2.0, dtype=torch.bfloat16)
        r, n, stats = L.block_norm(r0, r0, gate=r0, w_post=wp, w_pre=wn, scale=SCALE)
        dr, dy, du = L.block_norm_grad(n, r, r, stats, r0, gate=r0, w_post=wp, w_pre=wn, scale=SCALE, dw_post=dw[0], dw_pre=dw[1])
        L.embed_grad(dr, tok, dtable, scale=2.0)
        return r, n, dr, dy, du

    step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        held = step()
    torch.cuda.synchronize()
    for k in range(3):
        table.copy_(rnd(W, V, D, seed=10 + k))                         # replays read what is there now
        tok.copy_(draw_tokens(W, T, V, seed=20 + k))
        want = [t.clone() for t in step()] + [dtable.clone(), dw.clone()]
        dtable.fill_(7.0)
        dw.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, [*held, dtable, dw]):
            assert torch.equal(a, b)


def test_embedding_gradient_of_the_most_rows():
    V, T = (1 << 30) - 1, 9001
    tok, dout = draw_tokens(1, T, V, seed=5), rnd(1, T, 1, seed=6)
    tok[0, 7], tok[0, 8] = V - 1, V                                    # the last row, and one past it: padding
    dtable = torch.full((1, V, 1), 7.0, device=DEV)
    L.embed_grad(dout, tok, dtable)
    ok = (tok[0] >= 0) & (tok[0] < V)
    rows, at = tok[0, ok].long().unique(return_inverse=True)
    f = lambda: torch.zeros(len(rows), dtype=torch.float64, device=DEV)
    d = dout[0, ok, 0].double()
    ref, mag, n = f().index_add_(0, at, d), f().index_add_(0, at, d.abs()), f().index_add_(0, at, torch.ones_like(d))
    within(dtable[0, rows, 0], ref, mag * (n + 3) * EPS)
    dtable[0, rows] = 0.0
    assert int(dtable.count_nonzero()) == 0
