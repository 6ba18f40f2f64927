"""What mixes the positions of a population's token models, as cases to time and to compare.

A case is a dict of plain values.  `op` says which operator:

  qk          queries and keys before attention: each head's norm and the rotation by its position, in one pass
  qk_grad     its gradients: queries, keys, and both norms' weights
  attend      attention of queries to the keys of their entry: causal, or to another sequence's keys of another length, or of
              single new tokens to a long cache; fewer key heads than query heads; padded entries
  attend_grad its gradients: queries, keys, values

With `own` false `run` computes them from elementary torch operations in 32 bits (the angles of the rotation in 64); with
`own` true it calls the library.  `exact` is the definition in 64 bits.  Norms' weights are columns of the rows of a [W, ld]
fp32 matrix, as everywhere in the library; an entry of attention is a worker or one of its sequences.
"""
import math

import torch

own = False

DEV = "cuda:0"
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "bf16": 2}
EPS_NORM = 1e-6
PHI = 0.6180339887498949
BASE = 10000.0


# ------------------------------------------------------------------------------------------------
# the listed cases
# ------------------------------------------------------------------------------------------------
def listed():
    return [
        # serving: the new token of each worker, far into its text; the cost is the launch
        {"name": "qk_one_token", "op": "qk", "W": 4, "T": 1, "Hq": 16, "Hk": 4, "D": 64, "R": 64, "dtype": "bf16", "norm": True,
         "interleaved": False, "stretch": 1.0},
        # odd sizes; part of the head rotated, neighbours paired, positions stretched to a longer context
        {"name": "qk_odd", "op": "qk", "W": 3, "T": 517, "Hq": 9, "Hk": 3, "D": 72, "R": 36, "dtype": "fp32", "norm": True,
         "interleaved": True, "stretch": 4.0},
        # a large training batch
        {"name": "qk_large", "op": "qk", "W": 8, "T": 8192, "Hq": 32, "Hk": 8, "D": 128, "R": 128, "dtype": "bf16", "norm": True,
         "interleaved": False, "stretch": 1.0},
        # backward at odd sizes
        {"name": "qk_grad_odd", "op": "qk_grad", "W": 5, "T": 333, "Hq": 6, "Hk": 2, "D": 72, "R": 36, "dtype": "fp32", "norm": True,
         "interleaved": True, "stretch": 4.0},
        # backward of a large training batch
        {"name": "qk_grad_large", "op": "qk_grad", "W": 8, "T": 4096, "Hq": 32, "Hk": 8, "D": 128, "R": 128, "dtype": "bf16", "norm": True,
         "interleaved": False, "stretch": 1.0},
        # serving: one new token an entry against a short cache
        {"name": "attend_one_token", "op": "attend", "B": 4, "Tq": 1, "Tk": 517, "Hq": 16, "Hk": 4, "D": 64, "dtype": "bf16",
         "causal": True, "ragged": "keys"},
        # serving: one new token an entry against long caches of many lengths; the keys and values have to be read
        {"name": "attend_long_cache", "op": "attend", "B": 32, "Tq": 1, "Tk": 16384, "Hq": 32, "Hk": 8, "D": 128, "dtype": "bf16",
         "causal": True, "ragged": "keys"},
        # cross attention to encoded sequences of odd lengths, one of them empty
        {"name": "attend_cross_odd", "op": "attend", "B": 6, "Tq": 333, "Tk": 501, "Hq": 6, "Hk": 6, "D": 72, "dtype": "fp32",
         "causal": False, "ragged": "keys"},
        # an ordinary training batch of padded sequences
        {"name": "attend_batch", "op": "attend", "B": 64, "Tq": 512, "Tk": 512, "Hq": 16, "Hk": 16, "D": 64, "dtype": "bf16",
         "causal": True, "ragged": "both"},
        # long texts
        {"name": "attend_long", "op": "attend", "B": 2, "Tq": 8192, "Tk": 8192, "Hq": 32, "Hk": 8, "D": 128, "dtype": "bf16",
         "causal": True, "ragged": "no"},
        # backward of cross attention at odd sizes
        {"name": "attend_grad_odd", "op": "attend_grad", "B": 3, "Tq": 100, "Tk": 259, "Hq": 6, "Hk": 2, "D": 72, "dtype": "fp32",
         "causal": False, "ragged": "keys"},
        # backward of a large training batch
        {"name": "attend_grad_large", "op": "attend_grad", "B": 4, "Tq": 4096, "Tk": 4096, "Hq": 16, "Hk": 4, "D": 128, "dtype": "bf16",
         "causal": True, "ragged": "no"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    """(query heads, key heads, columns of a head)"""
    Hk, G = rng.choice([1, 2, 2, 4, 8]), rng.choice([1, 1, 2, 3, 4, 8])
    D = rng.choice([64, 128, 128, 32, 80, 96, rng.randint(8, 128)])
    return Hk * G, Hk, D


def _drawn(rng):
    op = rng.choice(["qk", "qk_grad", "attend", "attend", "attend", "attend_grad", "attend_grad"])
    kind = rng.choice(["fp32", "bf16", "bf16", "bf16"])
    Hq, Hk, D = _heads(rng)
    if op in ("qk", "qk_grad"):
        R = rng.choice([D // 2 * 2, D // 2 * 2, D // 4 * 2])
        return {"op": op, "W": rng.choice([1, 2, 3, 4, 8, 16]), "T": _log_int(rng, 1, 16384), "Hq": Hq, "Hk": Hk, "D": D, "R": R, "dtype": kind,
                "norm": rng.random() < 0.7, "interleaved": rng.random() < 0.4, "stretch": rng.choice([1.0, 1.0, 4.0])}
    way = rng.choice(["self", "self", "cross"] + (["cache"] if op == "attend" else []))
    B = _log_int(rng, 1, 64)
    if way == "self":
        T = _log_int(rng, 1, 8192)
        return {"op": op, "B": B, "Tq": T, "Tk": T, "Hq": Hq, "Hk": Hk, "D": D, "dtype": kind, "causal": True, "ragged": rng.choice(["no", "both"])}
    if way == "cross":
        return {"op": op, "B": B, "Tq": _log_int(rng, 1, 4096), "Tk": _log_int(rng, 1, 8192), "Hq": Hq, "Hk": Hk, "D": D, "dtype": kind,
                "causal": False, "ragged": rng.choice(["no", "keys"])}
    return {"op": op, "B": B, "Tq": rng.choice([1, 1, 1, 2, 4]), "Tk": _log_int(rng, 1, 65536), "Hq": Hq, "Hk": Hk, "D": D, "dtype": kind,
            "causal": True, "ragged": rng.choice(["no", "keys"])}


def _cost(case):
    """Bytes, products (one of fp32 is worth sixteen of bf16), and the scores that the plain form holds whole."""
    w = work(case)
    scores = 1.0 * case["B"] * case["Hq"] * case["Tq"] * case["Tk"] if case["op"].startswith("attend") else 0.0
    return w["bytes"], w["flops"] * (16 if case["dtype"] == "fp32" else 1), scores


def draw(rng):
    """One more case of the ranges above, in nothing larger than the listed ones of its operator."""
    largest = {}
    for c in listed():
        largest[c["op"]] = [max(p) for p in zip(largest.get(c["op"], (0, 0, 0)), _cost(c))]
    while True:
        c = _drawn(rng)
        if all(n <= most for n, most in zip(_cost(c), largest[c["op"]])):
            return c


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(1_000_003 * int(seed) + 31)
    return g


def _normal(shape, gen, std=1.0, dtype=torch.float32):
    return torch.empty(shape, device=DEV, dtype=dtype).normal_(std=std, generator=gen)


def _turns(case):
    """Turns per position of each pair of rotated columns."""
    R = case["R"]
    return [BASE ** (-2.0 * i / R) / (2.0 * math.pi * case["stretch"]) for i in range(R // 2)]


def _lengths(case):
    """Lengths of the entries' sequences: spread over the range, one full, and where there are several one empty."""
    B, T = case["B"], case["Tk"]
    if case["ragged"] == "no":
        return [T] * B
    out = [min(T, int(T * ((i * PHI) % 1.0)) + 1) for i in range(B)]
    out[-1] = T
    if B >= 4:
        out[0] = 0
    return out


def _weights(W, D, gen):
    """Both norms' weights: columns of wider rows."""
    w = torch.zeros((W, (2 * D + 63) // 64 * 64), device=DEV)
    w[:, :2 * D].normal_(mean=1.0, std=0.1, generator=gen)
    return w[:, :D], w[:, D:2 * D]


def _inputs(case, seed):
    gen = _gen(seed)
    op, dt, Hq, Hk, D = case["op"], DT[case["dtype"]], case["Hq"], case["Hk"], case["D"]
    d = {}
    if op in ("qk", "qk_grad"):
        W, T = case["W"], case["T"]
        qk = _normal((W, T, Hq + Hk, D), gen, 2.0, dt)                  # one projection makes both
        d["q"], d["k"] = qk[:, :, :Hq], qk[:, :, Hq:]
        d["w_q"], d["w_k"] = _weights(W, D, gen)
        start = torch.randint(0, 100000, (W, 1), device=DEV, generator=gen)
        d["positions"] = (start + torch.arange(T, device=DEV)).to(torch.int32)
        d["turns"] = torch.tensor(_turns(case), dtype=torch.float64, device=DEV)
        if op == "qk_grad":
            d["dq"], d["dk"] = _normal((W, T, Hq, D), gen, 1e-2, dt), _normal((W, T, Hk, D), gen, 1e-2, dt)
            d["stats"] = qk.float().square().mean(-1).add(EPS_NORM).rsqrt() if case["norm"] else None
            dw = torch.zeros((W, (2 * D + 63) // 64 * 64), device=DEV)
            d["dw_q"], d["dw_k"] = dw[:, :D], dw[:, D:2 * D]
        return d
    B, Tq, Tk = case["B"], case["Tq"], case["Tk"]
    d["q"] = _normal((B, Tq, Hq, D), gen, 1.5, dt)
    kv = _normal((B, Tk, 2, Hk, D), gen, 1.0, dt)
    d["k"], d["v"] = kv[:, :, 0], kv[:, :, 1]
    d["k_lens"] = d["q_lens"] = None
    if case["ragged"] != "no":
        n = _lengths(case)
        n = n[int(seed) % B:] + n[:int(seed) % B]
        d["k_lens"] = torch.tensor(n, dtype=torch.int32, device=DEV)
        if case["ragged"] == "both":
            d["q_lens"] = d["k_lens"].clone()
    d["scale"] = D ** -0.5
    if op == "attend_grad":
        d["dout"] = _normal((B, Tq, Hq, D), gen, 1e-2, dt)
        out, d["lse"] = _plain_attend(case, d)
        d["out"] = out.to(dt).contiguous()
    return d


def prepare(case, seed):
    return {"case": case, "in": _inputs(case, seed)}


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    import paper_1905_10395_amd as L
    case, d = s["case"], s["in"]
    op = case["op"]
    if op == "qk":
        q, k, stats = L.qk_rotary(d["q"], d["k"], d["positions"], d["turns"], w_q=d["w_q"], w_k=d["w_k"], norm=case["norm"], eps=EPS_NORM,
                                  interleaved=case["interleaved"])
        return {"q": q, "k": k, "stats": stats}
    if op == "qk_grad":
        dq, dk = L.qk_rotary_grad(d["dq"], d["dk"], d["q"], d["k"], d["stats"], d["positions"], d["turns"], w_q=d["w_q"], w_k=d["w_k"],
                                  norm=case["norm"], interleaved=case["interleaved"], dw_q=d["dw_q"], dw_k=d["dw_k"])
        return {"dq": dq, "dk": dk, "dw_q": d["dw_q"], "dw_k": d["dw_k"]}
    args = dict(causal=case["causal"], scale=d["scale"], q_lens=d["q_lens"], k_lens=d["k_lens"])
    if op == "attend":
        out, lse = L.attention(d["q"], d["k"], d["v"], with_lse=case["Tq"] > 1, **args)
        return {"out": out, "lse": lse}
    dq, dk, dv = L.attention_grad(d["dout"], d["q"], d["k"], d["v"], d["out"], d["lse"], **args)
    return {"dq": dq, "dk": dk, "dv": dv}


def _run_plain(s):
    case, d = s["case"], s["in"]
    op, dt = case["op"], DT[case["dtype"]]
    if op == "qk":
        (q, sq), (k, sk) = _plain_qk(case, d, "q"), _plain_qk(case, d, "k")
        return {"q": q.to(dt), "k": k.to(dt), "stats": torch.cat([sq, sk], 2) if case["norm"] else None}
    if op == "qk_grad":
        (dq, wq), (dk, wk) = _plain_qk_grad(case, d, "q", 0), _plain_qk_grad(case, d, "k", case["Hq"])
        d["dw_q"].copy_(wq)
        d["dw_k"].copy_(wk)
        return {"dq": dq.to(dt), "dk": dk.to(dt), "dw_q": d["dw_q"], "dw_k": d["dw_k"]}
    if op == "attend":
        out, lse = _plain_attend(case, d)
        return {"out": out.to(dt), "lse": lse if case["Tq"] > 1 else None}
    return _plain_attend_grad(case, d)


def _angles(d):
    """cos and sin of every position's angles [W, T, 1, R/2]: the angle in 64 bits, whole turns taken off."""
    a = d["positions"].double()[..., None] * d["turns"]
    a = (a - torch.round(a)) * (2.0 * math.pi)
    return torch.cos(a).float()[:, :, None], torch.sin(a).float()[:, :, None]


def _turned(case, x, c, s):
    """The first R columns of x turned by the angles; pairs are neighbours, or a half apart."""
    R = case["R"]
    if case["interleaved"]:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        return torch.cat([torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2), x[..., R:]], -1)
    a, b = x[..., :R // 2], x[..., R // 2:R]
    return torch.cat([a * c - b * s, a * s + b * c, x[..., R:]], -1)


def _plain_qk(case, d, which):
    x, q = d[which].float(), None
    if case["norm"]:
        q = torch.rsqrt((x * x).mean(-1) + EPS_NORM)
        x = x * q[..., None]
    x = x * d["w_" + which][:, None, None]
    return _turned(case, x, *_angles(d)), q


def _plain_qk_grad(case, d, which, first):
    c, s = _angles(d)
    dy = _turned(case, d["d" + which].float(), c, -s)
    x, w = d[which].float(), d["w_" + which][:, None, None]
    if not case["norm"]:
        return dy * w, (dy * x).sum((1, 2))
    q = d["stats"][:, :, first:first + x.shape[2], None]
    h, t = x * q, dy * w
    return q * (t - h * (t * h).mean(-1, keepdim=True)), (dy * h).sum((1, 2))


def _seen(case, d):
    """Which keys each query sees [B, 1, Tq, Tk]: those of its entry; causal: none behind its own, both sequences ending together."""
    B, Tq, Tk = case["B"], case["Tq"], case["Tk"]
    full = lambda t, n: torch.full((B,), n, device=DEV) if t is None else t.long()
    nq, nk = full(d["q_lens"], Tq)[:, None, None], full(d["k_lens"], Tk)[:, None, None]
    t, j = torch.arange(Tq, device=DEV)[:, None], torch.arange(Tk, device=DEV)[None]
    seen = (t < nq) & (j < nk)
    if case["causal"]:
        seen = seen & (j <= t + nk - nq)
    return seen[:, None]


def _by_head(case, x):
    """[B, T, H, D] as fp32 [B, Hq, T, D], key heads repeated for the query heads that share them."""
    x = x.float().transpose(1, 2)
    return x.repeat_interleave(case["Hq"] // x.shape[1], 1).contiguous()


def _plain_attend(case, d):
    q, k, v = (_by_head(case, d[n]) for n in ("q", "k", "v"))
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(d["scale"]).masked_fill_(~_seen(case, d), -math.inf)
    top = s.amax(-1, keepdim=True)
    s.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = s.sum(-1, keepdim=True)
    out = torch.matmul(s, v) / torch.where(total == 0, torch.ones_like(total), total)
    return out.transpose(1, 2), (top + torch.log(total))[..., 0]


def _plain_attend_grad(case, d):
    dt, B, Hk, Tk, D = DT[case["dtype"]], case["B"], case["Hk"], case["Tk"], case["D"]
    q, k, v, o, do = (_by_head(case, d[n]) for n in ("q", "k", "v", "out", "dout"))
    seen = _seen(case, d)
    lse = torch.where(d["lse"] == -math.inf, torch.zeros_like(d["lse"]), d["lse"])[..., None]
    p = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(d["scale"]).sub_(lse).masked_fill_(~seen, -math.inf).exp_()
    do = do.masked_fill(~seen.any(-1, keepdim=True), 0.0)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    ds = torch.matmul(do, v.transpose(2, 3).contiguous()).sub_((o * do).sum(-1, keepdim=True)).mul_(p).mul_(d["scale"])
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q)
    shared = lambda g: g.view(B, Hk, -1, Tk, D).sum(2).transpose(1, 2).to(dt)
    return {"dq": dq.transpose(1, 2).to(dt), "dk": shared(dk), "dv": shared(dv)}


# ------------------------------------------------------------------------------------------------
# what one pass cannot do without
# ------------------------------------------------------------------------------------------------
def _pairs(case):
    """Pairs of a query and a key that it sees, of one head, over all entries; keys of all entries."""
    pairs, keys = 0.0, 0
    for n in _lengths(case):
        nq = n if case["ragged"] == "both" else case["Tq"]
        keys += n
        if not case["causal"]:
            pairs += 1.0 * nq * n
        elif nq <= n:
            pairs += nq * (n - nq + 1) + nq * (nq - 1) / 2.0
        else:
            pairs += n * (n + 1) / 2.0
    return pairs, keys


def work(case):
    op, es, Hq, Hk, D = case["op"], SIZE[case["dtype"]], case["Hq"], case["Hk"], case["D"]
    if op in ("qk", "qk_grad"):
        rows = 1.0 * case["W"] * case["T"] * (Hq + Hk)
        streams = 2 if op == "qk" else 3
        return {"bytes": rows * (D * es * streams + (4.0 if case["norm"] else 0.0)) + 4.0 * case["W"] * (case["T"] + 2 * D * (1 if op == "qk" else 2)),
                "flops": rows * D * (9.0 if op == "qk" else 16.0)}
    pairs, keys = _pairs(case)
    queries = 1.0 * case["B"] * case["Tq"] * Hq * D * es
    cached = 2.0 * keys * Hk * D * es
    if op == "attend":
        return {"bytes": 2 * queries + cached, "flops": 4.0 * pairs * Hq * D}
    return {"bytes": 4 * queries + cached + 2.0 * case["B"] * case["Tk"] * Hk * D * es, "flops": 10.0 * pairs * Hq * D}


# ------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ------------------------------------------------------------------------------------------------
def exact(case, seed):
    d = _inputs(case, seed)
    op = case["op"]
    if op == "qk":
        q, k = _exact_qk(case, d, "q"), _exact_qk(case, d, "k")
        return {"q": q[0], "k": k[0], "stats": torch.cat([q[1], k[1]], 2) if case["norm"] else None}
    if op == "qk_grad":
        q, k = _exact_qk_grad(case, d, "q"), _exact_qk_grad(case, d, "k")
        return {"dq": q[0], "dk": k[0], "dw_q": q[1], "dw_k": k[1]}
    return _exact_attend(case, d)


def _rotation(case, d, w):
    """Worker w's turns as complex numbers [T, 1, R/2]."""
    a = 2.0 * math.pi * torch.frac(d["positions"][w].double()[:, None] * d["turns"][None])
    return torch.polar(torch.ones_like(a), a)[:, None]


def _pairs_of(case, x):
    R = case["R"]
    return torch.view_as_complex(x[..., :R].unflatten(-1, (R // 2, 2)).contiguous()) if case["interleaved"] else torch.complex(x[..., :R // 2], x[..., R // 2:R])


def _columns_of(case, z, x):
    z = torch.view_as_real(z).flatten(-2) if case["interleaved"] else torch.cat([z.real, z.imag], -1)
    return torch.cat([z, x[..., case["R"]:]], -1)


def _exact_qk(case, d, which):
    out, stats = [], []
    for w in range(case["W"]):
        x = d[which][w].double()
        q = (x.pow(2).sum(-1) / case["D"] + EPS_NORM).pow(-0.5)
        y = x * d["w_" + which][w].double()
        y = y * q[..., None] if case["norm"] else y
        out.append(_columns_of(case, _pairs_of(case, y) * _rotation(case, d, w), y))
        stats.append(q)
    return torch.stack(out), torch.stack(stats)


def _exact_qk_grad(case, d, which):
    """The rotation undone, then the Jacobian of x -> q x with q = (mean x^2 + eps)^-1/2 given: dq/dx = -q^3 x / D."""
    first = 0 if which == "q" else case["Hq"]
    dx, dw = [], []
    for w in range(case["W"]):
        g = d["d" + which][w].double()
        g = _columns_of(case, _pairs_of(case, g) * _rotation(case, d, w).conj(), g)
        x, t = d[which][w].double(), g * d["w_" + which][w].double()
        if case["norm"]:
            q = d["stats"][w, :, first:first + x.shape[1], None].double()
            dx.append(q * t - x * q.pow(3) * (t * x).sum(-1, keepdim=True) / case["D"])
            dw.append((g * x * q).sum((0, 1)))
        else:
            dx.append(t)
            dw.append((g * x).sum((0, 1)))
    return torch.stack(dx), torch.stack(dw)


def _exact_attend(case, d):
    """Entry by entry and head by head, each query's softmax over the keys that it sees."""
    B, Tq, Tk, Hq, G = case["B"], case["Tq"], case["Tk"], case["Hq"], case["Hq"] // case["Hk"]
    grad = case["op"] == "attend_grad"
    zeros = lambda n: torch.zeros(d[n].shape, dtype=torch.float64, device=DEV)
    out, dq, dk, dv = zeros("q"), zeros("q"), zeros("k"), zeros("v")
    lse = torch.full((B, Hq, Tq), -math.inf, dtype=torch.float64, device=DEV)
    for b in range(B):
        nk = Tk if d["k_lens"] is None else int(d["k_lens"][b])
        nq = Tq if d["q_lens"] is None else int(d["q_lens"][b])
        lo = max(0, nq - nk) if case["causal"] else 0                    # queries before the first key see nothing
        if nk == 0 or nq <= lo:
            continue
        hidden = torch.ones((nq - lo, nk), dtype=torch.bool, device=DEV).triu(nk - nq + lo + 1) if case["causal"] else None
        for h in range(Hq):
            q, k, v = d["q"][b, lo:nq, h].double(), d["k"][b, :nk, h // G].double(), d["v"][b, :nk, h // G].double()
            s = q @ k.t() * d["scale"]
            if hidden is not None:
                s.masked_fill_(hidden, -math.inf)
            if not grad:
                z = torch.logsumexp(s, -1)
                lse[b, h, lo:nq] = z
                out[b, lo:nq, h] = (s - z[:, None]).exp() @ v
                continue
            p = (s - d["lse"][b, h, lo:nq, None].double()).exp()
            do = d["dout"][b, lo:nq, h].double()
            dv[b, :nk, h // G] += p.t() @ do
            ds = p * (do @ v.t() - (do * d["out"][b, lo:nq, h].double()).sum(-1, keepdim=True)) * d["scale"]
            dq[b, lo:nq, h] = ds @ k
            dk[b, :nk, h // G] += ds.t() @ q
    if grad:
        return {"dq": dq, "dk": dk, "dv": dv}
    return {"out": out, "lse": lse if Tq > 1 else None}
