"""The operators a population of token models needs around its blocks' products, as cases to time and to compare.

A case is a dict of plain values.  `op` says which operator:

  lookup       rows of each worker's embedding table, scaled
  lookup_grad  the table's gradient from the gradient of the looked-up rows
  norm         after a block: post-norm, gate, scaled residual sum, and the next block's pre-norm in the same pass
  norm_grad    its gradients: residual stream, block output, gate, both norms' weights
  adamw        one AdamW step over every tensor of every worker, moments held in 32 or in 8 bits

With `own` false `run` computes them from elementary torch operations in 32 bits; with `own` true it calls the library.
`exact` is the definition in 64 bits.  Workers' parameters are columns of the rows of a [W, ld] fp32 matrix, as everywhere
in the library.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "bf16": 2}
EPS_NORM = 1e-6
LR, BETA1, BETA2, EPS, STEP, WD = 1e-3, 0.9, 0.999, 1e-8, 37, 0.1
BLOCK = 256                                          # elements that share a scale of the 8-bit moments
PHI = 0.6180339887498949


def _ld(P):
    """Row stride a program uses: rows padded to 256 bytes."""
    return (P + 63) // 64 * 64


# ------------------------------------------------------------------------------------------------
# the listed cases
# ------------------------------------------------------------------------------------------------
def listed():
    return [
        # serving: every worker looks up its one new token; the cost is the launch
        {"name": "lookup_one_token", "op": "lookup", "W": 4, "T": 1, "V": 1003, "D": 256, "table": "fp32", "out": "bf16"},
        # a training batch of 16 workers from the bf16 copy of the weights
        {"name": "lookup_batch", "op": "lookup", "W": 16, "T": 8192, "V": 32768, "D": 1024, "table": "bf16", "out": "bf16"},
        # a small character-like vocabulary of odd sizes: every table row gets several tokens
        {"name": "lookup_grad_odd", "op": "lookup_grad", "W": 3, "T": 517, "V": 131, "D": 101, "dtype": "fp32", "accumulate": False},
        # a vocabulary much larger than the batch, added to the gradient that tied output weights left there
        {"name": "lookup_grad_tied", "op": "lookup_grad", "W": 4, "T": 2048, "V": 65536, "D": 512, "dtype": "bf16",
         "accumulate": True},
        # a long batch whose frequent tokens come by the thousand; the whole table's gradient is written
        {"name": "lookup_grad_long", "op": "lookup_grad", "W": 8, "T": 32768, "V": 50000, "D": 1024, "dtype": "bf16",
         "accumulate": False},
        # serving: one new token a worker
        {"name": "norm_one_token", "op": "norm", "W": 4, "T": 1, "D": 1024, "dtype": "bf16", "gate": True},
        # a large training batch
        {"name": "norm_large", "op": "norm", "W": 8, "T": 8192, "D": 4096, "dtype": "bf16", "gate": True},
        # odd sizes without a gate
        {"name": "norm_grad_odd", "op": "norm_grad", "W": 5, "T": 333, "D": 1001, "dtype": "fp32", "gate": False},
        # backward of a large training batch
        {"name": "norm_grad_large", "op": "norm_grad", "W": 8, "T": 4096, "D": 2048, "dtype": "bf16", "gate": True},
        # a toy model: the cost of a step is its launches
        {"name": "adamw_tiny", "op": "adamw", "W": 4, "dims": "20-16-4", "bits": 32, "g": "fp32", "shadow": False},
        # a small classifier population of sizes that are no multiples of anything, moments in 8 bits
        {"name": "adamw_8bit_ragged", "op": "adamw", "W": 8, "dims": "785-301-100-10", "bits": 8, "g": "fp32", "shadow": False},
        # 268 M parameters, bf16 copy of the weights kept current
        {"name": "adamw_large", "op": "adamw", "W": 8, "dims": "4096-4096-4096-10", "bits": 32, "g": "fp32", "shadow": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Round widths are the common ones; odd ones have to work as well."""
    d = _log_int(rng, lo, hi)
    return d if rng.random() < 0.4 else max(64, (d + 63) // 64 * 64)


def _drawn(rng):
    op = rng.choice(["lookup", "lookup_grad", "lookup_grad", "norm", "norm_grad", "adamw", "adamw"])
    W = rng.choice([1, 2, 3, 4, 6, 8, 12, 16])
    kind = rng.choice(["fp32", "bf16", "bf16"])
    if op == "lookup":
        return {"op": op, "W": W, "T": _log_int(rng, 1, 16384), "V": _log_int(rng, 100, 65536), "D": _width(rng, 48, 2048),
                "table": rng.choice(["fp32", "bf16"]), "out": kind}
    if op == "lookup_grad":
        return {"op": op, "W": W, "T": _log_int(rng, 1, 65536), "V": _log_int(rng, 100, 65536), "D": _width(rng, 48, 2048),
                "dtype": kind, "accumulate": rng.random() < 0.5}
    if op in ("norm", "norm_grad"):
        return {"op": op, "W": W, "T": _log_int(rng, 1, 16384), "D": _width(rng, 48, 8192), "dtype": kind, "gate": rng.random() < 0.6}
    dims = [_log_int(rng, 16, 4096) for _ in range(rng.choice([2, 3, 4]))] + [rng.choice([10, 10, 2, 7, 100])]
    if rng.random() < 0.5:
        dims[:-1] = [max(64, (d + 63) // 64 * 64) for d in dims[:-1]]
    return {"op": op, "W": W, "dims": "-".join(str(d) for d in dims), "bits": rng.choice([32, 8]), "g": rng.choice(["fp32", "fp32", "bf16"]),
            "shadow": rng.random() < 0.4}


def draw(rng):
    """One more case of the ranges above, no larger than the largest listed one of its operator."""
    largest = {}
    for c in listed():
        largest[c["op"]] = max(largest.get(c["op"], 0.0), work(c)["bytes"])
    while True:
        c = _drawn(rng)
        if work(c)["bytes"] <= largest[c["op"]]:
            return c


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(1_000_003 * int(seed) + 29)
    return g


def _normal(shape, gen, std=1.0, dtype=torch.float32, mean=0.0):
    return torch.empty(shape, device=DEV, dtype=dtype).normal_(mean=mean, std=std, generator=gen)


def _rows(W, P, gen, std, dtype=torch.float32):
    t = torch.zeros((W, _ld(P)), device=DEV, dtype=dtype)
    t[:, :P].normal_(std=std, generator=gen)
    return t


def _tokens(W, T, V, gen):
    """Frequencies that fall as 1/rank, as tokens' do, and one place in fifty left as padding (-1)."""
    u = torch.rand((W, T), device=DEV, generator=gen, dtype=torch.float64)
    tok = (torch.exp(u * math.log(V + 1.0)) - 1.0).long().clamp(0, V - 1)
    pad = torch.rand((W, T), device=DEV, generator=gen) < 0.02
    return tok.masked_fill(pad, -1).to(torch.int32)


def _tensors(case):
    """(first column, elements, weight decay) of every weight matrix and bias in a worker's row, and the row's length."""
    dims = [int(v) for v in case["dims"].split("-")]
    at, out = 0, []
    for k in range(len(dims) - 1):
        out.append((at, dims[k] * dims[k + 1], WD))
        at += dims[k] * dims[k + 1]
        out.append((at, dims[k + 1], 0.0))
        at += dims[k + 1]
    return out, at


def _inputs(case, seed):
    gen = _gen(seed)
    W, op = case["W"], case["op"]
    d = {}
    if op == "lookup":
        V, D = case["V"], case["D"]
        x = _rows(W, V * D, gen, 0.02, DT[case["table"]])
        d["table"] = x[:, :V * D].unflatten(1, (V, D))
        d["tokens"] = _tokens(W, case["T"], V, gen)
        d["scale"] = math.sqrt(D)
    elif op == "lookup_grad":
        V, D = case["V"], case["D"]
        d["tokens"] = _tokens(W, case["T"], V, gen)
        d["dout"] = _normal((W, case["T"], D), gen, 1e-2, DT[case["dtype"]])
        g = _rows(W, V * D, gen, 1e-2)
        d["dtable"] = g[:, :V * D].unflatten(1, (V, D))
        d["scale"] = math.sqrt(D)
    elif op in ("norm", "norm_grad"):
        T, D, dt = case["T"], case["D"], DT[case["dtype"]]
        w = _rows(W, 2 * D, gen, 0.1)
        w[:, :2 * D] += 1.0
        d["w_post"], d["w_pre"] = w[:, :D], w[:, D:2 * D]
        d["scale"] = 0.5
        d["y"] = _normal((W, T, D), gen, 3.0, dt)
        d["gate"] = _normal((W, T, D), gen, 1.0, dt) if case["gate"] else None
        d["r"] = _normal((W, T, D), gen, 1.0, dt)            # norm_grad: the residual stream after the sum
        if op == "norm_grad":
            d["dn"] = _normal((W, T, D), gen, 1e-2, dt)
            d["dr_out"] = _normal((W, T, D), gen, 1e-2, dt)
            d["stats"] = torch.stack([d[k].float().square().mean(-1).add(EPS_NORM).rsqrt() for k in ("y", "r")])
            dw = torch.zeros((W, _ld(2 * D)), device=DEV)
            d["dw_post"], d["dw_pre"] = dw[:, :D], dw[:, D:2 * D]
    else:
        tensors, P = _tensors(case)
        d["x"] = _rows(W, P, gen, 0.05)
        d["g"] = _rows(W, P, gen, 1e-2, DT[case["g"]])
        d["xb"] = d["x"].to(torch.bfloat16) if case["shadow"] else None
        if case["bits"] == 32:
            d["m"] = _rows(W, P, gen, 3e-3)
            d["v"] = _rows(W, P, gen, 1e-2).square_()
        else:                                                # codes and scales as earlier steps leave them
            nb = sum(-(-n // BLOCK) for _, n, _ in tensors)
            d["m"] = torch.randint(-127, 128, d["x"].shape, device=DEV, generator=gen, dtype=torch.int8)
            d["v"] = torch.randint(1, 256, d["x"].shape, device=DEV, generator=gen, dtype=torch.uint8)
            d["m_scale"] = (torch.rand((W, nb), device=DEV, generator=gen) + 0.5) * (8e-3 / 127 ** 2)
            d["v_scale"] = (torch.rand((W, nb), device=DEV, generator=gen) + 0.5) * (3e-2 / 255 ** 2)
            d["m_values"], d["v_values"] = torch.zeros_like(d["x"]), torch.zeros_like(d["x"])
    return d


def prepare(case, seed):
    d = _inputs(case, seed)
    s = {"case": case, "in": d}
    if case["op"] == "adamw":
        tensors, P = _tensors(case)
        s["P"] = P
        s["decay"] = torch.cat([torch.full((n,), 1.0 - LR * wd, dtype=torch.float64) for _, n, wd in tensors]).float().to(DEV)
        if case["bits"] == 8:
            s["block"] = _blocks(tensors).to(DEV)
        if own:                                              # the handle a program keeps from step to step
            import paper_1905_10395_amd as L
            parts, b = [], 0
            for at, n, wd in tensors:
                cut = lambda k: None if d.get(k) is None else d[k][:, at:at + n]
                e = b + -(-n // BLOCK)
                sc = (lambda k: d[k][:, b:e]) if case["bits"] == 8 else (lambda k: None)
                parts.append(L.AdamWTensor(cut("x"), cut("g"), cut("m"), cut("v"), weight_decay=wd, x_bf16=cut("xb"), m_scale=sc("m_scale"),
                                           v_scale=sc("v_scale"), m_values=cut("m_values"), v_values=cut("v_values")))
                b = e
            s["opt"] = L.AdamW(parts, bits=case["bits"])
    return s


def _blocks(tensors):
    """Which block of the 8-bit moments each column belongs to: blocks start with their tensor."""
    out, b = [], 0
    for _, n, _ in tensors:
        out.append(b + torch.arange(n) // BLOCK)
        b += -(-n // BLOCK)
    return torch.cat(out)


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    import paper_1905_10395_amd as L
    case, d = s["case"], s["in"]
    op = case["op"]
    if op == "lookup":
        return {"out": L.embed_lookup(d["table"], d["tokens"], scale=d["scale"], dtype=DT[case["out"]])}
    if op == "lookup_grad":
        L.embed_grad(d["dout"], d["tokens"], d["dtable"], scale=d["scale"], accumulate=case["accumulate"])
        return {"dtable": d["dtable"]}
    if op == "norm":
        r, n, stats = L.block_norm(d["r"], d["y"], gate=d["gate"], w_post=d["w_post"], w_pre=d["w_pre"], scale=d["scale"], eps=EPS_NORM)
        return {"r": r, "n": n, "stats": stats}
    if op == "norm_grad":
        dr, dy, dgate = L.block_norm_grad(d["dn"], d["dr_out"], d["r"], d["stats"], d["y"], gate=d["gate"], w_post=d["w_post"],
                                          w_pre=d["w_pre"], scale=d["scale"], dw_post=d["dw_post"], dw_pre=d["dw_pre"])
        return {"dr": dr, "dy": dy, "dgate": dgate, "dw_post": d["dw_post"], "dw_pre": d["dw_pre"]}
    s["opt"].step(LR, STEP, beta1=BETA1, beta2=BETA2, eps=EPS)
    if case["bits"] == 8:
        s["opt"].moments()                                   # the values that the codes stand for
        return {"x": d["x"], "xb": d["xb"], "m": d["m_values"], "v": d["v_values"]}
    return {"x": d["x"], "xb": d["xb"], "m": d["m"], "v": d["v"]}


def _run_plain(s):
    case, d = s["case"], s["in"]
    op, W = case["op"], case["W"]
    if op == "lookup":
        tok = d["tokens"].long()
        rows = d["table"][torch.arange(W, device=DEV)[:, None], tok.clamp(min=0)].float() * d["scale"]
        return {"out": rows.masked_fill((tok < 0)[..., None], 0.0).to(DT[case["out"]])}
    if op == "lookup_grad":
        V, D = case["V"], case["D"]
        tok = d["tokens"].long()
        at = torch.where(tok < 0, W * V, tok + V * torch.arange(W, device=DEV)[:, None])     # padding: one row more
        g = torch.zeros((W * V + 1, D), device=DEV).index_add_(0, at.reshape(-1), d["dout"].float().reshape(-1, D) * d["scale"])
        g = g[:-1].view(W, V, D)
        d["dtable"].copy_(d["dtable"] + g if case["accumulate"] else g)
        return {"dtable": d["dtable"]}
    if op == "norm":
        y = d["y"].float()
        qy = torch.rsqrt((y * y).mean(-1) + EPS_NORM)
        b = y * qy[..., None] * d["w_post"][:, None]
        if d["gate"] is not None:
            b = b / (1.0 + torch.exp(-d["gate"].float()))
        r = d["r"].float() + d["scale"] * b
        qr = torch.rsqrt((r * r).mean(-1) + EPS_NORM)
        n = r * qr[..., None] * d["w_pre"][:, None]
        return {"r": r.to(d["r"].dtype), "n": n.to(d["r"].dtype), "stats": torch.stack([qy, qr])}
    if op == "norm_grad":
        dt = d["r"].dtype
        qy, qr = d["stats"][0][..., None], d["stats"][1][..., None]
        h, dn = d["r"].float() * qr, d["dn"].float()
        t = d["w_pre"][:, None] * dn
        dr = d["dr_out"].float() + qr * (t - h * (t * h).mean(-1, keepdim=True))
        z, e = d["y"].float() * qy, d["scale"] * dr
        dgate = None
        if d["gate"] is not None:
            a = 1.0 / (1.0 + torch.exp(-d["gate"].float()))
            dgate = (e * z * d["w_post"][:, None] * (a * (1.0 - a))).to(dt)
            e = e * a
        t = e * d["w_post"][:, None]
        dy = qy * (t - z * (t * z).mean(-1, keepdim=True))
        d["dw_pre"].copy_((dn * h).sum(1))
        d["dw_post"].copy_((e * z).sum(1))
        return {"dr": dr.to(dt), "dy": dy.to(dt), "dgate": dgate, "dw_post": d["dw_post"], "dw_pre": d["dw_pre"]}
    return _plain_adamw(s)


def _plain_adamw(s):
    case, d, P = s["case"], s["in"], s["P"]
    eight = case["bits"] == 8
    x, g = d["x"][:, :P], d["g"][:, :P].float()
    if eight:
        sm, sv = d["m_scale"][:, s["block"]], d["v_scale"][:, s["block"]]
        c = d["m"][:, :P].float()
        m = c * c.abs() * sm
        c = d["v"][:, :P].float()
        r = c * c * sv
        v = r * r
    else:
        m, v = d["m"][:, :P], d["v"][:, :P]
    m = BETA1 * m + (1.0 - BETA1) * g
    v = BETA2 * v + (1.0 - BETA2) * (g * g)
    r = torch.sqrt(v)
    den = r * (1.0 / math.sqrt(1.0 - BETA2 ** STEP)) + EPS
    x.copy_(x * s["decay"] - (m / den) * (LR / (1.0 - BETA1 ** STEP)))
    if d["xb"] is not None:
        d["xb"][:, :P].copy_(x)
    if not eight:
        d["m"][:, :P].copy_(m)
        d["v"][:, :P].copy_(v)
        return {"x": d["x"], "xb": d["xb"], "m": d["m"], "v": d["v"]}
    uv, um = (STEP * PHI) % 1.0, (STEP * PHI + 0.5) % 1.0
    W, nb = d["m_scale"].shape
    blk = s["block"].expand(W, P)
    y, sm, d["m_scale"] = _scaled(m.abs(), blk, nb, 127.0)
    c = _floor_root(y)
    c = c + (y - c * c > um * (2.0 * c + 1.0)).float()
    d["m"][:, :P].copy_(torch.where(m < 0, -c, c))
    d["m_values"][:, :P].copy_(torch.where(m < 0, -c, c) * c * sm)
    y, sv, d["v_scale"] = _scaled(r, blk, nb, 255.0)
    c = _floor_root(y)
    c2, d2 = c * c, (c + 1.0) * (c + 1.0)
    c = c + ((y - c2) * (y + c2) > uv * ((d2 - c2) * (d2 + c2))).float()
    c = torch.where((r > 0) & (sv > 0), c.clamp(min=1.0), c)
    d["v"][:, :P].copy_(c)
    r = c * c * sv
    d["v_values"][:, :P].copy_(r * r)
    return {"x": d["x"], "xb": d["xb"], "m": d["m_values"], "v": d["v_values"]}


def _scaled(a, blk, nb, top):
    """a over its block's scale (the block's largest value has the code `top`), the scale by column and by block."""
    big = torch.zeros((a.shape[0], nb), device=DEV, dtype=a.dtype).scatter_reduce_(1, blk, a, "amax")
    scale = big * (1.0 / (top * top))
    scale = torch.where(scale > 2.0 ** -100, scale, torch.zeros_like(scale))
    inv = torch.where(scale > 0, 1.0 / scale, torch.zeros_like(scale))
    return (a * inv.gather(1, blk)).clamp(max=top * top), scale.gather(1, blk), scale


def _floor_root(y):
    """The largest whole c with c * c <= y, whatever sqrt's last bit."""
    c = torch.floor(torch.sqrt(y))
    c = c - (c * c > y).float()
    return c + ((c + 1.0) * (c + 1.0) <= y).float()


# ------------------------------------------------------------------------------------------------
# what one pass cannot do without
# ------------------------------------------------------------------------------------------------
def _distinct(T, V):
    """Table rows that T drawn tokens touch, on average."""
    if T <= 0:
        return 0.0
    p = np.log1p(1.0 / (1.0 + np.arange(V, dtype=np.float64))) / math.log(V + 1.0)
    return float((1.0 - np.power(1.0 - p, 0.98 * T)).sum())


def work(case):
    W, op = case["W"], case["op"]
    if op == "lookup":
        T, V, D = case["T"], case["V"], case["D"]
        return {"bytes": W * (4.0 * T + D * (_distinct(T, V) * SIZE[case["table"]] + T * SIZE[case["out"]])), "flops": 1.0 * W * T * D}
    if op == "lookup_grad":
        T, V, D = case["T"], case["V"], case["D"]
        table = 8.0 * _distinct(T, V) if case["accumulate"] else 4.0 * V
        return {"bytes": W * (4.0 * T + D * (0.98 * T * SIZE[case["dtype"]] + table)), "flops": 1.0 * W * T * D}
    if op in ("norm", "norm_grad"):
        T, D, es = case["T"], case["D"], SIZE[case["dtype"]]
        streams = (4 if op == "norm" else 6) + (1 if op == "norm" else 2) * bool(case["gate"])
        return {"bytes": W * (1.0 * T * D * es * streams + 8.0 * T + 8.0 * D * (1 if op == "norm" else 2)),
                "flops": W * T * D * (14.0 if op == "norm" else 30.0)}
    tensors, P = _tensors(case)
    per = 8.0 + SIZE[case["g"]] + (2.0 if case["shadow"] else 0.0) + (16.0 if case["bits"] == 32 else 12.0)
    extra = 16.0 * sum(-(-n // BLOCK) for _, n, _ in tensors) if case["bits"] == 8 else 0.0
    return {"bytes": W * (P * per + extra), "flops": 20.0 * W * P}


# ------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ------------------------------------------------------------------------------------------------
def exact(case, seed):
    d = _inputs(case, seed)
    W, op = case["W"], case["op"]
    if op == "lookup":
        out = torch.zeros((W, case["T"], case["D"]), dtype=torch.float64, device=DEV)
        for w in range(W):
            used = (d["tokens"][w] >= 0).nonzero()[:, 0]
            out[w, used] = d["table"][w].double()[d["tokens"][w, used].long()] * d["scale"]
        return {"out": out}
    if op == "lookup_grad":
        out = torch.zeros((W, case["V"], case["D"]), dtype=torch.float64, device=DEV)
        for w in range(W):
            used = (d["tokens"][w] >= 0).nonzero()[:, 0]
            out[w].index_add_(0, d["tokens"][w, used].long(), d["dout"][w, used].double())
        out *= d["scale"]
        return {"dtable": out + d["dtable"].double() if case["accumulate"] else out}
    if op == "norm":
        out = {"r": [], "n": [], "stats": []}
        for w in range(W):
            y, r = d["y"][w].double(), d["r"][w].double()
            vy = y.pow(2).sum(1) / case["D"] + EPS_NORM
            b = d["scale"] * y * d["w_post"][w].double() / vy.sqrt()[:, None]
            r = r + (b if d["gate"] is None else b * torch.sigmoid(d["gate"][w].double()))
            vr = r.pow(2).sum(1) / case["D"] + EPS_NORM
            out["r"].append(r)
            out["n"].append(r / vr.sqrt()[:, None] * d["w_pre"][w].double())
            out["stats"].append(torch.stack([vy.pow(-0.5), vr.pow(-0.5)]))
        return {"r": torch.stack(out["r"]), "n": torch.stack(out["n"]), "stats": torch.stack(out["stats"], 1)}
    if op == "norm_grad":
        got = [_exact_norm_grad(case, d, w) for w in range(W)]
        return {k: None if got[0][k] is None else torch.stack([o[k] for o in got]) for k in got[0]}
    return _exact_adamw(case, d)


def _exact_norm_grad(case, d, w):
    """Row by row the Jacobians of x -> q x with q = (mean x^2 + eps)^-1/2 given: dq/dx = -q^3 x / D."""
    D = case["D"]
    dn, r, y = d["dn"][w].double(), d["r"][w].double(), d["y"][w].double()
    qy, qr = (d["stats"][k, w].double()[:, None] for k in (0, 1))
    wq, wr = d["w_post"][w].double(), d["w_pre"][w].double()
    a = torch.sigmoid(d["gate"][w].double()) if d["gate"] is not None else torch.ones_like(y)
    dr = d["dr_out"][w].double() + dn * wr * qr - r * qr.pow(3) / D * (dn * wr * r).sum(1, keepdim=True)
    db = d["scale"] * dr
    dz = db * a * wq
    return {"dr": dr, "dy": dz * qy - y * qy.pow(3) / D * (dz * y).sum(1, keepdim=True),
            "dgate": db * qy * y * wq * a * (1 - a) if d["gate"] is not None else None,
            "dw_post": (db * a * y * qy).sum(0), "dw_pre": (dn * r * qr).sum(0)}


def _exact_adamw(case, d):
    tensors, P = _tensors(case)
    x, ms, vs = d["x"].double(), [], []
    new_x = x.clone()
    b = 0
    for at, n, wd in tensors:
        cols, nb = slice(at, at + n), -(-n // BLOCK)
        g = d["g"][:, cols].double()
        if case["bits"] == 8:
            blk = b + torch.arange(n, device=DEV) // BLOCK
            c = d["m"][:, cols].double()
            m = c.sign() * c.pow(2) * d["m_scale"].double()[:, blk]
            v = (d["v"][:, cols].double().pow(2) * d["v_scale"].double()[:, blk]).pow(2)
        else:
            m, v = d["m"][:, cols].double(), d["v"][:, cols].double()
        m = m + (1 - BETA1) * (g - m)
        v = v + (1 - BETA2) * (g * g - v)
        step = (m / (1 - BETA1 ** STEP)) / ((v / (1 - BETA2 ** STEP)).sqrt() + EPS)
        new_x[:, cols] = x[:, cols] - LR * (step + wd * x[:, cols])
        if case["bits"] == 8:
            m, v = _exact_codes(m, v)
        ms.append(m)
        vs.append(v)
        b += nb
    pad = torch.zeros((case["W"], x.shape[1] - P), dtype=torch.float64, device=DEV)
    return {"x": new_x, "xb": new_x if case["shadow"] else None, "m": torch.cat(ms + [pad], 1), "v": torch.cat(vs + [pad], 1)}


def _exact_codes(m, v):
    """The values nearest below or above that 8 bits hold; which of the two is the step's threshold's to say."""
    W, n = m.shape
    fill = (-n) % BLOCK
    wide = lambda t: torch.cat([t, torch.zeros((W, fill), dtype=t.dtype, device=DEV)], 1).view(W, -1, BLOCK)
    m, r = wide(m), wide(v.sqrt())
    sm = m.abs().amax(2, keepdim=True) / 127.0 ** 2
    lo = (m.abs() / sm.clamp(min=1e-300)).sqrt().floor().clamp(max=127.0)
    up = m.abs() > (lo.pow(2) + ((STEP * PHI + 0.5) % 1.0) * ((lo + 1).pow(2) - lo.pow(2))) * sm
    m = m.sign() * (lo + up).clamp(max=127).pow(2) * sm
    sv = r.amax(2, keepdim=True) / 255.0 ** 2
    lo = (r / sv.clamp(min=1e-300)).sqrt().floor().clamp(max=255)
    up = r.pow(2) > (lo.pow(4) + ((STEP * PHI) % 1.0) * ((lo + 1).pow(4) - lo.pow(4))) * sv.pow(2)
    c = (lo + up).clamp(max=255)
    c = torch.where(r > 0, c.clamp(min=1), c)
    return m.reshape(W, -1)[:, :n], (c.pow(2) * sv).pow(2).reshape(W, -1)[:, :n]
