#!/usr/bin/env python3
"""A population of small token models trained on one GPU: embedding lookup, norms around a gated block, their gradients and
AdamW from this library, the block's matrix products from torch, leaders and communication pulls of Algorithm 1.

    python examples/token_population.py [--workers 8] [--steps 200] [--bits 8]

Each worker is a row of x[W, ld] with its own

    E [V, D]  embedding            v1 [D]  norm before the block       W1 [H, D], W2 [D, H], U [D, D]  block and its gate
    w [D]     norm after the block v2 [D]  norm before the output      O [V, D]  output

    r0 = sqrt(D) E[token];  n0 = norm(r0) v1;  y = relu(n0 W1') W2';  r1 = r0 + s sigmoid(n0 U') norm(y) w
    n1 = norm(r1) v2;  logits = n1 O';  loss: mean cross entropy of the next token

and learns a chain of tokens (next = 5 token + 3 mod V, replaced by a random one now and then).
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1905_10395_amd as L  # noqa: E402

SCALE = 0.5                                          # of the block's part of the residual sum


class Model:
    """Parameters, gradients, moments and the library's handles of W workers."""

    def __init__(self, W=8, V=96, D=64, H=128, groups=2, bits=8, seed=0, device="cuda:0"):
        self.W, self.V, self.D, self.H = W, V, D, H
        self.shapes = {"E": (V, D), "v1": (D,), "W1": (H, D), "W2": (D, H), "U": (D, D), "w": (D,), "v2": (D,), "O": (V, D)}
        P = sum(math.prod(s) for s in self.shapes.values())
        ld = (P + 63) // 64 * 64
        rows = lambda n=W, dtype=torch.float32: torch.zeros((n, ld), device=device, dtype=dtype)
        self.x, self.g = rows(), rows()
        self.m, self.v = rows(dtype=torch.int8 if bits == 8 else torch.float32), rows(dtype=torch.uint8 if bits == 8 else torch.float32)
        self.at, self.p, self.dp = {}, {}, {}
        gen = torch.Generator(device=device).manual_seed(seed)
        tensors, a = [], 0
        for name, shape in self.shapes.items():
            n = math.prod(shape)
            cols = slice(a, a + n)
            a += n
            self.at[name] = cols
            cut = lambda t: t[:, cols].unflatten(1, shape) if len(shape) > 1 else t[:, cols]
            self.p[name], self.dp[name] = cut(self.x), cut(self.g)
            vector = len(shape) == 1                     # norms start at one and do not decay
            if vector:
                self.p[name].fill_(1.0)
            else:
                self.x[:, cols].normal_(std=shape[1] ** -0.5 if name != "E" else 1.0 / math.sqrt(D), generator=gen)
            scales = torch.zeros((2, W, -(-n // L.ADAMW_BLOCK)), device=device) if bits == 8 else (None, None)
            tensors.append(L.AdamWTensor(self.x[:, cols], self.g[:, cols], self.m[:, cols], self.v[:, cols], weight_decay=0.0 if vector else 0.01,
                                         m_scale=scales[0], v_scale=scales[1]))
        self.opt = L.AdamW(tensors, bits=bits)
        # the handle that selects leaders and pulls towards them
        self.pop = L.Population(self.x, self.g, groups, z_snapshot=rows(groups + 1), P=P)

    def grad_loss(self, tokens, targets):
        """Fills g; losses [W].  tokens, targets: int32 [W, T]."""
        p, d, W, T = self.p, self.dp, self.W, tokens.shape[1]
        bmm = torch.bmm
        t = lambda a: a.transpose(1, 2).contiguous()
        r0 = L.embed_lookup(p["E"], tokens, scale=math.sqrt(self.D))
        _, n0, stats0 = L.block_norm(r0, w_pre=p["v1"])
        h = bmm(n0, t(p["W1"])).relu_()
        y, u = bmm(h, t(p["W2"])), bmm(n0, t(p["U"]))
        r1, n1, stats1 = L.block_norm(r0, y, gate=u, w_post=p["w"], w_pre=p["v2"], scale=SCALE)
        logits = bmm(n1, t(p["O"]))
        want = targets.long()[..., None]
        losses = (torch.logsumexp(logits, 2) - logits.gather(2, want)[..., 0]).mean(1)

        dl = torch.softmax(logits, 2)
        dl.scatter_add_(2, want, torch.full_like(want, -1, dtype=dl.dtype))
        dl /= T
        d["O"].copy_(bmm(t(dl), n1))
        dr, dy, du = L.block_norm_grad(bmm(dl, p["O"].contiguous()), None, r1, stats1, y, gate=u, w_post=p["w"], w_pre=p["v2"], scale=SCALE,
                                       dw_post=d["w"], dw_pre=d["v2"])
        dh = bmm(dy, p["W2"].contiguous()) * (h > 0)
        d["W2"].copy_(bmm(t(dy), h))
        d["W1"].copy_(bmm(t(dh), n0))
        d["U"].copy_(bmm(t(du), n0))
        dn0 = bmm(dh, p["W1"].contiguous()) + bmm(du, p["U"].contiguous())
        dr0, _, _ = L.block_norm_grad(dn0, dr, r0, stats0, w_pre=p["v1"], dw_pre=d["v1"], dr=dr)
        L.embed_grad(dr0, tokens, d["E"], scale=math.sqrt(self.D))
        return losses

    def step(self, k, tokens, targets, lr=3e-3, communicate=False, pull=(0.1, 0.05)):
        """Iteration k (from 1): a gradient step of every worker; at a communication leaders are chosen and followed."""
        losses = self.grad_loss(tokens, targets)
        self.opt.step(lr, k, beta2=0.99)
        if communicate:
            self.pop.select_leaders(losses)
            self.pop.leader_pull(*pull)
        return losses


def batch(W, T, V, gen, device="cuda:0"):
    """Chains of tokens: int32 [W, T] and what follows each."""
    tok = torch.empty((W, T + 1), dtype=torch.int64, device=device)
    tok[:, 0] = torch.randint(0, V, (W,), device=device, generator=gen)
    noise = torch.randint(0, V, (W, T), device=device, generator=gen)
    odd = torch.rand((W, T), device=device, generator=gen) < 0.05
    for i in range(T):
        tok[:, i + 1] = torch.where(odd[:, i], noise[:, i], (5 * tok[:, i] + 3) % V)
    return tok[:, :-1].to(torch.int32).contiguous(), tok[:, 1:].to(torch.int32).contiguous()


def train(steps=200, W=8, T=64, tau=10, bits=8, report=0, **kw):
    """Losses [steps, W]."""
    model = Model(W=W, bits=bits, **kw)
    gen = torch.Generator(device="cuda:0").manual_seed(1)
    out = []
    for k in range(1, steps + 1):
        tokens, targets = batch(W, T, model.V, gen)
        out.append(model.step(k, tokens, targets, communicate=k % tau == 0))
        if report and (k % report == 0 or k == 1):
            print(f"step {k:4d}  loss of the best worker {float(out[-1].min()):.3f}, of all {float(out[-1].mean()):.3f}", flush=True)
    return torch.stack(out)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--workers", type=int, default=8)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--bits", type=int, default=8, choices=(8, 32))
    a = ap.parse_args()
    train(a.steps, W=a.workers, bits=a.bits, report=20)
