#!/usr/bin/env python3
"""A population of small token models with attention, trained on one GPU and then asked to go on with a text: embedding lookup, norms, rotation of
queries and keys, attention, their gradients and AdamW from this library, the matrix products from torch, leaders and pulls of Algorithm 1.

    python examples/attention_population.py [--workers 8] [--steps 200]

Each worker is a row of x[W, ld] with its own

    E [V, D]  embedding            v1 [D]  norm before the block       A [(Hq + 2 Hk) K, D]  queries, keys, values
    wq, wk [K] norms of a head     B [D, Hq K]  after attention        w [D]  norm after the block
    v2 [D]    norm before the output                                   O [V, D]  output

    r0 = sqrt(D) E[token];  n0 = norm(r0) v1;  q, k, v = n0 A';  q, k = rotated norm(q) wq, norm(k) wk
    y = attention(q, k, v) B';  r1 = r0 + norm(y) w;  logits = norm(r1) v2 O'

and learns texts whose second half repeats the first; then it is given the first half and a token, and goes on one token at a time.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1905_10395_amd as L  # noqa: E402


class Model:
    """Parameters, gradients, moments and the library's handles of W workers."""

    def __init__(self, W=8, V=32, D=64, Hq=4, Hk=2, K=32, groups=2, seed=0, device="cuda:0"):
        self.W, self.V, self.D, self.Hq, self.Hk, self.K, self.device = W, V, D, Hq, Hk, K, device
        self.shapes = {"E": (V, D), "v1": (D,), "A": ((Hq + 2 * Hk) * K, D), "wq": (K,), "wk": (K,), "B": (D, Hq * K), "w": (D,), "v2": (D,), "O": (V, D)}
        P = sum(math.prod(s) for s in self.shapes.values())
        ld = (P + 63) // 64 * 64
        rows = lambda n=W: torch.zeros((n, ld), device=device)
        self.x, self.g, m, v = rows(), rows(), rows(), rows()
        self.p, self.dp = {}, {}
        gen = torch.Generator(device=device).manual_seed(seed)
        tensors, a = [], 0
        for name, shape in self.shapes.items():
            n = math.prod(shape)
            cols = slice(a, a + n)
            a += n
            cut = lambda t: t[:, cols].unflatten(1, shape) if len(shape) > 1 else t[:, cols]
            self.p[name], self.dp[name] = cut(self.x), cut(self.g)
            if len(shape) == 1:                      # norms start at one and do not decay
                self.p[name].fill_(1.0)
            else:
                self.x[:, cols].normal_(std=shape[1] ** -0.5, generator=gen)
            tensors.append(L.AdamWTensor(self.x[:, cols], self.g[:, cols], m[:, cols], v[:, cols], weight_decay=0.0 if len(shape) == 1 else 0.01))
        self.opt = L.AdamW(tensors)
        self.turns = L.rotary_turns(K, device=device)
        # the handle that selects leaders and pulls towards them
        self.pop = L.Population(self.x, self.g, groups, z_snapshot=rows(groups + 1), P=P)

    def _heads(self, n0):
        """Queries, keys and values [W, tokens, heads, K], parts of one projection."""
        qkv = torch.bmm(n0, self.p["A"].transpose(1, 2).contiguous()).unflatten(2, (-1, self.K))
        return qkv, qkv[:, :, :self.Hq], qkv[:, :, self.Hq:self.Hq + self.Hk], qkv[:, :, self.Hq + self.Hk:]

    def _of_texts(self, t, S):
        """[W, S T, heads, K] as [W S, T, heads, K]."""
        return t.unflatten(1, (S, -1)).flatten(0, 1)

    def _output(self, r0, a):
        """What follows attention: the block's output, the residual stream, its norm, and the logits."""
        y = torch.bmm(a, self.p["B"].transpose(1, 2).contiguous())
        r1, n1, stats1 = L.block_norm(r0, y, w_post=self.p["w"], w_pre=self.p["v2"])
        return y, r1, n1, stats1, torch.bmm(n1, self.p["O"].transpose(1, 2).contiguous())

    def grad_loss(self, tokens, targets, S):
        """Fills g; losses [W].  tokens, targets: int32 [W, S T], S texts a worker; a target of -1 does not count."""
        p, d, W, n = self.p, self.dp, self.W, tokens.shape[1]
        bmm = torch.bmm
        t = lambda a: a.transpose(1, 2).contiguous()
        pos = torch.arange(n // S, dtype=torch.int32, device=self.device).repeat(S)[None]
        r0 = L.embed_lookup(p["E"], tokens, scale=math.sqrt(self.D))
        _, n0, stats0 = L.block_norm(r0, w_pre=p["v1"])
        qkv, q, k, v = self._heads(n0)
        qr, kr, stats = L.qk_rotary(q, k, pos, self.turns, w_q=p["wq"], w_k=p["wk"])
        qt, kt, vt = (self._of_texts(x, S) for x in (qr, kr, v))
        at, lse = L.attention(qt, kt, vt, causal=True)
        a = at.flatten(2).view(W, n, -1)
        y, r1, n1, stats1, logits = self._output(r0, a)
        want = targets.long().clamp(min=0)[..., None]
        counts = (targets >= 0).float() / (targets >= 0).sum(1, keepdim=True)
        losses = ((torch.logsumexp(logits, 2) - logits.gather(2, want)[..., 0]) * counts).sum(1)

        dl = torch.softmax(logits, 2)
        dl.scatter_add_(2, want, torch.full_like(want, -1, dtype=dl.dtype))
        dl *= counts[..., None]
        d["O"].copy_(bmm(t(dl), n1))
        dr, dy, _ = L.block_norm_grad(bmm(dl, p["O"].contiguous()), None, r1, stats1, y, w_post=p["w"], w_pre=p["v2"], dw_post=d["w"], dw_pre=d["v2"])
        d["B"].copy_(bmm(t(dy), a))
        da = self._of_texts(bmm(dy, p["B"].contiguous()).unflatten(2, (-1, self.K)), S)
        dqkv = torch.empty_like(qkv)
        dq, dk, dv = dqkv[:, :, :self.Hq], dqkv[:, :, self.Hq:self.Hq + self.Hk], dqkv[:, :, self.Hq + self.Hk:]
        L.attention_grad(da, qt, kt, vt, at, lse, causal=True, dq=self._of_texts(dq, S), dk=self._of_texts(dk, S), dv=self._of_texts(dv, S))
        L.qk_rotary_grad(dq, dk, q, k, stats, pos, self.turns, w_q=p["wq"], w_k=p["wk"], dw_q=d["wq"], dw_k=d["wk"], dq=dq, dk=dk)
        dqkv = dqkv.flatten(2)
        d["A"].copy_(bmm(t(dqkv), n0))
        dr0, _, _ = L.block_norm_grad(bmm(dqkv, p["A"].contiguous()), dr, r0, stats0, w_pre=p["v1"], dw_pre=d["v1"], dr=dr)
        L.embed_grad(dr0, tokens, d["E"], scale=math.sqrt(self.D))
        return losses

    def step(self, i, tokens, targets, S, lr=3e-3, communicate=False, pull=(0.1, 0.05)):
        """Iteration i (from 1): a gradient step of every worker; at a communication leaders are chosen and followed."""
        losses = self.grad_loss(tokens, targets, S)
        self.opt.step(lr, i, beta2=0.99)
        if communicate:
            self.pop.select_leaders(losses)
            self.pop.leader_pull(*pull)
        return losses

    def generate(self, prompt, steps):
        """Goes on with one text a worker, the likeliest token at a time.  prompt: int32 [W, T]; returns tokens [W, T + steps] and the logits
        [W, T + steps - 1, V] that each position gave."""
        W, T = prompt.shape
        cache_k, cache_v = (torch.zeros((W, T + steps, self.Hk, self.K), device=self.device) for _ in range(2))
        tokens, out, at = prompt, [], 0
        while True:
            new = tokens[:, at:]                     # the prompt, then one token at a time
            end = tokens.shape[1]
            pos = torch.arange(at, end, dtype=torch.int32, device=self.device)[None]
            r0 = L.embed_lookup(self.p["E"], new.contiguous(), scale=math.sqrt(self.D))
            _, n0, _ = L.block_norm(r0, w_pre=self.p["v1"])
            _, q, k, v = self._heads(n0)
            q, _, _ = L.qk_rotary(q, k, pos, self.turns, w_q=self.p["wq"], w_k=self.p["wk"], k_out=cache_k[:, at:end])
            cache_v[:, at:end] = v
            a, _ = L.attention(q, cache_k[:, :end], cache_v[:, :end], causal=True, with_lse=False)
            logits = self._output(r0, a.flatten(2))[4]
            out.append(logits)
            if end == T + steps:
                return tokens, torch.cat(out, 1)[:, :-1]
            tokens = torch.cat([tokens, logits[:, -1].argmax(1, keepdim=True).to(torch.int32)], 1)
            at = end


def batch(W, S, half, V, gen, device="cuda:0"):
    """Texts whose second half repeats the first: tokens [W, S (2 half - 1)] and what follows each, -1 where it cannot be known."""
    first = torch.randint(0, V, (W, S, half), device=device, generator=gen)
    text = torch.cat([first, first], 2)
    follows = text[:, :, 1:].clone()
    follows[:, :, :half - 1] = -1
    return text[:, :, :-1].flatten(1).to(torch.int32).contiguous(), follows.flatten(1).to(torch.int32).contiguous()


def train(steps=200, W=8, S=16, half=12, tau=10, report=0, **kw):
    """The model and losses [steps, W]."""
    model = Model(W=W, **kw)
    gen = torch.Generator(device="cuda:0").manual_seed(1)
    out = []
    for i in range(1, steps + 1):
        tokens, targets = batch(W, S, half, model.V, gen)
        out.append(model.step(i, tokens, targets, S, communicate=i % tau == 0))
        if report and (i % report == 0 or i == 1):
            print(f"step {i:4d}  loss of the best worker {float(out[-1].min()):.3f}, of all {float(out[-1].mean()):.3f}", flush=True)
    return model, torch.stack(out)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--workers", type=int, default=8)
    ap.add_argument("--steps", type=int, default=200)
    a = ap.parse_args()
    model, losses = train(a.steps, W=a.workers, report=20)
    best = int(losses[-1].argmin())
    tokens, _ = batch(a.workers, 1, 12, model.V, torch.Generator(device="cuda:0").manual_seed(7))
    text, _ = model.generate(tokens[:, :13].contiguous(), 10)
    print("worker", best, "was given", text[best, :13].tolist(), "and went on with", text[best, 13:].tolist())
