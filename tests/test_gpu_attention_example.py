"""The example that runs the attention operators together, forward, backward and token by token: its gradient against differentiation by torch
in 64 bits, its steps with a cache against the whole text at once, and that it runs."""
import math
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def rotated(x, pos, turns):
    a = 2 * math.pi * pos[:, None].double() * turns[None]
    c, s = torch.cos(a)[:, None], torch.sin(a)[:, None]
    n = turns.numel()
    u, v = x[..., :n], x[..., n:2 * n]
    return torch.cat([u * c - v * s, u * s + v * c], -1)


def logits_of(model, p, tokens, S):
    """The model's formulas in 64 bits, differentiated by torch."""
    W, n = tokens.shape
    Hq, Hk, K = model.Hq, model.Hk, model.K
    T = n // S
    norm = lambda a, w: a * (a.pow(2).mean(-1, keepdim=True) + 1e-6).rsqrt() * w
    r0 = math.sqrt(model.D) * p["E"][torch.arange(W)[:, None], tokens]
    qkv = (norm(r0, p["v1"][:, None]) @ p["A"].transpose(1, 2)).view(W, S, T, Hq + 2 * Hk, K)
    q, k, v = qkv[:, :, :, :Hq], qkv[:, :, :, Hq:Hq + Hk], qkv[:, :, :, Hq + Hk:]
    pos, turns = torch.arange(T), model.turns.cpu()
    q, k = rotated(norm(q, p["wq"][:, None, None, None]), pos, turns), rotated(norm(k, p["wk"][:, None, None, None]), pos, turns)
    k, v = (x.repeat_interleave(Hq // Hk, 3) for x in (k, v))
    q, k, v = (x.transpose(2, 3) for x in (q, k, v))
    s = (q @ k.transpose(3, 4)) * K ** -0.5
    s = s.masked_fill(torch.ones((T, T), dtype=torch.bool).triu(1), -math.inf)
    a = (torch.softmax(s, -1) @ v).transpose(2, 3).reshape(W, n, Hq * K)
    r1 = r0 + norm(a @ p["B"].transpose(1, 2), p["w"][:, None])
    return norm(r1, p["v2"][:, None]) @ p["O"].transpose(1, 2)


def fresh(ex, **kw):
    model = ex.Model(W=3, V=19, D=24, Hq=6, Hk=2, K=20, groups=1, **kw)
    gen = torch.Generator(device="cuda:0").manual_seed(3)
    for k in ("v1", "wq", "wk", "w", "v2"):
        model.p[k].normal_(mean=1.0, std=0.2, generator=gen)
    return model, gen


def test_gradient():
    import attention_population as ex
    model, gen = fresh(ex)
    S = 2
    tokens, targets = ex.batch(3, S, 9, model.V, gen)
    losses = model.grad_loss(tokens, targets, S)
    p = {k: t.detach().cpu().double().requires_grad_() for k, t in model.p.items()}
    logits = logits_of(model, p, tokens.cpu().long(), S)
    tg = targets.cpu().long()
    lost = -torch.log_softmax(logits, 2).gather(2, tg.clamp(min=0)[..., None])[..., 0] * (tg >= 0)
    ref = lost.sum(1) / (tg >= 0).sum(1)
    ref.sum().backward()
    assert torch.allclose(losses.cpu().double(), ref, rtol=1e-5, atol=0)
    # fp32 through three norms, a softmax and five products of at most 120 terms: some hundred roundings of the gradient's size
    for k in p:
        got, g = model.dp[k].cpu().double(), p[k].grad
        assert float((got - g).norm() / g.norm()) <= 200 * 2.0 ** -24 * 4, k


def test_one_token_at_a_time_is_the_whole_text():
    import attention_population as ex
    model, gen = fresh(ex)
    prompt = torch.randint(0, model.V, (3, 7), device="cuda:0", generator=gen).to(torch.int32)
    text, logits = model.generate(prompt, 6)
    assert text.shape == (3, 13) and torch.equal(text[:, :7], prompt)
    want = logits_of(model, {k: t.detach().cpu().double() for k, t in model.p.items()}, text.cpu().long()[:, :-1], 1)
    # logits of size 5 through some hundred roundings of fp32
    assert float((logits.cpu().double() - want).abs().max()) <= 5 * 200 * 2.0 ** -24 * 4
    assert torch.equal(text[:, 7:].cpu().long(), want[:, 6:].argmax(2))


def test_it_runs():
    import attention_population as ex
    model, losses = ex.train(steps=12, W=4, S=4, half=6, tau=5)
    assert losses.shape == (12, 4) and bool(torch.isfinite(losses).all()) and bool(torch.isfinite(model.x).all())
