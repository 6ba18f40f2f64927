"""The example that runs the token-model operators together: its gradient against differentiation by torch in 64 bits, and that it
learns with moments in 32 and in 8 bits."""
import math
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_gradient():
    import token_population as ex
    W, T = 3, 37
    model = ex.Model(W=W, V=41, D=24, H=40, groups=1)
    gen = torch.Generator(device="cuda:0").manual_seed(3)
    for k in ("v1", "w", "v2"):
        model.p[k].normal_(mean=1.0, std=0.2, generator=gen)
    tokens, targets = ex.batch(W, T, model.V, gen)
    losses = model.grad_loss(tokens, targets)

    p = {k: t.detach().cpu().double().requires_grad_() for k, t in model.p.items()}
    tok, want = tokens.cpu().long(), targets.cpu().long()
    norm = lambda a, s: a * (a.pow(2).mean(2, keepdim=True) + 1e-6).rsqrt() * s[:, None]
    r0 = math.sqrt(model.D) * p["E"][torch.arange(W)[:, None], tok]
    n0 = norm(r0, p["v1"])
    y = torch.relu(n0 @ p["W1"].transpose(1, 2)) @ p["W2"].transpose(1, 2)
    r1 = r0 + ex.SCALE * torch.sigmoid(n0 @ p["U"].transpose(1, 2)) * norm(y, p["w"])
    logits = norm(r1, p["v2"]) @ p["O"].transpose(1, 2)
    ref = -torch.log_softmax(logits, 2).gather(2, want[..., None])[..., 0].mean(1)
    ref.sum().backward()
    assert torch.allclose(losses.cpu().double(), ref, rtol=1e-5, atol=0)
    # fp32 through two norms and three products of at most 41 terms: some hundred roundings of the gradient's size
    for k in p:
        got, g = model.dp[k].cpu().double(), p[k].grad
        assert float((got - g).norm() / g.norm()) <= 100 * 2.0 ** -24 * 4, k


@pytest.mark.parametrize("bits", [32, 8])
def test_it_learns(bits):
    import token_population as ex
    losses = ex.train(steps=150, W=4, T=64, bits=bits, groups=2).cpu()
    assert bool(torch.isfinite(losses).all())
    # a fresh model guesses: log 96 = 4.6; the chain's own entropy is 0.05 (log 96 + ...) + ... = 0.4
    assert float(losses[0].mean()) > 4.0 and float(losses[-10:].mean()) < 1.5
