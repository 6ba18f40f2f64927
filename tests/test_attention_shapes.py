"""The binding takes statistics of attention and of the rotation's norm in their own layout only: these calls need no GPU."""
import pytest
import torch

import paper_1905_10395_amd as L
from paper_1905_10395_amd import binding as b


@pytest.fixture
def as_if_on_a_gpu(monkeypatch):
    monkeypatch.setattr(b, "_gpu", lambda who, first, tensors: -1)
    monkeypatch.setattr(b, "_call", lambda *a: None)


def f(*shape):
    return torch.zeros(shape)


B, Tq, Tk, Hq, Hk, D = 2, 3, 5, 4, 2, 8


def test_lse_has_its_own_layout(as_if_on_a_gpu):
    q, k = f(B, Tq, Hq, D), f(B, Tk, Hk, D)
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    for lse in (f(B, Tq, Hq), f(B, Hq * Tq), f(B * Hq, Tq), f(B, Hq, Tq, 1), f(Hq, B, Tq)):
        with pytest.raises(ValueError, match=r"lse must be .*\[2, 4, 3\]"):
            L.attention_grad(q, q, k, k, q, lse, workspace=ws)
        with pytest.raises(ValueError, match=r"lse must be .*\[2, 4, 3\]"):
            L.attention(q, k, k, lse=lse)
    L.attention_grad(q, q, k, k, q, f(B, Hq, Tq), workspace=ws)
    assert L.attention(q, k, k, lse=f(B, Hq, Tq))[1].shape == (B, Hq, Tq)


def test_stats_have_their_own_layout(as_if_on_a_gpu):
    q, k = f(B, Tq, Hq, D), f(B, Tq, Hk, D)
    for stats in (f(B, Hq + Hk, Tq), f(B * Tq, Hq + Hk), f(B, Tq * (Hq + Hk)), f(Tq, B, Hq + Hk), f(1, B, Tq, Hq + Hk)):
        with pytest.raises(ValueError, match=r"stats must be .*\[2, 3, 6\]"):
            L.qk_rotary_grad(q, k, q, k, stats)
        with pytest.raises(ValueError, match=r"stats must be .*\[2, 3, 6\]"):
            L.qk_rotary(q, k, stats=stats)
    L.qk_rotary_grad(q, k, q, k, f(B, Tq, Hq + Hk))
    assert L.qk_rotary(q, k, stats=f(B, Tq, Hq + Hk))[2].shape == (B, Tq, Hq + Hk)


def test_heads_without_columns_are_refused(as_if_on_a_gpu):
    q, k = f(B, Tq, Hq, 0), f(B, Tk, Hk, 0)
    for call in (lambda: L.attention(q, k, k), lambda: L.attention_grad(q, q, k, k, q, f(B, Hq, Tq))):
        with pytest.raises(ValueError, match="columns"):
            call()
