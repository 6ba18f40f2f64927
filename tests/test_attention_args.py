"""Arguments of the attention operators are checked before any device work: these calls need no GPU."""
import pytest
import torch

import paper_1905_10395_amd as L
from paper_1905_10395_amd import binding as b

OK, INVALID, SHAPE, STATE, UNSUPPORTED, HIP, NOMEM = range(7)
P = 4096                                              # never followed
NONE = (0, 0, 0, 0)


def error():
    return b.lib().lsgd_last_error().decode()


def heads(T, H, D, p=P):
    return (p, T * H * D, H * D, D)


def test_argument_structs_have_the_headers_layout():
    """Offsets as the C compiler lays them out: ints and floats, padding to 8, lsgd_heads of 32 bytes, then pointers and strides."""
    assert b._QK_ROTARY.size == 48 + 4 * 32 + 8 * 8
    assert b._QK_ROTARY_GRAD.size == 48 + 6 * 32 + 12 * 8
    assert b._ATTENTION.size == 40 + 4 * 32 + 3 * 8
    assert b._ATTENTION_GRAD.size == 40 + 8 * 32 + 3 * 8


def qk(W=2, T=3, Hq=4, Hk=2, D=8, R=8, bf16=0, norm=1, interleaved=0, eps=1e-6, magnitude=1.0, q=None, k=None, q_out=None, k_out=None, pos=P, ld_pos=3,
       turns=P, wq=P, wk=P, lq=8, lk=8, stats=P):
    at = lambda v, H: heads(T, H, D) if v is None else v
    return b._QK_ROTARY.pack(W, T, Hq, Hk, D, R, bf16, norm, interleaved, eps, magnitude, *at(q, Hq), *at(k, Hk), *at(q_out, Hq), *at(k_out, Hk), pos, ld_pos, turns,
                             wq, wk, lq, lk, stats)


def test_qk_rotary_arguments():
    f = b.lib().lsgd_qk_rotary
    for bad, status, word in (
            (dict(W=0), SHAPE, "W="), (dict(T=-1), SHAPE, "T="), (dict(T=2 ** 24 + 1), SHAPE, "T="), (dict(Hq=0), SHAPE, "Hq="), (dict(Hk=-1), SHAPE, "Hk="),
            (dict(Hq=1025), SHAPE, "1024"), (dict(D=0), SHAPE, "D="), (dict(D=257), UNSUPPORTED, "256"), (dict(R=7), SHAPE, "R="), (dict(R=10), SHAPE, "R="),
            (dict(bf16=2), INVALID, "is_bf16"), (dict(norm=-1), INVALID, "norm"), (dict(interleaved=3), INVALID, "interleaved"),
            (dict(eps=0.0), INVALID, "eps"), (dict(eps=float("nan")), INVALID, "eps"), (dict(magnitude=float("inf")), INVALID, "magnitude"),
            (dict(q=NONE), INVALID, "q is required"), (dict(k=NONE), INVALID, "k is required"), (dict(k_out=NONE), INVALID, "k_out is required"),
            (dict(Hk=0), INVALID, "k has no meaning"), (dict(turns=0), INVALID, "turns are required"), (dict(turns=P + 4), INVALID, "turns are not aligned"),
            (dict(pos=P + 2), INVALID, "positions"), (dict(ld_pos=2), SHAPE, "ld_positions"), (dict(wq=P + 1), INVALID, "w_q"), (dict(lk=-1), SHAPE, "w_k"),
            (dict(stats=P + 2), INVALID, "stats"), (dict(q=heads(3, 4, 8, P + 2)), INVALID, "q is not aligned"),
            (dict(q_out=(P, 96, 32, 7)), SHAPE, "q_out overlap"), (dict(q_out=(P, 95, 32, 8)), SHAPE, "q_out overlap"), (dict(k=(P, -48, 16, 8)), SHAPE, "negative"),
            (dict(k_out=(P, 0, 16, 8)), SHAPE, "k_out overlap")):
        assert f(qk(**bad), None) == status and word in error(), (bad, error())
    assert f(None, None) == INVALID
    assert f(qk(T=0), None) == OK
    assert f(qk(W=32768, T=2 ** 24, Hq=1, Hk=0, k=NONE, k_out=NONE, wk=0, D=1, R=0, turns=0, ld_pos=0, q=(P, 2 ** 24, 1, 1), q_out=(P, 2 ** 24, 1, 1)), None) == SHAPE
    assert "too large" in error()
    # without a norm eps has no meaning, without a rotation turns have none
    assert f(qk(T=0, norm=0, eps=0.0, R=0, turns=0), None) == OK


def test_qk_rotary_grad_arguments():
    f, size = b.lib().lsgd_qk_rotary_grad, b.lib().lsgd_qk_rotary_grad_workspace_bytes
    assert size(2, 300, 4, 2, 64, 64, 1) >= 2 * 2 * 64 * 4 and size(2, 0, 4, 2, 64, 64, 1) > 0
    for bad in ((0, 3, 4, 2, 8, 8, 0), (2, 3, 0, 2, 8, 8, 0), (2, 3, 4, 2, 300, 8, 0), (2, 3, 4, 2, 8, 9, 0)):
        assert size(*bad) == 0 and "qk_rotary_grad" in error()
    W, T, Hq, Hk, D = 2, 3, 4, 2, 8

    def call(norm=1, accumulate=0, dq_out=None, dk_out=None, q=None, k=None, dq=None, dk=None, stats=P, dwq=P, dwk=P, ldq=8, hk=Hk, ws=P, nbytes=1 << 20):
        at = lambda v, H: heads(T, H, D) if v is None else v
        a = b._QK_ROTARY_GRAD.pack(W, T, Hq, hk, D, 8, 0, norm, 0, accumulate, 1.0, *at(dq_out, Hq), *at(dk_out, hk), *at(q, Hq), *at(k, hk), *at(dq, Hq), *at(dk, hk),
                                   P, T, P, P, P, 8, 8, stats, dwq, dwk, ldq, 8)
        return f(a, ws, nbytes, None)
    for bad, status, word in (
            (dict(accumulate=2), INVALID, "accumulate"), (dict(dq_out=NONE), INVALID, "dq_out is required"), (dict(q=NONE), INVALID, "q is required"),
            (dict(norm=0, k=NONE), INVALID, "k is required"), (dict(stats=0), INVALID, "stats are required"), (dict(ldq=7), SHAPE, "dw_q"),
            (dict(ws=None), INVALID, "workspace"), (dict(ws=P + 8), INVALID, "256"), (dict(nbytes=100), NOMEM, "workspace"),
            (dict(dk=(P, 48, 16, 4)), SHAPE, "dk overlap"), (dict(hk=0), INVALID, "dw_k has no meaning")):
        assert call(**bad) == status and word in error(), (bad, error())
    assert f(None, None, 0, None) == INVALID


def attention(B=2, Tq=3, Tk=5, Hq=4, Hk=2, D=8, bf16=0, causal=0, scale=1.0, q=None, k=None, v=None, out=None, q_lens=0, k_lens=0, lse=P):
    at = lambda x, T, H: heads(T, H, D) if x is None else x
    return b._ATTENTION.pack(B, Tq, Tk, Hq, Hk, D, bf16, causal, scale, *at(q, Tq, Hq), *at(k, Tk, Hk), *at(v, Tk, Hk), *at(out, Tq, Hq), q_lens, k_lens, lse)


BAD = [(dict(B=0), SHAPE, "B="), (dict(B=2 ** 20 + 1), SHAPE, "B="), (dict(Tq=-1), SHAPE, "Tq="), (dict(Tk=2 ** 24 + 1), SHAPE, "Tk="), (dict(Hk=0), SHAPE, "Hk="),
       (dict(Hq=5), SHAPE, "multiple"), (dict(Hq=2048), SHAPE, "Hq="), (dict(D=0), SHAPE, "D="), (dict(D=129), UNSUPPORTED, "128"), (dict(bf16=2), INVALID, "is_bf16"),
       (dict(causal=-1), INVALID, "causal"), (dict(scale=0.0), INVALID, "scale"), (dict(scale=-1.0), INVALID, "scale"), (dict(scale=float("inf")), INVALID, "scale"), (dict(scale=float("nan")), INVALID, "scale"),
       (dict(scale=1e-39), INVALID, "scale"),
       (dict(q=NONE), INVALID, "q is required"), (dict(v=NONE), INVALID, "v is required"), (dict(k=heads(5, 2, 8, P + 2)), INVALID, "k is not aligned"),
       (dict(k=(P, 80, -16, 8)), SHAPE, "negative"), (dict(q_lens=P + 2), INVALID, "q_lens"), (dict(k_lens=P + 1), INVALID, "k_lens"),
       (dict(Hq=1024, Hk=1, Tq=2 ** 21), SHAPE, "too large"), (dict(B=2 ** 20, Tq=2 ** 20), SHAPE, "too large")]


def test_attention_arguments():
    f, size = b.lib().lsgd_attention, b.lib().lsgd_attention_workspace_bytes
    for bad, status, word in BAD + [(dict(out=NONE), INVALID, "out is required"), (dict(out=(P, 96, 32, 7)), SHAPE, "out overlap"), (dict(lse=P + 2), INVALID, "lse")]:
        assert f(attention(**bad), P, 1 << 40, None) == status and word in error(), (bad, error())
    assert f(None, None, 0, None) == INVALID
    assert f(attention(Tq=0), None, 0, None) == OK
    assert size(2, 3, 5, 4, 2, 8, 0) == 256 and size(0, 3, 5, 4, 2, 8, 0) == 0 and size(2, 3, 5, 3, 2, 8, 0) == 0
    # few queries, long keys: in parts, and those need their room
    need = size(1, 1, 100000, 4, 1, 64, 1)
    assert need > 256
    long = dict(B=1, Tq=1, Tk=100000, Hq=4, Hk=1, D=64, bf16=1)
    assert f(attention(**long), None, 0, None) == INVALID and "workspace" in error()
    assert f(attention(**long), P + 16, need, None) == INVALID and "256" in error()
    assert f(attention(**long), P, need - 1, None) == NOMEM


def test_no_queries_need_no_parts():
    size = b.lib().lsgd_attention_workspace_bytes
    for Tk in (0, 5, 1024, 1025, 100000):
        assert size(2, 0, Tk, 4, 2, 64, 1) == 256


def test_attention_grad_arguments():
    f, size = b.lib().lsgd_attention_grad, b.lib().lsgd_attention_grad_workspace_bytes

    def call(B=2, Tq=3, Tk=5, Hq=4, Hk=2, D=8, bf16=0, causal=0, scale=1.0, q_lens=0, k_lens=0, lse=P, ws=P, nbytes=1 << 50, **t):
        at = lambda n, T, H: t.get(n) or heads(T, H, D)
        a = b._ATTENTION_GRAD.pack(B, Tq, Tk, Hq, Hk, D, bf16, causal, scale, *at("dout", Tq, Hq), *at("q", Tq, Hq), *at("k", Tk, Hk), *at("v", Tk, Hk),
                                   *at("out", Tq, Hq), *at("dq", Tq, Hq), *at("dk", Tk, Hk), *at("dv", Tk, Hk), q_lens, k_lens, lse)
        return f(a, ws, nbytes, None)
    for bad, status, word in BAD + [(dict(dout=NONE), INVALID, "dout is required"), (dict(out=NONE), INVALID, "out is required"), (dict(dk=NONE), INVALID, "dk is required"),
                                    (dict(dv=(P, 80, 15, 8)), SHAPE, "dv overlap"), (dict(lse=0), INVALID, "lse is required"), (dict(ws=None), INVALID, "workspace"),
                                    (dict(ws=P + 128), INVALID, "256"), (dict(nbytes=64), NOMEM, "workspace")]:
        assert call(**bad) == status and word in error(), (bad, error())
    assert call(Tq=0, Tk=0) == OK
    assert size(2, 3, 5, 4, 2, 8, 0) >= 2 * 2 * 2 * 6 * 4 and size(2, 3, 5, 4, 2, 129, 0) == 0
    assert f(None, None, 0, None) == INVALID


def test_tensors_on_the_cpu_are_refused():
    q, k = torch.zeros((2, 3, 4, 8)), torch.zeros((2, 5, 2, 8))
    for call in (lambda: L.qk_rotary(q), lambda: L.qk_rotary_grad(q, norm=False), lambda: L.attention(q, k, k), lambda: L.attention_grad(q, q, k, k, q, q)):
        with pytest.raises(ValueError, match="not on a GPU"):
            call()


def test_the_binding_names_what_is_wrong(monkeypatch):
    monkeypatch.setattr(b, "_gpu", lambda who, first, tensors: -1)   # as if the first were on a GPU, as the others are
    f = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype)
    q, k = f(2, 3, 4, 8), f(2, 3, 2, 8)
    for call, word in (
            (lambda: L.qk_rotary(q.half()), "float32 or bfloat16"), (lambda: L.qk_rotary(q, k[:, :2]), "k must be"), (lambda: L.qk_rotary(q, k.bfloat16()), "k must be"),
            (lambda: L.qk_rotary(q, w_k=f(2, 8)), "need k"), (lambda: L.qk_rotary(q, turns=f(5, dtype=torch.float64)), "more turns"),
            (lambda: L.qk_rotary(q, turns=f(4)), "turns must be"), (lambda: L.qk_rotary(q, positions=f(2, 3)), "positions must be int32"),
            (lambda: L.qk_rotary(q, positions=f(2, 4, dtype=torch.int32)), "positions must be"), (lambda: L.qk_rotary(q, w_q=f(2, 7)), "w_q must be"),
            (lambda: L.qk_rotary(q, norm=False, stats=f(2, 3, 4)), "stats need"), (lambda: L.qk_rotary(q.transpose(2, 3)), "columns of q"),
            (lambda: L.qk_rotary_grad(q, None, q, k, f(2, 3, 4)), "need dk_out"), (lambda: L.qk_rotary_grad(q, q=q), "needs stats"),
            (lambda: L.qk_rotary_grad(q, q=q, stats=f(2, 3, 5)), "stats must be"),
            (lambda: L.attention(q[0], k, k), "q must be"), (lambda: L.attention(q, k[:1], k), "k must be"), (lambda: L.attention(q, k, k[:, :2]), "v must be"),
            (lambda: L.attention(q, k, k, k_lens=f(2)), "k_lens must be"), (lambda: L.attention(q, k, k, q_lens=f(3, dtype=torch.int32)), "q_lens must be"),
            (lambda: L.attention(q, k, k, lse=f(2, 3, 4, dtype=torch.float64)), "lse must be"), (lambda: L.attention(q, k, k, out=q[:, :2]), "out must be"),
            (lambda: L.attention_grad(q[:, :2], q, k, k, q, f(2, 4, 3)), "dout must be"), (lambda: L.attention_grad(q, q, k, k, q, f(2, 4, 2)), "lse must be"),
            (lambda: L.rotary_turns(7, device="cpu"), "even"), (lambda: L.rotary_turns(8, stretch=0.0, device="cpu"), "positive"),
            (lambda: L.rotary_turns(8, keep=(100, 2.0, 1.0), device="cpu"), "keep")):
        with pytest.raises(ValueError, match=word):
            call()
