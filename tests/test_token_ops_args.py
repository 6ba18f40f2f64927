"""Arguments of the token-model operators are checked before any device work: these calls need no GPU."""
import ctypes as C

import pytest
import torch

import paper_1905_10395_amd as L
from paper_1905_10395_amd import binding as b

OK, INVALID, SHAPE, STATE, UNSUPPORTED, HIP, NOMEM = range(7)


def error():
    return b.lib().lsgd_last_error().decode()


def test_embed_workspace():
    f = b.lib().lsgd_embed_grad_workspace_bytes
    assert f(4, 10, 100, 8) > 0 and f(4, 0, 100, 8) > 0
    # keys, places and their copies, and room for partial sums
    assert f(2, 100000, 70000, 64) >= 2 * 100000 * 4 * 4
    for bad in ((0, 10, 100, 8), (4, -1, 100, 8), (4, 10, 0, 8), (4, 10, 100, 0), (40000, 1, 1, 1)):
        assert f(*bad) == 0 and "SHAPE" not in error() and "embed_grad" in error()
    assert f(1, 2 ** 24 + 1, 10, 8) == 0 and "beyond" in error()
    assert f(1, 10, 2 ** 30, 8) == 0 and f(1, 10, 10, 2 ** 20 + 1) == 0 and "beyond" in error()


def test_embed_arguments():
    f = b.lib().lsgd_embed_lookup
    p = 4096                                          # never followed
    assert f(2, 3, 5, 4, None, 20, 0, p, 3, 1.0, p, 12, 0, None) == INVALID and "required" in error()
    assert f(2, 3, 5, 4, p, 20, 2, p, 3, 1.0, p, 12, 0, None) == INVALID
    assert f(2, 3, 5, 4, p, 20, 0, p, 3, float("inf"), p, 12, 0, None) == INVALID and "scale" in error()
    assert f(2, 3, 5, 4, p, 20, 0, p, 2, 1.0, p, 12, 0, None) == SHAPE and "ld_tokens" in error()
    assert f(2, 3, 5, 4, p, 20, 0, p, 3, 1.0, p, 11, 0, None) == SHAPE
    assert f(2, 3, 5, 4, p + 2, 20, 0, p, 3, 1.0, p, 12, 0, None) == INVALID and "aligned" in error()
    assert f(2, 0, 5, 4, None, 20, 0, None, 3, 1.0, None, 12, 0, None) == OK
    g = b.lib().lsgd_embed_grad
    assert g(2, 3, 5, 4, p, 12, 0, p, 3, 1.0, 0, None, 20, p, 1 << 20, None) == INVALID
    assert g(2, 3, 5, 4, p, 12, 0, p, 3, 1.0, 0, p, 19, p, 1 << 20, None) == SHAPE and "overlap" in error()
    assert g(2, 3, 5, 4, p, 12, 0, p, 3, 1.0, 2, p, 20, p, 1 << 20, None) == INVALID
    assert g(2, 9000, 5, 4, p, 36000, 0, p, 9000, 1.0, 0, p, 20, None, 0, None) == INVALID and "workspace" in error()
    assert g(2, 9000, 5, 4, p, 36000, 0, p, 9000, 1.0, 0, p, 20, p, 1000, None) == NOMEM
    assert g(2, 9000, 5, 4, p, 36000, 0, p, 9000, 1.0, 0, p, 20, p + 16, 1 << 30, None) == INVALID and "256" in error()


def norm_args(W=2, T=3, D=8, bf16=0, post=1, scale=1.0, eps=1e-6, r=None, y=None, gate=None, r_out=None, n=None):
    at = lambda v: (4096, T * D, D) if v is None else v
    return b._BLOCK_NORM.pack(W, T, D, bf16, post, scale, eps, *at(r), *at(y), *(gate or (0, 0, 0)), *at(r_out), *at(n), 0, 0, 0, 0, 0, 0)


def test_block_norm_arguments():
    f = b.lib().lsgd_block_norm
    none = (0, 0, 0)
    for bad, status, word in (
            (dict(W=0), SHAPE, "W="), (dict(D=0), SHAPE, "D="), (dict(D=16385), UNSUPPORTED, "16384"), (dict(bf16=2), INVALID, "is_bf16"),
            (dict(scale=float("nan")), INVALID, "scale"), (dict(eps=0.0), INVALID, "eps"), (dict(r=none), INVALID, "r is required"),
            (dict(r_out=none), INVALID, "r_out is required"), (dict(y=none), INVALID, "r_out has no meaning"),
            (dict(y=none, r_out=none, gate=(4096, 24, 8)), INVALID, "gate has no meaning"), (dict(y=none, r_out=none, n=none), INVALID, "n is required"),
            (dict(r_out=(4096, 24, 7)), SHAPE, "overlap"), (dict(n=(4096, 20, 8)), SHAPE, "overlap"), (dict(n=(4098, 24, 8)), INVALID, "aligned"),
            (dict(r=(4096, -24, 8)), SHAPE, "negative")):
        assert f(norm_args(**bad), None) == status and word in error(), (bad, error())
    assert f(None, None) == INVALID
    assert f(norm_args(T=0), None) == OK
    assert b.lib().lsgd_block_norm_grad_workspace_bytes(2, 100, 64) >= 2 * 2 * 64 * 4
    assert b.lib().lsgd_block_norm_grad_workspace_bytes(2, 100, 20000) == 0


def test_argument_structs_have_the_headers_layout():
    """Offsets as the C compiler lays lsgd_block_norm_args out: five ints, two floats, padding, five triples of 24 bytes."""
    assert b._BLOCK_NORM.size == 32 + 5 * 24 + 6 * 8
    assert b._BLOCK_NORM_GRAD.size == 32 + 8 * 24 + 10 * 8
    assert C.sizeof(b._AdamWTensor) == 9 * 8 + 8 * 8 + 2 * 8


def adamw_tensor(**kw):
    p = 4096
    d = dict(x=p, g=p, m=p, v=p, m_scale=None, v_scale=None, m_values=None, v_values=None, x_bf16=None, rows=2, n=300, ld_x=300, ld_g=300,
             ld_state=300, ld_scale=2, ld_values=300, ld_bf16=300, weight_decay=0.0, lr_mult=1.0)
    d.update(kw)
    return (b._AdamWTensor * 1)(b._AdamWTensor(*[d[k] for k, _ in b._AdamWTensor._fields_]))


def test_adamw_arguments():
    f = b.lib().lsgd_adamw_workspace_bytes
    assert f(adamw_tensor(), 1, 32, 0) > 0 and f(adamw_tensor(n=0), 1, 32, 0) > 0 and f(None, 0, 32, 0) > 0
    for bad, bits, word in ((dict(x=None), 32, "required"), (dict(ld_g=299), 32, "stride"), (dict(n=-1), 32, "negative"),
                            (dict(weight_decay=float("nan")), 32, "finite"), (dict(), 8, "m_scale"), (dict(m_scale=4096, v_scale=4096, ld_scale=1), 8, "blocks"),
                            (dict(m_scale=4096, v_scale=4096, m_values=4096), 8, "both"), (dict(x=4097), 32, "aligned"), (dict(), 16, "neither"),
                            (dict(n=2 ** 42, ld_x=2 ** 42, ld_g=2 ** 42, ld_state=2 ** 42), 32, "too large")):
        assert f(adamw_tensor(**bad), 1, bits, 0) == 0 and word in error(), (bad, error())
    h = C.c_void_p()
    assert b.lib().lsgd_adamw_create(adamw_tensor(), 1, 32, 0, None, 0, None, C.byref(h)) == INVALID and not h.value
    assert b.lib().lsgd_adamw_create(adamw_tensor(), 1, 32, 0, 4096, 16, None, C.byref(h)) == NOMEM
    assert b.lib().lsgd_adamw_step(None, 0.1, 0.9, 0.99, 1e-8, 1, 1.0) == INVALID
    assert b.lib().lsgd_adamw_moments(None) == INVALID


def test_tensors_on_the_cpu_are_refused():
    t = torch.zeros((2, 5, 8))
    tok = torch.zeros((2, 3), dtype=torch.int32)
    for call in (lambda: L.embed_lookup(t, tok), lambda: L.embed_grad(t[:, :3], tok, t), lambda: L.block_norm(t),
                 lambda: L.block_norm_grad(t, None, t, torch.zeros((2, 2, 5))), lambda: L.AdamW([L.AdamWTensor(t, t, t, t)])):
        with pytest.raises(ValueError, match="not on a GPU"):
            call()


def test_embed_launches_are_of_fewer_than_2_to_the_32_threads():
    f, g, p = b.lib().lsgd_embed_lookup, b.lib().lsgd_embed_grad, 4096          # never followed
    T = 1 << 24
    for D, table, out in ((1 << 12, 0, 0), (1 << 13, 1, 1), (1 << 13, 0, 1), (1 << 16, 1, 0)):
        assert f(1, T, 5, D, p, 5 * D, table, p, T, 1.0, p, T * D, out, None) == SHAPE and "too large" in error()
    for D, bf16 in ((1 << 14, 0), (1 << 15, 1)):                                # 2^20 spans of 64 teams of 64 lanes
        assert g(1, T, 5, D, p, T * D, bf16, p, T, 1.0, 0, p, 5 * D, p, 1 << 60, None) == SHAPE and "too large" in error()


def test_adamw_stream_needs_a_handle():
    assert b.lib().lsgd_adamw_set_stream(None, None) == INVALID and "NULL" in error()


def test_adamw_scales_without_a_copy():
    """Scales of any shape but [rows, blocks] have to lie in memory as one row: a copy's memory would be gone before the first step."""
    f = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype)
    x, sm = f(2, 5, 100), f(2, 2)                                     # 1000 elements: 4 blocks
    make = lambda a, v: L.AdamWTensor(x, x, f(2, 5, 100, dtype=torch.int8), f(2, 5, 100, dtype=torch.uint8), m_scale=a, v_scale=v)._c(0, 8, torch.float32)
    assert make(f(4), f(4)).ld_scale == 4
    c = make(sm[None], sm[None])
    assert c.m_scale == c.v_scale == sm.data_ptr()
    with pytest.raises(ValueError, match="m_scale must be contiguous"):
        make(sm.t()[None], sm[None])


def test_adamw_names_what_is_missing(monkeypatch):
    monkeypatch.setattr(b, "_gpu", lambda who, first, tensors: 0)     # as if the others were on a GPU
    t = torch.zeros((2, 8))
    for name in ("x", "g", "m", "v"):
        with pytest.raises(ValueError, match=f"tensor 0: {name} is missing"):
            L.AdamW([L.AdamWTensor(**{k: None if k == name else t for k in ("x", "g", "m", "v")})])
    with pytest.raises(ValueError, match="no tensors"):
        L.AdamW([])
