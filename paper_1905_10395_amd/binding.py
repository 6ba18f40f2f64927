"""ctypes marshalling for include/lsgd.h.  Same names as the C entry points:
lsgd_create_population, lsgd_grad_loss, lsgd_select_leaders, lsgd_pull_update,
lsgd_step (+ helpers).  No arithmetic of the method happens in Python."""
from __future__ import annotations

import ctypes as C
import math
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))

NESTEROV = 1
LEADER_EXEMPT = 2
PULL_UNSCALED_BY_ETA = 4
MOMENTUM_GRAD_ONLY = 8
WRITE_BF16_SHADOW = 16
FUSED_MLP_UPDATE = 32
COMM_LOCAL = 1
COMM_GLOBAL = 2

BATCH_EXTERNAL, BATCH_MC, BATCH_MLP = 0, 1, 2

_STATUS = {0: "OK", 1: "INVALID_ARG", 2: "SHAPE", 3: "STATE", 4: "UNSUPPORTED", 5: "HIP", 6: "NOMEM"}


class LsgdError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"LSGD_ERR_{_STATUS.get(status, status)}: {msg}")
        self.status = status


class _Config(C.Structure):
    _fields_ = [("W", C.c_int32), ("P", C.c_int64), ("ld", C.c_int64), ("n_groups", C.c_int32),
                ("group_offsets", C.POINTER(C.c_int32)), ("momentum", C.c_float), ("flags", C.c_int32),
                ("weight_decay", C.c_float)]


class _External(C.Structure):
    _fields_ = [("losses", C.c_void_p)]


class _MC(C.Structure):
    _fields_ = [("m", C.c_int32), ("n", C.c_int32), ("r", C.c_int32), ("rows", C.c_void_p), ("cols", C.c_void_p),
                ("vals", C.c_void_p), ("n_obs", C.c_int64), ("batch_idx", C.c_void_p), ("B", C.c_int64),
                ("c", C.c_float), ("entries", C.c_void_p)]


class _MLP(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("dims", C.POINTER(C.c_int32)), ("X", C.c_void_p), ("y", C.c_void_p),
                ("B", C.c_int32), ("x_is_fp32", C.c_int32)]


class _Batch(C.Structure):
    _fields_ = [("kind", C.c_int32), ("desc", C.c_void_p)]


# lsgd_block_norm_args, lsgd_block_norm_grad_args (native layout): sizes and flags, factors, lsgd_rows triples, pointers and strides
_BLOCK_NORM = struct.Struct("@5i2f" + "P2q" * 5 + "2P2q2P")
_BLOCK_NORM_GRAD = struct.Struct("@6if" + "P2q" * 8 + "2P2q2P2P2q")

# lsgd_qk_rotary_args, lsgd_qk_rotary_grad_args, lsgd_attention_args, lsgd_attention_grad_args; lsgd_heads are a pointer and three strides
_QK_ROTARY = struct.Struct("@9i2f" + "P3q" * 4 + "PqP2P2qP")
_QK_ROTARY_GRAD = struct.Struct("@10if" + "P3q" * 6 + "PqP2P2qP2P2q")
_ATTENTION = struct.Struct("@8if" + "P3q" * 4 + "3P")
_ATTENTION_GRAD = struct.Struct("@8if" + "P3q" * 8 + "3P")


class _AdamWTensor(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in ("x", "g", "m", "v", "m_scale", "v_scale", "m_values", "v_values", "x_bf16")] + \
               [(k, C.c_int64) for k in ("rows", "n", "ld_x", "ld_g", "ld_state", "ld_scale", "ld_values", "ld_bf16")] + \
               [("weight_decay", C.c_double), ("lr_mult", C.c_double)]


def lib_path() -> str:
    return os.path.join(_HERE, "liblsgd.so")


_lib = None


def lib():
    """Loads liblsgd.so; raises if it has not been built (there is no fallback)."""
    global _lib
    if _lib is None:
        path = lib_path()
        if not os.path.exists(path):
            raise ImportError(f"{path} is missing: run `python -m paper_1905_10395_amd.build` "
                              "(or __graft_entry__.build()) first")
        L = C.CDLL(path)
        L.lsgd_last_error.restype = C.c_char_p
        L.lsgd_workspace_bytes.restype = C.c_size_t
        L.lsgd_workspace_bytes.argtypes = [C.POINTER(_Config), C.POINTER(_Batch)]
        L.lsgd_create_population.argtypes = [C.POINTER(_Config), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                             C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.POINTER(C.c_void_p)]
        L.lsgd_destroy_population.argtypes = [C.c_void_p]
        L.lsgd_grad_loss.argtypes = [C.c_void_p, C.POINTER(_Batch), C.c_void_p]
        L.lsgd_select_leaders.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_uint8), C.c_int]
        L.lsgd_pull_update.argtypes = [C.c_void_p, C.c_float, C.c_float, C.c_float]
        L.lsgd_step.argtypes = [C.c_void_p, C.POINTER(_Batch), C.c_float, C.c_float, C.c_float,
                                C.POINTER(C.c_uint8), C.c_int]
        L.lsgd_leader_pull.argtypes = [C.c_void_p, C.c_float, C.c_float]
        L.lsgd_step_alg1.argtypes = [C.c_void_p, C.POINTER(_Batch), C.c_float, C.c_float, C.c_float, C.c_float, C.c_float,
                                     C.c_int, C.POINTER(C.c_uint8)]
        L.lsgd_smooth_losses.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int64, C.c_void_p, C.c_void_p]
        L.lsgd_center.argtypes = [C.c_void_p, C.c_void_p]
        L.lsgd_easgd_update.argtypes = [C.c_void_p, C.c_void_p, C.c_float, C.c_float]
        L.lsgd_easgd_step.argtypes = [C.c_void_p, C.POINTER(_Batch), C.c_void_p, C.c_float, C.c_float]
        L.lsgd_sync_shadow.argtypes = [C.c_void_p]
        L.lsgd_mc_pack_entries.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
        L.lsgd_select_pull_static.argtypes = [C.c_int32, C.c_int64, C.c_int64, C.c_int32, C.POINTER(C.c_int32), C.c_void_p,
                                              C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_float, C.c_float,
                                              C.c_float, C.c_float, C.c_float, C.c_int32, C.c_void_p]
        L.lsgd_stream_probe.argtypes = [C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]
        L.lsgd_get_leaders.argtypes = [C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
        L.lsgd_get_losses.argtypes = [C.c_void_p, C.POINTER(C.c_float)]
        L.lsgd_set_leaders.argtypes = [C.c_void_p, C.POINTER(C.c_int32), C.c_int32]
        L.lsgd_embed_lookup.argtypes = [C.c_int32] * 4 + [C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.c_int64, C.c_float, C.c_void_p,
                                                          C.c_int64, C.c_int32, C.c_void_p]
        L.lsgd_embed_grad_workspace_bytes.restype = C.c_size_t
        L.lsgd_embed_grad_workspace_bytes.argtypes = [C.c_int32] * 4
        L.lsgd_embed_grad.argtypes = [C.c_int32] * 4 + [C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.c_int64, C.c_float, C.c_int32,
                                                        C.c_void_p, C.c_int64, C.c_void_p, C.c_size_t, C.c_void_p]
        L.lsgd_block_norm.argtypes = [C.c_char_p, C.c_void_p]
        L.lsgd_block_norm_grad_workspace_bytes.restype = C.c_size_t
        L.lsgd_block_norm_grad_workspace_bytes.argtypes = [C.c_int32] * 3
        L.lsgd_block_norm_grad.argtypes = [C.c_char_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.lsgd_qk_rotary.argtypes = [C.c_char_p, C.c_void_p]
        L.lsgd_qk_rotary_grad_workspace_bytes.restype = C.c_size_t
        L.lsgd_qk_rotary_grad_workspace_bytes.argtypes = [C.c_int32] * 7
        L.lsgd_qk_rotary_grad.argtypes = [C.c_char_p, C.c_void_p, C.c_size_t, C.c_void_p]
        for f in ("attention", "attention_grad"):
            size, call = getattr(L, f"lsgd_{f}_workspace_bytes"), getattr(L, f"lsgd_{f}")
            size.restype, size.argtypes = C.c_size_t, [C.c_int32] * 7
            call.argtypes = [C.c_char_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.lsgd_adamw_workspace_bytes.restype = C.c_size_t
        L.lsgd_adamw_workspace_bytes.argtypes = [C.POINTER(_AdamWTensor), C.c_int32, C.c_int32, C.c_int32]
        L.lsgd_adamw_create.argtypes = [C.POINTER(_AdamWTensor), C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p,
                                        C.POINTER(C.c_void_p)]
        L.lsgd_adamw_destroy.argtypes = [C.c_void_p]
        L.lsgd_adamw_set_stream.argtypes = [C.c_void_p, C.c_void_p]
        L.lsgd_adamw_step.argtypes = [C.c_void_p, C.c_double, C.c_double, C.c_double, C.c_double, C.c_int64, C.c_double]
        L.lsgd_adamw_moments.argtypes = [C.c_void_p]
        _lib = L
    return _lib


def _check(status):
    if status != 0:
        raise LsgdError(status, lib().lsgd_last_error().decode())


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


class ExternalBatch:
    """Gradient already in g; losses: device float32 [W]."""

    def __init__(self, losses):
        self.losses = losses
        self._d = _External(losses.data_ptr())
        self.c = _Batch(BATCH_EXTERNAL, C.cast(C.pointer(self._d), C.c_void_p))


class MCBatch:
    """rows, cols: int32 [n_obs]; vals: float32 [n_obs]; batch_idx: int32 [W,B] or None (all entries);
    entries: optional int32 [n_obs, 4] from mc_pack_entries (read instead of rows/cols/vals)."""

    def __init__(self, m, n, r, rows, cols, vals, batch_idx, c, entries=None):
        B = 0 if batch_idx is None else int(batch_idx.shape[-1])
        idx_ptr = None
        if batch_idx is not None:
            # an empty tensor has a NULL data pointer, which the C side reads as "all entries"
            anchor = batch_idx if batch_idx.numel() else torch.zeros(1, dtype=torch.int32, device=rows.device)
            idx_ptr = anchor.data_ptr()
            batch_idx = anchor
        self.keep = (rows, cols, vals, batch_idx, entries)
        self._d = _MC(m, n, r, rows.data_ptr(), cols.data_ptr(), vals.data_ptr(), int(rows.numel()),
                      idx_ptr, B, float(c), None if entries is None else entries.data_ptr())
        self.c = _Batch(BATCH_MC, C.cast(C.pointer(self._d), C.c_void_p))


class MLPBatch:
    """dims: [d0..dL]; X: bfloat16 (or int16/uint16 bit patterns) or float32 [W,B,d0]; y: int32 [W,B]."""

    def __init__(self, dims, X, y):
        self.keep = (X, y)
        self._dims = (C.c_int32 * len(dims))(*[int(d) for d in dims])
        self._d = _MLP(len(dims) - 1, self._dims, X.data_ptr(), y.data_ptr(), int(y.shape[-1]),
                       1 if X.dtype == torch.float32 else 0)
        self.c = _Batch(BATCH_MLP, C.cast(C.pointer(self._d), C.c_void_p))


def mc_pack_entries(rows, cols, vals, stream=None):
    """lsgd_mc_pack_entries: returns an int32 [n_obs, 4] tensor of 16-byte records {row, col, val bits, 0}."""
    n = int(rows.numel())
    out = torch.empty((n, 4), dtype=torch.int32, device=rows.device)
    st = torch.cuda.current_stream(rows.device) if stream is None else stream
    _check(lib().lsgd_mc_pack_entries(_ptr(rows), _ptr(cols), _ptr(vals), n, _ptr(out), C.c_void_p(st.cuda_stream)))
    return out


def _config(W, P, ld, n_groups, group_offsets, momentum, flags, weight_decay):
    off = None
    if group_offsets is not None:
        off = (C.c_int32 * len(group_offsets))(*[int(v) for v in group_offsets])
    cfg = _Config(W, P, ld, n_groups, off, momentum, flags, weight_decay)
    return cfg, off


def workspace_bytes(W, P, ld, n_groups, group_offsets=None, momentum=0.0, flags=0, weight_decay=0.0, batch=None):
    cfg, _keep = _config(W, P, ld, n_groups, group_offsets, momentum, flags, weight_decay)
    n = lib().lsgd_workspace_bytes(C.byref(cfg), None if batch is None else C.byref(batch.c))
    if n == 0:
        raise LsgdError(-1, lib().lsgd_last_error().decode())
    return n


PROBE_READ, PROBE_COPY, PROBE_UPDATE = 0, 1, 2


def stream_probe(kind, a, b, c=None, stream=None):
    """lsgd_stream_probe over the whole of the (contiguous, equally sized) float32 tensors a, b, c."""
    assert a.is_contiguous() and b.is_contiguous() and a.numel() == b.numel() and (c is None or c.numel() == a.numel())
    st = torch.cuda.current_stream(a.device) if stream is None else stream
    _check(lib().lsgd_stream_probe(int(kind), _ptr(a), _ptr(b), _ptr(c), a.numel(), C.c_void_p(st.cuda_stream)))


STATIC_MAX_WORKERS, STATIC_MAX_GROUPS = 1024, 64


def select_pull_static(x, g, losses, n_groups, eta, lambda_L, lambda_G, m=None, P=None, group_offsets=None, momentum=0.0,
                       weight_decay=0.0, flags=0, leaders=None, stream=None):
    """lsgd_select_pull_static: selection over all groups + pull update with no handle, workspace or allocation.
    x, g, m: float32 [W, ld]; losses: float32 [W]; leaders: optional int32 [n_groups+1] output."""
    W, ld = x.shape
    off = None if group_offsets is None else (C.c_int32 * len(group_offsets))(*[int(v) for v in group_offsets])
    st = torch.cuda.current_stream(x.device) if stream is None else stream
    _check(lib().lsgd_select_pull_static(W, ld if P is None else int(P), ld, int(n_groups), off, _ptr(x), _ptr(g), _ptr(m),
                                         _ptr(losses), _ptr(leaders), eta, lambda_L, lambda_G, momentum, weight_decay,
                                         int(flags), C.c_void_p(st.cuda_stream)))


class Population:
    """Handle over caller-owned torch CUDA tensors (lsgd_create_population).

    x, g: float32 [W, ld]; m: float32 [W, ld] or None; z_snapshot: float32 [G+1, ld] or None;
    x_bf16: bfloat16 [W, ld] or None.  P defaults to ld.
    """

    def __init__(self, x, g, n_groups, m=None, z_snapshot=None, x_bf16=None, P=None, group_offsets=None,
                 momentum=0.0, flags=0, weight_decay=0.0, largest_batch=None, stream=None, workspace=None):
        assert x.is_cuda and x.dtype == torch.float32 and x.dim() == 2 and x.is_contiguous()
        W, ld = x.shape
        self.W, self.ld, self.P, self.G = W, ld, (ld if P is None else int(P)), int(n_groups)
        self.x, self.g, self.m, self.Z, self.xb = x, g, m, z_snapshot, x_bf16
        cfg, self._off = _config(W, self.P, ld, n_groups, group_offsets, momentum, flags, weight_decay)
        if workspace is None:
            nbytes = lib().lsgd_workspace_bytes(C.byref(cfg), None if largest_batch is None else C.byref(largest_batch.c))
            if nbytes == 0:
                raise LsgdError(-1, lib().lsgd_last_error().decode())
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=x.device)
        self.workspace = workspace
        self.stream = torch.cuda.current_stream(x.device) if stream is None else stream
        h = C.c_void_p()
        _check(lib().lsgd_create_population(C.byref(cfg), _ptr(x), _ptr(g), _ptr(m), _ptr(z_snapshot), _ptr(x_bf16),
                                            _ptr(workspace), workspace.numel(), C.c_void_p(self.stream.cuda_stream),
                                            C.byref(h)))
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            lib().lsgd_destroy_population(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @staticmethod
    def _mask(refresh_local):
        if refresh_local is None:
            return None
        return (C.c_uint8 * len(refresh_local))(*[int(v) for v in refresh_local])

    def grad_loss(self, batch, losses=None):
        _check(lib().lsgd_grad_loss(self._h, C.byref(batch.c), _ptr(losses)))

    def loss(self, batch, losses=None):
        _check(lib().lsgd_loss(self._h, C.byref(batch.c), _ptr(losses)))

    def select_leaders(self, losses=None, refresh_local=None, refresh_global=1):
        _check(lib().lsgd_select_leaders(self._h, _ptr(losses), self._mask(refresh_local), int(refresh_global)))

    def pull_update(self, eta, lambda_L, lambda_G):
        _check(lib().lsgd_pull_update(self._h, eta, lambda_L, lambda_G))

    def step(self, batch, eta, lambda_L, lambda_G, refresh_local=None, refresh_global=1):
        _check(lib().lsgd_step(self._h, C.byref(batch.c), eta, lambda_L, lambda_G, self._mask(refresh_local),
                               int(refresh_global)))

    def leader_pull(self, lambda_L, lambda_G):
        _check(lib().lsgd_leader_pull(self._h, lambda_L, lambda_G))

    def step_alg1(self, batch, eta, gamma_L, gamma_G, lambda_L, lambda_G, comm=0, comm_local_mask=None):
        _check(lib().lsgd_step_alg1(self._h, C.byref(batch.c), eta, gamma_L, gamma_G, lambda_L, lambda_G, int(comm),
                                    self._mask(comm_local_mask)))

    def smooth_losses(self, window, t, losses=None, out=None):
        """window: device float32 [K, W] ring."""
        assert window.dtype == torch.float32 and window.is_contiguous() and window.shape[1] == self.W
        _check(lib().lsgd_smooth_losses(self._h, _ptr(window), int(window.shape[0]), int(t), _ptr(losses), _ptr(out)))

    def center(self, out):
        assert out.dtype == torch.float32 and out.is_contiguous() and out.numel() >= self.P
        _check(lib().lsgd_center(self._h, _ptr(out)))

    def easgd_update(self, center, eta, lam):
        assert center.dtype == torch.float32 and center.is_contiguous() and center.numel() >= self.ld
        _check(lib().lsgd_easgd_update(self._h, _ptr(center), eta, lam))

    def easgd_step(self, batch, center, eta, lam):
        assert center.dtype == torch.float32 and center.is_contiguous() and center.numel() >= self.ld
        _check(lib().lsgd_easgd_step(self._h, C.byref(batch.c), _ptr(center), eta, lam))

    def sync_shadow(self):
        _check(lib().lsgd_sync_shadow(self._h))

    def get_leaders(self):
        lead = (C.c_int32 * self.G)()
        gl = C.c_int32()
        _check(lib().lsgd_get_leaders(self._h, lead, C.byref(gl)))
        return list(lead), int(gl.value)

    def set_leaders(self, local_leaders, global_leader):
        arr = (C.c_int32 * self.G)(*[int(v) for v in local_leaders])
        _check(lib().lsgd_set_leaders(self._h, arr, int(global_leader)))

    def get_losses(self):
        out = (C.c_float * self.W)()
        _check(lib().lsgd_get_losses(self._h, out))
        return list(out)


# ------------------------------------------------------------------------------------------------
# operators of token models: plain functions over memory.  Results carry no autograd graph, whatever the inputs require:
# embed_grad and block_norm_grad are how gradients come about (in the backward of a torch.autograd.Function, say).
# ------------------------------------------------------------------------------------------------
ADAMW_BLOCK = 256

EMBED_GRAD_ONE_LAUNCH = 8192

ATTENTION_ONE_LAUNCH = 1024

_F32, _BF16, _I32 = torch.float32, torch.bfloat16, torch.int32
_FLOATS = (_F32, _BF16)
# the handle alone: a torch.cuda.Stream object takes longer to make than a small call
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)


def _need(ok, msg):
    if not ok:
        raise ValueError(msg)


def _gpu(who, first, tensors):
    """Index of the GPU that `first` and all given (name, tensor) pairs lie on."""
    i = first.get_device()
    for name, t in tensors:
        if t is not None and t.get_device() != i or i < 0:
            raise ValueError(f"{who}: {name} is not on {'a GPU' if t is None or t.get_device() < 0 or i < 0 else 'the GPU of the others'}")
    return i


def _call(index, stream, f, *args):
    """f(*args, stream) with the tensors' GPU current."""
    if torch.cuda.current_device() == index:
        status = f(*args, _raw_stream(index) if stream is None else stream.cuda_stream)
    else:
        with torch.cuda.device(index):
            status = f(*args, _raw_stream(index) if stream is None else stream.cuda_stream)
    if status != 0:
        _check(status)


def _fresh(like, shape, dtype, stream):
    """Memory of the stream that the call runs on, as under torch.cuda.stream(stream): whoever used it before, or will after it is
    freed, is ordered on that stream too."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _workspace(who, nbytes, like, workspace, stream):
    """The caller's, or memory of this call's own."""
    if nbytes == 0:
        raise LsgdError(-1, lib().lsgd_last_error().decode())
    if workspace is None:
        return _fresh(like, (nbytes,), torch.uint8, stream), nbytes
    _need(workspace.device == like.device and workspace.is_contiguous(), f"{who}: workspace must be contiguous and on {like.device}")
    return workspace, workspace.numel() * workspace.element_size()


def _worker_stride(who, name, t, rule):
    """Row stride of a tensor whose dimensions after the first lie in memory without gaps (of a single row any will do)."""
    st, sh = t.stride(), t.shape
    want = 1
    for d in range(len(sh) - 1, 0, -1):
        if sh[d] > 1 and st[d] != want and t.numel():
            raise ValueError(f"{who}: {name} {rule}")
        want *= sh[d]
    return st[0] if sh[0] > 1 else want


def embed_lookup(table, tokens, scale=1.0, dtype=None, out=None, stream=None):
    """lsgd_embed_lookup: scale * table[w, tokens[w, t]] as [W, T, D]; zeros where a token lies outside [0, V).  Not recorded by
    autograd: embed_grad is its gradient.
    table: float32 or bfloat16 [W, V, D], dense within a worker (columns of x: x[:, a:a + V * D].unflatten(1, (V, D)));
    tokens: int32 [W, T]; dtype: of the result (the table's if None); out: optional result buffer."""
    who = "embed_lookup"
    index = _gpu(who, table, (("table", table), ("tokens", tokens), ("out", out)))
    _need(tokens.dtype is _I32 and tokens.dim() == 2, "embed_lookup: tokens must be int32 [W, T]")
    _need(table.dim() == 3 and table.dtype in _FLOATS, "embed_lookup: table must be float32 or bfloat16 [W, V, D]")
    W, V, D = table.shape
    rows, T = tokens.shape
    if rows != W:
        raise ValueError(f"{who}: {rows} rows of tokens for {W} workers")
    ld_table = _worker_stride(who, "table", table, "must be dense within a worker")
    ld_tokens = _worker_stride(who, "tokens", tokens, "must be dense within a worker")
    if out is None:
        dtype = table.dtype if dtype is None else dtype
        _need(dtype in _FLOATS, "embed_lookup: dtype must be float32 or bfloat16")
        out = _fresh(table, (W, T, D), dtype, stream)
        ld_out = T * D
    else:
        _need(out.shape == (W, T, D) and out.dtype in _FLOATS and (dtype is None or out.dtype == dtype), "embed_lookup: out must be [W, T, D] of dtype")
        ld_out = _worker_stride(who, "out", out, "must be dense within a worker")
    if T:
        _call(index, stream, lib().lsgd_embed_lookup, W, T, V, D, table.data_ptr(), ld_table, table.dtype is _BF16, tokens.data_ptr(), ld_tokens,
              scale, out.data_ptr(), ld_out, out.dtype is _BF16)
    return out


def embed_grad(dout, tokens, dtable, scale=1.0, accumulate=False, workspace=None, stream=None):
    """lsgd_embed_grad: the table's gradient of embed_lookup, into dtable (float32 [W, V, D], dense within a worker).
    dout: float32 or bfloat16 [W, T, D], dense within a worker; accumulate: add to dtable instead of writing all of it."""
    who = "embed_grad"
    index = _gpu(who, dtable, (("dout", dout), ("tokens", tokens), ("dtable", dtable)))
    _need(tokens.dtype is _I32 and tokens.dim() == 2, "embed_grad: tokens must be int32 [W, T]")
    _need(dtable.dim() == 3 and dtable.dtype is _F32, "embed_grad: dtable must be float32 [W, V, D]")
    W, V, D = dtable.shape
    rows, T = tokens.shape
    _need(rows == W and dout.shape == (W, T, D) and dout.dtype in _FLOATS, "embed_grad: dout must be float32 or bfloat16 [W, T, D] and tokens [W, T]")
    ld_table = _worker_stride(who, "dtable", dtable, "must be dense within a worker")
    ld_dout = _worker_stride(who, "dout", dout, "must be dense within a worker (an expanded gradient needs .contiguous())")
    ld_tokens = _worker_stride(who, "tokens", tokens, "must be dense within a worker")
    L = lib()
    ws, nbytes = None, 0
    if T > EMBED_GRAD_ONE_LAUNCH or workspace is not None:
        workspace, nbytes = _workspace(who, L.lsgd_embed_grad_workspace_bytes(W, T, V, D), dtable, workspace, stream)
        ws = workspace.data_ptr()
    _call(index, stream, L.lsgd_embed_grad, W, T, V, D, dout.data_ptr(), ld_dout, dout.dtype is _BF16, tokens.data_ptr(), ld_tokens, scale,
          bool(accumulate), dtable.data_ptr(), ld_table, ws, nbytes)


_NO_ROWS = (0, 0, 0)


def _rows(who, name, t, shape, dtype, index):
    """lsgd_rows of an activation tensor."""
    if t is None:
        return _NO_ROWS
    if t.shape != shape or t.dtype is not dtype:
        raise ValueError(f"{who}: {name} must be {dtype} {list(shape)}")
    if t.get_device() != index:
        raise ValueError(f"{who}: {name} is not on the GPU of the others")
    W, T, D = shape
    sw, st, sd = t.stride()
    if sd != 1 and D > 1 and t.numel():
        raise ValueError(f"{who}: rows of {name} must be dense")
    # a dimension of one element has no stride that means anything
    return t.data_ptr(), sw if W > 1 else T * D, st if T > 1 else D


def _weights(who, name, w, W, D, index):
    if w is None:
        return 0, 0
    if w.dtype is not _F32 or w.shape != (W, D) or w.get_device() != index or (D > 1 and w.stride(1) != 1):
        raise ValueError(f"{who}: {name} must be float32 [W, D] with dense rows, on the GPU of the others")
    return w.data_ptr(), w.stride(0) if W > 1 else D


def _stats(who, stats, W, T, index):
    _need(stats.dtype is _F32 and stats.shape == (2, W, T) and stats.is_contiguous() and stats.get_device() == index,
          f"{who}: stats must be contiguous float32 [2, W, T], on the GPU of the others")
    p = stats.data_ptr()
    return p, p + 4 * W * T if p else 0


def block_norm(r, y=None, gate=None, w_post=None, w_pre=None, scale=1.0, eps=1e-6, post_norm=True, pre_norm=True, r_out=None, n=None,
               stats=None, stream=None):
    """lsgd_block_norm: r_out = r + scale * sigmoid(gate) * norm(y) * w_post, n = norm(r_out) * w_pre.  Not recorded by autograd:
    block_norm_grad is its gradient.
    r, y, gate: float32 or bfloat16 [W, T, D] with dense rows; w_post, w_pre: float32 [W, D] (columns of x) or None (ones).
    y None: only n = norm(r) * w_pre.  post_norm False: y itself instead of norm(y).  pre_norm False: no n.
    Returns (r_out, n, stats); stats: float32 [2, W, T], what block_norm_grad needs.  r_out, n, stats: optional buffers (r_out
    may be r)."""
    who = "block_norm"
    dt = r.dtype
    _need(r.dim() == 3 and dt in _FLOATS, "block_norm: r must be float32 or bfloat16 [W, T, D]")
    index = _gpu(who, r, (("r", r),))
    shape = r.shape
    W, T, D = shape
    _need(y is not None or pre_norm, "block_norm: neither y nor a norm after it: nothing to do")
    _need(y is not None or (gate is None and r_out is None and w_post is None), "block_norm: gate, w_post and r_out need y")
    _need(pre_norm or (n is None and w_pre is None), "block_norm: n and w_pre need pre_norm")
    if y is not None and r_out is None:
        r_out = _fresh(r, shape, dt, stream)
    if pre_norm and n is None:
        n = _fresh(r, shape, dt, stream)
    if stats is None:
        stats = _fresh(r, (2, W, T), _F32, stream)
    q_post, q_pre = _stats(who, stats, W, T, index)
    wp, lp = _weights(who, "w_post", w_post, W, D, index)
    wn, ln = _weights(who, "w_pre", w_pre, W, D, index)
    a = _BLOCK_NORM.pack(W, T, D, dt is _BF16, bool(post_norm), scale, eps, *_rows(who, "r", r, shape, dt, index), *_rows(who, "y", y, shape, dt, index),
                         *_rows(who, "gate", gate, shape, dt, index), *_rows(who, "r_out", r_out, shape, dt, index), *_rows(who, "n", n, shape, dt, index),
                         wp, wn, lp, ln, q_post if y is not None else 0, q_pre)
    _call(index, stream, lib().lsgd_block_norm, a)
    return (r if y is None else r_out), n, stats


def block_norm_grad(dn, dr_out, r_out, stats, y=None, gate=None, w_post=None, w_pre=None, scale=1.0, post_norm=True, dw_post=None,
                    dw_pre=None, accumulate=False, dr=None, dy=None, dgate=None, workspace=None, stream=None):
    """lsgd_block_norm_grad: (dr, dy, dgate) from dn (gradient of n, or None) and dr_out (gradient of r_out past the next
    block, or None); r_out, stats: what block_norm returned; the rest as given to it.  dw_post, dw_pre: float32 [W, D]
    (columns of g) that receive the weights' gradients, added to what is there if accumulate; dr, dy, dgate: optional buffers."""
    who = "block_norm_grad"
    dt = r_out.dtype
    _need(r_out.dim() == 3 and dt in _FLOATS, "block_norm_grad: r_out must be float32 or bfloat16 [W, T, D]")
    index = _gpu(who, r_out, (("r_out", r_out),))
    shape = r_out.shape
    W, T, D = shape
    _need(dn is not None or dr_out is not None, "block_norm_grad: neither dn nor dr_out is given")
    _need(y is not None or (gate is None and dw_post is None and dy is None and dgate is None), "block_norm_grad: gate, dw_post, dy and dgate need y")
    _need(gate is not None or dgate is None, "block_norm_grad: dgate needs gate")
    if dr is None:
        dr = _fresh(r_out, shape, dt, stream)
    if y is not None and dy is None:
        dy = _fresh(r_out, shape, dt, stream)
    if gate is not None and dgate is None:
        dgate = _fresh(r_out, shape, dt, stream)
    q_post, q_pre = _stats(who, stats, W, T, index)
    wp, lp = _weights(who, "w_post", w_post, W, D, index)
    wn, ln = _weights(who, "w_pre", w_pre, W, D, index)
    dwp, ldp = _weights(who, "dw_post", dw_post, W, D, index)
    dwn, ldn = _weights(who, "dw_pre", dw_pre, W, D, index)
    a = _BLOCK_NORM_GRAD.pack(W, T, D, dt is _BF16, bool(post_norm), bool(accumulate), scale, *_rows(who, "dn", dn, shape, dt, index),
                              *_rows(who, "dr_out", dr_out, shape, dt, index), *_rows(who, "r_out", r_out, shape, dt, index),
                              *_rows(who, "y", y, shape, dt, index), *_rows(who, "gate", gate, shape, dt, index), *_rows(who, "dr", dr, shape, dt, index),
                              *_rows(who, "dy", dy, shape, dt, index), *_rows(who, "dgate", dgate, shape, dt, index), wp, wn, lp, ln, q_post, q_pre,
                              dwp, dwn, ldp, ldn)
    L = lib()
    ws, nbytes = None, 0
    if dwp or dwn:
        workspace, nbytes = _workspace(who, L.lsgd_block_norm_grad_workspace_bytes(W, T, D), r_out, workspace, stream)
        ws = workspace.data_ptr()
    _call(index, stream, L.lsgd_block_norm_grad, a, ws, nbytes)
    return dr, dy, dgate


_NO_HEADS = (0, 0, 0, 0)


def _heads(who, name, t, shape, dtype, index):
    """lsgd_heads of an activation tensor [B, T, H, D] (strides of a dimension of one element mean nothing, and are not looked at)."""
    if t is None:
        return _NO_HEADS
    if t.shape != shape or t.dtype is not dtype:
        raise ValueError(f"{who}: {name} must be {dtype} {list(shape)}")
    if t.get_device() != index:
        raise ValueError(f"{who}: {name} is not on the GPU of the others")
    sb, st, sh, sd = t.stride()
    if sd != 1 and shape[3] > 1 and t.numel():
        raise ValueError(f"{who}: columns of {name} must be dense")
    return t.data_ptr(), sb, st, sh


def _new_heads(like, shape, dtype, stream):
    """A result of the call's own, and its lsgd_heads."""
    t = _fresh(like, shape, dtype, stream)
    row = shape[2] * shape[3]
    return t, (t.data_ptr(), shape[1] * row, row, shape[3])


def _vector(who, name, t, dtype, n, index):
    """Address of a dense vector, or of n things in any shape."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.numel() != n or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{who}: {name} must be {n} contiguous {dtype}, on the GPU of the others")
    return t.data_ptr()


def _statistics(who, name, t, shape, index):
    """Address of float32 statistics without gaps, laid out as one of these calls writes them."""
    if t is None:
        return 0
    if t.shape != shape or t.dtype is not _F32 or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{who}: {name} must be contiguous {_F32} {list(shape)}, on the GPU of the others")
    return t.data_ptr()


def _positions(who, t, W, T, index):
    if t is None:
        return 0, 0
    if t.dtype is not _I32 or t.get_device() != index or t.shape not in ((W, T), (1, T)):
        raise ValueError(f"{who}: positions must be int32 [W, T] or [1, T], on the GPU of the others")
    ld, st = t.stride()
    if st != 1 and T > 1:
        raise ValueError(f"{who}: positions must be dense within a worker")
    return t.data_ptr(), ld if t.shape[0] > 1 else 0


def _head_weights(who, name, w, W, D, index):
    """[W, D], or [1, D] for all workers."""
    if w is None:
        return 0, 0
    if w.dtype is not _F32 or w.get_device() != index or w.shape not in ((W, D), (1, D)):
        raise ValueError(f"{who}: {name} must be float32 [W, D] or [1, D], on the GPU of the others")
    ld, sd = w.stride()
    if sd != 1 and D > 1:
        raise ValueError(f"{who}: rows of {name} must be dense")
    return w.data_ptr(), ld if w.shape[0] > 1 else 0


def rotary_turns(columns, base=10000.0, stretch=1.0, keep=None, device="cuda"):
    """Turns per position of the pairs of `columns` rotated columns, float64 [columns / 2] on device, for qk_rotary: pair i makes
    base^(-2 i / columns) / (2 pi).
    stretch > 1 serves contexts that much longer than those trained on.  keep None: every pair turns that much slower.  keep =
    (length, low, high): a pair that makes at least `high` turns over the trained length keeps its pace, one that makes at most `low` is
    slowed by the whole factor, between them a share in proportion."""
    _need(columns >= 0 and columns % 2 == 0, "rotary_turns: columns must be even")
    _need(base > 0 and stretch > 0, "rotary_turns: base and stretch must be positive")
    turns = torch.tensor([base ** (-2.0 * i / columns) / (2.0 * math.pi) for i in range(columns // 2)], dtype=torch.float64)
    if keep is None:
        turns = turns / stretch
    else:
        length, low, high = keep
        _need(length > 0 and 0 <= low < high, "rotary_turns: keep must be (length, low, high) with 0 <= low < high")
        share = ((turns * length - low) / (high - low)).clamp(0.0, 1.0)
        turns = share * turns + (1.0 - share) * (turns / stretch)
    return turns.to(device)


def qk_rotary(q, k=None, positions=None, turns=None, w_q=None, w_k=None, norm=True, eps=1e-6, interleaved=False, magnitude=1.0, q_out=None,
              k_out=None, stats=None, stream=None):
    """lsgd_qk_rotary: each head's norm and its rotation by the token's position, of queries and keys in one pass.  Not recorded by
    autograd: qk_rotary_grad is its gradient.
    q, k: float32 or bfloat16 [W, T, Hq, D], [W, T, Hk, D] with dense columns (views of one projection will do); positions: int32 [W, T] or
    [1, T], None: 0 .. T-1; turns: float64 [R / 2] on the GPU (rotary_turns), None: no rotation; w_q, w_k: float32 [W, D] (columns of x)
    or [1, D], None: ones; norm False: no norm; interleaved: pairs are neighbours, not a half apart; magnitude: of the rotated columns.
    Returns (q_out, k_out, stats); stats: float32 [W, T, Hq + Hk], what the gradient needs, None without a norm.  q_out, k_out, stats:
    optional buffers (q_out may be q, k_out may be k; a slice of a cache)."""
    who = "qk_rotary"
    dt = q.dtype
    _need(q.dim() == 4 and dt in _FLOATS, "qk_rotary: q must be float32 or bfloat16 [W, T, H, D]")
    index = q.get_device()
    if index < 0:
        index = _gpu(who, q, (("q", q),))
    W, T, Hq, D = shape = q.shape
    _need(k is None or k.dim() == 4, "qk_rotary: k must be [W, T, H, D]")
    _need(k is not None or (w_k is None and k_out is None), "qk_rotary: w_k and k_out need k")
    _need(norm or stats is None, "qk_rotary: stats need a norm")
    Hk = 0 if k is None else k.shape[2]
    kshape = (W, T, Hk, D)
    half = 0 if turns is None else turns.numel()
    _need(half * 2 <= D, "qk_rotary: more turns than pairs of columns")
    if q_out is None:
        q_out, to_q = _new_heads(q, shape, dt, stream)
    else:
        to_q = _heads(who, "q_out", q_out, shape, dt, index)
    if Hk and k_out is None:
        k_out, to_k = _new_heads(q, kshape, dt, stream)
    else:
        to_k = _heads(who, "k_out", k_out, kshape, dt, index)
    if norm and stats is None:
        stats = _fresh(q, (W, T, Hq + Hk), _F32, stream)
    wq, lq = _head_weights(who, "w_q", w_q, W, D, index)
    wk, lk = _head_weights(who, "w_k", w_k, W, D, index)
    if T:
        a = _QK_ROTARY.pack(W, T, Hq, Hk, D, 2 * half, dt is _BF16, bool(norm), bool(interleaved), eps, magnitude, *_heads(who, "q", q, shape, dt, index),
                            *_heads(who, "k", k, kshape, dt, index), *to_q, *to_k, *_positions(who, positions, W, T, index),
                            _vector(who, "turns", turns, torch.float64, half, index), wq, wk, lq, lk,
                            _statistics(who, "stats", stats, (W, T, Hq + Hk), index))
        _call(index, stream, lib().lsgd_qk_rotary, a)
    return q_out, k_out, stats


def qk_rotary_grad(dq_out, dk_out=None, q=None, k=None, stats=None, positions=None, turns=None, w_q=None, w_k=None, norm=True, interleaved=False,
                   magnitude=1.0, dw_q=None, dw_k=None, accumulate=False, dq=None, dk=None, workspace=None, stream=None):
    """lsgd_qk_rotary_grad: (dq, dk) from dq_out, dk_out (gradients of qk_rotary's results); q, k, stats and the rest as it had or gave
    them (q, k None: neither a norm nor dw_q, dw_k).  dw_q, dw_k: float32 [W, D] (columns of g) that receive the weights' gradients, added to
    what is there if accumulate; weights shared by workers have theirs worker by worker.  dq, dk: optional buffers."""
    who = "qk_rotary_grad"
    dt = dq_out.dtype
    _need(dq_out.dim() == 4 and dt in _FLOATS, "qk_rotary_grad: dq_out must be float32 or bfloat16 [W, T, H, D]")
    index = dq_out.get_device()
    if index < 0:
        index = _gpu(who, dq_out, (("dq_out", dq_out),))
    W, T, Hq, D = shape = dq_out.shape
    _need(dk_out is None or dk_out.dim() == 4, "qk_rotary_grad: dk_out must be [W, T, H, D]")
    _need(dk_out is not None or (k is None and w_k is None and dw_k is None and dk is None), "qk_rotary_grad: k, w_k, dw_k and dk need dk_out")
    _need(not norm or stats is not None, "qk_rotary_grad: a norm's gradient needs stats")
    Hk = 0 if dk_out is None else dk_out.shape[2]
    kshape = (W, T, Hk, D)
    half = 0 if turns is None else turns.numel()
    _need(half * 2 <= D, "qk_rotary_grad: more turns than pairs of columns")
    if dq is None:
        dq, to_q = _new_heads(dq_out, shape, dt, stream)
    else:
        to_q = _heads(who, "dq", dq, shape, dt, index)
    if Hk and dk is None:
        dk, to_k = _new_heads(dq_out, kshape, dt, stream)
    else:
        to_k = _heads(who, "dk", dk, kshape, dt, index)
    wq, lq = _head_weights(who, "w_q", w_q, W, D, index)
    wk, lk = _head_weights(who, "w_k", w_k, W, D, index)
    dwq, ldq = _weights(who, "dw_q", dw_q, W, D, index)
    dwk, ldk = _weights(who, "dw_k", dw_k, W, D, index)
    a = _QK_ROTARY_GRAD.pack(W, T, Hq, Hk, D, 2 * half, dt is _BF16, bool(norm), bool(interleaved), bool(accumulate), magnitude,
                             *_heads(who, "dq_out", dq_out, shape, dt, index), *_heads(who, "dk_out", dk_out, kshape, dt, index),
                             *_heads(who, "q", q, shape, dt, index), *_heads(who, "k", k, kshape, dt, index), *to_q, *to_k, *_positions(who, positions, W, T, index),
                             _vector(who, "turns", turns, torch.float64, half, index), wq, wk, lq, lk,
                             _statistics(who, "stats", stats, (W, T, Hq + Hk), index) if norm else 0, dwq, dwk, ldq, ldk)
    L = lib()
    ws, nbytes = None, 0
    if T and (dwq or dwk):
        workspace, nbytes = _workspace(who, L.lsgd_qk_rotary_grad_workspace_bytes(W, T, Hq, Hk, D, 2 * half, dt is _BF16), dq_out, workspace, stream)
        ws = workspace.data_ptr()
    _call(index, stream, L.lsgd_qk_rotary_grad, a, ws, nbytes)
    return dq, dk


def _attention_shapes(who, q, k):
    qs, ks = q.shape, k.shape
    if len(qs) != 4 or q.dtype not in _FLOATS:
        raise ValueError(f"{who}: q must be float32 or bfloat16 [B, Tq, Hq, D]")
    if len(ks) != 4 or ks[0] != qs[0] or ks[3] != qs[3]:
        raise ValueError(f"{who}: k must be [B, Tk, Hk, D] beside q")
    if qs[3] == 0:
        raise ValueError(f"{who}: q has no columns")
    return qs, ks


def attention(q, k, v, causal=False, scale=None, q_lens=None, k_lens=None, with_lse=True, out=None, lse=None, workspace=None, stream=None):
    """lsgd_attention: softmax(scale q k') v.  Not recorded by autograd: attention_grad is its gradient.
    q: float32 or bfloat16 [B, Tq, Hq, D], k, v: [B, Tk, Hk, D] with dense columns, Hk a divisor of Hq (query heads that share a key head are
    adjacent); an entry is a worker, or one of its sequences.  q_lens, k_lens: int32 [B] on the GPU, lengths of the entries' sequences
    (None: full); causal: a query sees the keys up to its own place, both sequences ending together; scale: 1 / sqrt(D) if None.
    Returns (out, lse): out like q, lse float32 [B, Hq, Tq], which the gradient needs (None if not with_lse).  Queries that see nothing have zeros
    and -inf.  out, lse: optional buffers."""
    who = "attention"
    shape, kshape = _attention_shapes(who, q, k)
    (B, Tq, Hq, D), (_, Tk, Hk, _) = shape, kshape
    dt = q.dtype
    index = q.get_device()
    if index < 0:
        index = _gpu(who, q, (("q", q),))
    if scale is None:
        scale = D ** -0.5
    if out is None:
        out, to = _new_heads(q, shape, dt, stream)
    else:
        to = _heads(who, "out", out, shape, dt, index)
    if lse is None and with_lse:
        lse = _fresh(q, (B, Hq, Tq), _F32, stream)
    a = _ATTENTION.pack(B, Tq, Tk, Hq, Hk, D, dt is _BF16, bool(causal), scale, *_heads(who, "q", q, shape, dt, index),
                        *_heads(who, "k", k, kshape, dt, index), *_heads(who, "v", v, kshape, dt, index), *to,
                        _vector(who, "q_lens", q_lens, _I32, B, index), _vector(who, "k_lens", k_lens, _I32, B, index),
                        _statistics(who, "lse", lse, (B, Hq, Tq), index))
    L = lib()
    ws, nbytes = None, 0
    if Tk > ATTENTION_ONE_LAUNCH or workspace is not None:
        workspace, nbytes = _workspace(who, L.lsgd_attention_workspace_bytes(B, Tq, Tk, Hq, Hk, D, dt is _BF16), q, workspace, stream)
        ws = workspace.data_ptr()
    _call(index, stream, L.lsgd_attention, a, ws, nbytes)
    return out, lse


def attention_grad(dout, q, k, v, out, lse, causal=False, scale=None, q_lens=None, k_lens=None, dq=None, dk=None, dv=None, workspace=None, stream=None):
    """lsgd_attention_grad: (dq, dk, dv) from dout; out, lse: what attention returned; the rest as given to it.  dq, dk, dv: optional
    buffers (parts of one projection's gradient will do)."""
    who = "attention_grad"
    shape, kshape = _attention_shapes(who, q, k)
    (B, Tq, Hq, D), (_, Tk, Hk, _) = shape, kshape
    dt = q.dtype
    index = q.get_device()
    if index < 0:
        index = _gpu(who, q, (("q", q),))
    if scale is None:
        scale = D ** -0.5
    dq, to_q = _new_heads(q, shape, dt, stream) if dq is None else (dq, _heads(who, "dq", dq, shape, dt, index))
    dk, to_k = _new_heads(q, kshape, dt, stream) if dk is None else (dk, _heads(who, "dk", dk, kshape, dt, index))
    dv, to_v = _new_heads(q, kshape, dt, stream) if dv is None else (dv, _heads(who, "dv", dv, kshape, dt, index))
    a = _ATTENTION_GRAD.pack(B, Tq, Tk, Hq, Hk, D, dt is _BF16, bool(causal), scale, *_heads(who, "dout", dout, shape, dt, index),
                             *_heads(who, "q", q, shape, dt, index), *_heads(who, "k", k, kshape, dt, index), *_heads(who, "v", v, kshape, dt, index),
                             *_heads(who, "out", out, shape, dt, index), *to_q, *to_k, *to_v,
                             _vector(who, "q_lens", q_lens, _I32, B, index), _vector(who, "k_lens", k_lens, _I32, B, index),
                             _statistics(who, "lse", lse, (B, Hq, Tq), index))
    L = lib()
    workspace, nbytes = _workspace(who, L.lsgd_attention_grad_workspace_bytes(B, Tq, Tk, Hq, Hk, D, dt is _BF16), q, workspace, stream)
    _call(index, stream, L.lsgd_attention_grad, a, workspace.data_ptr(), nbytes)
    return dq, dk, dv


class AdamWTensor:
    """One tensor of an AdamW step: float32 x and its gradient g (float32 or bfloat16), both [rows, n] with dense rows (columns of a
    population's x and g, or any dense tensor, which counts as one row).  Moments m, v of the same shape: float32 for 32 bits;
    int8 and uint8 for 8 bits with float32 scales m_scale, v_scale [rows, ceil(n / ADAMW_BLOCK)].  x_bf16: optional bfloat16 copy
    of x that the step keeps current (a Population over the same x does so at its updates and pulls if it has x_bf16 and
    WRITE_BF16_SHADOW; else Population.sync_shadow before the copy is read).  m_values, v_values: optional float32 tensors that
    AdamW.moments() fills."""

    def __init__(self, x, g, m, v, weight_decay=0.0, lr_mult=1.0, x_bf16=None, m_scale=None, v_scale=None, m_values=None, v_values=None):
        self.t = dict(x=x, g=g, m=m, v=v, m_scale=m_scale, v_scale=v_scale, m_values=m_values, v_values=v_values, x_bf16=x_bf16)
        self.weight_decay, self.lr_mult = float(weight_decay), float(lr_mult)

    def _c(self, k, bits, g_dtype):
        who = f"AdamW: tensor {k}"
        x = self.t["x"]
        types = {"x": torch.float32, "g": g_dtype, "m": torch.float32 if bits == 32 else torch.int8, "v": torch.float32 if bits == 32 else torch.uint8,
                 "m_scale": torch.float32, "v_scale": torch.float32, "m_values": torch.float32, "v_values": torch.float32, "x_bf16": torch.bfloat16}
        two = x.dim() == 2
        rows, n = (x.shape if two else (1, x.numel()))
        got, ld = {}, {}
        for name, t in self.t.items():
            if t is None or (bits == 32 and name in ("m_scale", "v_scale", "m_values", "v_values")):
                got[name], ld[name] = None, 0
                continue
            _need(t.dtype == types[name], f"{who}: {name} must be {types[name]}, is {t.dtype}")
            if name in ("m_scale", "v_scale"):
                nb = -(-n // ADAMW_BLOCK)
                if t.dim() != 2:
                    _need(t.is_contiguous(), f"{who}: {name} must be contiguous or [{rows}, {nb}]")
                    t = t.view(1, -1)
                _need(tuple(t.shape) == (rows, nb), f"{who}: {name} must be [{rows}, {nb}]")
            else:
                _need(t.shape == x.shape, f"{who}: {name} has shape {list(t.shape)}, x has {list(x.shape)}")
                if not two:
                    _need(t.is_contiguous(), f"{who}: {name} must be contiguous")
                    t = t.view(1, -1)
            _need(t.numel() == 0 or t.shape[1] == 1 or t.stride(1) == 1, f"{who}: rows of {name} must be dense")
            got[name], ld[name] = t.data_ptr() or None, (t.stride(0) if t.shape[0] > 1 else t.shape[1])
        _need(ld["m"] == ld["v"] and ld["m_scale"] == ld["v_scale"] and ld["m_values"] == ld["v_values"],
              f"{who}: m and v (their scales, their values) must have the same row stride")
        return _AdamWTensor(got["x"], got["g"], got["m"], got["v"], got["m_scale"], got["v_scale"], got["m_values"], got["v_values"], got["x_bf16"],
                            rows, n, ld["x"], ld["g"], ld["m"], ld["m_scale"], ld["m_values"], ld["x_bf16"], self.weight_decay, self.lr_mult)


class AdamW:
    """lsgd_adamw_create over a list of AdamWTensor; bits: 32 or 8, how the moments are held.  Keeps the tensors alive.
    Calls run on `stream`, or where none is given on the stream that is current at each call, as the other operators do."""

    def __init__(self, tensors, bits=32, stream=None, workspace=None):
        self._h = None
        self.tensors = list(tensors)
        _need(len(self.tensors) > 0, "AdamW: no tensors")
        for k, a in enumerate(self.tensors):
            for name in ("x", "g", "m", "v"):
                _need(a.t[name] is not None, f"AdamW: tensor {k}: {name} is missing")
        self._index = _gpu("AdamW", self.tensors[0].t["x"], [(f"{name} of tensor {k}", t) for k, a in enumerate(self.tensors) for name, t in a.t.items()])
        dev = self.tensors[0].t["x"].device
        g_dtype = self.tensors[0].t["g"].dtype
        _need(g_dtype in _FLOATS, "AdamW: g must be float32 or bfloat16")
        arr = (_AdamWTensor * len(self.tensors))(*[a._c(k, bits, g_dtype) for k, a in enumerate(self.tensors)])
        self._follows = stream is None
        self.stream = torch.cuda.current_stream(dev) if stream is None else stream
        self._raw = self.stream.cuda_stream
        self._step = lib().lsgd_adamw_step
        bf = int(g_dtype == torch.bfloat16)
        with torch.cuda.device(dev):
            self.workspace, nbytes = _workspace("AdamW", lib().lsgd_adamw_workspace_bytes(arr, len(arr), bits, bf), self.tensors[0].t["x"], workspace, stream)
            h = C.c_void_p()
            _check(lib().lsgd_adamw_create(arr, len(arr), bits, bf, _ptr(self.workspace), nbytes, C.c_void_p(self.stream.cuda_stream), C.byref(h)))
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            lib().lsgd_adamw_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def step(self, lr, step, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0):
        """One step; `step` counts from 1.  Captured in a graph, it is replayed with the rates and the step number of its call."""
        self._call(self._step, lr, beta1, beta2, eps, int(step), grad_scale)

    def moments(self):
        """8 bits: fills m_values and v_values of the tensors that have them."""
        self._call(lib().lsgd_adamw_moments)

    def _call(self, f, *args):
        if self._follows and _raw_stream(self._index) != self._raw:
            self.stream = torch.cuda.current_stream(self._index)
            self._raw = self.stream.cuda_stream
            _check(lib().lsgd_adamw_set_stream(self._h, self._raw))
            self.workspace.record_stream(self.stream)        # its memory is another stream's
        if torch.cuda.current_device() == self._index:
            status = f(self._h, *args)
        else:
            with torch.cuda.device(self._index):
                status = f(self._h, *args)
        if status != 0:
            _check(status)
