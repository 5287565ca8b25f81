"""Thin Python binding of the C ABI in include/flce.h: argument marshalling only.

Every step of the path (projection, cross entropy, both gradients, the chunk
loop) runs inside libflce.so; PyTorch is used for device memory and streams.
There is no fallback: if the library is missing or a call fails, this raises.
"""
from __future__ import annotations

import array
import ctypes
import os

import torch  # imported before the library so both share one HIP runtime

from . import _build

FLCE_F32, FLCE_BF16 = 0, 1
SKIP_DX, SKIP_DW = 1, 2
_DTYPES = {torch.float32: FLCE_F32, torch.bfloat16: FLCE_BF16}

_lib = None


class FlceError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: status {status} ({status_string(status)})")
        self.status = status


def lib() -> ctypes.CDLL:
    """Loads libflce.so, building it first when there is none or when a kernel source or
    the header is newer than the built library (so an edited kernel is never tested
    against an old binary)."""
    global _lib
    if _lib is None:
        if _build.is_stale():
            _build.build()
        L = ctypes.CDLL(_build.LIB_PATH)
        p, i64, sz, ci, u = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_int, ctypes.c_uint
        sigs = {
            "flce_fwd_bwd": ([p, p, p, i64, i64, i64, i64, ci, p, p, p, p], ci),
            "flce_fwd_bwd_ex": ([p, p, p, i64, i64, i64, i64, ci, p, p, p, u, p], ci),
            "flce_fwd_bwd_opt": ([p, p, p, i64, i64, i64, i64, ci, p, p, p, p, p], ci),
            "flce_default_options": ([p], None),
            "flce_workspace_bytes_opt": ([i64, i64, i64, ci, p], sz),
            "flce_multihead_fwd_bwd": ([p, p, p, p, ci, i64, i64, i64, i64, ci, p, p, p, p, u, p], ci),
            "flce_rmsnorm_fwd_bwd": ([p, p, ctypes.c_float, p, p, i64, i64, i64, i64, ci, p, p, p, p, u, p], ci),
            "flce_rmsnorm_workspace_bytes": ([i64, i64, i64, ci], sz),
            "flce_cross_entropy_inplace": ([p, p, i64, i64, i64, i64, ci, p, p], ci),
            "flce_cross_entropy_inplace_noalloc": ([p, p, i64, i64, i64, i64, ci, p, p], ci),
            "flce_block_norm_fwd": ([p] * 9, ci),
            "flce_block_norm_bwd": ([p] * 14, ci),
            "flce_block_norm_workspace_bytes": ([p], sz),
            "flce_grad_norm": ([p, p, p, ci, ci, p, p, sz, p], ci),
            "flce_grad_clip": ([p, p, p, p, ci, p, ctypes.c_float, p], ci),
            "flce_clip_grad_norm": ([p, p, p, p, ci, ci, ctypes.c_float, p, p, sz, p], ci),
            "flce_grad_norm_workspace_bytes": ([ci], sz),
            "flce_layer_norm_fwd": ([p] * 8, ci),
            "flce_layer_norm_bwd": ([p] * 9, ci),
            "flce_layer_norm_workspace_bytes": ([p], sz),
            "flce_orthogonalize": ([p, p, ci, p, p], ci),
            "flce_orthogonalize_workspace_bytes": ([ci, p], sz),
            "flce_embedding_fwd": ([p] * 5, ci),
            "flce_embedding_bwd": ([p] * 5, ci),
            "flce_embedding_workspace_bytes": ([p], sz),
            "flce_workspace_bytes": ([i64, i64, i64, ci], sz),
            "flce_workspace_bytes_max": ([i64, i64, ci], sz),
            "flce_set_workspace": ([p, sz], ci),
            "flce_release_workspace": ([], ci),
            "flce_set_logits_budget_bytes": ([sz], ci),
            "flce_get_logits_budget_bytes": ([], sz),
            "flce_set_row_compaction": ([ci], ci),
            "flce_get_row_compaction": ([], ci),
            "flce_logits_budget_for_workspace": ([i64, i64, i64, ci, sz], sz),
            "flce_chunk_rows": ([i64, i64, i64, ci], i64),
            "flce_num_chunks": ([i64, i64, i64, ci], i64),
            "flce_dx_k_ranges": ([i64, i64, i64, ci], ci),
            "flce_paper_chunk_rows": ([i64, i64, i64], i64),
            "flce_full_logits_bytes": ([i64, i64, ci], sz),
            "flce_mfma_ceiling_launch": ([ci, ci, ci, ctypes.c_float, p, sz, p], ci),
            "flce_timing_enable": ([ci], ci),
            "flce_timing_collect": ([p, p], ci),
            "flce_status_string": ([ci], ctypes.c_char_p),
        }
        for name, (args, res) in sigs.items():
            fn = getattr(L, name)
            fn.argtypes, fn.restype = args, res
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().flce_status_string(int(status)).decode()


def _check(status: int, what: str):
    if status != 0:
        raise FlceError(status, what)


def _dtype_code(t: torch.Tensor) -> int:
    try:
        return _DTYPES[t.dtype]
    except KeyError:
        raise TypeError(f"unsupported dtype {t.dtype}; use float32 or bfloat16") from None


def _dev_ptr(t: torch.Tensor | None, name: str) -> int | None:
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous (dense row-major)")
    return t.data_ptr()


def _stream_handle(stream, device) -> int:
    if stream is None:   # (the handle alone: current_stream() builds an object around it)
        return _raw_stream(device.index)
    return stream.cuda_stream


try:
    _raw_stream = torch._C._cuda_getCurrentRawStream
except AttributeError:   # a build without GPU support
    def _raw_stream(index):
        return torch.cuda.current_stream(index).cuda_stream


class _OnDevice:
    """torch.cuda.device that switches only when it has to.  With the stream's handle taken directly, a
    stand-alone cross entropy of 32 rows is issued in 6.4-7.2 us instead of 11."""
    __slots__ = ("index", "before")

    def __init__(self, device):
        if device.type != "cuda":
            raise ValueError(f"Expected a cuda device, but got: {device}")
        self.index = device.index

    def __enter__(self):
        self.before = torch.cuda.current_device()
        if self.before != self.index:
            torch.cuda.set_device(self.index)

    def __exit__(self, *exc):
        if self.before != self.index:
            torch.cuda.set_device(self.before)
        return False


def flce_fwd_bwd(X, W, targets, ignore_index=-100, loss=None, dX=None, dW=None, flags=0,
                 stream=None):
    """loss, dX, dW of mean cross_entropy(X @ W.T, targets) on the GPU, chunked.

    X [BT, H], W [V, H] (float32 or bfloat16, same dtype), targets [BT] int64,
    all contiguous CUDA tensors.  Outputs are allocated when not passed.
    Asynchronous on `stream` (default: torch's current stream).
    """
    code = _dtype_code(X)
    if W.dtype != X.dtype:
        raise TypeError("X and W must have the same dtype")
    if X.dim() != 2 or W.dim() != 2 or X.shape[1] != W.shape[1] or targets.shape != (X.shape[0],):
        raise ValueError("expected X [BT, H], W [V, H], targets [BT]")
    if targets.dtype != torch.int64:
        raise TypeError("targets must be int64")
    BT, H = X.shape
    V = W.shape[0]
    if loss is None:
        loss = torch.empty((), dtype=torch.float32, device=X.device)
    if dX is None and not (flags & SKIP_DX):
        dX = torch.empty_like(X)
    if dW is None and not (flags & SKIP_DW):
        dW = torch.empty_like(W)
    for name, t, ref in (("dX", dX, X), ("dW", dW, W)):
        if t is not None and (t.shape != ref.shape or t.dtype != ref.dtype):
            raise ValueError(f"{name} must match its input in shape and dtype")
    with _OnDevice(X.device):
        st = lib().flce_fwd_bwd_ex(_dev_ptr(X, "X"), _dev_ptr(W, "W"), _dev_ptr(targets, "targets"),
                                   BT, H, V, int(ignore_index), code, _dev_ptr(loss, "loss"),
                                   _dev_ptr(dX, "dX"), _dev_ptr(dW, "dW"), int(flags),
                                   _stream_handle(stream, X.device))
    _check(st, "flce_fwd_bwd")
    return loss, dX, dW


class FlceOptions(ctypes.Structure):
    """flce_options of include/flce.h."""
    _fields_ = [("size", ctypes.c_size_t), ("logits_budget_bytes", ctypes.c_size_t),
                ("row_compaction", ctypes.c_int), ("flags", ctypes.c_uint),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


def flce_options(logits_budget_bytes=None, row_compaction=None, flags=0, workspace=None) -> FlceOptions:
    """The process-wide settings (flce_default_options) with the given fields replaced.
    workspace: a device tensor the call uses as its scratch memory instead of the device's
    shared workspace (kept alive by the returned struct)."""
    o = FlceOptions()
    lib().flce_default_options(ctypes.byref(o))
    if workspace is not None:
        o.workspace = _dev_ptr(workspace, "workspace")
        o.workspace_bytes = workspace.numel() * workspace.element_size()
        o._workspace_tensor = workspace
    if logits_budget_bytes is not None:
        o.logits_budget_bytes = int(logits_budget_bytes)
    if row_compaction is not None:
        o.row_compaction = 1 if row_compaction else 0
    o.flags = int(flags)
    return o


def flce_fwd_bwd_opt(X, W, targets, options: FlceOptions, ignore_index=-100, loss=None, dX=None,
                     dW=None, stream=None):
    """flce_fwd_bwd with its settings passed along (see flce_options)."""
    code = _dtype_code(X)
    if W.dtype != X.dtype or targets.dtype != torch.int64:
        raise TypeError("X and W must have the same dtype, targets must be int64")
    if X.dim() != 2 or W.dim() != 2 or X.shape[1] != W.shape[1] or targets.shape != (X.shape[0],):
        raise ValueError("expected X [BT, H], W [V, H], targets [BT]")
    BT, H = X.shape
    V = W.shape[0]
    if loss is None:
        loss = torch.empty((), dtype=torch.float32, device=X.device)
    if dX is None and not (options.flags & SKIP_DX):
        dX = torch.empty_like(X)
    if dW is None and not (options.flags & SKIP_DW):
        dW = torch.empty_like(W)
    with _OnDevice(X.device):
        st = lib().flce_fwd_bwd_opt(_dev_ptr(X, "X"), _dev_ptr(W, "W"), _dev_ptr(targets, "targets"),
                                    BT, H, V, int(ignore_index), code, _dev_ptr(loss, "loss"),
                                    _dev_ptr(dX, "dX"), _dev_ptr(dW, "dW"), ctypes.byref(options),
                                    _stream_handle(stream, X.device))
    _check(st, "flce_fwd_bwd_opt")
    return loss, dX, dW


def flce_workspace_bytes_opt(BT, H, V, dtype, options: FlceOptions) -> int:
    return int(lib().flce_workspace_bytes_opt(BT, H, V, _DTYPES.get(dtype, dtype), ctypes.byref(options)))


def flce_multihead_fwd_bwd(X, Ws, targets, weights=None, ignore_index=-100, loss=None,
                           head_losses=None, dX=None, dWs=None, flags=0, stream=None):
    """Several heads on shared hidden states: loss = sum_j weights[j] * CE_j.

    X [BT, H]; Ws, targets: sequences of n_heads tensors W_j [V, H] and int64
    targets_j [BT]; weights: n_heads floats or None (all 1).  Returns
    (loss, head_losses [n_heads], dX, [dW_j]).  Outputs are allocated when not passed.
    """
    code = _dtype_code(X)
    n = len(Ws)
    if n < 1 or len(targets) != n or (weights is not None and len(weights) != n):
        raise ValueError("Ws, targets and weights must have one entry per head")
    if X.dim() != 2:
        raise ValueError("expected X [BT, H]")
    BT, H = X.shape
    V = Ws[0].shape[0]
    for W, t in zip(Ws, targets):
        if W.dtype != X.dtype or t.dtype != torch.int64:
            raise TypeError("every W must have X's dtype and every targets tensor must be int64")
        if W.shape != (V, H) or t.shape != (BT,):
            raise ValueError("expected every W [V, H] and every targets [BT]")
    if loss is None:
        loss = torch.empty((), dtype=torch.float32, device=X.device)
    if head_losses is None:
        head_losses = torch.empty(n, dtype=torch.float32, device=X.device)
    if head_losses.shape != (n,) or head_losses.dtype != torch.float32:
        raise ValueError("head_losses must be n_heads float32 values")
    if dX is None and not (flags & SKIP_DX):
        dX = torch.empty_like(X)
    if dX is not None and (dX.shape != X.shape or dX.dtype != X.dtype):
        raise ValueError("dX must match X in shape and dtype")
    if dWs is None and not (flags & SKIP_DW):
        dWs = [torch.empty_like(W) for W in Ws]
    if dWs is not None:
        if len(dWs) != n or any(d.shape != (V, H) or d.dtype != X.dtype for d in dWs):
            raise ValueError("dWs must hold one [V, H] tensor of X's dtype per head")
    ptr_array = ctypes.c_void_p * n
    w_arr = ptr_array(*[_dev_ptr(W, "W") for W in Ws])
    t_arr = ptr_array(*[_dev_ptr(t, "targets") for t in targets])
    dw_arr = ptr_array(*[_dev_ptr(d, "dW") for d in dWs]) if dWs is not None else None
    wt_arr = (ctypes.c_float * n)(*[float(w) for w in weights]) if weights is not None else None
    with _OnDevice(X.device):
        st = lib().flce_multihead_fwd_bwd(_dev_ptr(X, "X"), w_arr, t_arr, wt_arr, n, BT, H, V,
                                          int(ignore_index), code, _dev_ptr(loss, "loss"),
                                          _dev_ptr(head_losses, "head_losses"), _dev_ptr(dX, "dX"),
                                          dw_arr, int(flags), _stream_handle(stream, X.device))
    _check(st, "flce_multihead_fwd_bwd")
    return loss, head_losses, dX, dWs


def flce_rmsnorm_fwd_bwd(h, gamma, eps, W, targets, ignore_index=-100, loss=None, dh=None,
                         dgamma=None, dW=None, flags=0, stream=None):
    """loss, dh, dgamma, dW of mean cross_entropy(rmsnorm(h; gamma, eps) @ W.T, targets)."""
    code = _dtype_code(h)
    if W.dtype != h.dtype or gamma.dtype != h.dtype:
        raise TypeError("h, gamma and W must have the same dtype")
    if h.dim() != 2 or W.dim() != 2 or h.shape[1] != W.shape[1] or gamma.shape != (h.shape[1],) \
            or targets.shape != (h.shape[0],):
        raise ValueError("expected h [BT, H], gamma [H], W [V, H], targets [BT]")
    if targets.dtype != torch.int64:
        raise TypeError("targets must be int64")
    BT, H = h.shape
    V = W.shape[0]
    if loss is None:
        loss = torch.empty((), dtype=torch.float32, device=h.device)
    if not (flags & SKIP_DX):
        dh = torch.empty_like(h) if dh is None else dh
        dgamma = torch.empty_like(gamma) if dgamma is None else dgamma
    if dW is None and not (flags & SKIP_DW):
        dW = torch.empty_like(W)
    for name, t, ref in (("dh", dh, h), ("dgamma", dgamma, gamma), ("dW", dW, W)):
        if t is not None and (t.shape != ref.shape or t.dtype != ref.dtype):
            raise ValueError(f"{name} must match its input in shape and dtype")
    with _OnDevice(h.device):
        st = lib().flce_rmsnorm_fwd_bwd(_dev_ptr(h, "h"), _dev_ptr(gamma, "gamma"), float(eps),
                                        _dev_ptr(W, "W"), _dev_ptr(targets, "targets"), BT, H, V,
                                        int(ignore_index), code, _dev_ptr(loss, "loss"),
                                        _dev_ptr(dh, "dh"), _dev_ptr(dgamma, "dgamma"),
                                        _dev_ptr(dW, "dW"), int(flags), _stream_handle(stream, h.device))
    _check(st, "flce_rmsnorm_fwd_bwd")
    return loss, dh, dgamma, dW


def flce_rmsnorm_workspace_bytes(BT, H, V, dtype) -> int:
    return int(lib().flce_rmsnorm_workspace_bytes(BT, H, V, _DTYPES.get(dtype, dtype)))


class FlceBlockNorm(ctypes.Structure):
    """flce_block_norm of include/flce.h."""
    _fields_ = [("size", ctypes.c_size_t), ("rows", ctypes.c_int64), ("H", ctypes.c_int64),
                ("dtype", ctypes.c_int), ("gate_act", ctypes.c_int), ("rows_per_gate", ctypes.c_int64),
                ("scale", ctypes.c_float), ("eps", ctypes.c_float)] + \
               [(ld, ctypes.c_int64) for ld in ("ldx", "ldy", "ldh", "ldn", "ldgate",
                                                "lddx", "lddy", "lddh", "lddn", "lddgate")] + \
               [("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


GATE_ACTS = ("linear", "sigmoid", "silu", "tanh")


def _refuse(t, name, like, shape):
    if t.device != like.device:
        raise ValueError(f"{name} must live on {like.device}")
    if t.dtype != like.dtype:
        raise TypeError(f"{name} must have dtype {like.dtype}")
    raise ValueError(f"{name} must be {tuple(shape)}")


def _rows_ptr(t, name, like, shape, dtype, index):
    """Pointer and row stride (0: dense) of a matrix whose rows may be apart, or of a vector; dtype, index: those of
    `like` and its device, asked for once."""
    if t is None:
        return None, 0
    if t.shape != shape or t.dtype is not dtype or t.get_device() != index:
        _refuse(t, name, like, shape)
    if t.is_contiguous():
        return t.data_ptr(), 0
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name} must have unit column stride")
    if t.dim() == 1 or t.shape[0] == 1:
        return t.data_ptr(), 0
    if t.stride(0) < t.shape[1]:
        raise ValueError(f"the rows of {name} must not overlap")
    return t.data_ptr(), t.stride(0)


def _gate_shape(gate, shape, rows_per_gate):
    if rows_per_gate < 0:
        raise ValueError("rows_per_gate must be 0 (one gate row for all) or positive")
    if gate is None:
        return shape
    return ((shape[0] + rows_per_gate - 1) // rows_per_gate, shape[1]) if rows_per_gate else shape[1:]


def _gate_act(kind) -> int:
    try:
        return GATE_ACTS.index(kind)
    except ValueError:
        raise ValueError(f"gate_act must be one of {GATE_ACTS}") from None


_BLOCK_NORM_BYTES = ctypes.sizeof(FlceBlockNorm)


def flce_block_norm_fwd(x, y=None, gamma_pre=None, gamma_post=None, gate=None, gate_act="linear", rows_per_gate=0,
                        scale=1.0, eps=1e-6, h=None, n=None, stream=None):
    """h = x + scale * a(gate) * z and n = rmsnorm(h; gamma_pre), z = y or rmsnorm(y; gamma_post).

    x, y [rows, H] (float32 or bfloat16; rows may be apart), gammas [H], gate [H] (rows_per_gate = 0) or
    [ceil(rows / rows_per_gate), H].  x may be None (no residual), y too (n alone).  Returns (h, n), None for
    what there is not; outputs are allocated when not passed, h may be x itself.
    """
    like = x if x is not None else y
    if like is None:
        raise ValueError("x or y is needed")
    if not like.is_cuda:
        raise ValueError("x and y must live on the GPU")
    shape = like.shape
    if len(shape) != 2:
        raise ValueError("expected [rows, H]")
    code, vec, device = _dtype_code(like), shape[1:], like.device
    dtype, index = like.dtype, device.index
    if y is not None and h is None:
        h = torch.empty_like(like)   # (dense, also where `like` is not; a third of the time of torch.empty)
    if gamma_pre is not None and n is None:
        n = torch.empty_like(like)
    px, ldx = _rows_ptr(x, "x", like, shape, dtype, index)
    py, ldy = _rows_ptr(y, "y", like, shape, dtype, index)
    pg, ldg = _rows_ptr(gate, "gate", like, _gate_shape(gate, shape, rows_per_gate), dtype, index)
    ph, ldh = _rows_ptr(h, "h", like, shape, dtype, index)
    pn, ldn = _rows_ptr(n, "n", like, shape, dtype, index)
    args = FlceBlockNorm(_BLOCK_NORM_BYTES, shape[0], shape[1], code, _gate_act(gate_act), int(rows_per_gate), scale, eps,
                         ldx, ldy, ldh, ldn, ldg)
    with _OnDevice(device):
        st = lib().flce_block_norm_fwd(px, py, pg, _rows_ptr(gamma_post, "gamma_post", like, vec, dtype, index)[0],
                                       _rows_ptr(gamma_pre, "gamma_pre", like, vec, dtype, index)[0], ctypes.byref(args), ph, pn,
                                       _stream_handle(stream, device))
    _check(st, "flce_block_norm_fwd")
    return h, n


def flce_block_norm_bwd(h=None, dn=None, dh=None, y=None, gamma_pre=None, gamma_post=None, gate=None,
                        gate_act="linear", rows_per_gate=0, scale=1.0, eps=1e-6, dx=None, dy=None, dgate=None,
                        dgamma_post=None, dgamma_pre=None, flags=0, workspace=None, stream=None):
    """Gradients of flce_block_norm_fwd from its h and y and the gradients dn of n, dh of h (None = zero).

    Returns (dx, dy, dgate, dgamma_post, dgamma_pre), None for what there is not.  Outputs are allocated when
    not passed; dx may be dh itself, and without gamma_pre it is dh (nothing is computed for it).
    flags: SKIP_DX leaves dx out, SKIP_DW the gradients of the gammas and the gate.
    """
    like = dn if dn is not None else dh
    if like is None:
        raise ValueError("dn or dh is needed")
    if not like.is_cuda:
        raise ValueError("dn and dh must live on the GPU")
    if flags & ~(SKIP_DX | SKIP_DW):
        raise ValueError("unknown flags")
    shape = like.shape
    if len(shape) != 2:
        raise ValueError("expected [rows, H]")
    code, vec, device = _dtype_code(like), shape[1:], like.device
    dtype, index = like.dtype, device.index
    gshape = _gate_shape(gate, shape, rows_per_gate)
    want_dx, want_dw = not flags & SKIP_DX, not flags & SKIP_DW
    passed_on = want_dx and gamma_pre is None and dx is None
    if passed_on and y is None:
        raise ValueError("without y and gamma_pre there is nothing to compute")

    def output(given, of, wanted, name, size):   # of: the input it is the gradient of
        if of is None and given is not None:
            raise ValueError(f"{name} is the gradient of an input that is not there")
        if of is None or not wanted:
            return None, None, 0
        if given is None:
            given = torch.empty_like(of)
            return given, given.data_ptr(), 0
        return given, *_rows_ptr(given, name, like, size, dtype, index)

    dx, pdx, lddx = output(dx, like, want_dx and not passed_on, "dx", shape)
    dy, pdy, lddy = output(dy, y, True, "dy", shape)
    dgate, pdg, lddg = output(dgate, gate, want_dw, "dgate", gshape)
    dgamma_post, pdpost, _ = output(dgamma_post, gamma_post, want_dw, "dgamma_post", vec)
    dgamma_pre, pdpre, _ = output(dgamma_pre, gamma_pre, want_dw, "dgamma_pre", vec)
    ph, ldh = _rows_ptr(h, "h", like, shape, dtype, index)
    pdn, lddn = _rows_ptr(dn, "dn", like, shape, dtype, index)
    pdh, lddh = _rows_ptr(dh, "dh", like, shape, dtype, index)
    py, ldy = _rows_ptr(y, "y", like, shape, dtype, index)
    pg, ldg = _rows_ptr(gate, "gate", like, gshape, dtype, index)
    args = FlceBlockNorm(_BLOCK_NORM_BYTES, shape[0], shape[1], code, _gate_act(gate_act), int(rows_per_gate), scale, eps,
                         0, ldy, ldh, 0, ldg, lddx, lddy, lddh, lddn, lddg, *_workspace_args(workspace, device))
    with _OnDevice(device):
        st = lib().flce_block_norm_bwd(ph, pdn, pdh, py, pg, _rows_ptr(gamma_post, "gamma_post", like, vec, dtype, index)[0],
                                       _rows_ptr(gamma_pre, "gamma_pre", like, vec, dtype, index)[0], ctypes.byref(args), pdx, pdy, pdg,
                                       pdpost, pdpre, _stream_handle(stream, device))
    _check(st, "flce_block_norm_bwd")
    return dh if passed_on else dx, dy, dgate, dgamma_post, dgamma_pre


def flce_block_norm_workspace_bytes(rows, H, dtype, rows_per_gate=0) -> int:
    """Bytes flce_block_norm_bwd uses at most for this shape (with both gammas and a gate)."""
    b = FlceBlockNorm()
    b.size, b.rows, b.H, b.dtype = ctypes.sizeof(FlceBlockNorm), rows, H, _DTYPES.get(dtype, dtype)
    b.rows_per_gate = rows_per_gate
    return int(lib().flce_block_norm_workspace_bytes(ctypes.byref(b)))


def flce_grad_norm_workspace_bytes(n_tensors) -> int:
    """Bytes flce_grad_norm and flce_clip_grad_norm use for a list of that many tensors."""
    return int(lib().flce_grad_norm_workspace_bytes(int(n_tensors)))


NORM_TYPES = {2.0: 0, float("inf"): 1}


def _tensor_list(grads):
    """(device, host arrays of pointers, element counts and dtypes) of a list of dense tensors on one GPU.
    (Attribute by attribute over the whole list: a call over 300 tensors spends most of its time here.)"""
    T = torch.Tensor
    if not grads:
        return None, None, None, None
    device = grads[0].device
    index = device.index if device.type == "cuda" else -1
    if index < 0 or any(map(index.__ne__, map(T.get_device, grads))):
        raise ValueError("every tensor must live on the same GPU")
    if not all(map(T.is_contiguous, grads)):
        raise ValueError("every tensor must be contiguous")
    try:
        dtypes = array.array("i", map(_DTYPES.__getitem__, map(T.dtype.__get__, grads)))
    except KeyError as e:
        raise TypeError(f"unsupported dtype {e.args[0]}; use float32 or bfloat16") from None
    return device, array.array("Q", map(T.data_ptr, grads)), array.array("q", map(T.numel, grads)), dtypes


def _at(a):
    """The address of an array's elements."""
    return a.buffer_info()[0] if a is not None else None


def _norm_out(norm, device):
    if norm is None:
        if device is None:
            raise ValueError("an empty list needs `norm`")
        return torch.empty((), dtype=torch.float32, device=device)
    if norm.dtype != torch.float32 or norm.numel() != 1 or not norm.is_cuda or device not in (None, norm.device):
        raise ValueError("norm must be one float32 value on the tensors' GPU")
    return norm


def _norm_type(norm_type) -> int:
    try:
        return NORM_TYPES[float(norm_type)]
    except KeyError:
        raise ValueError("norm_type must be 2 or inf") from None


def _out_list(outs, device, counts, dtypes):
    if outs is None:
        return None
    outs = list(outs)
    out_device, ptrs, out_counts, out_dtypes = _tensor_list(outs)
    if (out_device, out_counts, out_dtypes) != (device, counts, dtypes):
        raise ValueError("outs must hold one tensor per gradient, of its size and dtype and on its GPU")
    return ptrs


def _workspace_args(workspace, device):
    if workspace is None:
        return None, 0
    if workspace.device != device:
        raise ValueError(f"workspace must live on {device}")
    return _dev_ptr(workspace, "workspace"), workspace.numel() * workspace.element_size()


def flce_grad_norm(grads, norm_type=2.0, norm=None, workspace=None, stream=None):
    """Norm (2 or inf) over all elements of a list of tensors (float32 and bfloat16 mixed): one float32 on the GPU."""
    grads = list(grads)
    device, ptrs, counts, dtypes = _tensor_list(grads)
    norm = _norm_out(norm, device)
    with _OnDevice(norm.device):
        st = lib().flce_grad_norm(_at(ptrs), _at(counts), _at(dtypes), len(grads), _norm_type(norm_type), norm.data_ptr(),
                                  *_workspace_args(workspace, norm.device), _stream_handle(stream, norm.device))
    _check(st, "flce_grad_norm")
    return norm


def flce_grad_clip(grads, norm, max_norm, outs=None, stream=None):
    """Scales a list of tensors by min(1, max_norm / (norm + 1e-6)), in place or into `outs`; norm: one float32 on
    the GPU, e.g. over all shards of a model."""
    if norm is None:   # (_norm_out makes one for the calls that write it)
        raise ValueError("norm must be one float32 value on the tensors' GPU")
    grads = list(grads)
    device, ptrs, counts, dtypes = _tensor_list(grads)
    norm = _norm_out(norm, device)
    to = _out_list(outs, device, counts, dtypes)
    with _OnDevice(norm.device):
        st = lib().flce_grad_clip(_at(ptrs), _at(to), _at(counts), _at(dtypes), len(grads), norm.data_ptr(),
                                  float(max_norm), _stream_handle(stream, norm.device))
    _check(st, "flce_grad_clip")


def flce_clip_grad_norm(grads, max_norm, norm_type=2.0, outs=None, norm=None, workspace=None, stream=None):
    """flce_grad_norm, then flce_grad_clip by it; returns the norm before clipping (one float32 on the GPU)."""
    grads = list(grads)
    device, ptrs, counts, dtypes = _tensor_list(grads)
    norm = _norm_out(norm, device)
    to = _out_list(outs, device, counts, dtypes)
    with _OnDevice(norm.device):
        st = lib().flce_clip_grad_norm(_at(ptrs), _at(to), _at(counts), _at(dtypes), len(grads),
                                       _norm_type(norm_type), float(max_norm), norm.data_ptr(),
                                       *_workspace_args(workspace, norm.device), _stream_handle(stream, norm.device))
    _check(st, "flce_clip_grad_norm")
    return norm


class FlceLayerNorm(ctypes.Structure):
    """flce_layer_norm of include/flce.h."""
    _fields_ = [("size", ctypes.c_size_t), ("rows", ctypes.c_int64), ("H", ctypes.c_int64), ("dtype", ctypes.c_int),
                ("eps", ctypes.c_float)] + \
               [(ld, ctypes.c_int64) for ld in ("ldx", "ldy", "ldh", "ldn", "lddx", "lddh", "lddn")] + \
               [("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


_LAYER_NORM_BYTES = ctypes.sizeof(FlceLayerNorm)


def flce_layer_norm_fwd(x, y=None, gamma=None, beta=None, eps=1e-5, h=None, n=None, stream=None):
    """h = x + y and n = (h - mean) / sqrt(var + eps) * gamma + beta, row by row.

    x, y [rows, H] (float32 or bfloat16; rows may be apart), gamma, beta [H] or None.  Returns (h, n), h None without
    y; outputs are allocated when not passed, h may be x itself.
    """
    if not x.is_cuda:
        raise ValueError("x must live on the GPU")
    shape = x.shape
    if len(shape) != 2:
        raise ValueError("expected [rows, H]")
    code, vec, device = _dtype_code(x), shape[1:], x.device
    dtype, index = x.dtype, device.index
    if y is not None and h is None:
        h = torch.empty_like(x)
    if n is None:
        n = torch.empty_like(x)
    px, ldx = _rows_ptr(x, "x", x, shape, dtype, index)
    py, ldy = _rows_ptr(y, "y", x, shape, dtype, index)
    ph, ldh = _rows_ptr(h, "h", x, shape, dtype, index)
    pn, ldn = _rows_ptr(n, "n", x, shape, dtype, index)
    args = FlceLayerNorm(_LAYER_NORM_BYTES, shape[0], shape[1], code, eps, ldx, ldy, ldh, ldn)
    with _OnDevice(device):
        st = lib().flce_layer_norm_fwd(px, py, _rows_ptr(gamma, "gamma", x, vec, dtype, index)[0],
                                       _rows_ptr(beta, "beta", x, vec, dtype, index)[0], ctypes.byref(args), ph, pn,
                                       _stream_handle(stream, device))
    _check(st, "flce_layer_norm_fwd")
    return h, n


def flce_layer_norm_bwd(h, dn, dh=None, gamma=None, bias=True, eps=1e-5, dx=None, dgamma=None, dbeta=None, flags=0,
                        workspace=None, stream=None):
    """Gradients of flce_layer_norm_fwd from its h (x where there was no y) and the gradients dn of n, dh of h (None =
    zero).  bias: the forward had a beta.

    Returns (dx, dgamma, dbeta), None for what there is not.  Outputs are allocated when not passed; dx may be dh
    itself.  flags: SKIP_DX leaves dx out, SKIP_DW the gradients of gamma and beta.
    """
    if not h.is_cuda:
        raise ValueError("h must live on the GPU")
    if flags & ~(SKIP_DX | SKIP_DW):
        raise ValueError("unknown flags")
    shape = h.shape
    if len(shape) != 2:
        raise ValueError("expected [rows, H]")
    code, vec, device = _dtype_code(h), shape[1:], h.device
    dtype, index = h.dtype, device.index
    want_dw = not flags & SKIP_DW
    if (gamma is None and dgamma is not None) or (not bias and dbeta is not None):
        raise ValueError("the gradient of an input that is not there")

    def output(given, wanted, name, size):
        if not wanted:
            return None, None, 0
        if given is None:
            given = torch.empty(size, dtype=dtype, device=device) if len(size) == 1 else torch.empty_like(h)
            return given, given.data_ptr(), 0
        return given, *_rows_ptr(given, name, h, size, dtype, index)

    dx, pdx, lddx = output(dx, not flags & SKIP_DX, "dx", shape)
    dgamma, pdg, _ = output(dgamma, gamma is not None and want_dw, "dgamma", vec)
    dbeta, pdb, _ = output(dbeta, bias and want_dw, "dbeta", vec)
    ph, ldh = _rows_ptr(h, "h", h, shape, dtype, index)
    pdn, lddn = _rows_ptr(dn, "dn", h, shape, dtype, index)
    pdh, lddh = _rows_ptr(dh, "dh", h, shape, dtype, index)
    args = FlceLayerNorm(_LAYER_NORM_BYTES, shape[0], shape[1], code, eps, 0, 0, ldh, 0, lddx, lddh, lddn,
                         *_workspace_args(workspace, device))
    with _OnDevice(device):
        st = lib().flce_layer_norm_bwd(ph, pdn, pdh, _rows_ptr(gamma, "gamma", h, vec, dtype, index)[0], ctypes.byref(args),
                                       pdx, pdg, pdb, _stream_handle(stream, device))
    _check(st, "flce_layer_norm_bwd")
    return dx, dgamma, dbeta


def flce_layer_norm_workspace_bytes(rows, H, dtype) -> int:
    """Bytes flce_layer_norm_bwd uses at most for this shape."""
    b = FlceLayerNorm(size=_LAYER_NORM_BYTES, rows=rows, H=H, dtype=_DTYPES.get(dtype, dtype))
    return int(lib().flce_layer_norm_workspace_bytes(ctypes.byref(b)))


class FlceOrthogonalizeArgs(ctypes.Structure):
    """flce_orthogonalize_args of include/flce.h."""
    _fields_ = [("size", ctypes.c_size_t), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("dtype", ctypes.c_int),
                ("steps", ctypes.c_int), ("coefficients", ctypes.c_void_p), ("per_step", ctypes.c_int),
                ("scale", ctypes.c_float), ("eps", ctypes.c_float), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t)]


def _orthogonalize_args(rows, cols, code, steps, coefficients, scale, eps) -> FlceOrthogonalizeArgs:
    args = FlceOrthogonalizeArgs(ctypes.sizeof(FlceOrthogonalizeArgs), rows, cols, code, steps, None, 0, scale, eps)
    if coefficients is not None:
        triples = coefficients.tolist() if hasattr(coefficients, "tolist") else list(coefficients)   # (tensors, arrays)
        args.per_step = 1 if triples and hasattr(triples[0], "__len__") else 0
        flat = [float(x) for t in triples for x in t] if args.per_step else [float(x) for x in triples]
        if len(flat) != 3 * (steps if args.per_step else 1):
            raise ValueError("coefficients must be three numbers, or three for each step")
        args._coefficients = (ctypes.c_float * len(flat))(*flat)   # (kept alive by the struct)
        args.coefficients = ctypes.addressof(args._coefficients)
    return args


def flce_orthogonalize(updates, outs=None, steps=5, coefficients=None, scale=1.0, eps=1e-7, workspace=None, stream=None):
    """scale * (each matrix of the list with its singular values driven towards 1 by `steps` Newton-Schulz steps).

    updates: dense [rows, cols] tensors of one shape and dtype (float32 or bfloat16) on one GPU; outs: as many, or
    None for in place.  coefficients: (a, b, c), a triple for each step, or None for (3.4445, -4.7750, 2.0315).
    Returns outs.
    """
    updates = list(updates)
    if not updates:
        return []
    first = updates[0]
    if first.dim() != 2 or any(t.shape != first.shape or t.dtype != first.dtype for t in updates):
        raise ValueError("updates must be matrices of one shape and dtype")
    outs = updates if outs is None else list(outs)
    if any(t.shape != first.shape for t in outs):
        raise ValueError("outs must hold one tensor per update, of its size and dtype and on its GPU")
    device, ptrs, counts, dtypes = _tensor_list(updates)
    to = None if outs is updates else _out_list(outs, device, counts, dtypes)
    args = _orthogonalize_args(first.shape[0], first.shape[1], _dtype_code(first), int(steps), coefficients, scale, eps)
    args.workspace, args.workspace_bytes = _workspace_args(workspace, device)
    with _OnDevice(device):
        st = lib().flce_orthogonalize(_at(ptrs), _at(to), len(updates), ctypes.byref(args), _stream_handle(stream, device))
    _check(st, "flce_orthogonalize")
    return outs


def flce_orthogonalize_workspace_bytes(n_matrices, rows, cols, dtype) -> int:
    """Bytes flce_orthogonalize uses at most for a list of that many matrices."""
    args = _orthogonalize_args(rows, cols, _DTYPES.get(dtype, dtype), 1, None, 1.0, 0.0)
    return int(lib().flce_orthogonalize_workspace_bytes(int(n_matrices), ctypes.byref(args)))


class FlceEmbedding(ctypes.Structure):
    """flce_embedding of include/flce.h."""
    _fields_ = [("size", ctypes.c_size_t), ("rows", ctypes.c_int64), ("V", ctypes.c_int64), ("H", ctypes.c_int64),
                ("dtype", ctypes.c_int), ("accumulate", ctypes.c_int), ("first_token", ctypes.c_int64),
                ("ignore_index", ctypes.c_int64), ("scale", ctypes.c_float), ("ldtable", ctypes.c_int64),
                ("ldrows", ctypes.c_int64), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


_EMBEDDING_BYTES = ctypes.sizeof(FlceEmbedding)


def _tokens_ptr(tokens, device):
    if tokens.dtype != torch.int64:
        raise TypeError("tokens must be int64")
    if tokens.device != device:
        raise ValueError(f"tokens must live on {device}")
    return _dev_ptr(tokens, "tokens")


def flce_embedding_fwd(table, tokens, scale=1.0, ignore_index=-100, first_token=0, out=None, stream=None):
    """out[i] = scale * table[tokens[i] - first_token]; zeros where that is no row of the table or ignore_index.

    table [V, H] (float32 or bfloat16; rows may be apart), tokens int64 of any shape.  Returns out
    [*tokens.shape, H]; where it is passed: [tokens.numel(), H], rows may be apart.
    """
    code = _dtype_code(table)
    if table.dim() != 2 or not table.is_cuda:
        raise ValueError("expected table [V, H] on the GPU")
    V, H = table.shape
    rows, device = tokens.numel(), table.device
    pt = _tokens_ptr(tokens, device)
    ptab, ldt = _rows_ptr(table, "table", table, table.shape, table.dtype, device.index)
    if out is None:
        out = torch.empty((*tokens.shape, H), dtype=table.dtype, device=device)
        po, ldo = out.data_ptr(), 0
    else:
        po, ldo = _rows_ptr(out, "out", table, (rows, H), table.dtype, device.index)
    args = FlceEmbedding(_EMBEDDING_BYTES, rows, V, H, code, 0, first_token, ignore_index, scale, ldt, ldo)
    with _OnDevice(device):
        st = lib().flce_embedding_fwd(ptab, pt, ctypes.byref(args), po, _stream_handle(stream, device))
    _check(st, "flce_embedding_fwd")
    return out


def flce_embedding_bwd(dout, tokens, V, scale=1.0, ignore_index=-100, first_token=0, dtable=None, accumulate=False,
                       workspace=None, stream=None):
    """Gradient [V, H] of flce_embedding_fwd's table from dout [tokens.numel(), H] (rows may be apart) or
    [*tokens.shape, H] (dense).  accumulate: it is added to what dtable holds (the head's dW, where both share the
    matrix)."""
    code = _dtype_code(dout)
    if not dout.is_cuda or dout.dim() < 2:
        raise ValueError("expected dout [rows, H] on the GPU")
    rows, H, device = tokens.numel(), dout.shape[-1], dout.device
    pt = _tokens_ptr(tokens, device)
    if dout.dim() > 2 or tokens.dim() != 1:
        if dout.shape != (*tokens.shape, H) and dout.shape != (rows, H):
            raise ValueError("expected dout [*tokens.shape, H]")
        dout = dout.view(rows, H)
    pd, ldd = _rows_ptr(dout, "dout", dout, (rows, H), dout.dtype, device.index)
    if dtable is None:
        if accumulate:
            raise ValueError("accumulate needs dtable")
        dtable = torch.empty((V, H), dtype=dout.dtype, device=device)
    pg, ldg = _rows_ptr(dtable, "dtable", dout, (V, H), dout.dtype, device.index)
    args = FlceEmbedding(_EMBEDDING_BYTES, rows, V, H, code, 1 if accumulate else 0, first_token, ignore_index, scale, ldg, ldd,
                         *_workspace_args(workspace, device))
    with _OnDevice(device):
        st = lib().flce_embedding_bwd(pd, pt, ctypes.byref(args), pg, _stream_handle(stream, device))
    _check(st, "flce_embedding_bwd")
    return dtable


def flce_embedding_workspace_bytes(rows, V, H, dtype) -> int:
    """Bytes of scratch flce_embedding_bwd uses for this shape."""
    b = FlceEmbedding(size=_EMBEDDING_BYTES, rows=rows, V=V, H=H, dtype=_DTYPES.get(dtype, dtype))
    return int(lib().flce_embedding_workspace_bytes(ctypes.byref(b)))


CE_NOALLOC_MAX_ROWS = 65536


def flce_cross_entropy_inplace(Z, targets, ignore_index=-100, loss=None, stream=None, noalloc=False):
    """Replaces logits Z [BT, V] (row stride Z.stride(0)) by dL/dZ; returns the mean loss.
    noalloc=True calls flce_cross_entropy_inplace_noalloc (pass `loss`: this wrapper
    would otherwise allocate it)."""
    code = _dtype_code(Z)
    if Z.dim() != 2 or Z.stride(1) != 1 or targets.shape != (Z.shape[0],):
        raise ValueError("expected Z [BT, V] with unit column stride, targets [BT]")
    if targets.dtype != torch.int64 or not Z.is_cuda:
        raise TypeError("targets must be int64 and Z on the GPU")
    BT, V = Z.shape
    if loss is None:
        loss = torch.empty((), dtype=torch.float32, device=Z.device)
    with _OnDevice(Z.device):
        fn = lib().flce_cross_entropy_inplace_noalloc if noalloc else lib().flce_cross_entropy_inplace
        st = fn(Z.data_ptr(), _dev_ptr(targets, "targets"), BT, V,
                Z.stride(0) if BT > 1 else max(V, Z.stride(0)), int(ignore_index), code,
                _dev_ptr(loss, "loss"), _stream_handle(stream, Z.device))
    _check(st, "flce_cross_entropy_inplace_noalloc" if noalloc else "flce_cross_entropy_inplace")
    return loss


def flce_cross_entropy_inplace_noalloc(Z, targets, ignore_index=-100, loss=None, stream=None):
    return flce_cross_entropy_inplace(Z, targets, ignore_index, loss, stream, noalloc=True)


def flce_workspace_bytes(BT, H, V, dtype) -> int:
    return int(lib().flce_workspace_bytes(BT, H, V, _DTYPES.get(dtype, dtype)))


def flce_workspace_bytes_max(H, V, dtype) -> int:
    return int(lib().flce_workspace_bytes_max(H, V, _DTYPES.get(dtype, dtype)))


def flce_set_workspace(ws: torch.Tensor | None):
    if ws is None:
        _check(lib().flce_set_workspace(None, 0), "flce_set_workspace")
    else:
        with _OnDevice(ws.device):
            _check(lib().flce_set_workspace(ws.data_ptr(), ws.numel() * ws.element_size()),
                   "flce_set_workspace")


def flce_release_workspace():
    _check(lib().flce_release_workspace(), "flce_release_workspace")


def flce_set_logits_budget_bytes(n: int):
    _check(lib().flce_set_logits_budget_bytes(int(n)), "flce_set_logits_budget_bytes")


def flce_get_logits_budget_bytes() -> int:
    return int(lib().flce_get_logits_budget_bytes())


def flce_set_row_compaction(on: bool):
    _check(lib().flce_set_row_compaction(1 if on else 0), "flce_set_row_compaction")


def flce_get_row_compaction() -> bool:
    return bool(lib().flce_get_row_compaction())


def flce_logits_budget_for_workspace(BT, H, V, dtype, max_workspace_bytes) -> int:
    return int(lib().flce_logits_budget_for_workspace(BT, H, V, _DTYPES.get(dtype, dtype), int(max_workspace_bytes)))


def flce_chunk_rows(BT, H, V, dtype) -> int:
    return int(lib().flce_chunk_rows(BT, H, V, _DTYPES.get(dtype, dtype)))


def flce_num_chunks(BT, H, V, dtype) -> int:
    return int(lib().flce_num_chunks(BT, H, V, _DTYPES.get(dtype, dtype)))


def flce_dx_k_ranges(BT, H, V, dtype) -> int:
    return int(lib().flce_dx_k_ranges(BT, H, V, _DTYPES.get(dtype, dtype)))


def flce_paper_chunk_rows(BT, H, V) -> int:
    return int(lib().flce_paper_chunk_rows(BT, H, V))


def flce_full_logits_bytes(BT, V, dtype) -> int:
    return int(lib().flce_full_logits_bytes(BT, V, _DTYPES.get(dtype, dtype)))


KERNEL_KINDS = ("logits_gemm", "ce_rows", "dx_gemm", "dw_gemm", "other")


def flce_mfma_ceiling_launch(pattern: int, workgroups: int, iters: int, std_b: float, out, stream=None):
    """Enqueues the MFMA-only loop (see include/flce.h); `out` is a float32 CUDA tensor
    of at least workgroups * 256 elements.  Returns the flops of the launch."""
    if out.dtype != torch.float32 or not out.is_cuda or not out.is_contiguous():
        raise ValueError("out must be a contiguous float32 CUDA tensor")
    here = torch.device("cuda", torch.cuda.current_device())
    _check(lib().flce_mfma_ceiling_launch(int(pattern), int(workgroups), int(iters), float(std_b),
                                          out.data_ptr(), out.numel(), _stream_handle(stream, here)),
           "flce_mfma_ceiling_launch")
    return workgroups * 4 * iters * 16 * 32768.0


def flce_timing_enable(on: bool):
    _check(lib().flce_timing_enable(1 if on else 0), "flce_timing_enable")


def flce_timing_collect() -> dict:
    """{kind: (total_ms, launches)} of the launches recorded since the last collect."""
    n = len(KERNEL_KINDS)
    ms = (ctypes.c_double * n)()
    cnt = (ctypes.c_int64 * n)()
    _check(lib().flce_timing_collect(ctypes.addressof(ms), ctypes.addressof(cnt)), "flce_timing_collect")
    return {k: (float(ms[i]), int(cnt[i])) for i, k in enumerate(KERNEL_KINDS)}
