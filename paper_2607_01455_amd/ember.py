"""Python binding of libember.so: argument marshalling only.

Each function has the name of the C entry point it calls (include/ember.h) and
passes torch tensors as raw device pointers plus sizes, on the current torch
stream.  Every step of the Ember update runs in the library's HIP kernels;
there is no other implementation here.  Importing this module fails loudly if
the library has not been built.
"""
from __future__ import annotations

import ctypes
import os

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libember.so")

EMBER_F32 = 0
EMBER_BF16 = 1

EMBER_OK = 0
EMBER_ERR_ARG = -1
EMBER_ERR_SHAPE = -2
EMBER_ERR_ALIGN = -3
EMBER_ERR_DTYPE = -4
EMBER_ERR_WORKSPACE = -5
EMBER_ERR_INDEX = -6
EMBER_ERR_HIP = -7
EMBER_ERR_DEVICE = -8

# Every function the C header declares, checked by the CPU test suite.
EXPORTED = ("ember_workspace_bytes", "ember_init_state", "ember_step_dense",
            "ember_step_sparse_rows", "ember_rowonly_init_state", "ember_rowonly_step_dense",
            "ember_rowonly_step_sparse_rows", "ember_step_sparse_rows_devn",
            "ember_rowonly_step_sparse_rows_devn", "ember_coalesce_workspace_bytes", "ember_coalesce_rows",
            "ember_lmhead_step", "ember_rmsnorm", "ember_rmsnorm_grad_workspace_bytes", "ember_rmsnorm_grad",
            "ember_quantize_rows", "ember_logits_q8", "ember_quantize_rows_q4", "ember_rows_q4", "ember_logits_q4",
            "ember_sample_workspace_bytes", "ember_sample", "ember_clip_workspace_bytes", "ember_clip_grads",
            "ember_step_multi", "ember_get_error", "ember_strerror",
            "ember_profile_enable", "ember_profile_collect", "ember_stream_probe",
            "ember_set_barrier_wait_ticks",
            "ember_step_sparse_rows_static")


class EmberError(RuntimeError):
    def __init__(self, status: int, where: str):
        super().__init__(f"{where}: {ember_strerror(status)} (status {status})")
        self.status = status


EMBER_MAX_TABLES = 8


class TableStep(ctypes.Structure):
    """One table of ember_step_multi (the C struct ember_table_step)."""
    _fields_ = [("W", ctypes.c_void_p), ("w_dtype", ctypes.c_int), ("ldw", ctypes.c_int64),
                ("G", ctypes.c_void_p), ("g_dtype", ctypes.c_int), ("ldg", ctypes.c_int64),
                ("sparse", ctypes.c_int), ("row_only", ctypes.c_int), ("idx", ctypes.c_void_p),
                ("n_idx", ctypes.c_int64),
                ("n_idx_dev", ctypes.c_void_p), ("r", ctypes.c_void_p), ("c", ctypes.c_void_p),
                ("V", ctypes.c_int64), ("D", ctypes.c_int64), ("t", ctypes.c_int64),
                ("lr", ctypes.c_float), ("beta2", ctypes.c_float), ("eps", ctypes.c_float),
                ("maximize", ctypes.c_int), ("ws", ctypes.c_void_p), ("ws_bytes", ctypes.c_size_t)]


class Grad(ctypes.Structure):
    """One tensor of ember_clip_grads (the C struct ember_grad)."""
    _fields_ = [("src", ctypes.c_void_p), ("src_dtype", ctypes.c_int), ("lds", ctypes.c_int64),
                ("dst", ctypes.c_void_p), ("dst_dtype", ctypes.c_int), ("ldd", ctypes.c_int64),
                ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("rows_dev", ctypes.c_void_p)]


class _KernelStat(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char_p), ("launches", ctypes.c_int64), ("total_ms", ctypes.c_double)]


def _load(path: str = _LIB_PATH) -> ctypes.CDLL:
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with `python -m paper_2607_01455_amd.build`")
    lib = ctypes.CDLL(path)
    vp, i64, f32, i32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_float, ctypes.c_int, ctypes.c_size_t
    lib.ember_workspace_bytes.argtypes = [i64, i64, ctypes.POINTER(sz)]
    lib.ember_init_state.argtypes = [vp, vp, i64, i64, vp, sz, vp]
    lib.ember_step_dense.argtypes = [vp, i32, i64, vp, i32, i64, vp, vp, i64, i64, i64,
                                     f32, f32, f32, i32, vp, sz, vp]
    lib.ember_step_sparse_rows.argtypes = [vp, i32, i64, vp, i32, i64, vp, i64, vp, vp, i64, i64, i64,
                                           f32, f32, f32, i32, vp, sz, vp]
    lib.ember_rowonly_init_state.argtypes = [vp, i64, i64, vp, sz, vp]
    lib.ember_rowonly_step_dense.argtypes = [vp, i32, i64, vp, i32, i64, vp, i64, i64, i64,
                                             f32, f32, f32, i32, vp, sz, vp]
    lib.ember_rowonly_step_sparse_rows.argtypes = [vp, i32, i64, vp, i32, i64, vp, i64, vp, i64, i64, i64,
                                                   f32, f32, f32, i32, vp, sz, vp]
    lib.ember_step_sparse_rows_devn.argtypes = [vp, i32, i64, vp, i32, i64, vp, vp, i64, vp, vp, i64, i64, i64,
                                                f32, f32, f32, i32, vp, sz, vp]
    lib.ember_rowonly_step_sparse_rows_devn.argtypes = [vp, i32, i64, vp, i32, i64, vp, vp, i64, vp, i64, i64,
                                                        i64, f32, f32, f32, i32, vp, sz, vp]
    lib.ember_coalesce_workspace_bytes.argtypes = [i64, i64, i64, ctypes.POINTER(sz)]
    lib.ember_coalesce_rows.argtypes = [vp, i64, vp, i32, i64, i64, i64, vp, vp, i32, i64, vp, vp, sz, vp]
    lib.ember_lmhead_step.argtypes = [vp, i32, i64, vp, i64, vp, i64, i64, vp, i32, i64, vp, vp, i64, i64, i64,
                                      f32, f32, f32, i32, vp, sz, vp]
    lib.ember_rmsnorm.argtypes = [vp, i32, i64, vp, i64, vp, i32, f32, i64, i64, vp, i64, vp, i32, i64, vp, i64,
                                  vp, vp, vp]
    lib.ember_rmsnorm_grad_workspace_bytes.argtypes = [i64, i64, ctypes.POINTER(sz)]
    lib.ember_rmsnorm_grad.argtypes = [vp, i64, vp, i32, i64, vp, i32, vp, vp, i64, i64, i64, vp, i64, vp, vp, sz, vp]
    lib.ember_quantize_rows.argtypes = [vp, i32, i64, i64, i64, vp, i64, vp, vp]
    lib.ember_logits_q8.argtypes = [vp, i64, vp, vp, i64, vp, vp, i64, i64, i64, vp, i32, i64, vp]
    lib.ember_quantize_rows_q4.argtypes = [vp, i32, i64, i64, i64, i32, vp, i64, vp, i64, vp]
    lib.ember_rows_q4.argtypes = [vp, i64, vp, i64, i32, i64, i64, vp, i64, vp, i32, i64, vp]
    lib.ember_logits_q4.argtypes = [vp, i64, vp, vp, i64, vp, i64, i32, vp, i64, i64, i64, vp, i32, i64, vp]
    lib.ember_sample_workspace_bytes.argtypes = [i64, i64, ctypes.POINTER(sz)]
    lib.ember_sample.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.ember_clip_workspace_bytes.argtypes = [i64, ctypes.POINTER(sz)]
    lib.ember_clip_grads.argtypes = [ctypes.POINTER(Grad), i64, f32, vp, vp, sz, vp]
    lib.ember_step_multi.argtypes = [ctypes.POINTER(TableStep), i32, vp]
    lib.ember_get_error.argtypes = [vp, vp, ctypes.POINTER(i32)]
    lib.ember_strerror.argtypes = [i32]
    lib.ember_strerror.restype = ctypes.c_char_p
    lib.ember_profile_enable.argtypes = [i32]
    lib.ember_set_barrier_wait_ticks.argtypes = [ctypes.c_int64]
    lib.ember_profile_collect.argtypes = [ctypes.POINTER(_KernelStat), i32, ctypes.POINTER(i32)]
    lib.ember_stream_probe.argtypes = [i32, vp, vp, vp, sz, vp]
    lib.ember_step_sparse_rows_static.argtypes = [vp, i32, i64, vp, i32, i64, vp, i64, vp, vp, i64, i64, i64,
                                                  f32, f32, f32, i32, vp, vp]
    for name in EXPORTED:
        if name != "ember_strerror":
            getattr(lib, name).restype = i32
    return lib


LIB = _load()


_DTYPES = {torch.float32: EMBER_F32, torch.bfloat16: EMBER_BF16}
_CHUNK = {torch.float32: 4, torch.bfloat16: 8, torch.int8: 16, torch.uint8: 16}   # elements of 16 bytes


def _dtype(t: torch.Tensor) -> int:
    return _DTYPES.get(t.dtype, 99)  # 99: rejected by the library with EMBER_ERR_DTYPE


def _ld(t: torch.Tensor) -> int:
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or (shape[1] > 1 and stride[1] != 1):
        raise TypeError("a 2-D tensor with unit column stride is required")
    if shape[0] > 1:
        return stride[0]
    # one row: the stride is never used to address a second row; give the
    # smallest one that keeps the library's 16-byte row rule
    q = max(1, 16 // t.element_size())
    return (shape[1] + q - 1) // q * q


def _ptr(t):
    return None if t is None or t.numel() == 0 else t.data_ptr()


def _stream(t: torch.Tensor):
    """Handle of the current stream of t's device: what
    torch.cuda.current_stream(t.device).cuda_stream gives, by torch's raw query
    (not part of its public interface), which takes 0.2 us; making a Stream
    object for it takes 1.9 us of a small step's ~15."""
    if not t.is_cuda:
        return torch.cuda.current_stream(t.device).cuda_stream   # refuses a host tensor
    return torch._C._cuda_getCurrentRawStream(t.get_device())


def _check(status: int, where: str) -> None:
    if status != EMBER_OK:
        raise EmberError(status, where)


def ember_strerror(status: int) -> str:
    return LIB.ember_strerror(int(status)).decode()


def ember_workspace_bytes(V: int, D: int) -> int:
    out = ctypes.c_size_t(0)
    _check(LIB.ember_workspace_bytes(int(V), int(D), ctypes.byref(out)), "ember_workspace_bytes")
    return out.value


def ember_init_state(r: torch.Tensor, c: torch.Tensor, ws: torch.Tensor) -> None:
    _check(LIB.ember_init_state(_ptr(r), _ptr(c), r.numel(), c.numel(), _ptr(ws),
                                ws.numel() * ws.element_size(), _stream(r)), "ember_init_state")


def ember_step_dense(W: torch.Tensor, G: torch.Tensor, r: torch.Tensor, c: torch.Tensor, t: int,
                     lr: float = 1e-3, beta2: float = 0.999, eps: float = 1e-8,
                     maximize: bool = False, ws: torch.Tensor | None = None) -> None:
    V, D = W.shape
    _check(LIB.ember_step_dense(_ptr(W), _dtype(W), _ld(W), _ptr(G), _dtype(G), _ld(G),
                                _ptr(r), _ptr(c), V, D, int(t), float(lr), float(beta2), float(eps),
                                int(bool(maximize)), _ptr(ws), ws.numel() * ws.element_size(),
                                _stream(W)), "ember_step_dense")


def ember_step_sparse_rows(W: torch.Tensor, G_rows: torch.Tensor, idx: torch.Tensor,
                           r: torch.Tensor, c: torch.Tensor, t: int,
                           lr: float = 1e-3, beta2: float = 0.999, eps: float = 1e-8,
                           maximize: bool = False, ws: torch.Tensor | None = None) -> None:
    V, D = W.shape
    n = idx.numel()
    if idx.dtype != torch.int64:
        raise TypeError("idx must be int64")
    ldg = _ld(G_rows) if G_rows.numel() else D
    _check(LIB.ember_step_sparse_rows(_ptr(W), _dtype(W), _ld(W), _ptr(G_rows), _dtype(G_rows), ldg,
                                      _ptr(idx), n, _ptr(r), _ptr(c), V, D, int(t), float(lr),
                                      float(beta2), float(eps), int(bool(maximize)), _ptr(ws),
                                      ws.numel() * ws.element_size(), _stream(W)),
           "ember_step_sparse_rows")


def ember_step_sparse_rows_static(W: torch.Tensor, G_rows: torch.Tensor, idx: torch.Tensor,
                                  r: torch.Tensor, c: torch.Tensor, t: int, status: torch.Tensor,
                                  lr: float = 1e-3, beta2: float = 0.999, eps: float = 1e-8,
                                  maximize: bool = False) -> None:
    """Sparse-row step whose scratch is the library's own array (no workspace);
    status: a device int32 tensor of one element that receives the error bits."""
    V, D = W.shape
    n = idx.numel()
    if idx.dtype != torch.int64 or status.dtype != torch.int32:
        raise TypeError("idx must be int64 and status int32")
    ldg = _ld(G_rows) if G_rows.numel() else D
    _check(LIB.ember_step_sparse_rows_static(_ptr(W), _dtype(W), _ld(W), _ptr(G_rows), _dtype(G_rows), ldg,
                                             _ptr(idx), n, _ptr(r), _ptr(c), V, D, int(t), float(lr),
                                             float(beta2), float(eps), int(bool(maximize)), status.data_ptr(),
                                             _stream(W)), "ember_step_sparse_rows_static")


def ember_rowonly_init_state(r: torch.Tensor, D: int, ws: torch.Tensor) -> None:
    _check(LIB.ember_rowonly_init_state(_ptr(r), r.numel(), int(D), _ptr(ws),
                                        ws.numel() * ws.element_size(), _stream(r)),
           "ember_rowonly_init_state")


def ember_rowonly_step_dense(W: torch.Tensor, G: torch.Tensor, r: torch.Tensor, t: int,
                             lr: float = 1e-3, beta2: float = 0.999, eps: float = 1e-8,
                             maximize: bool = False, ws: torch.Tensor | None = None) -> None:
    V, D = W.shape
    _check(LIB.ember_rowonly_step_dense(_ptr(W), _dtype(W), _ld(W), _ptr(G), _dtype(G), _ld(G),
                                        _ptr(r), V, D, int(t), float(lr), float(beta2), float(eps),
                                        int(bool(maximize)), _ptr(ws), ws.numel() * ws.element_size(),
                                        _stream(W)), "ember_rowonly_step_dense")


def ember_rowonly_step_sparse_rows(W: torch.Tensor, G_rows: torch.Tensor, idx: torch.Tensor,
                                   r: torch.Tensor, t: int,
                                   lr: float = 1e-3, beta2: float = 0.999, eps: float = 1e-8,
                                   maximize: bool = False, ws: torch.Tensor | None = None) -> None:
    V, D = W.shape
    n = idx.numel()
    if idx.dtype != torch.int64:
        raise TypeError("idx must be int64")
    ldg = _ld(G_rows) if G_rows.numel() else D
    _check(LIB.ember_rowonly_step_sparse_rows(_ptr(W), _dtype(W), _ld(W), _ptr(G_rows), _dtype(G_rows),
                                              ldg, _ptr(idx), n, _ptr(r), V, D, int(t), float(lr),
                                              float(beta2), float(eps), int(bool(maximize)), _ptr(ws),
                                              ws.numel() * ws.element_size(), _stream(W)),
           "ember_rowonly_step_sparse_rows")


def ember_step_sparse_rows_devn(W: torch.Tensor, G_rows: torch.Tensor, idx: torch.Tensor, n_dev: torch.Tensor,
                                r: torch.Tensor, c, t: int, lr: float = 1e-3, beta2: float = 0.999,
                                eps: float = 1e-8, maximize: bool = False, ws: torch.Tensor | None = None,
                                row_only: bool = False) -> None:
    """Sparse step whose row count n is the int64 in device tensor n_dev; G_rows
    and idx hold the maximum count of rows (their first dimension)."""
    V, D = W.shape
    if idx.dtype != torch.int64 or n_dev.dtype != torch.int64:
        raise TypeError("idx and n_dev must be int64")
    max_rows = idx.numel()
    ldg = _ld(G_rows) if G_rows.numel() else D
    if row_only:
        st = LIB.ember_rowonly_step_sparse_rows_devn(
            _ptr(W), _dtype(W), _ld(W), _ptr(G_rows), _dtype(G_rows), ldg, _ptr(idx), n_dev.data_ptr(), max_rows,
            _ptr(r), V, D, int(t), float(lr), float(beta2), float(eps), int(bool(maximize)), _ptr(ws),
            ws.numel() * ws.element_size(), _stream(W))
    else:
        st = LIB.ember_step_sparse_rows_devn(
            _ptr(W), _dtype(W), _ld(W), _ptr(G_rows), _dtype(G_rows), ldg, _ptr(idx), n_dev.data_ptr(), max_rows,
            _ptr(r), _ptr(c), V, D, int(t), float(lr), float(beta2), float(eps), int(bool(maximize)), _ptr(ws),
            ws.numel() * ws.element_size(), _stream(W))
    _check(st, "ember_step_sparse_rows_devn")


def ember_coalesce_workspace_bytes(max_tokens: int, V: int, D: int) -> int:
    out = ctypes.c_size_t(0)
    _check(LIB.ember_coalesce_workspace_bytes(int(max_tokens), int(V), int(D), ctypes.byref(out)),
           "ember_coalesce_workspace_bytes")
    return out.value


def ember_coalesce_rows(tok: torch.Tensor, U: torch.Tensor, V: int, idx: torch.Tensor, G_rows: torch.Tensor,
                        n_out: torch.Tensor, ws: torch.Tensor) -> None:
    """Enqueue the coalescing of (tok, U) into (idx, G_rows, n_out) on the current
    stream; n_out is a device int64 tensor of one element."""
    if tok.dtype != torch.int64 or idx.dtype != torch.int64 or n_out.dtype != torch.int64:
        raise TypeError("tok, idx and n_out must be int64")
    P = tok.numel()
    D = U.shape[1]
    ldu = _ld(U) if P else D
    ldg = _ld(G_rows) if G_rows.numel() else D
    _check(LIB.ember_coalesce_rows(_ptr(tok), P, _ptr(U), _dtype(U), ldu, int(V), D, _ptr(idx),
                                   _ptr(G_rows), _dtype(G_rows), ldg, n_out.data_ptr(), _ptr(ws),
                                   ws.numel() * ws.element_size(), _stream(n_out)), "ember_coalesce_rows")


class Coalescer:
    """Workspace and outputs for coalescing batches of up to max_tokens token
    gradients of a V-row, D-column table."""

    def __init__(self, max_tokens: int, V: int, D: int, dtype=torch.bfloat16, device="cuda"):
        self.max_tokens, self.V, self.D = int(max_tokens), int(V), int(D)
        n = max(self.max_tokens, 1)
        q = 16 // torch.empty(0, dtype=dtype).element_size()
        ld = (self.D + q - 1) // q * q   # rows start on 16-byte boundaries
        self.idx = torch.empty(n, dtype=torch.int64, device=device)
        self.G_rows = torch.empty(n, ld, dtype=dtype, device=device)[:, :self.D]
        self.n_out = torch.zeros(1, dtype=torch.int64, device=device)
        nbytes = ember_coalesce_workspace_bytes(self.max_tokens, self.V, self.D)
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device=device)

    def enqueue(self, tok: torch.Tensor, U: torch.Tensor) -> None:
        """Coalesce one batch on the current stream without reading n back:
        self.idx, self.G_rows and self.n_out then feed a step with a device
        row count (EmberTable.step_tokens)."""
        if tok.numel() > self.max_tokens:
            raise ValueError("batch larger than max_tokens")
        ember_coalesce_rows(tok, U, self.V, self.idx, self.G_rows, self.n_out, self.ws)

    def __call__(self, tok: torch.Tensor, U: torch.Tensor):
        """Coalesce one batch; synchronises to read n.  Returns (idx, G_rows)
        views of the first n rows."""
        if tok.numel() > self.max_tokens:
            raise ValueError("batch larger than max_tokens")
        ember_coalesce_rows(tok, U, self.V, self.idx, self.G_rows, self.n_out, self.ws)
        _check(ember_get_error(self.ws), "ember_coalesce_rows (device)")
        n = int(self.n_out.item())
        return self.idx[:n], self.G_rows[:n]


def ember_lmhead_step(W: torch.Tensor, dY: torch.Tensor, H: torch.Tensor, G: torch.Tensor,
                      r: torch.Tensor, c: torch.Tensor, t: int,
                      lr: float = 1e-3, beta2: float = 0.999, eps: float = 1e-8,
                      maximize: bool = False, ws: torch.Tensor | None = None) -> None:
    """LM-head step: G = dY^T H (dY: T x V logits gradient, H: T x D hidden
    states, both bf16) written to G, and the dense Ember step on W with it."""
    V, D = W.shape
    T = dY.shape[0]
    if dY.dim() != 2 or H.dim() != 2 or dY.shape[1] != V or H.shape[0] != T or H.shape[1] != D:
        raise ValueError(f"shapes: dY {tuple(dY.shape)}, H {tuple(H.shape)} for W {tuple(W.shape)}")
    if tuple(G.shape) != (V, D):
        raise ValueError(f"G must be {V} x {D}")
    if T and (dY.dtype != torch.bfloat16 or H.dtype != torch.bfloat16):
        raise TypeError("dY and H must be bfloat16")
    ldy = _ld(dY) if T else V
    ldh = _ld(H) if T else D
    _check(LIB.ember_lmhead_step(_ptr(W), _dtype(W), _ld(W), _ptr(dY), ldy, _ptr(H), ldh, T,
                                 _ptr(G), _dtype(G), _ld(G), _ptr(r), _ptr(c), V, D, int(t), float(lr),
                                 float(beta2), float(eps), int(bool(maximize)), _ptr(ws),
                                 ws.numel() * ws.element_size(), _stream(W)), "ember_lmhead_step")


# The C entry points know pointers and the sizes they are given, not what memory
# lies behind them: these refuse a tensor that would be indexed past its end, and one
# that is not on the call's GPU.

def _misfit(what, t, shape, device, dtype):
    if t.get_device() != device:
        raise ValueError(f"{what}: on {t.device}, the call's tensors are on " +
                         (f"cuda:{device}" if device >= 0 else "the host"))
    if t.shape != shape:
        raise ValueError(f"{what}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    raise TypeError(f"{what}: a contiguous {dtype or 'tensor'} is required" if len(shape) == 1 else
                    f"{what}: {t.dtype}, expected {dtype}")


def _matrix(what, t, shape, device, dtype=None):
    """(address, row stride) of a 2-D tensor of this shape and type on this GPU (its
    index); None: no tensor."""
    if t is None:
        return None, 0
    if t.shape != shape or t.get_device() != device or (dtype is not None and t.dtype is not dtype):
        _misfit(what, t, shape, device, dtype)
    if len(shape) == 2:
        ld, unit = t.stride()
        if unit == 1:
            if shape[0] > 1:
                return t.data_ptr(), ld
            q = _CHUNK.get(t.dtype)
            if q is not None:   # one row, as _ld has it
                return t.data_ptr(), (shape[1] + q - 1) // q * q
    return t.data_ptr(), _ld(t)


def _vector(what, t, shape, device, dtype=torch.float32):
    """Address of a contiguous 1-D tensor of this shape and type on this GPU; None: no tensor."""
    if t is None:
        return None
    if t.shape != shape or t.get_device() != device or (dtype is not None and t.dtype is not dtype) or \
            not t.is_contiguous():
        _misfit(what, t, shape, device, dtype)
    return t.data_ptr()


def _workspace(ws, device):
    """Address and bytes of a workspace on this GPU."""
    if ws.get_device() != device:
        _misfit("ws", ws, ws.shape, device, None)
    return ws.data_ptr(), ws.numel() * ws.element_size()


def ember_rmsnorm(X: torch.Tensor, gain: torch.Tensor, eps: float = 1e-6, R: torch.Tensor | None = None,
                  S: torch.Tensor | None = None, Y: torch.Tensor | None = None, Q: torch.Tensor | None = None,
                  qscale: torch.Tensor | None = None, rstd: torch.Tensor | None = None) -> None:
    """S = X + R and its root-mean-square norm with gains, to Y and, in 8 bits
    with one scale a row, to (Q, qscale); rstd is kept for the gradient."""
    shape, dtype, dev = X.shape, X.dtype, X.get_device()
    x, ldx = _matrix("X", X, shape, dev)
    r, ldr = _matrix("R", R, shape, dev, dtype)
    sm, lds = _matrix("S", S, shape, dev, dtype)
    y, ldy = _matrix("Y", Y, shape, dev)
    q, ldq = _matrix("Q", Q, shape, dev, torch.int8)
    T, D = shape
    rows = (T,)
    _check(LIB.ember_rmsnorm(x, _DTYPES.get(dtype, 99), ldx, r, ldr, _vector("gain", gain, (D,), dev, None),
                             _dtype(gain), eps, T, D, sm, lds, y, EMBER_F32 if Y is None else _dtype(Y), ldy, q, ldq,
                             _vector("qscale", qscale, rows, dev), _vector("rstd", rstd, rows, dev), _stream(X)),
           "ember_rmsnorm")


def ember_rmsnorm_grad_workspace_bytes(max_tokens: int, D: int) -> int:
    out = ctypes.c_size_t(0)
    _check(LIB.ember_rmsnorm_grad_workspace_bytes(int(max_tokens), int(D), ctypes.byref(out)),
           "ember_rmsnorm_grad_workspace_bytes")
    return out.value


def ember_rmsnorm_grad(dY: torch.Tensor, S: torch.Tensor, gain: torch.Tensor, rstd: torch.Tensor,
                       dX: torch.Tensor, dgain: torch.Tensor, ws: torch.Tensor,
                       dS: torch.Tensor | None = None) -> None:
    """Gradient of ember_rmsnorm: dX (of X and of R) and dgain from dY, the sum S
    and rstd of the forward call, plus dS, the sum's gradient by other ways."""
    shape, dtype, dev = S.shape, S.dtype, S.get_device()
    s, lds = _matrix("S", S, shape, dev)
    dy, lddy = _matrix("dY", dY, shape, dev, dtype)
    dx, lddx = _matrix("dX", dX, shape, dev, dtype)
    ds, ldds = _matrix("dS", dS, shape, dev, dtype)
    T, D = shape
    cols = (D,)
    w, w_bytes = _workspace(ws, dev)
    _check(LIB.ember_rmsnorm_grad(dy, lddy, s, _DTYPES.get(dtype, 99), lds, _vector("gain", gain, cols, dev, None),
                                  _dtype(gain), _vector("rstd", rstd, (T,), dev), ds, ldds, T, D, dx, lddx,
                                  _vector("dgain", dgain, cols, dev), w, w_bytes, _stream(dgain)),
           "ember_rmsnorm_grad")


def ember_quantize_rows(X: torch.Tensor, Q: torch.Tensor, qscale: torch.Tensor) -> None:
    """Rows of X in 8 bits: codes Q and one scale a row."""
    shape, dev = X.shape, X.get_device()
    x, ldx = _matrix("X", X, shape, dev)
    q, ldq = _matrix("Q", Q, shape, dev, torch.int8)
    rows, D = shape
    _check(LIB.ember_quantize_rows(x, _dtype(X), ldx, rows, D, q, ldq, _vector("qscale", qscale, (rows,), dev),
                                   _stream(X)), "ember_quantize_rows")


def ember_logits_q8(Xq: torch.Tensor, xscale: torch.Tensor, Wq: torch.Tensor, wscale: torch.Tensor,
                    Y: torch.Tensor, bias: torch.Tensor | None = None) -> None:
    """Y = (Xq Wq^T) xscale wscale + bias: logits of T tokens from 8-bit hidden
    states and an 8-bit table, each with one scale a row."""
    T, D = Xq.shape
    V, dev = wscale.numel(), Wq.get_device()
    x, ldx = _matrix("Xq", Xq, (T, D), dev, torch.int8)
    w, ldw = _matrix("Wq", Wq, (V, D), dev, torch.int8)
    y, ldy = _matrix("Y", Y, (T, V), dev)
    _check(LIB.ember_logits_q8(x, ldx, _vector("xscale", xscale, (T,), dev), w, ldw,
                               _vector("wscale", wscale, (V,), dev), _vector("bias", bias, (V,), dev), T, V, D, y,
                               _dtype(Y), ldy, _stream(Wq)),
           "ember_logits_q8")


def _run(where, dev, f, *args):
    """The entry point f with the GPU dev current: a launch on the null stream goes to the current one."""
    if torch._C._cuda_getDevice() == dev:
        st = f(*args)
    else:
        with torch.cuda.device(dev):
            st = f(*args)
    _check(st, where)


def q4_shapes(V: int, D: int, group: int):
    """Shapes of a V x D table's codes (uint8) and scales (bf16) in 4 bits; rows of
    either start on 16-byte boundaries."""
    if group not in (32, 64, 128):
        raise ValueError(f"group {group}: 32, 64 or 128 columns share a scale")
    return (V, (D + 127) // 128 * 64), (V, (D + group - 1) // group)


def _table4(Wq, wscale, V, D, group, dev):
    """Addresses and row strides of a table's codes and scales."""
    codes, scales = q4_shapes(V, D, group)
    return *_matrix("Wq", Wq, codes, dev, torch.uint8), *_matrix("wscale", wscale, scales, dev, torch.bfloat16)


def ember_quantize_rows_q4(X: torch.Tensor, Q: torch.Tensor, gscale: torch.Tensor, group: int) -> None:
    """Rows of X in 4 bits: codes Q, packed, and a bf16 scale for each group of columns."""
    (rows, D), dev = X.shape, X.get_device()
    x, ldx = _matrix("X", X, X.shape, dev)
    q, ldq, s, lds = _table4(Q, gscale, rows, D, group, dev)
    _run("ember_quantize_rows_q4", dev, LIB.ember_quantize_rows_q4, x, _dtype(X), ldx, rows, D, group, q, ldq, s, lds,
         _stream(X))


def ember_rows_q4(Wq: torch.Tensor, wscale: torch.Tensor, Y: torch.Tensor, group: int,
                  tok: torch.Tensor | None = None) -> None:
    """Y = the rows of a 4-bit table that tok (int64) names, or (None) its first ones."""
    V, dev = Wq.shape[0], Wq.get_device()
    n, D = Y.shape
    w, ldw, s, lds = _table4(Wq, wscale, V, D, group, dev)
    y, ldy = _matrix("Y", Y, Y.shape, dev)
    _run("ember_rows_q4", dev, LIB.ember_rows_q4, w, ldw, s, lds, group, V, D,
         _vector("tok", tok, (n,), dev, torch.int64), n, y, _dtype(Y), ldy, _stream(Wq))


def ember_logits_q4(Xq: torch.Tensor, xscale: torch.Tensor, Wq: torch.Tensor, wscale: torch.Tensor,
                    Y: torch.Tensor, group: int, bias: torch.Tensor | None = None) -> None:
    """Logits of T tokens from 8-bit hidden states and a table in 4 bits with a scale
    a group of columns."""
    T, D = Xq.shape
    V, dev = Wq.shape[0], Wq.get_device()
    x, ldx = _matrix("Xq", Xq, (T, D), dev, torch.int8)
    w, ldw, s, lds = _table4(Wq, wscale, V, D, group, dev)
    y, ldy = _matrix("Y", Y, (T, V), dev)
    _run("ember_logits_q4", dev, LIB.ember_logits_q4, x, ldx, _vector("xscale", xscale, (T,), dev), w, ldw, s, lds,
         group, _vector("bias", bias, (V,), dev), T, V, D, y, _dtype(Y), ldy, _stream(Wq))


def ember_sample_workspace_bytes(max_tokens: int, V: int) -> int:
    out = ctypes.c_size_t(0)
    _check(LIB.ember_sample_workspace_bytes(int(max_tokens), int(V), ctypes.byref(out)),
           "ember_sample_workspace_bytes")
    return out.value


def ember_sample(L: torch.Tensor, u: torch.Tensor, ids: torch.Tensor, ws: torch.Tensor,
                 temperature: torch.Tensor | None = None, top_k: torch.Tensor | None = None,
                 top_p: torch.Tensor | None = None, min_p: torch.Tensor | None = None,
                 logp: torch.Tensor | None = None, kept: torch.Tensor | None = None) -> None:
    """A token of each row of logits L, drawn with the random numbers u in [0, 1): ids
    (int64), and, where wanted, their log-probabilities before the filters and the
    number of tokens that the filters keep (int32).  Parameters: a value a row, on the
    device (top_k int32)."""
    (T, V), dev = L.shape, L.get_device()
    l, ldl = _matrix("L", L, L.shape, dev)
    rows = (T,)
    w, w_bytes = _workspace(ws, dev)
    _run("ember_sample", dev, LIB.ember_sample, l, _dtype(L), ldl, T, V, _vector("temperature", temperature, rows, dev),
         _vector("top_k", top_k, rows, dev, torch.int32), _vector("top_p", top_p, rows, dev),
         _vector("min_p", min_p, rows, dev), _vector("u", u, rows, dev), _vector("ids", ids, rows, dev, torch.int64),
         _vector("logp", logp, rows, dev), _vector("kept", kept, rows, dev, torch.int32), w, w_bytes, _stream(L))


def ember_clip_workspace_bytes(n_grads: int) -> int:
    out = ctypes.c_size_t(0)
    _check(LIB.ember_clip_workspace_bytes(int(n_grads), ctypes.byref(out)), "ember_clip_workspace_bytes")
    return out.value


def grad_entry(src: torch.Tensor, dst: torch.Tensor | None = None, rows_dev: torch.Tensor | None = None) -> Grad:
    """One entry of ember_clip_grads: the gradient src, written clipped to dst
    (None: in place); rows_dev: a device int64 of one element that says how many
    of its rows hold a gradient (the others become zeros), all of them on one GPU.  A 2-D tensor with
    unit column stride, or any contiguous one.  The tensors must stay alive until the call has run."""
    if dst is None:
        dst = src
    dev = src.get_device()
    for what, t in (("gradient", src), ("destination", dst), ("rows_dev", rows_dev)):
        if t is not None and (dev < 0 or t.get_device() != dev):
            raise ValueError(f"{what}: on {t.device}; a gradient, its destination and its count are on one GPU")
    if dst.shape != src.shape:
        raise ValueError(f"gradient {tuple(src.shape)} does not fit its destination {tuple(dst.shape)}")
    if rows_dev is not None and (rows_dev.dtype != torch.int64 or rows_dev.numel() != 1 or src.dim() != 2):
        raise TypeError("rows_dev must be one int64 and its gradient 2-D")
    if src.dim() == 2:
        (rows, cols), lds, ldd = src.shape, src.stride(0), dst.stride(0)
        for t in (src, dst):
            if cols > 1 and t.stride(1) != 1 and t.numel():
                raise TypeError("a 2-D gradient needs unit column stride")
        if rows == 1:
            lds = ldd = cols
    else:
        if not (src.is_contiguous() and dst.is_contiguous()):
            raise TypeError("a gradient that is not 2-D must be contiguous")
        rows, cols = 1, src.numel()
        lds = ldd = cols
    entry = Grad(_ptr(src), _dtype(src), lds, _ptr(dst), _dtype(dst), ldd, rows, cols, _ptr(rows_dev))
    entry.device = dev
    return entry


def _grad_array(entries, device):
    """The ctypes array of grad_entry's entries, all of them on this GPU."""
    for i, e in enumerate(entries):
        if getattr(e, "device", device) != device:
            raise ValueError(f"gradient {i}: on cuda:{e.device}, the call's tensors are on cuda:{device}")
    return (Grad * len(entries))(*entries)


def ember_clip_grads(grads, max_norm: float, out: torch.Tensor, ws: torch.Tensor) -> None:
    """Clip gradients (a ctypes array of Grad entries, or a list of them) by
    their global norm; out (device, two floats) receives the norm and the factor."""
    dev = out.get_device()
    arr = grads if isinstance(grads, ctypes.Array) else _grad_array(grads, dev)
    w, w_bytes = _workspace(ws, dev)
    _check(LIB.ember_clip_grads(arr, len(arr), float(max_norm), _vector("out", out, (2,), dev), w, w_bytes,
                                _stream(out)), "ember_clip_grads")


class HeadNorm:
    """The final norm of a model: its gains (D values), eps and the workspace of
    its gradient for up to max_tokens tokens.  Call it for the norm; ``grad`` is
    its gradient."""

    def __init__(self, gain: torch.Tensor, eps: float = 1e-6, max_tokens: int = 0):
        self.gain, self.eps, self.max_tokens = gain, float(eps), int(max_tokens)
        self.D = gain.numel()
        nbytes = ember_rmsnorm_grad_workspace_bytes(self.max_tokens, self.D)
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device=gain.device)

    def __call__(self, X, R=None, S=None, Y=None, Q=None, qscale=None, rstd=None) -> None:
        ember_rmsnorm(X, self.gain, self.eps, R, S, Y, Q, qscale, rstd)

    def grad(self, dY, S, rstd, dX, dgain, dS=None) -> None:
        ember_rmsnorm_grad(dY, S, self.gain, rstd, dX, dgain, self.ws, dS)


class HeadQ8:
    """An LM head in 8 bits: codes Wq (V x D, rows on 16-byte boundaries), one
    scale a row and, if the head has one, a bias."""

    def __init__(self, Wq: torch.Tensor, wscale: torch.Tensor, bias: torch.Tensor | None = None):
        self.Wq, self.wscale, self.bias = Wq, wscale, bias

    @classmethod
    def from_table(cls, W: torch.Tensor, bias: torch.Tensor | None = None) -> "HeadQ8":
        """The head of a table (V x D, fp32 or bf16)."""
        V, D = W.shape
        # wide rows on the memory's 128-byte lines (211 tokens x 36770 x 2896 43 us, on 16 bytes 50)
        pad = 128 if D >= 1024 else 16
        Wq = torch.empty(V, (D + pad - 1) // pad * pad, dtype=torch.int8, device=W.device)[:, :D]
        head = cls(Wq, torch.empty(V, dtype=torch.float32, device=W.device), bias)
        head.load(W)
        return head

    def load(self, W: torch.Tensor) -> None:
        """Take the table's present rows (after steps on it)."""
        ember_quantize_rows(W, self.Wq, self.wscale)

    def logits(self, Xq: torch.Tensor, xscale: torch.Tensor, Y: torch.Tensor) -> None:
        ember_logits_q8(Xq, xscale, self.Wq, self.wscale, Y, self.bias)


class HeadQ4:
    """A token table in 4 bits, an LM head's or an embedding's (or one for both): packed
    codes Wq and the scales wscale of groups of columns, D columns, and, if the head has
    one, a bias."""

    def __init__(self, Wq: torch.Tensor, wscale: torch.Tensor, D: int, group: int = 128,
                 bias: torch.Tensor | None = None):
        self.Wq, self.wscale, self.D, self.group, self.bias = Wq, wscale, int(D), int(group), bias
        self.V = Wq.shape[0]

    @classmethod
    def from_table(cls, W: torch.Tensor, group: int = 128, bias: torch.Tensor | None = None) -> "HeadQ4":
        """The head of a table (V x D, fp32 or bf16)."""
        codes, (V, groups) = q4_shapes(*W.shape, group)
        Wq = torch.empty(codes, dtype=torch.uint8, device=W.device)
        wscale = torch.empty(V, (groups + 7) // 8 * 8, dtype=torch.bfloat16, device=W.device)[:, :groups]
        head = cls(Wq, wscale, W.shape[1], group, bias)
        head.load(W)
        return head

    def load(self, W: torch.Tensor) -> None:
        """Take the table's present rows (after steps on it)."""
        if W.shape[1] != self.D:
            raise ValueError(f"W has {W.shape[1]} columns, the table {self.D}")
        ember_quantize_rows_q4(W, self.Wq, self.wscale, self.group)

    def logits(self, Xq: torch.Tensor, xscale: torch.Tensor, Y: torch.Tensor) -> None:
        if Xq.shape[1] != self.D:
            raise ValueError(f"Xq has {Xq.shape[1]} columns, the head {self.D}")
        ember_logits_q4(Xq, xscale, self.Wq, self.wscale, Y, self.group, self.bias)

    def rows(self, tok: torch.Tensor | None, Y: torch.Tensor) -> None:
        """Y = the rows of the tokens tok (int64), or (None) the first ones."""
        if Y.shape[1] != self.D:
            raise ValueError(f"Y has {Y.shape[1]} columns, the table {self.D}")
        ember_rows_q4(self.Wq, self.wscale, Y, self.group, tok)


class Sampler:
    """Draws a token from each of up to max_tokens rows of V logits; holds the
    workspace.  Call it as ember_sample, without the workspace."""

    def __init__(self, max_tokens: int, V: int, device="cuda"):
        self.max_tokens, self.V = int(max_tokens), int(V)
        nbytes = ember_sample_workspace_bytes(self.max_tokens, self.V)
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device=device)

    def __call__(self, L: torch.Tensor, u: torch.Tensor, ids: torch.Tensor, temperature=None, top_k=None, top_p=None,
                 min_p=None, logp=None, kept=None) -> None:
        ember_sample(L, u, ids, self.ws, temperature, top_k, top_p, min_p, logp, kept)


class GradClipper:
    """Clips a fixed list of gradient tensors by their global norm.  out: where
    each goes (None: in place), counts: for each None or its device row count.
    Call it with the largest norm allowed; it returns the norm and the factor,
    scalars on the device that the next call overwrites."""

    def __init__(self, grads, out=None, counts=None):
        grads = list(grads)
        out = [None] * len(grads) if out is None else list(out)
        counts = [None] * len(grads) if counts is None else list(counts)
        if not grads or len(out) != len(grads) or len(counts) != len(grads):
            raise ValueError("one gradient at least, and out and counts as long as the list")
        self.tensors = (grads, out, counts)    # kept alive: the entries hold their addresses
        self.entries = _grad_array([grad_entry(*x) for x in zip(grads, out, counts)], grads[0].get_device())
        self.out = torch.zeros(2, dtype=torch.float32, device=grads[0].device)
        self.norm, self.factor = self.out[0], self.out[1]
        nbytes = ember_clip_workspace_bytes(len(grads))
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device=grads[0].device)

    def __call__(self, max_norm: float):
        ember_clip_grads(self.entries, max_norm, self.out, self.ws)
        return self.norm, self.factor


def table_step(W: torch.Tensor, G: torch.Tensor | None, r: torch.Tensor, c: torch.Tensor | None, t: int,
               ws: torch.Tensor, idx: torch.Tensor | None = None, n_idx_dev: torch.Tensor | None = None,
               lr: float = 1e-3, beta2: float = 0.999, eps: float = 1e-8,
               maximize: bool = False, row_only: bool = False) -> TableStep:
    """One entry of ember_step_multi: a dense step when idx is None, else a
    sparse-row step on the rows idx lists (with n_idx_dev: the row count in
    device memory, idx.numel() its maximum); row_only: the row-only step (c
    unused).  The tensors must stay alive until the step has run."""
    V, D = W.shape
    sparse = idx is not None
    if sparse and idx.dtype != torch.int64:
        raise TypeError("idx must be int64")
    n = idx.numel() if sparse else 0
    ldg = _ld(G) if G is not None and G.numel() else D
    return TableStep(_ptr(W), _dtype(W), _ld(W), _ptr(G), _dtype(G) if G is not None else _dtype(W), ldg,
                     int(sparse), int(bool(row_only)), _ptr(idx) if sparse else None, n, _ptr(n_idx_dev),
                     _ptr(r), _ptr(c),
                     V, D, int(t), float(lr), float(beta2), float(eps), int(bool(maximize)), _ptr(ws),
                     ws.numel() * ws.element_size())


def ember_step_multi(steps, stream_of: torch.Tensor) -> None:
    """Enqueue the steps of several tables (TableStep entries) on the current
    stream of stream_of's device, in shared launches (a sparse table whose
    rows fit on chip takes its one-launch step)."""
    arr = (TableStep * len(steps))(*steps)
    _check(LIB.ember_step_multi(arr, len(steps), _stream(stream_of)), "ember_step_multi")


def step_tables(items) -> None:
    """Ember steps of several tables in one call.  items: tuples (EmberTable,
    W, G) for a dense step or (EmberTable, W, G_rows, idx) for a sparse-row
    step; each table takes its canonical or row-only step; every table
    advances t by one."""
    steps = []
    for it in items:
        tab, W, G = it[0], it[1], it[2]
        idx = it[3] if len(it) > 3 else None
        steps.append(table_step(W, G, tab.r, tab.c, tab.t + 1, tab.ws, idx=idx, lr=tab.lr, beta2=tab.beta2,
                                eps=tab.eps, maximize=tab.maximize, row_only=tab.row_only))
    ember_step_multi(steps, items[0][1])
    for it in items:
        it[0].t += 1


def ember_get_error(ws: torch.Tensor) -> int:
    """Device status of the last step on this workspace (synchronises the stream)."""
    st = ctypes.c_int(0)
    _check(LIB.ember_get_error(_ptr(ws), _stream(ws), ctypes.byref(st)), "ember_get_error")
    return st.value


def ember_set_barrier_wait_ticks(ticks: int) -> None:
    """Bound of the one-launch sparse step's grid-barrier waits in 100 MHz
    ticks (diagnostics; 0 restores the default of about one second)."""
    _check(LIB.ember_set_barrier_wait_ticks(int(ticks)), "ember_set_barrier_wait_ticks")


def ember_profile_enable(enable: bool) -> None:
    _check(LIB.ember_profile_enable(int(bool(enable))), "ember_profile_enable")


def ember_profile_collect() -> dict:
    """{kernel name: (launches, total milliseconds)} since the last collect."""
    buf = (_KernelStat * 64)()    # more than the library has names
    n = ctypes.c_int(0)
    _check(LIB.ember_profile_collect(buf, len(buf), ctypes.byref(n)), "ember_profile_collect")
    return {buf[k].name.decode(): (buf[k].launches, buf[k].total_ms) for k in range(n.value)}


def ember_stream_probe(mode: int, dst: torch.Tensor, a: torch.Tensor, b: torch.Tensor | None = None) -> None:
    """Streaming probe over a's bytes: 0 read a, 1 copy a to dst, 2 dst = a + b
    (32-bit integer lanes)."""
    nbytes = a.numel() * a.element_size()
    _check(LIB.ember_stream_probe(int(mode), _ptr(dst), _ptr(a), _ptr(b), nbytes, _stream(a)),
           "ember_stream_probe")


class EmberTable:
    """Ember state of one V x D token table on one device: r, c, workspace, t.

    A convenience holder around the C entry points (Algorithm 1: r_0 = 0,
    c_0 = 0, t = 0, then t += 1 before each update).  ``row_only`` selects the
    row-only variant of Section 2.1 (no c).
    """

    def __init__(self, V: int, D: int, device="cuda", lr: float = 1e-3, beta2: float = 0.999,
                 eps: float = 1e-8, maximize: bool = False, row_only: bool = False):
        self.V, self.D = int(V), int(D)
        self.lr, self.beta2, self.eps, self.maximize = lr, beta2, eps, maximize
        self.row_only = bool(row_only)
        self.r = torch.empty(self.V, dtype=torch.float32, device=device)
        self.c = None if self.row_only else torch.empty(self.D, dtype=torch.float32, device=device)
        nbytes = ember_workspace_bytes(self.V, self.D)
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.t = 0
        if self.row_only:
            ember_rowonly_init_state(self.r, self.D, self.ws)
        else:
            ember_init_state(self.r, self.c, self.ws)

    def step(self, W: torch.Tensor, G: torch.Tensor) -> None:
        if self.row_only:
            ember_rowonly_step_dense(W, G, self.r, self.t + 1, self.lr, self.beta2, self.eps,
                                     self.maximize, self.ws)
        else:
            ember_step_dense(W, G, self.r, self.c, self.t + 1, self.lr, self.beta2, self.eps,
                             self.maximize, self.ws)
        self.t += 1

    def step_lmhead(self, W: torch.Tensor, dY: torch.Tensor, H: torch.Tensor, G: torch.Tensor) -> None:
        """LM-head step from the logits gradient dY [T, V] and hidden states
        H [T, D] (bf16): G = dY^T H is written to G and the step takes its
        statistics from the GEMM's epilogue (canonical Ember only)."""
        if self.row_only:
            raise ValueError("the fused LM-head step is the canonical (row and column) step")
        ember_lmhead_step(W, dY, H, G, self.r, self.c, self.t + 1, self.lr, self.beta2, self.eps,
                          self.maximize, self.ws)
        self.t += 1

    def step_tokens(self, W: torch.Tensor, tok: torch.Tensor, U: torch.Tensor, coalescer: "Coalescer") -> None:
        """Sparse step from token ids and per-position gradient rows: coalescing
        and the step are enqueued back to back with the row count kept in
        device memory (no host synchronisation; capturable in a HIP graph).
        Index errors of either call show in ember_get_error of its workspace."""
        coalescer.enqueue(tok, U)
        ember_step_sparse_rows_devn(W, coalescer.G_rows, coalescer.idx, coalescer.n_out, self.r, self.c,
                                    self.t + 1, self.lr, self.beta2, self.eps, self.maximize, self.ws,
                                    row_only=self.row_only)
        self.t += 1

    def step_sparse_rows(self, W: torch.Tensor, G_rows: torch.Tensor, idx: torch.Tensor,
                         check: bool = False) -> None:
        """Sparse-row step.  With check=True the index status is read back (a
        stream sync) and t advances only if idx was valid."""
        if self.row_only:
            ember_rowonly_step_sparse_rows(W, G_rows, idx, self.r, self.t + 1, self.lr, self.beta2,
                                           self.eps, self.maximize, self.ws)
        else:
            ember_step_sparse_rows(W, G_rows, idx, self.r, self.c, self.t + 1, self.lr, self.beta2,
                                   self.eps, self.maximize, self.ws)
        if check:
            _check(ember_get_error(self.ws), "ember_step_sparse_rows (device)")
        self.t += 1
