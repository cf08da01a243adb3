"""ctypes binding of libcsrtrain.so (include/csrtrain.h).

Argument marshalling only: every function takes torch tensors that already
live on the GPU, checks dtype / shape / contiguity, and passes raw device
pointers and sizes to the C ABI on the current (or given) CUDA stream. All
arithmetic runs in the CUDA library; there is no CPU fallback, and loading
fails loudly if the library has not been built.
"""

from __future__ import annotations

import ctypes
import os
import struct
import threading
from ctypes import POINTER, c_float, c_int8, c_int32, c_int64, c_size_t, c_void_p

import torch

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_lib", "libcsrtrain.so")

CSRT_OK, CSRT_ERR_ARG, CSRT_ERR_CUDA, CSRT_ERR_WORKSPACE = 0, 1, 2, 3
CSRT_DEV_CAPACITY, CSRT_DEV_TIMEOUT, CSRT_DEV_NONFINITE, CSRT_DEV_INVALID = 1, 2, 4, 8
CSRT_PREC_FP32, CSRT_PREC_TF32 = 0, 1
CSRT_DT_F32, CSRT_DT_BF16, CSRT_DT_F16 = 0, 1, 2
CSRT_ACT_NONE, CSRT_ACT_RELU, CSRT_ACT_GELU, CSRT_ACT_SILU = 0, 1, 2, 3
CSRT_NORM_SCALE, CSRT_NORM_RMS, CSRT_NORM_LAYER = 0, 1, 2
CSRT_GATE_NONE, CSRT_GATE_SIGMOID, CSRT_GATE_SILU = 0, 1, 2


class csrt_csr(ctypes.Structure):
    _fields_ = [
        ("rows", c_int32), ("cols", c_int32), ("capacity", c_int64),
        ("row_ptr", c_void_p), ("col_idx", c_void_p), ("val", c_void_p),
        ("t_row_ptr", c_void_p), ("t_col_idx", c_void_p), ("t_val", c_void_p),
        ("t_pos", c_void_p),
    ]


class csrt_mat(ctypes.Structure):
    _fields_ = [("data", c_void_p), ("rows", c_int32), ("cols", c_int32), ("ld", c_int64), ("dtype", c_int32)]


class csrt_norm(ctypes.Structure):
    _fields_ = [("kind", c_int32), ("eps", c_float), ("weight", c_void_p), ("bias", c_void_p), ("mean", c_void_p),
                ("rstd", c_void_p), ("dweight", c_void_p), ("dbias", c_void_p)]


class CsrtError(RuntimeError):
    pass


_LIB = None

_SIGS = {
    "csrt_workspace_bytes": [c_int32, c_int32, c_int32, POINTER(c_size_t)],
    "csrt_workspace_init": [c_void_p, c_size_t, c_void_p],
    "csrt_get_status": [c_void_p, POINTER(c_int32), POINTER(c_int64), c_void_p],
    "csrt_clear_status": [c_void_p, c_void_p],
    "csrt_validate_csr": [POINTER(csrt_csr), c_void_p, c_size_t, c_void_p],
    "csrt_get_invalid_row": [c_void_p, POINTER(c_int64), c_void_p],
    "csr_from_dense": [c_void_p, c_int32, c_int32, POINTER(csrt_csr), c_void_p, c_size_t, c_void_p],
    "csr_transpose": [POINTER(csrt_csr), c_void_p, c_size_t, c_void_p],
    "spmm_fwd": [POINTER(csrt_csr), c_void_p, c_int32, c_void_p, c_void_p, c_size_t, c_void_p],
    "spmm_bwd_t": [POINTER(csrt_csr), c_void_p, c_int32, c_void_p, c_void_p, c_size_t, c_void_p],
    "spmm_fwd_bias_act": [POINTER(csrt_csr), c_void_p, c_int32, c_void_p, c_int32, c_void_p, c_void_p, c_size_t,
                          c_void_p],
    "spmm_bwd_t_relu": [POINTER(csrt_csr), c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p],
    "spmm_fwd_noalloc": [POINTER(csrt_csr), c_void_p, c_int32, c_void_p, c_void_p],
    "spmm_fwd_noalloc_status": [POINTER(c_int32), c_int32, c_void_p],
    "weight_grad_dense": [c_void_p, c_void_p, c_int32, c_int32, c_int32, c_void_p, c_int32, c_void_p,
                          c_size_t, c_void_p],
    "weight_grad_sddmm": [POINTER(csrt_csr), c_void_p, c_void_p, c_int32, c_void_p, c_void_p, c_size_t,
                          c_void_p],
    "prox_update_compact": [POINTER(csrt_csr), c_void_p, c_float, c_float, POINTER(csrt_csr), c_void_p,
                            c_size_t, c_void_p],
    "debias_update": [POINTER(csrt_csr), c_void_p, c_float, c_void_p],
    "prox_rmsprop_update_compact": [POINTER(csrt_csr), c_void_p, c_void_p, c_float, c_float, c_float, c_float,
                                    POINTER(csrt_csr), c_void_p, c_size_t, c_void_p],
    "prox_adam_update_compact": [POINTER(csrt_csr), c_void_p, c_void_p, c_void_p, c_int32, c_float, c_float,
                                 c_float, c_float, c_float, POINTER(csrt_csr), c_void_p, c_size_t, c_void_p],
    "weight_grad_prox_update": [POINTER(csrt_csr), c_void_p, c_void_p, c_int32, c_float, c_float, c_int32, c_void_p,
                                POINTER(csrt_csr), c_void_p, c_size_t, c_void_p],
    "csrt_dense_workspace_bytes": [c_int32, c_int32, c_int32, POINTER(c_size_t)],
    "csrt_dense_fwd": [POINTER(csrt_mat), POINTER(csrt_mat), c_void_p, c_int32, POINTER(csrt_mat), POINTER(csrt_mat),
                       POINTER(csrt_mat), c_void_p, c_size_t, c_void_p],
    "csrt_dense_bwd_x": [POINTER(csrt_mat), POINTER(csrt_mat), POINTER(csrt_mat), c_int32, POINTER(csrt_mat),
                         POINTER(csrt_mat), c_void_p, c_size_t, c_void_p],
    "csrt_dense_bwd_w": [POINTER(csrt_mat), POINTER(csrt_mat), c_int32, POINTER(csrt_mat), c_void_p, c_void_p, c_size_t,
                         c_void_p],
    "csrt_dense_act_bwd": [POINTER(csrt_mat), POINTER(csrt_mat), c_int32, POINTER(csrt_mat), c_void_p],
    "csrt_dense_update": [POINTER(csrt_mat), POINTER(csrt_mat), c_float, c_float, POINTER(csrt_mat), c_void_p],
    "csrt_orthogonalize_workspace_bytes": [c_int32, c_int32, c_int32, POINTER(c_size_t)],
    "csrt_orthogonalize": [POINTER(csrt_mat), c_int64, c_int32, c_void_p, c_float, c_int32, c_int32, c_float, c_float,
                           POINTER(csrt_mat), c_int64, c_void_p, c_size_t, c_void_p],
    "csrt_block_norm_fwd": [POINTER(csrt_mat), POINTER(csrt_norm), POINTER(csrt_mat), c_int32, POINTER(csrt_mat), c_float,
                            POINTER(csrt_norm), POINTER(csrt_mat), POINTER(csrt_mat), c_void_p],
    "csrt_block_norm_workspace_bytes": [c_int32, c_int32, POINTER(c_size_t)],
    "csrt_block_norm_bwd": [POINTER(csrt_mat), POINTER(csrt_mat), POINTER(csrt_mat), POINTER(csrt_norm),
                            POINTER(csrt_mat), POINTER(csrt_norm), POINTER(csrt_mat), c_int32, c_float, c_int32,
                            POINTER(csrt_mat), POINTER(csrt_mat), POINTER(csrt_mat), c_void_p, c_size_t, c_void_p],
    "csrt_embed_workspace_bytes": [c_int32, c_int32, c_int32, POINTER(c_size_t)],
    "csrt_embed_fwd": [POINTER(csrt_mat), c_void_p, c_float, POINTER(csrt_mat), c_void_p, c_size_t, c_void_p],
    "csrt_embed_bwd": [POINTER(csrt_mat), c_void_p, c_float, c_int32, POINTER(csrt_mat), c_void_p, c_size_t, c_void_p],
    "csrt_grad_workspace_bytes": [POINTER(c_size_t)],
    "csrt_grad_norm": [POINTER(csrt_mat), c_int32, c_void_p, c_void_p, c_size_t, c_void_p],
    "csrt_grad_clip": [POINTER(csrt_mat), c_int32, c_float, POINTER(csrt_mat), c_void_p, c_void_p, c_size_t, c_void_p],
    "csrt_bias_act_fwd": [c_void_p, c_void_p, c_int32, c_int32, c_int32, c_void_p],
    "csrt_relu_bwd": [c_void_p, c_void_p, c_int64, c_void_p],
    "csrt_bias_grad_sgd": [c_void_p, c_int32, c_int32, c_void_p, c_float, c_void_p, c_void_p],
    "csrt_softmax_xent": [c_void_p, c_void_p, c_int32, c_int32, c_void_p, c_void_p, c_void_p],
    "csrt_im2col": [c_void_p, c_int32, c_int32, c_int32, c_int32, c_int32, c_void_p, c_void_p],
    "csrt_col2im": [c_void_p, c_int32, c_int32, c_int32, c_int32, c_int32, c_void_p, c_void_p],
    "csrt_check_bounded_waits": [c_void_p, c_size_t, c_void_p],
    "csrt_fma_peak_run": [c_void_p, c_int32, c_int32, ctypes.POINTER(ctypes.c_double), c_void_p],
    "csrt_conv2d_sparse_fwd": [POINTER(csrt_csr), c_void_p, c_int32, c_int32, c_int32, c_int32, c_int32, c_void_p,
                               c_int32, c_void_p, c_void_p],
    "csrt_maxpool2_fwd": [c_void_p, c_int32, c_int32, c_int32, c_int32, c_void_p, c_void_p, c_void_p],
    "csrt_maxpool2_bwd": [c_void_p, c_void_p, c_int32, c_int32, c_int32, c_int32, c_void_p, c_void_p],
    "csrt_flatten": [c_void_p, c_int32, c_int32, c_int32, c_void_p, c_void_p],
    "csrt_unflatten": [c_void_p, c_int32, c_int32, c_int32, c_void_p, c_void_p],
}


def lib():
    """Load libcsrtrain.so once; raise if it has not been built."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise CsrtError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
        L = ctypes.CDLL(LIB_PATH)
        for name, args in _SIGS.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = c_int32
        L.csrt_last_error.argtypes = []
        L.csrt_last_error.restype = ctypes.c_char_p
        L.csrt_launch_count.argtypes = [c_int32]
        L.csrt_launch_count.restype = c_int64
        _LIB = L
    return _LIB


def exported_symbols():
    """The entry points this binding expects the library to export."""
    return sorted(list(_SIGS) + ["csrt_last_error", "csrt_launch_count"])


def _check(rc: int, what: str):
    if rc != CSRT_OK:
        msg = lib().csrt_last_error().decode(errors="replace")
        raise CsrtError(f"{what} failed with code {rc}: {msg}")


# The current stream's handle without building a Stream object (3 us a call); the fallback is for torch builds
# without the accessors.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None and _raw_device is not None:
            return c_void_p(_raw_stream(_raw_device()))
        stream = torch.cuda.current_stream()
    return c_void_p(stream.cuda_stream)


def _ptr(t):
    return None if t is None else c_void_p(t.data_ptr())


def _f32(t, name, numel=None):
    if t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous float32 CUDA tensor")
    if numel is not None and t.numel() < numel:
        raise ValueError(f"{name} has {t.numel()} elements, needs {numel}")
    return t


def launch_count(reset: bool = False) -> int:
    return int(lib().csrt_launch_count(1 if reset else 0))


# ---------------------------------------------------------------------------
# Owned device objects
# ---------------------------------------------------------------------------

class CSR:
    """A device CSR matrix (caller-owned torch buffers) with optional
    transposed arrays, mirroring ``csrt_csr``."""

    def __init__(self, rows: int, cols: int, capacity: int | None = None, transposed: bool = True,
                 device="cuda"):
        self.rows, self.cols = int(rows), int(cols)
        self.capacity = int(rows * cols if capacity is None else capacity)
        cap = max(self.capacity, 1)
        i32 = dict(dtype=torch.int32, device=device)
        self.row_ptr = torch.zeros(self.rows + 1, **i32)
        self.col_idx = torch.zeros(cap, **i32)
        self.val = torch.zeros(cap, dtype=torch.float32, device=device)
        self.transposed = transposed
        if transposed:
            self.t_row_ptr = torch.zeros(self.cols + 1, **i32)
            self.t_col_idx = torch.zeros(cap, **i32)
            self.t_val = torch.zeros(cap, dtype=torch.float32, device=device)
            self.t_pos = torch.zeros(cap, **i32)
        else:
            self.t_row_ptr = self.t_col_idx = self.t_val = self.t_pos = None
        self._s = csrt_csr(self.rows, self.cols, self.capacity, _ptr(self.row_ptr), _ptr(self.col_idx),
                           _ptr(self.val), _ptr(self.t_row_ptr), _ptr(self.t_col_idx), _ptr(self.t_val),
                           _ptr(self.t_pos))

    @property
    def struct(self):
        return ctypes.byref(self._s)

    def nnz(self) -> int:
        return int(self.row_ptr[self.rows].item())

    def copy_from(self, other: "CSR"):
        """Device-to-device copy of another CSR of the same shape (nnz entries)."""
        self.row_ptr.copy_(other.row_ptr)
        n = other.nnz()
        self.col_idx[:n].copy_(other.col_idx[:n])
        self.val[:n].copy_(other.val[:n])
        if self.transposed and other.transposed:
            self.t_row_ptr.copy_(other.t_row_ptr)
            self.t_col_idx[:n].copy_(other.t_col_idx[:n])
            self.t_val[:n].copy_(other.t_val[:n])
            self.t_pos[:n].copy_(other.t_pos[:n])

    def to_host(self):
        """(row_ptr, col_idx, val) as numpy arrays trimmed to nnz, and the
        transposed arrays (or None)."""
        n = self.nnz()
        main = (self.row_ptr.cpu().numpy(), self.col_idx[:n].cpu().numpy(), self.val[:n].cpu().numpy())
        if not self.transposed:
            return main, None
        t = (self.t_row_ptr.cpu().numpy(), self.t_col_idx[:n].cpu().numpy(), self.t_val[:n].cpu().numpy(),
             self.t_pos[:n].cpu().numpy())
        return main, t


class Workspace:
    """Device scratch + status word (csrt_workspace_bytes / csrt_workspace_init)."""

    def __init__(self, rows: int, cols: int, max_n: int, device="cuda", stream=None):
        nbytes = c_size_t(0)
        _check(lib().csrt_workspace_bytes(int(rows), int(cols), int(max_n), ctypes.byref(nbytes)),
               "csrt_workspace_bytes")
        self._init(nbytes.value, device, stream)

    def _init(self, nbytes, device, stream):
        self.nbytes = int(nbytes)
        self.buf = torch.empty(self.nbytes, dtype=torch.uint8, device=device)
        self.ptr = _ptr(self.buf)
        _check(lib().csrt_workspace_init(_ptr(self.buf), self.nbytes, _stream(stream)), "csrt_workspace_init")

    def status(self, stream=None):
        flags, req = c_int32(0), c_int64(0)
        _check(lib().csrt_get_status(self.ptr, ctypes.byref(flags), ctypes.byref(req), _stream(stream)),
               "csrt_get_status")
        return int(flags.value), int(req.value)

    def clear_status(self, stream=None):
        _check(lib().csrt_clear_status(self.ptr, _stream(stream)), "csrt_clear_status")


# ---------------------------------------------------------------------------
# The training-step calls
# ---------------------------------------------------------------------------

def csr_from_dense(dense: torch.Tensor, out: CSR, ws: Workspace, stream=None):
    _f32(dense, "dense", out.rows * out.cols)
    _check(lib().csr_from_dense(_ptr(dense), out.rows, out.cols, out.struct, ws.ptr, ws.nbytes, _stream(stream)),
           "csr_from_dense")


def validate_csr(w: CSR, ws: Workspace, stream=None):
    """Structural check of w (and its transposed copy). Returns the first row
    with a broken invariant (see csrt_get_invalid_row), or None. Synchronises;
    leaves CSRT_DEV_INVALID set in the status word when it finds one."""
    _check(lib().csrt_validate_csr(w.struct, ws.ptr, ws.nbytes, _stream(stream)), "csrt_validate_csr")
    row = c_int64(0)
    _check(lib().csrt_get_invalid_row(ws.ptr, ctypes.byref(row), _stream(stream)), "csrt_get_invalid_row")
    return None if row.value < 0 else int(row.value)


def csr_transpose(w: CSR, ws: Workspace, stream=None):
    _check(lib().csr_transpose(w.struct, ws.ptr, ws.nbytes, _stream(stream)), "csr_transpose")


def spmm_fwd(w: CSR, x: torch.Tensor, y: torch.Tensor, ws: Workspace, stream=None):
    n = x.shape[1] if x.dim() == 2 else x.numel() // max(w.cols, 1)
    _f32(x, "X", w.cols * n)
    _f32(y, "Y", w.rows * n)
    _check(lib().spmm_fwd(w.struct, _ptr(x), n, _ptr(y), ws.ptr, ws.nbytes, _stream(stream)), "spmm_fwd")


def spmm_bwd_t(w: CSR, dy: torch.Tensor, dx: torch.Tensor, ws: Workspace, stream=None):
    n = dy.shape[1] if dy.dim() == 2 else dy.numel() // max(w.rows, 1)
    _f32(dy, "dY", w.rows * n)
    _f32(dx, "dX", w.cols * n)
    _check(lib().spmm_bwd_t(w.struct, _ptr(dy), n, _ptr(dx), ws.ptr, ws.nbytes, _stream(stream)), "spmm_bwd_t")


def spmm_fwd_bias_act(w: CSR, x: torch.Tensor, bias, relu: bool, y: torch.Tensor, ws: Workspace, stream=None):
    n = x.shape[1] if x.dim() == 2 else x.numel() // max(w.cols, 1)
    _f32(x, "X", w.cols * n)
    _f32(y, "Y", w.rows * n)
    if bias is not None:
        _f32(bias, "bias", w.rows)
    _check(lib().spmm_fwd_bias_act(w.struct, _ptr(x), n, _ptr(bias), 1 if relu else 0, _ptr(y), ws.ptr, ws.nbytes,
                                   _stream(stream)), "spmm_fwd_bias_act")


def spmm_bwd_t_relu(w: CSR, dy: torch.Tensor, y_below: torch.Tensor, dx: torch.Tensor, ws: Workspace, stream=None):
    n = dy.shape[1] if dy.dim() == 2 else dy.numel() // max(w.rows, 1)
    _f32(dy, "dY", w.rows * n)
    _f32(dx, "dX", w.cols * n)
    _f32(y_below, "y_below", w.cols * n)
    _check(lib().spmm_bwd_t_relu(w.struct, _ptr(dy), n, _ptr(y_below), _ptr(dx), ws.ptr, ws.nbytes, _stream(stream)),
           "spmm_bwd_t_relu")


def spmm_fwd_noalloc(w: CSR, x: torch.Tensor, y: torch.Tensor, stream=None):
    """spmm_fwd without a workspace (the library's own fixed device scratch)."""
    n = x.shape[1] if x.dim() == 2 else x.numel() // max(w.cols, 1)
    _f32(x, "X", w.cols * n)
    _f32(y, "Y", w.rows * n)
    _check(lib().spmm_fwd_noalloc(w.struct, _ptr(x), n, _ptr(y), _stream(stream)), "spmm_fwd_noalloc")


def weight_grad_dense(dy: torch.Tensor, x: torch.Tensor, g: torch.Tensor, ws: Workspace,
                      precision: int = CSRT_PREC_FP32, stream=None):
    m, n = dy.shape
    k = x.shape[0]
    if x.shape[1] != n:
        raise ValueError("dY and X must have the same number of columns")
    _f32(dy, "dY")
    _f32(x, "X")
    _f32(g, "G", m * k)
    _check(lib().weight_grad_dense(_ptr(dy), _ptr(x), m, k, n, _ptr(g), int(precision), ws.ptr, ws.nbytes,
                                   _stream(stream)), "weight_grad_dense")


def weight_grad_sddmm(w: CSR, dy: torch.Tensor, x: torch.Tensor, g: torch.Tensor, ws: Workspace, stream=None):
    n = dy.shape[1]
    _f32(dy, "dY", w.rows * n)
    _f32(x, "X", w.cols * n)
    _f32(g, "g", 1)
    _check(lib().weight_grad_sddmm(w.struct, _ptr(dy), _ptr(x), n, _ptr(g), ws.ptr, ws.nbytes, _stream(stream)),
           "weight_grad_sddmm")


def prox_update_compact(w_in: CSR, g: torch.Tensor, eta: float, lam: float, w_out: CSR, ws: Workspace,
                        stream=None):
    _f32(g, "G", w_in.rows * w_in.cols)
    _check(lib().prox_update_compact(w_in.struct, _ptr(g), float(eta), float(lam), w_out.struct, ws.ptr,
                                     ws.nbytes, _stream(stream)), "prox_update_compact")


def prox_rmsprop_update_compact(w_in: CSR, g: torch.Tensor, v: torch.Tensor, eta: float, lam: float, beta: float,
                                eps: float, w_out: CSR, ws: Workspace, stream=None):
    """One Prox-RMSProp step (Algorithm 1); v (M x K) is updated in place."""
    _f32(g, "G", w_in.rows * w_in.cols)
    _f32(v, "v", w_in.rows * w_in.cols)
    _check(lib().prox_rmsprop_update_compact(w_in.struct, _ptr(g), _ptr(v), float(eta), float(lam), float(beta),
                                             float(eps), w_out.struct, ws.ptr, ws.nbytes, _stream(stream)),
           "prox_rmsprop_update_compact")


def prox_adam_update_compact(w_in: CSR, g: torch.Tensor, m: torch.Tensor, v: torch.Tensor, t: int, eta: float,
                             lam: float, beta1: float, beta2: float, eps: float, w_out: CSR, ws: Workspace,
                             stream=None):
    """Step t >= 1 of Prox-ADAM (Algorithm 2); m and v (M x K) are updated in place."""
    _f32(g, "G", w_in.rows * w_in.cols)
    _f32(m, "m", w_in.rows * w_in.cols)
    _f32(v, "v", w_in.rows * w_in.cols)
    _check(lib().prox_adam_update_compact(w_in.struct, _ptr(g), _ptr(m), _ptr(v), int(t), float(eta), float(lam),
                                          float(beta1), float(beta2), float(eps), w_out.struct, ws.ptr, ws.nbytes,
                                          _stream(stream)), "prox_adam_update_compact")


def weight_grad_prox_update(w_in: CSR, dy: torch.Tensor, x: torch.Tensor, eta: float, lam: float, w_out: CSR,
                            ws: Workspace, precision: int = CSRT_PREC_TF32, g_scratch=None, stream=None):
    n = dy.shape[1]
    _f32(dy, "dY", w_in.rows * n)
    _f32(x, "X", w_in.cols * n)
    if g_scratch is not None:
        _f32(g_scratch, "g_scratch", w_in.rows * w_in.cols)
    _check(lib().weight_grad_prox_update(w_in.struct, _ptr(dy), _ptr(x), n, float(eta), float(lam), int(precision),
                                         _ptr(g_scratch), w_out.struct, ws.ptr, ws.nbytes, _stream(stream)),
           "weight_grad_prox_update")


def debias_update(w: CSR, g: torch.Tensor, eta: float, stream=None):
    _f32(g, "g", 1)
    _check(lib().debias_update(w.struct, _ptr(g), float(eta), _stream(stream)), "debias_update")


# ---------------------------------------------------------------------------
# Dense layers and the orthogonalised update
# ---------------------------------------------------------------------------

_DTYPES = {torch.float32: CSRT_DT_F32, torch.bfloat16: CSRT_DT_BF16, torch.float16: CSRT_DT_F16}
_ACTS = {"none": CSRT_ACT_NONE, "relu": CSRT_ACT_RELU, "gelu": CSRT_ACT_GELU, "silu": CSRT_ACT_SILU}


class DenseWorkspace(Workspace):
    """Workspace of the dense-layer calls on a layer of m outputs and k inputs
    with at most max_n columns."""

    def __init__(self, m: int, k: int, max_n: int, device="cuda", stream=None):
        nbytes = c_size_t(0)
        _check(lib().csrt_dense_workspace_bytes(int(m), int(k), int(max_n), ctypes.byref(nbytes)),
               "csrt_dense_workspace_bytes")
        self._init(nbytes.value, device, stream)


class OrthogonalizeWorkspace(Workspace):
    """Workspace of orthogonalize for `batch` matrices of rows x cols."""

    def __init__(self, batch: int, rows: int, cols: int, device="cuda", stream=None):
        nbytes = c_size_t(0)
        _check(lib().csrt_orthogonalize_workspace_bytes(int(batch), int(rows), int(cols), ctypes.byref(nbytes)),
               "csrt_orthogonalize_workspace_bytes")
        self._init(nbytes.value, device, stream)


def _mat(t, name):
    """csrt_mat of a 2-D CUDA tensor whose rows are contiguous (any row stride
    of at least a row)."""
    if not t.is_cuda or t.dim() != 2:
        raise ValueError(f"{name} must be a 2-D CUDA tensor")
    rows, cols = t.shape
    ld, inner = t.stride()
    if inner != 1 and cols > 1:
        raise ValueError(f"{name}: the elements of a row must be contiguous")
    if ld < cols:
        if rows > 1:
            raise ValueError(f"{name}: rows overlap")
        ld = cols
    dtype = _DTYPES.get(t.dtype)
    if dtype is None:
        raise ValueError(f"{name}: {t.dtype} is not supported")
    return csrt_mat(t.data_ptr(), rows, cols, ld, dtype)


def _act(act):
    if act not in _ACTS:
        raise ValueError(f"unknown activation {act!r}")
    return _ACTS[act]


def dense_fwd(w, x, y, ws: Workspace, bias=None, act: str = "none", residual=None, z=None, stream=None):
    """y = act(w x + bias) + residual; z (optional) receives w x + bias."""
    if bias is not None:
        _f32(bias, "bias", w.shape[0])
    _check(lib().csrt_dense_fwd(_mat(w, "w"), _mat(x, "x"), _ptr(bias), _act(act),
                                None if residual is None else _mat(residual, "residual"),
                                None if z is None else _mat(z, "z"), _mat(y, "y"), ws.ptr, ws.nbytes,
                                _stream(stream)), "csrt_dense_fwd")


def dense_bwd_x(w, dy, dx, ws: Workspace, z_below=None, act: str = "none", residual=None, stream=None):
    """dx = (w^T dy) * act'(z_below) + residual."""
    _check(lib().csrt_dense_bwd_x(_mat(w, "w"), _mat(dy, "dy"), None if z_below is None else _mat(z_below, "z_below"),
                                  _act(act), None if residual is None else _mat(residual, "residual"), _mat(dx, "dx"),
                                  ws.ptr, ws.nbytes, _stream(stream)), "csrt_dense_bwd_x")


def dense_bwd_w(dy, x, dw, ws: Workspace, db=None, accumulate: bool = False, stream=None):
    """dw = dy x^T and db = the row sums of dy (both added to what is there with accumulate)."""
    if db is not None:
        _f32(db, "db", dy.shape[0])
    _check(lib().csrt_dense_bwd_w(_mat(dy, "dy"), _mat(x, "x"), 1 if accumulate else 0, _mat(dw, "dw"), _ptr(db),
                                  ws.ptr, ws.nbytes, _stream(stream)), "csrt_dense_bwd_w")


def dense_act_bwd(dy, z, act: str, dpre, stream=None):
    """dpre = dy * act'(z); a conversion with act "none" (z may then be None)."""
    _check(lib().csrt_dense_act_bwd(_mat(dy, "dy"), None if z is None else _mat(z, "z"), _act(act), _mat(dpre, "dpre"),
                                    _stream(stream)), "csrt_dense_act_bwd")


def dense_update(w, d, eta: float, decay: float = 0.0, w16=None, stream=None):
    """w <- w (1 - eta decay) - eta d for the float32 w; w16 (optional) receives its 16-bit copy."""
    _check(lib().csrt_dense_update(_mat(w, "w"), _mat(d, "d"), float(eta), float(decay),
                                   None if w16 is None else _mat(w16, "w16"), _stream(stream)), "csrt_dense_update")


def orthogonalize(g, o, ws: Workspace, momentum=None, beta: float = 0.95, nesterov: bool = True, steps: int = 5,
                  eps: float = 1e-7, scale: float = 1.0, stream=None):
    """o = scale * the Newton-Schulz orthogonalisation of the momentum direction
    of g. g and o are rows x cols, or batch x rows x cols; momentum (float32,
    contiguous, g's shape) is updated in place, None orthogonalises g itself."""
    if g.dim() not in (2, 3) or g.shape != o.shape:
        raise ValueError("g and o must have one shape, rows x cols or batch x rows x cols")
    batch = 1
    g_stride = o_stride = 0
    g2, o2 = g, o
    if g.dim() == 3:
        batch = g.shape[0]
        if batch == 0:
            return
        g_stride, o_stride = g.stride(0), o.stride(0)
        g2, o2 = g[0], o[0]
    if momentum is not None:
        if momentum.shape != g.shape:
            raise ValueError("momentum must have g's shape")
        _f32(momentum, "momentum")
    _check(lib().csrt_orthogonalize(_mat(g2, "g"), g_stride, batch, _ptr(momentum), float(beta), 1 if nesterov else 0,
                                    int(steps), float(eps), float(scale), _mat(o2, "o"), o_stride, ws.ptr, ws.nbytes,
                                    _stream(stream)), "csrt_orthogonalize")


# ---------------------------------------------------------------------------
# Norms around a block, token embedding, gradient clipping
# ---------------------------------------------------------------------------

_NORMS = {"scale": CSRT_NORM_SCALE, "rms": CSRT_NORM_RMS, "layer": CSRT_NORM_LAYER}
_GATES = {"none": CSRT_GATE_NONE, "sigmoid": CSRT_GATE_SIGMOID, "silu": CSRT_GATE_SILU}


class BlockNormWorkspace(Workspace):
    """Workspace of block_norm_bwd for d features and at most max_n tokens."""

    def __init__(self, d: int, max_n: int, device="cuda", stream=None):
        nbytes = c_size_t(0)
        _check(lib().csrt_block_norm_workspace_bytes(int(d), int(max_n), ctypes.byref(nbytes)),
               "csrt_block_norm_workspace_bytes")
        self._init(nbytes.value, device, stream)


class EmbedWorkspace(Workspace):
    """Workspace of the embedding calls for a table of vocab rows of d features and at most max_n tokens (lookups alone: 0
    serves any number)."""

    def __init__(self, vocab: int, d: int, max_n: int, device="cuda", stream=None):
        nbytes = c_size_t(0)
        _check(lib().csrt_embed_workspace_bytes(int(vocab), int(d), int(max_n), ctypes.byref(nbytes)),
               "csrt_embed_workspace_bytes")
        self._init(nbytes.value, device, stream)


class GradWorkspace(Workspace):
    """Workspace of grad_norm and grad_clip (any number of tensors)."""

    def __init__(self, device="cuda", stream=None):
        nbytes = c_size_t(0)
        _check(lib().csrt_grad_workspace_bytes(ctypes.byref(nbytes)), "csrt_grad_workspace_bytes")
        self._init(nbytes.value, device, stream)


class Norm:
    """A norm over the d features of n tokens (csrt_norm): kind "rms", "layer"
    or "scale"; weight and bias (d floats, or None: ones, zeros); mean and rstd
    (n floats: statistics that the forward call writes, if given, and the
    backward call reads); dweight and dbias (d floats: gradients that the
    backward call writes, if given). The tensors are kept."""

    def __init__(self, kind: str, weight=None, bias=None, eps: float = 1e-5, mean=None, rstd=None, dweight=None,
                 dbias=None):
        if kind not in _NORMS:
            raise ValueError(f"unknown norm {kind!r}")
        self.kind, self.eps = kind, float(eps)
        for name, t in (("weight", weight), ("bias", bias), ("mean", mean), ("rstd", rstd), ("dweight", dweight),
                        ("dbias", dbias)):
            if t is not None:
                _f32(t, name)
        # the fewest elements of what is per feature, and per token
        self._features = min((t.numel() for t in (weight, bias, dweight, dbias) if t is not None), default=2 ** 31)
        self._tokens = min((t.numel() for t in (mean, rstd) if t is not None), default=2 ** 31)
        self.weight, self.bias, self.mean, self.rstd, self.dweight, self.dbias = weight, bias, mean, rstd, dweight, dbias
        self._s = csrt_norm(_NORMS[kind], self.eps, _ptr(weight), _ptr(bias), _ptr(mean), _ptr(rstd), _ptr(dweight),
                            _ptr(dbias))

    def struct(self, d: int, n: int):
        if self._features < d:
            raise ValueError(f"the norm has {self._features} features, needs {d}")
        if self._tokens < n:
            raise ValueError(f"the norm has statistics of {self._tokens} tokens, needs {n}")
        return self._s


def _gate(act):
    if act not in _GATES:
        raise ValueError(f"unknown gate activation {act!r}")
    return _GATES[act]


class _Slots(threading.local):
    """A thread's csrt_mat structures for one call: filled by packing, a third of the time of making new ones (a call of
    eight matrices is bound by the host up to 15 us)."""

    def __init__(self):
        self.buf = bytearray(12 * ctypes.sizeof(csrt_mat))
        self.mats = [csrt_mat.from_buffer(self.buf, k * ctypes.sizeof(csrt_mat)) for k in range(12)]


_slots = _Slots()
_pack_mat = struct.Struct("=Qiiqi4x").pack_into
assert ctypes.sizeof(csrt_mat) == 32


def _puts(tensors, names):
    """_mat of each of up to 12 tensors, in this thread's slots; None stays None."""
    slots = _slots
    buf, mats, types, pack = slots.buf, slots.mats, _DTYPES, _pack_mat
    out = []
    for k, t in enumerate(tensors):
        if t is None:
            out.append(None)
            continue
        shape, stride = t.shape, t.stride()
        if len(shape) != 2 or not t.is_cuda:
            raise ValueError(f"{names[k]} must be a 2-D CUDA tensor")
        rows, cols = shape
        ld, inner = stride
        dtype = types.get(t.dtype)
        if inner != 1 or ld < cols or dtype is None:   # what is left of the checks, and single rows and columns
            m = _mat(t, names[k])
            ld, dtype = m.ld, m.dtype
        pack(buf, 32 * k, t.data_ptr(), rows, cols, ld, dtype)
        out.append(mats[k])
    return out


def _int32(t, name):
    if t.dtype != torch.int32 or not t.is_cuda or not t.is_contiguous() or t.dim() != 1:
        raise ValueError(f"{name} must be a contiguous 1-D int32 CUDA tensor")
    return t


def block_norm_fwd(y, r, h, v, post: Norm | None = None, pre: Norm | None = None, gate=None, gate_act: str = "none",
                   r_scale: float = 1.0, stream=None):
    """t = post(y), h = r_scale r + a(gate) t, v = pre(h): what lies between two
    blocks of a residual network. None leaves out any of y, r, h, post, gate,
    and pre with v."""
    first = y if y is not None else r
    d, n = first.shape if first is not None else (0, 0)
    y, gate, r, h, v = _puts((y, gate, r, h, v), ("y", "gate", "r", "h", "v"))
    _check(lib().csrt_block_norm_fwd(y, None if post is None else post.struct(d, n), gate, _gate(gate_act), r, float(r_scale),
                                     None if pre is None else pre.struct(d, n), h, v, _stream(stream)),
           "csrt_block_norm_fwd")


def block_norm_bwd(dv, dh, h, y, dr, dy, ws: Workspace, post: Norm | None = None, pre: Norm | None = None, gate=None,
                   gate_act: str = "none", dgate=None, r_scale: float = 1.0, accumulate: bool = False, stream=None):
    """The gradients dr, dy and dgate (None: not wanted) from dv and dh (either
    may be None), and the norms' dweight and dbias (added to with accumulate)."""
    first = dv if dv is not None else dh
    d, n = first.shape if first is not None else (0, 0)
    dv, dh, h, y, gate, dr, dy, dgate = _puts((dv, dh, h, y, gate, dr, dy, dgate),
                                              ("dv", "dh", "h", "y", "gate", "dr", "dy", "dgate"))
    _check(lib().csrt_block_norm_bwd(dv, dh, h, None if pre is None else pre.struct(d, n), y,
                                     None if post is None else post.struct(d, n), gate, _gate(gate_act), float(r_scale),
                                     1 if accumulate else 0, dr, dy, dgate, ws.ptr, ws.nbytes, _stream(stream)),
           "csrt_block_norm_bwd")


def embed_fwd(table, tokens, x, ws: Workspace, scale: float = 1.0, stream=None):
    """x[:, c] = scale * table[tokens[c]]; a negative token gives a column of zeros."""
    if _int32(tokens, "tokens").numel() < x.shape[-1]:
        raise ValueError(f"tokens has {tokens.numel()} elements, needs {x.shape[-1]}")
    mtable, mx = _puts((table, x), ("table", "x"))
    _check(lib().csrt_embed_fwd(mtable, tokens.data_ptr(), float(scale), mx, ws.ptr, ws.nbytes, _stream(stream)),
           "csrt_embed_fwd")


def embed_bwd(dx, tokens, dtable, ws: Workspace, scale: float = 1.0, accumulate: bool = False, stream=None):
    """dtable[v] = scale * the sum of dx[:, c] over the tokens c that are v (with
    accumulate: added to it, rows without tokens left as they are)."""
    if _int32(tokens, "tokens").numel() < dx.shape[-1]:
        raise ValueError(f"tokens has {tokens.numel()} elements, needs {dx.shape[-1]}")
    mdx, mtable = _puts((dx, dtable), ("dx", "dtable"))
    _check(lib().csrt_embed_bwd(mdx, tokens.data_ptr(), float(scale), 1 if accumulate else 0, mtable, ws.ptr, ws.nbytes,
                                _stream(stream)), "csrt_embed_bwd")


class TensorList:
    """Tensors that grad_norm and grad_clip take together, described once: 2-D
    ones with contiguous rows, or contiguous ones of any shape. The tensors are
    kept; their storage must stay where it is. Lists that grad_clip writes to
    hold no two tensors of one memory (columns of one buffer count as such)."""

    def __init__(self, tensors):
        self.tensors = list(tensors)
        self._s = (csrt_mat * max(1, len(self.tensors)))()
        for k, t in enumerate(self.tensors):
            name = f"tensor {k}"
            if t.dim() != 2:
                if not t.is_contiguous():
                    raise ValueError(f"{name} must be contiguous (or 2-D with contiguous rows)")
                if t.numel() >= 2 ** 31:
                    t = t.flatten(0, -2) if t.dim() > 2 else t
                else:
                    t = t.reshape(1, -1)
            if t.dim() != 2 or max(t.shape) >= 2 ** 31:
                raise ValueError(f"{name} has a side of 2^31 or more")
            self._s[k] = _mat(t, name)
        # two tensors of one memory: fine to read, not to write
        extents = sorted((m.data or 0, (m.data or 0) + ((m.rows - 1) * m.ld + m.cols) * (4 if m.dtype == CSRT_DT_F32 else 2),
                          k) for k, m in enumerate(self._s[:len(self.tensors)]) if m.rows and m.cols)
        self.overlap = next(((a[2], b[2]) for a, b in zip(extents, extents[1:]) if b[0] < a[1]), None)

    def __len__(self):
        return len(self.tensors)


def _tensor_list(x):
    return x if isinstance(x, TensorList) else TensorList(x)


def grad_norm(grads, norm, ws: Workspace, stream=None):
    """norm[0] = the square root of the sum of squares over all tensors (a TensorList, or a list of tensors)."""
    grads = _tensor_list(grads)
    _f32(norm, "norm", 2)
    _check(lib().csrt_grad_norm(grads._s, len(grads), _ptr(norm), ws.ptr, ws.nbytes, _stream(stream)), "csrt_grad_norm")


def grad_clip(grads, max_norm: float, norm, ws: Workspace, out=None, stream=None):
    """grad_norm, norm[1] = min(1, max_norm / norm[0]) and out = grads * norm[1] (out None: in place)."""
    grads = _tensor_list(grads)
    out = None if out is None else _tensor_list(out)
    if out is not None and len(out) != len(grads):
        raise ValueError("out must have one tensor for each of grads")
    _f32(norm, "norm", 2)
    overlap = (grads if out is None else out).overlap
    if overlap is not None:
        raise ValueError("tensors %d and %d of %s overlap" % (*sorted(overlap), "grads" if out is None else "out"))
    _check(lib().csrt_grad_clip(grads._s, len(grads), float(max_norm), None if out is None else out._s, norm.data_ptr(),
                                ws.ptr, ws.nbytes, _stream(stream)), "csrt_grad_clip")


# ---------------------------------------------------------------------------
# Glue
# ---------------------------------------------------------------------------

def bias_act_fwd(y, bias, relu: bool, stream=None):
    m, n = y.shape
    _f32(y, "y")
    _check(lib().csrt_bias_act_fwd(_ptr(y), _ptr(bias), m, n, 1 if relu else 0, _stream(stream)),
           "csrt_bias_act_fwd")


def relu_bwd(dy, y, stream=None):
    _f32(dy, "dy")
    _f32(y, "y", dy.numel())
    _check(lib().csrt_relu_bwd(_ptr(dy), _ptr(y), dy.numel(), _stream(stream)), "csrt_relu_bwd")


def bias_grad_sgd(dy, bias, eta: float, gb=None, stream=None):
    m, n = dy.shape
    _f32(dy, "dy")
    _check(lib().csrt_bias_grad_sgd(_ptr(dy), m, n, _ptr(bias), float(eta), _ptr(gb), _stream(stream)),
           "csrt_bias_grad_sgd")


def softmax_xent(z, labels, dz, loss, stream=None):
    c, n = z.shape
    _f32(z, "z")
    _f32(dz, "dz", c * n)
    _f32(loss, "loss", n + 1)
    if labels.dtype != torch.int32 or not labels.is_cuda:
        raise ValueError("labels must be int32 CUDA")
    _check(lib().csrt_softmax_xent(_ptr(z), _ptr(labels), c, n, _ptr(dz), _ptr(loss), _stream(stream)),
           "csrt_softmax_xent")


def im2col(x, c, b, h, w, k, cols, stream=None):
    _check(lib().csrt_im2col(_ptr(_f32(x, "x")), c, b, h, w, k, _ptr(_f32(cols, "cols")), _stream(stream)),
           "csrt_im2col")


def check_bounded_waits(ws: Workspace, stream=None):
    """Run the library's bounded waits against events that never happen; they
    must give up and set CSRT_DEV_TIMEOUT (read it with ws.status())."""
    _check(lib().csrt_check_bounded_waits(ws.ptr, ws.nbytes, _stream(stream)), "csrt_check_bounded_waits")


def fma_peak_tflops(reps: int = 5) -> float:
    """Measured FP32 FMA throughput of the current GPU (TFLOP/s): the median of
    `reps` timed runs of the library's FMA probe (two waves of blocks per SM,
    after a warm-up run), timed with CUDA events on the current stream."""
    sms = torch.cuda.get_device_properties(torch.cuda.current_device()).multi_processor_count
    blocks, iters = 4 * sms, 1 << 15
    out = torch.empty(blocks * 512, dtype=torch.float32, device="cuda")
    flops = ctypes.c_double(0.0)
    s = torch.cuda.current_stream()

    def run():
        _check(lib().csrt_fma_peak_run(_ptr(out), blocks, iters, ctypes.byref(flops), _stream(s)),
               "csrt_fma_peak_run")

    run()
    times = []
    for _ in range(reps):
        st, en = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        st.record(s)
        run()
        en.record(s)
        en.synchronize()
        times.append(st.elapsed_time(en) / 1e3)
    times.sort()
    return flops.value / times[len(times) // 2] / 1e12


def conv2d_sparse_fwd(w: CSR, x, c, b, h, wd, k, bias, relu, y, stream=None):
    """Convolution with CSR filters read straight from the input (no unfolded matrix)."""
    _f32(x, "x", c * b * h * wd)
    _f32(y, "y", w.rows * b * (h - k + 1) * (wd - k + 1))
    bp = _ptr(_f32(bias, "bias", w.rows)) if bias is not None else None
    _check(lib().csrt_conv2d_sparse_fwd(w.struct, _ptr(x), c, b, h, wd, k, bp, int(bool(relu)), _ptr(y),
                                        _stream(stream)), "csrt_conv2d_sparse_fwd")


def col2im(dcols, c, b, h, w, k, dx, stream=None):
    _check(lib().csrt_col2im(_ptr(_f32(dcols, "dcols")), c, b, h, w, k, _ptr(_f32(dx, "dx")), _stream(stream)),
           "csrt_col2im")


def maxpool2_fwd(x, c, b, h, w, y, idx, stream=None):
    _check(lib().csrt_maxpool2_fwd(_ptr(_f32(x, "x")), c, b, h, w, _ptr(_f32(y, "y")), _ptr(idx), _stream(stream)),
           "csrt_maxpool2_fwd")


def maxpool2_bwd(dy, idx, c, b, h, w, dx, stream=None):
    _check(lib().csrt_maxpool2_bwd(_ptr(_f32(dy, "dy")), _ptr(idx), c, b, h, w, _ptr(_f32(dx, "dx")),
                                   _stream(stream)), "csrt_maxpool2_bwd")


def flatten(x, c, b, hw, xf, stream=None):
    _check(lib().csrt_flatten(_ptr(_f32(x, "x")), c, b, hw, _ptr(_f32(xf, "xf")), _stream(stream)), "csrt_flatten")


def unflatten(xf, c, b, hw, x, stream=None):
    _check(lib().csrt_unflatten(_ptr(_f32(xf, "xf")), c, b, hw, _ptr(_f32(x, "x")), _stream(stream)),
           "csrt_unflatten")
