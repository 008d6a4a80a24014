"""ctypes binding of the C ABI declared in ``include/nvfp4.h``.

Argument marshalling only: every function here passes device pointers of torch tensors (torch is used
for device memory and streams) straight to the C entry point of the same name.  There is no CPU or
PyTorch fallback: if the CUDA library is missing and cannot be built, loading fails loudly.
"""
from __future__ import annotations

import ctypes
import struct
from dataclasses import dataclass
from typing import Optional

import torch

from . import build as _build

OK = 0
ROUND_NEAREST_EVEN, ROUND_STOCHASTIC = 0, 1
SF_LINEAR, SF_SWIZZLED = 0, 1
SR_INDEPENDENT_COPIES, AMAX_PROVIDED, INPUT_FP32, LINEAR_ROW_SCALES = 1, 2, 4, 8
FORMAT_NVFP4, FORMAT_MXFP4, FORMAT_NVFP4_ROWSCALE, FORMAT_MXFP8 = 0, 1, 2, 3
ACT_NONE, ACT_RELU2, ACT_SILU, ACT_GELU = 0, 1, 2, 3

EXPORTED = (
    "nvfp4_quantize", "nvfp4_gemm", "nvfp4_linear_fwd_workspace_bytes", "nvfp4_linear_bwd_workspace_bytes",
    "nvfp4_linear_fwd", "nvfp4_linear_bwd", "nvfp4_dequantize", "nvfp4_rht16", "nvfp4_e2m1_sr", "nvfp4_test_wait_timeout",
    "nvfp4_test_cluster_leave", "nvfp4_device_status",
    "nvfp4_set_gemm_tile_n", "nvfp4_gemm_tile", "nvfp4_set_gemm_experiment", "nvfp4_status_string", "nvfp4_launch_count",
    "nvfp4_linear_fwd_noalloc", "nvfp4_linear_fwd_noalloc_max_bytes",
    "nvfp4_gemm_bf16", "nvfp4_linear_bf16_fwd", "nvfp4_linear_bf16_bwd", "nvfp4_quant_error", "nvfp4_sq_error",
    "nvfp4_dequantize_bf16", "nvfp4_rmsnorm_fwd", "nvfp4_rmsnorm_bwd_workspace_bytes", "nvfp4_rmsnorm_bwd",
    "nvfp4_gemm_bf16_epilogue", "nvfp4_act_bwd_workspace_bytes", "nvfp4_act_bwd", "nvfp4_linear_bf16_bwd8_workspace_bytes",
    "nvfp4_linear_bf16_bwd8",
    "nvfp4_headnorm_fwd", "nvfp4_headnorm_bwd_workspace_bytes", "nvfp4_headnorm_bwd",
    "nvfp4_embedding_fwd", "nvfp4_embedding_bwd_workspace_bytes", "nvfp4_embedding_bwd", "nvfp4_logprob_fwd", "nvfp4_logprob_bwd",
    "nvfp4_grad_sq_norm_workspace_bytes", "nvfp4_grad_sq_norm", "nvfp4_grad_clip",
)


class CTensor(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("global_", ctypes.c_void_p),
                ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("sf_layout", ctypes.c_int32),
                ("format", ctypes.c_int32)]

    @property
    def _as_parameter_(self):  # a struct itself may be passed where its address is wanted
        return ctypes.byref(self)


class CQuantOpts(ctypes.Structure):
    _fields_ = [("block_rows", ctypes.c_int32), ("rounding", ctypes.c_int32), ("rht_rowwise", ctypes.c_int32),
                ("rht_colwise", ctypes.c_int32), ("rht_sign_mask", ctypes.c_uint32), ("flags", ctypes.c_int32),
                ("seed", ctypes.c_uint64), ("sr_offset", ctypes.c_uint64), ("rht_dim", ctypes.c_int32),
                ("rht_sign_mask_ext", ctypes.c_uint32 * 3)]


class NVFP4Error(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


_lib = None


def lib() -> ctypes.CDLL:
    """Load (building first if the in-tree library is missing or stale) the C-ABI library."""
    global _lib
    if _lib is None:
        path = _build.build()
        L = ctypes.CDLL(path)
        c = ctypes
        vp, i64, i32, u32 = c.c_void_p, c.c_int64, c.c_int32, c.c_uint32
        TP, OP = c.c_void_p, c.POINTER(CQuantOpts)  # (tensor structs go by address: see NVFP4Tensor.packed)
        L.nvfp4_quantize.restype, L.nvfp4_quantize.argtypes = i32, [vp, i64, i64, i64, OP, TP, TP, vp]
        L.nvfp4_gemm.restype, L.nvfp4_gemm.argtypes = i32, [TP, TP, vp, i32, i64, i32, vp]
        L.nvfp4_linear_fwd_workspace_bytes.restype = c.c_size_t
        L.nvfp4_linear_fwd_workspace_bytes.argtypes = [i64, i64]
        L.nvfp4_linear_bwd_workspace_bytes.restype = c.c_size_t
        L.nvfp4_linear_bwd_workspace_bytes.argtypes = [i64, i64]
        L.nvfp4_linear_fwd.restype = i32
        L.nvfp4_linear_fwd.argtypes = [vp, vp, i64, i64, i64, OP, vp, TP, TP, TP, i32, vp, c.c_size_t, vp]
        L.nvfp4_linear_fwd_noalloc.restype = i32
        L.nvfp4_linear_fwd_noalloc.argtypes = [vp, vp, i64, i64, i64, OP, vp, TP, TP, TP, i32, vp]
        L.nvfp4_linear_fwd_noalloc_max_bytes.restype, L.nvfp4_linear_fwd_noalloc_max_bytes.argtypes = c.c_size_t, []
        L.nvfp4_linear_bwd.restype = i32
        L.nvfp4_linear_bwd.argtypes = [vp, TP, TP, i64, i64, i64, OP, vp, vp, i32, vp, c.c_size_t, vp]
        L.nvfp4_gemm_bf16.restype = i32
        L.nvfp4_gemm_bf16.argtypes = [vp, i32, i64, vp, i32, i64, i64, i64, i64, vp, i32, i64, i32, vp]
        L.nvfp4_linear_bf16_fwd.restype, L.nvfp4_linear_bf16_fwd.argtypes = i32, [vp, vp, i64, i64, i64, vp, vp]
        L.nvfp4_linear_bf16_bwd.restype = i32
        L.nvfp4_linear_bf16_bwd.argtypes = [vp, vp, vp, i64, i64, i64, vp, vp, i32, vp]
        L.nvfp4_quant_error.restype, L.nvfp4_quant_error.argtypes = i32, [vp, i64, i64, i64, TP, vp, vp]
        L.nvfp4_sq_error.restype = i32
        L.nvfp4_sq_error.argtypes = [vp, i32, i64, vp, i32, i64, i64, i64, vp, vp]
        sz, f32 = c.c_size_t, c.c_float
        L.nvfp4_dequantize_bf16.restype, L.nvfp4_dequantize_bf16.argtypes = i32, [TP, vp, i64, vp]
        L.nvfp4_rmsnorm_fwd.restype = i32
        L.nvfp4_rmsnorm_fwd.argtypes = [vp, i64, vp, i64, i32, vp, i64, i64, f32, vp, i64, vp, i64, TP, TP, vp, vp]
        L.nvfp4_rmsnorm_bwd.restype = i32
        L.nvfp4_rmsnorm_bwd.argtypes = [vp, i64, vp, i64, i32, TP, vp, vp, i64, i64, vp, i64, vp, i64, i32, vp, i32, vp, sz, vp]
        L.nvfp4_gemm_bf16_epilogue.restype = i32
        L.nvfp4_gemm_bf16_epilogue.argtypes = [vp, i64, vp, i64, i64, i64, i64, vp, vp, i64, vp]
        L.nvfp4_act_bwd.restype = i32
        L.nvfp4_act_bwd.argtypes = [vp, i64, vp, i64, TP, i32, i64, i64, vp, i64, vp, i64, vp, i32, vp, sz, vp]
        L.nvfp4_linear_bf16_bwd8.restype, L.nvfp4_linear_bf16_bwd8.argtypes = i32, [vp, TP, vp, i64, i64, i64, vp, vp, i32, vp, sz, vp]
        for name in ("nvfp4_rmsnorm_bwd", "nvfp4_act_bwd", "nvfp4_linear_bf16_bwd8"):
            fn = getattr(L, name + "_workspace_bytes")
            fn.restype, fn.argtypes = sz, [i64, i64]
        L.nvfp4_headnorm_fwd.restype = i32
        L.nvfp4_headnorm_fwd.argtypes = [vp, i64, i64, i32, i32, i32, vp, vp, f32, vp, i32, i32, vp, i32, vp, i64, vp]
        L.nvfp4_headnorm_bwd_workspace_bytes.restype, L.nvfp4_headnorm_bwd_workspace_bytes.argtypes = sz, [i64, i32, i32, i32]
        L.nvfp4_headnorm_bwd.restype = i32
        L.nvfp4_headnorm_bwd.argtypes = [vp, i64, vp, i64, i64, i32, i32, i32, vp, vp, f32, vp, i32, i32, vp, i32, vp, i64, vp, vp, i32, vp, sz, vp]
        L.nvfp4_embedding_fwd.restype = i32
        L.nvfp4_embedding_fwd.argtypes = [vp, i32, i64, vp, i32, i64, i64, i64, f32, vp, i32, i64, vp]
        L.nvfp4_embedding_bwd_workspace_bytes.restype, L.nvfp4_embedding_bwd_workspace_bytes.argtypes = sz, [i64, i64, i64]
        L.nvfp4_embedding_bwd.restype = i32
        L.nvfp4_embedding_bwd.argtypes = [vp, i32, i64, vp, i32, i64, i64, i64, f32, vp, i64, i32, vp, sz, vp]
        L.nvfp4_logprob_fwd.restype = i32
        L.nvfp4_logprob_fwd.argtypes = [vp, i32, i64, i64, i64, vp, i32, f32, vp, vp, vp, vp, i32, vp, vp, vp]
        L.nvfp4_logprob_bwd.restype = i32
        L.nvfp4_logprob_bwd.argtypes = [vp, i32, i64, i64, i64, vp, i32, f32, vp, vp, vp, vp, vp, i32, i64, i64, vp]
        L.nvfp4_grad_sq_norm_workspace_bytes.restype, L.nvfp4_grad_sq_norm_workspace_bytes.argtypes = sz, []
        L.nvfp4_grad_sq_norm.restype, L.nvfp4_grad_sq_norm.argtypes = i32, [vp, i32, vp, i32, vp, sz, vp]
        L.nvfp4_grad_clip.restype, L.nvfp4_grad_clip.argtypes = i32, [vp, i32, vp, f32, vp, vp]
        L.nvfp4_dequantize.restype, L.nvfp4_dequantize.argtypes = i32, [TP, vp, vp]
        L.nvfp4_rht16.restype, L.nvfp4_rht16.argtypes = i32, [vp, i64, i64, i64, i32, u32, vp, vp]
        L.nvfp4_e2m1_sr.restype, L.nvfp4_e2m1_sr.argtypes = i32, [vp, vp, i64, vp, vp]
        L.nvfp4_test_wait_timeout.restype, L.nvfp4_test_wait_timeout.argtypes = i32, [ctypes.c_uint64, vp]
        L.nvfp4_test_cluster_leave.restype, L.nvfp4_test_cluster_leave.argtypes = i32, [ctypes.c_uint64, vp, vp]
        L.nvfp4_device_status.restype, L.nvfp4_device_status.argtypes = i32, [vp, c.POINTER(u32)]
        L.nvfp4_set_gemm_tile_n.restype, L.nvfp4_set_gemm_tile_n.argtypes = i32, [i32]
        L.nvfp4_gemm_tile.restype, L.nvfp4_gemm_tile.argtypes = i32, [i32, i64, i64, i64, i32]
        L.nvfp4_set_gemm_experiment.restype, L.nvfp4_set_gemm_experiment.argtypes = i32, [i32, i32, vp]
        L.nvfp4_status_string.restype, L.nvfp4_status_string.argtypes = c.c_char_p, [i32]
        L.nvfp4_launch_count.restype, L.nvfp4_launch_count.argtypes = c.c_uint64, []
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().nvfp4_status_string(status).decode()


def _check(status: int, where: str) -> None:
    if status != OK:
        raise NVFP4Error(status, where)


# torch.cuda.current_stream() builds a Stream object around the handle, 3 us of host time per call; these return it as it is, where
# this torch has them
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_get_device = getattr(torch._C, "_cuda_getDevice", None)


_stream_is_raw = False


def _stream() -> int:
    global _stream_is_raw
    if not _stream_is_raw:  # asked until CUDA is initialised: the answer stays, and asking costs 0.15 us a call
        _stream_is_raw = _raw_stream is not None and _get_device is not None and torch.cuda.is_initialized()
        if not _stream_is_raw:
            return torch.cuda.current_stream().cuda_stream  # (initialises CUDA)
    return _raw_stream(_get_device())


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return t.data_ptr() if t is not None else None


_TENSOR_FIELDS = struct.Struct("PPPqqii")  # nvfp4_tensor
assert _TENSOR_FIELDS.size == ctypes.sizeof(CTensor)


@dataclass
class NVFP4Tensor:
    """Device buffers of one quantized copy ([rows x cols], cols = contraction dimension)."""
    codes: torch.Tensor   # uint8 [rows, cols/2]
    scales: torch.Tensor  # uint8 [rows * cols/16] (linear: viewable as [rows, cols/16])
    glob: Optional[torch.Tensor]  # float32 [2] = {amax, s_dec}
    rows: int
    cols: int
    sf_layout: int = SF_SWIZZLED
    format: int = FORMAT_NVFP4  # FORMAT_MXFP4: scales are rows * cols/32 UE8M0 bytes, glob unused ({0, 1})
    # FORMAT_MXFP8: codes uint8 [rows, cols] (E4M3), scales uint8 [rows, ceil(cols/32)] (UE8M0), glob unused (may be None), SF_LINEAR

    def c(self) -> CTensor:
        return CTensor(self.codes.data_ptr(), self.scales.data_ptr(), _ptr(self.glob), self.rows, self.cols,
                       self.sf_layout, self.format)

    def packed(self) -> bytes:
        """The C struct as bytes; ctypes passes their address.  Half the host time of building a ctypes structure."""
        return _TENSOR_FIELDS.pack(self.codes.data_ptr(), self.scales.data_ptr(), _ptr(self.glob) or 0, self.rows,
                                   self.cols, self.sf_layout, self.format)


def alloc_tensor(rows: int, cols: int, sf_layout: int = SF_SWIZZLED, device="cuda",
                 format: int = FORMAT_NVFP4) -> NVFP4Tensor:
    if format == FORMAT_MXFP8:  # (row by row whatever the layout asked for: it is no operand of the block-scaled product)
        return NVFP4Tensor(torch.empty((rows, cols), dtype=torch.uint8, device=device),
                           torch.empty((rows, (cols + 31) // 32), dtype=torch.uint8, device=device), None, rows, cols, SF_LINEAR, format)
    block = 32 if format == FORMAT_MXFP4 else 16
    glob = torch.zeros((2 * rows if format == FORMAT_NVFP4_ROWSCALE else 2,), dtype=torch.float32, device=device)
    if format == FORMAT_MXFP4:
        glob[1] = 1.0
    return NVFP4Tensor(torch.empty((rows, cols // 2), dtype=torch.uint8, device=device),
                       torch.empty((rows * cols // block,), dtype=torch.uint8, device=device),
                       glob, rows, cols, sf_layout, format)


def quant_opts(block_rows=1, rounding=ROUND_NEAREST_EVEN, rht_rowwise=False, rht_colwise=False, rht_sign_mask=0,
               flags=0, seed=0, sr_offset=0, rht_dim=0) -> CQuantOpts:
    """rht_sign_mask: up to 128 sign bits (bit j negates input j of a chunk); rht_dim: 0 = the format's own size."""
    ext = (ctypes.c_uint32 * 3)(*[(rht_sign_mask >> (32 * i)) & 0xFFFFFFFF for i in (1, 2, 3)])
    return CQuantOpts(block_rows, rounding, int(rht_rowwise), int(rht_colwise), rht_sign_mask & 0xFFFFFFFF, flags, seed,
                      sr_offset, rht_dim, ext)


def _ref(t: Optional[NVFP4Tensor]):
    return t.packed() if t is not None else None


def nvfp4_quantize(x: torch.Tensor, opts: CQuantOpts, rowwise: Optional[NVFP4Tensor] = None,
                   colwise: Optional[NVFP4Tensor] = None) -> None:
    assert x.is_cuda and x.dtype in (torch.bfloat16, torch.float32) and x.dim() == 2 and x.stride(1) == 1
    if x.dtype == torch.float32 and not (opts.flags & INPUT_FP32):  # a binary32 source is announced by a flag
        opts = CQuantOpts.from_buffer_copy(opts)
        opts.flags |= INPUT_FP32
    assert (x.dtype == torch.float32) == bool(opts.flags & INPUT_FP32)
    _check(lib().nvfp4_quantize(x.data_ptr(), x.shape[0], x.shape[1], x.stride(0), ctypes.byref(opts), _ref(rowwise),
                                _ref(colwise), _stream()), "nvfp4_quantize")


def nvfp4_gemm(A: NVFP4Tensor, B: NVFP4Tensor, D: torch.Tensor, accumulate: bool = False) -> None:
    assert D.is_cuda and D.dim() == 2 and D.stride(1) == 1 and D.dtype in (torch.bfloat16, torch.float32)
    _check(lib().nvfp4_gemm(_ref(A), _ref(B), D.data_ptr(), int(D.dtype == torch.float32), D.stride(0),
                            int(accumulate), _stream()), "nvfp4_gemm")


def nvfp4_linear_fwd_workspace_bytes(M: int, K: int) -> int:
    return int(lib().nvfp4_linear_fwd_workspace_bytes(M, K))


def nvfp4_linear_bwd_workspace_bytes(M: int, N: int) -> int:
    return int(lib().nvfp4_linear_bwd_workspace_bytes(M, N))


def nvfp4_linear_fwd(X: torch.Tensor, W: Optional[torch.Tensor], opts: CQuantOpts, Y: torch.Tensor,
                     X_col_saved: Optional[NVFP4Tensor], W_row: NVFP4Tensor, W_col_saved: Optional[NVFP4Tensor],
                     w_is_cached: bool, workspace: torch.Tensor) -> None:
    M, K = X.shape
    N = W_row.rows
    assert X.is_contiguous() and Y.is_contiguous() and Y.dtype == torch.bfloat16 and tuple(Y.shape) == (M, N)
    assert W is None or (W.is_contiguous() and tuple(W.shape) == (N, K))
    _check(lib().nvfp4_linear_fwd(X.data_ptr(), W.data_ptr() if W is not None else None, M, N, K, ctypes.byref(opts),
                                  Y.data_ptr(), _ref(X_col_saved), _ref(W_row), _ref(W_col_saved), int(w_is_cached),
                                  workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream()),
           "nvfp4_linear_fwd")


def nvfp4_linear_fwd_noalloc_max_bytes() -> int:
    return int(lib().nvfp4_linear_fwd_noalloc_max_bytes())


def nvfp4_linear_fwd_noalloc(X: torch.Tensor, W: Optional[torch.Tensor], opts: CQuantOpts, Y: torch.Tensor,
                             X_col_saved: Optional[NVFP4Tensor], W_row: NVFP4Tensor,
                             W_col_saved: Optional[NVFP4Tensor], w_is_cached: bool) -> None:
    """Forward pass for callers that cannot allocate device memory: same as nvfp4_linear_fwd, but the scratch copy
    of X sits in an array built into the library (16 MiB limit; calls must not overlap on the GPU)."""
    M, K = X.shape
    N = W_row.rows
    assert X.is_contiguous() and Y.is_contiguous() and Y.dtype == torch.bfloat16 and tuple(Y.shape) == (M, N)
    assert W is None or (W.is_contiguous() and tuple(W.shape) == (N, K))
    _check(lib().nvfp4_linear_fwd_noalloc(X.data_ptr(), W.data_ptr() if W is not None else None, M, N, K,
                                          ctypes.byref(opts), Y.data_ptr(), _ref(X_col_saved), _ref(W_row),
                                          _ref(W_col_saved), int(w_is_cached), _stream()),
           "nvfp4_linear_fwd_noalloc")


def nvfp4_linear_bwd(dY: torch.Tensor, X_col_saved: Optional[NVFP4Tensor], W_col_saved: Optional[NVFP4Tensor], K: int,
                     opts: CQuantOpts, dX: Optional[torch.Tensor], dW: Optional[torch.Tensor], accumulate_dw: bool,
                     workspace: torch.Tensor) -> None:
    M, N = dY.shape
    assert dY.is_contiguous()
    assert dX is None or (dX.is_contiguous() and dX.dtype == torch.bfloat16 and tuple(dX.shape) == (M, K))
    assert dW is None or (dW.is_contiguous() and dW.dtype == torch.float32 and tuple(dW.shape) == (N, K))
    _check(lib().nvfp4_linear_bwd(dY.data_ptr(), _ref(X_col_saved), _ref(W_col_saved), M, N, K, ctypes.byref(opts),
                                  dX.data_ptr() if dX is not None else None,
                                  dW.data_ptr() if dW is not None else None, int(accumulate_dw),
                                  workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream()),
           "nvfp4_linear_bwd")


K_MAJOR, MN_MAJOR = 0, 1


def nvfp4_gemm_bf16(A: torch.Tensor, B: torch.Tensor, D: torch.Tensor, a_layout: int = K_MAJOR,
                    b_layout: int = K_MAJOR, accumulate: bool = False) -> None:
    """D[M x N] = op(A) op(B)^T in BF16.  K_MAJOR: the operand is [M or N][K]; MN_MAJOR: it is [K][M or N]."""
    for t in (A, B):
        assert t.is_cuda and t.dim() == 2 and t.stride(1) == 1 and t.dtype == torch.bfloat16
    assert D.is_cuda and D.dim() == 2 and D.stride(1) == 1 and D.dtype in (torch.bfloat16, torch.float32)
    M, N = D.shape
    K = A.shape[0] if a_layout == MN_MAJOR else A.shape[1]
    assert tuple(A.shape) == ((K, M) if a_layout == MN_MAJOR else (M, K))
    assert tuple(B.shape) == ((K, N) if b_layout == MN_MAJOR else (N, K))
    _check(lib().nvfp4_gemm_bf16(A.data_ptr(), a_layout, A.stride(0), B.data_ptr(), b_layout, B.stride(0), M, N, K,
                                 D.data_ptr(), int(D.dtype == torch.float32), D.stride(0), int(accumulate), _stream()),
           "nvfp4_gemm_bf16")


def nvfp4_linear_bf16_fwd(X: torch.Tensor, W: torch.Tensor, Y: torch.Tensor) -> None:
    M, K = X.shape
    N = W.shape[0]
    assert X.is_contiguous() and W.is_contiguous() and Y.is_contiguous() and tuple(W.shape) == (N, K)
    assert X.dtype == W.dtype == Y.dtype == torch.bfloat16 and tuple(Y.shape) == (M, N)
    _check(lib().nvfp4_linear_bf16_fwd(X.data_ptr(), W.data_ptr(), M, N, K, Y.data_ptr(), _stream()),
           "nvfp4_linear_bf16_fwd")


def nvfp4_linear_bf16_bwd(dY: torch.Tensor, X: Optional[torch.Tensor], W: Optional[torch.Tensor], K: int,
                          dX: Optional[torch.Tensor], dW: Optional[torch.Tensor], accumulate_dw: bool = False) -> None:
    M, N = dY.shape
    assert dY.is_contiguous() and dY.dtype == torch.bfloat16
    assert dX is None or (W is not None and W.is_contiguous() and tuple(W.shape) == (N, K) and dX.is_contiguous()
                          and dX.dtype == torch.bfloat16 and tuple(dX.shape) == (M, K))
    assert dW is None or (X is not None and X.is_contiguous() and tuple(X.shape) == (M, K) and dW.is_contiguous()
                          and dW.dtype == torch.float32 and tuple(dW.shape) == (N, K))
    _check(lib().nvfp4_linear_bf16_bwd(dY.data_ptr(), X.data_ptr() if X is not None else None,
                                       W.data_ptr() if W is not None else None, M, N, K,
                                       dX.data_ptr() if dX is not None else None,
                                       dW.data_ptr() if dW is not None else None, int(accumulate_dw), _stream()),
           "nvfp4_linear_bf16_bwd")


def nvfp4_quant_error(x: torch.Tensor, q: NVFP4Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Device tensor {sum (x - decode(q))^2, sum x^2} (float64) for the row-wise copy q of x."""
    assert x.is_cuda and x.dim() == 2 and x.stride(1) == 1 and x.dtype == torch.bfloat16
    out = torch.empty(2, dtype=torch.float64, device=x.device) if out is None else out
    _check(lib().nvfp4_quant_error(x.data_ptr(), x.shape[0], x.shape[1], x.stride(0), _ref(q), out.data_ptr(),
                                   _stream()), "nvfp4_quant_error")
    return out


def nvfp4_sq_error(ref: torch.Tensor, test: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Device tensor {sum (ref - test)^2, sum ref^2} (float64) of two 2-D tensors, each bf16 or fp32."""
    for t in (ref, test):
        assert t.is_cuda and t.dim() == 2 and t.stride(1) == 1 and t.dtype in (torch.bfloat16, torch.float32)
    assert ref.shape == test.shape
    out = torch.empty(2, dtype=torch.float64, device=ref.device) if out is None else out
    _check(lib().nvfp4_sq_error(ref.data_ptr(), int(ref.dtype == torch.float32), ref.stride(0), test.data_ptr(),
                                int(test.dtype == torch.float32), test.stride(0), ref.shape[0], ref.shape[1],
                                out.data_ptr(), _stream()), "nvfp4_sq_error")
    return out


def nvfp4_dequantize(t: NVFP4Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    if out is None:
        out = torch.empty((t.rows, t.cols), dtype=torch.float32, device=t.codes.device)
    _check(lib().nvfp4_dequantize(_ref(t), out.data_ptr(), _stream()), "nvfp4_dequantize")
    return out


# ---- around the linear layers -------------------------------------------------------------------------------------------
_BF16, _BF16_OR_FP32 = (torch.bfloat16,), (torch.bfloat16, torch.float32)


def _device() -> int:
    """The current device, which the calls launch on."""
    return _get_device() if _get_device is not None else torch.cuda.current_device()


def _refuse(t, what: str) -> None:
    raise AssertionError(f"{what} on the current device is wanted, not {tuple(t.shape)} {t.dtype} with strides {t.stride()} on {t.device}")


# (The checks are written for the host's time: a call's launch takes 3 us, and an attribute of a tensor 0.1.)
def _matrix(t: torch.Tensor, shape, device: int, dtypes=_BF16, unit: int = 1) -> int:
    """Checks a row-major matrix on the current device and returns its leading dimension (of a single row: its columns, rounded up to `unit`)."""
    if t.shape != shape or t.dtype not in dtypes or t.get_device() != device:
        _refuse(t, f"a row-major {tuple(shape)} matrix of {dtypes}")
    ld, inner = t.stride()
    if inner != 1:
        _refuse(t, f"a row-major {tuple(shape)} matrix of {dtypes}")
    return ld if shape[0] > 1 else -(-shape[1] // unit) * unit  # (a single row's stride says nothing)


def _vector(t: Optional[torch.Tensor], n: int, device: int) -> Optional[int]:
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.numel() != n or t.dim() != 1 or t.get_device() != device or not t.is_contiguous():
        _refuse(t, f"a binary32 vector of {n}")
    return t.data_ptr()


def _copy8(t: NVFP4Tensor, device: int) -> bytes:
    assert t.codes.get_device() == device and t.scales.get_device() == device, "a copy on the current device is wanted"
    assert t.codes.is_contiguous() and t.scales.is_contiguous()
    assert t.codes.numel() >= t.rows * t.cols and t.scales.numel() >= t.rows * ((t.cols + 31) // 32)
    return _TENSOR_FIELDS.pack(t.codes.data_ptr(), t.scales.data_ptr(), 0, t.rows, t.cols, t.sf_layout, t.format)


def _scratch(t: Optional[torch.Tensor], device: int):
    """Address and size of a workspace."""
    if t is None:
        return None, 0
    assert t.get_device() == device and t.is_contiguous()
    return t.data_ptr(), t.numel() * t.element_size()


def nvfp4_dequantize_bf16(t: NVFP4Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The values of an MXFP8 copy in bf16."""
    if out is None:
        out = torch.empty((t.rows, t.cols), dtype=torch.bfloat16, device=t.codes.device)
    dev = _device()
    _check(lib().nvfp4_dequantize_bf16(_copy8(t, dev), out.data_ptr(), _matrix(out, (t.rows, t.cols), dev), _stream()),
           "nvfp4_dequantize_bf16")
    return out


def nvfp4_rmsnorm_fwd(x: torch.Tensor, gain: Optional[torch.Tensor], eps: float, y: Optional[torch.Tensor] = None,
                      rstd: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None,
                      h: Optional[torch.Tensor] = None, y8: Optional[NVFP4Tensor] = None,
                      h8: Optional[NVFP4Tensor] = None) -> None:
    """h = x + residual, y = h / sqrt(mean(h^2) + eps) * gain; y8, h8: MXFP8 copies of y and h."""
    dev, shape = _device(), x.shape
    rows, cols = shape
    ldx = _matrix(x, shape, dev)
    pr = ldr = fp32 = ph = ldh = py = ldy = 0
    if residual is not None:
        pr, ldr, fp32 = residual.data_ptr(), _matrix(residual, shape, dev, _BF16_OR_FP32), residual.dtype == torch.float32
    if h is not None:
        assert residual is None or h.dtype == residual.dtype
        ph, ldh = h.data_ptr(), _matrix(h, shape, dev, _BF16_OR_FP32)
    if y is not None:
        py, ldy = y.data_ptr(), _matrix(y, shape, dev)
    _check(lib().nvfp4_rmsnorm_fwd(x.data_ptr(), ldx, pr, ldr, fp32, _vector(gain, cols, dev), rows, cols, eps, ph, ldh, py, ldy,
                                   _copy8(y8, dev) if y8 is not None else None, _copy8(h8, dev) if h8 is not None else None,
                                   _vector(rstd, rows, dev), _stream()), "nvfp4_rmsnorm_fwd")


def nvfp4_rmsnorm_bwd_workspace_bytes(rows: int, cols: int) -> int:
    return int(lib().nvfp4_rmsnorm_bwd_workspace_bytes(rows, cols))


def nvfp4_rmsnorm_bwd(dy: torch.Tensor, h, gain: Optional[torch.Tensor], rstd: torch.Tensor, dh: torch.Tensor,
                      dgain: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                      residual_grad: Optional[torch.Tensor] = None, accumulate_dgain: bool = False) -> None:
    """h: the kept sum, a bf16 or binary32 tensor or its MXFP8 copy."""
    dev, shape = _device(), dy.shape
    rows, cols = shape
    lddy = _matrix(dy, shape, dev)
    ph = ldh = h32 = prg = ldrg = 0
    h8 = None
    if isinstance(h, NVFP4Tensor):
        h8 = _copy8(h, dev)
    else:
        ph, ldh, h32 = h.data_ptr(), _matrix(h, shape, dev, _BF16_OR_FP32), h.dtype == torch.float32
    if residual_grad is not None:
        assert residual_grad.dtype == dh.dtype
        prg, ldrg = residual_grad.data_ptr(), _matrix(residual_grad, shape, dev, _BF16_OR_FP32)
    ws, nws = _scratch(workspace, dev)
    _check(lib().nvfp4_rmsnorm_bwd(dy.data_ptr(), lddy, ph, ldh, h32, h8, _vector(gain, cols, dev), _vector(rstd, rows, dev), rows, cols,
                                   prg, ldrg, dh.data_ptr(), _matrix(dh, shape, dev, _BF16_OR_FP32), dh.dtype == torch.float32,
                                   _vector(dgain, cols, dev), accumulate_dgain, ws, nws, _stream()), "nvfp4_rmsnorm_bwd")


_EPILOGUE_FIELDS = struct.Struct("PPqPqPii")  # nvfp4_epilogue


def nvfp4_gemm_bf16_epilogue(A: torch.Tensor, B: torch.Tensor, D: torch.Tensor, bias: Optional[torch.Tensor] = None,
                             act: int = ACT_NONE, residual: Optional[torch.Tensor] = None, z=None) -> None:
    """z = A B^T + bias, D = act(z) + residual (A [M x K], B [N x K]); z: a bf16 tensor or an MXFP8 copy that is to keep it."""
    dev, shape = _device(), D.shape
    M, N = shape
    K = A.shape[1]
    pr = ldr = pz = ldz = pz8 = 0
    if residual is not None:
        pr, ldr = residual.data_ptr(), _matrix(residual, shape, dev)
    if isinstance(z, NVFP4Tensor):
        held = ctypes.create_string_buffer(_copy8(z, dev))  # (held until the call returns)
        pz8 = ctypes.addressof(held)
    elif z is not None:
        pz, ldz = z.data_ptr(), _matrix(z, shape, dev)
    epilogue = _EPILOGUE_FIELDS.pack(_vector(bias, N, dev) or 0, pr, ldr, pz, ldz, pz8, act, 0)
    _check(lib().nvfp4_gemm_bf16_epilogue(A.data_ptr(), _matrix(A, (M, K), dev), B.data_ptr(), _matrix(B, (N, K), dev), M, N, K,
                                          epilogue, D.data_ptr(), _matrix(D, shape, dev), _stream()), "nvfp4_gemm_bf16_epilogue")


def nvfp4_act_bwd_workspace_bytes(rows: int, cols: int) -> int:
    return int(lib().nvfp4_act_bwd_workspace_bytes(rows, cols))


def nvfp4_act_bwd(da: torch.Tensor, z, act: int, dz: Optional[torch.Tensor] = None, a: Optional[torch.Tensor] = None,
                  dbias: Optional[torch.Tensor] = None, accumulate_dbias: bool = False,
                  workspace: Optional[torch.Tensor] = None) -> None:
    """dz = da act'(z), a = act(z), dbias = column sums of dz; z: a bf16 tensor, its MXFP8 copy, or None where nothing needs it."""
    dev, shape = _device(), da.shape
    rows, cols = shape
    ldda = _matrix(da, shape, dev)
    pz = ldz = pdz = lddz = pa = lda = 0
    z8 = None
    if isinstance(z, NVFP4Tensor):
        z8 = _copy8(z, dev)
    elif z is not None:
        pz, ldz = z.data_ptr(), _matrix(z, shape, dev)
    if dz is not None:
        pdz, lddz = dz.data_ptr(), _matrix(dz, shape, dev)
    if a is not None:
        pa, lda = a.data_ptr(), _matrix(a, shape, dev)
    ws, nws = _scratch(workspace, dev)
    _check(lib().nvfp4_act_bwd(da.data_ptr(), ldda, pz, ldz, z8, act, rows, cols, pdz, lddz, pa, lda, _vector(dbias, cols, dev),
                               accumulate_dbias, ws, nws, _stream()), "nvfp4_act_bwd")


def nvfp4_linear_bf16_bwd8_workspace_bytes(M: int, K: int) -> int:
    return int(lib().nvfp4_linear_bf16_bwd8_workspace_bytes(M, K))


def nvfp4_linear_bf16_bwd8(dY: torch.Tensor, X8: Optional[NVFP4Tensor], W: Optional[torch.Tensor], dX: Optional[torch.Tensor],
                           dW: Optional[torch.Tensor], workspace: Optional[torch.Tensor] = None, accumulate_dw: bool = False) -> None:
    """Both gradients of a BF16 layer whose input was kept as an MXFP8 copy."""
    dev = _device()
    M, N = dY.shape
    K = X8.cols if X8 is not None else W.shape[1]
    assert dY.is_contiguous() and _matrix(dY, (M, N), dev) == N
    pw = pdx = pdw = 0
    if dX is not None:
        assert W is not None and W.is_contiguous() and dX.is_contiguous() and _matrix(W, (N, K), dev) == K and _matrix(dX, (M, K), dev) == K
        pw, pdx = W.data_ptr(), dX.data_ptr()
    if dW is not None:
        assert X8 is not None and dW.is_contiguous() and _matrix(dW, (N, K), dev, (torch.float32,)) == K
        pdw = dW.data_ptr()
    ws, nws = _scratch(workspace, dev)
    _check(lib().nvfp4_linear_bf16_bwd8(dY.data_ptr(), _copy8(X8, dev) if X8 is not None else None, pw, M, N, K, pdx, pdw,
                                        int(accumulate_dw), ws, nws, _stream()), "nvfp4_linear_bf16_bwd8")


# ---- the ends of a training step ------------------------------------------------------------------------------------------
def _indices(t: torch.Tensor, n: int, device: int, what: str):
    """Address of n tokens, targets or positions, and whether they are int64."""
    wide = t.dtype is torch.int64
    if t.shape != (n,) or not (wide or t.dtype is torch.int32) or t.get_device() != device or not t.is_contiguous():
        _refuse(t, f"an int32 or int64 vector of {n} {what}")
    return t.data_ptr(), wide


def _heads(x: torch.Tensor, heads_q: int, heads_k: int, inv_freq, positions, device: int):
    shape = x.shape
    rows, cols = shape
    heads = heads_q + heads_k
    assert heads > 0 and cols % heads == 0, f"{cols} columns are not {heads_q} + {heads_k} heads of one width"
    dim, rotary, pf, pp, wide = cols // heads, 0, 0, 0, False
    if inv_freq is not None:
        rotary = 2 * inv_freq.numel()
        pf = _vector(inv_freq, rotary // 2, device)
    if positions is not None:
        pp, wide = _indices(positions, rows, device, "positions")
    return shape, rows, dim, rotary, pf, pp, wide


def nvfp4_headnorm_fwd(x: torch.Tensor, heads_q: int, heads_k: int, y: torch.Tensor, gain_q: Optional[torch.Tensor] = None,
                       gain_k: Optional[torch.Tensor] = None, eps: float = 1e-5, inv_freq: Optional[torch.Tensor] = None,
                       positions: Optional[torch.Tensor] = None, interleaved: bool = False) -> None:
    """Norm, gain and rotation of the heads in x [rows x (heads_q + heads_k) * dim], the query heads first; y may be x.  Twice as many
    elements of a head turn as inv_freq has (None: none), by positions (None: the row) times inv_freq."""
    dev = _device()
    shape, rows, dim, rotary, pf, pp, wide = _heads(x, heads_q, heads_k, inv_freq, positions, dev)
    _check(lib().nvfp4_headnorm_fwd(x.data_ptr(), _matrix(x, shape, dev), rows, heads_q, heads_k, dim, _vector(gain_q, dim, dev),
                                    _vector(gain_k, dim, dev), eps, pf, rotary, interleaved, pp, wide, y.data_ptr(),
                                    _matrix(y, shape, dev), _stream()), "nvfp4_headnorm_fwd")


def nvfp4_headnorm_bwd_workspace_bytes(rows: int, heads_q: int, heads_k: int, head_dim: int) -> int:
    return int(lib().nvfp4_headnorm_bwd_workspace_bytes(rows, heads_q, heads_k, head_dim))


def nvfp4_headnorm_bwd(dy: torch.Tensor, x: torch.Tensor, heads_q: int, heads_k: int, dx: torch.Tensor,
                       gain_q: Optional[torch.Tensor] = None, gain_k: Optional[torch.Tensor] = None, eps: float = 1e-5,
                       dgain_q: Optional[torch.Tensor] = None, dgain_k: Optional[torch.Tensor] = None,
                       workspace: Optional[torch.Tensor] = None, inv_freq: Optional[torch.Tensor] = None,
                       positions: Optional[torch.Tensor] = None, interleaved: bool = False, accumulate_dgain: bool = False) -> None:
    """The gradient of nvfp4_headnorm_fwd from its input x; dx may be dy or x."""
    dev = _device()
    shape, rows, dim, rotary, pf, pp, wide = _heads(x, heads_q, heads_k, inv_freq, positions, dev)
    ws, nws = _scratch(workspace, dev)
    _check(lib().nvfp4_headnorm_bwd(dy.data_ptr(), _matrix(dy, shape, dev), x.data_ptr(), _matrix(x, shape, dev), rows, heads_q, heads_k, dim,
                                    _vector(gain_q, dim, dev), _vector(gain_k, dim, dev), eps, pf, rotary, interleaved, pp, wide,
                                    dx.data_ptr(), _matrix(dx, shape, dev), _vector(dgain_q, dim, dev), _vector(dgain_k, dim, dev),
                                    accumulate_dgain, ws, nws, _stream()), "nvfp4_headnorm_bwd")


def nvfp4_embedding_fwd(tokens: torch.Tensor, table: torch.Tensor, out: torch.Tensor, scale: float = 1.0) -> None:
    """out[i] = scale * table[tokens[i]], zeros for a token outside of the table."""
    dev = _device()
    (vocab, cols), n = table.shape, tokens.shape[0]
    pt, wide = _indices(tokens, n, dev, "tokens")
    _check(lib().nvfp4_embedding_fwd(pt, wide, n, table.data_ptr(), table.dtype is torch.float32,
                                     _matrix(table, table.shape, dev, _BF16_OR_FP32), vocab, cols, scale, out.data_ptr(),
                                     out.dtype is torch.float32, _matrix(out, (n, cols), dev, _BF16_OR_FP32), _stream()),
           "nvfp4_embedding_fwd")


def nvfp4_embedding_bwd_workspace_bytes(n: int, vocab: int, cols: int) -> int:
    return int(lib().nvfp4_embedding_bwd_workspace_bytes(n, vocab, cols))


def nvfp4_embedding_bwd(tokens: torch.Tensor, dout: torch.Tensor, dtable: torch.Tensor, workspace: torch.Tensor, scale: float = 1.0,
                        accumulate: bool = False) -> None:
    """dtable (+)= scale * the sums of dout's rows by token; without accumulate all of dtable is written."""
    dev = _device()
    (vocab, cols), n = dtable.shape, tokens.shape[0]
    pt, wide = _indices(tokens, n, dev, "tokens")
    ws, nws = _scratch(workspace, dev)
    _check(lib().nvfp4_embedding_bwd(pt, wide, n, dout.data_ptr(), dout.dtype is torch.float32, _matrix(dout, (n, cols), dev, _BF16_OR_FP32),
                                     vocab, cols, scale, dtable.data_ptr(), _matrix(dtable, dtable.shape, dev, (torch.float32,)), accumulate,
                                     ws, nws, _stream()), "nvfp4_embedding_bwd")


def _row_stats(t: Optional[torch.Tensor], rows: int, device: int) -> Optional[int]:
    if t is None:
        return None
    if t.shape != (rows, 2) or t.dtype is not torch.float32 or t.get_device() != device or not t.is_contiguous():
        _refuse(t, f"a contiguous binary32 ({rows}, 2) tensor")
    return t.data_ptr()


def nvfp4_logprob_fwd(logits: torch.Tensor, targets: Optional[torch.Tensor] = None, logprob: Optional[torch.Tensor] = None,
                      lse: Optional[torch.Tensor] = None, stats: Optional[torch.Tensor] = None, entropy: Optional[torch.Tensor] = None,
                      top_ids: Optional[torch.Tensor] = None, top_logprobs: Optional[torch.Tensor] = None, scale: float = 1.0) -> None:
    """Log probabilities of the targets under the softmax of scale * logits, ln of the sum, entropy, and the likeliest tokens (top_ids
    int32, top_logprobs binary32, both [rows x top]).  stats [rows x 2] is what nvfp4_logprob_bwd takes."""
    dev = _device()
    rows, vocab = logits.shape
    pt, wide, top, pid, ptl = 0, False, 0, 0, 0
    if targets is not None:
        pt, wide = _indices(targets, rows, dev, "targets")
    for t, dtype in ((top_ids, torch.int32), (top_logprobs, torch.float32)):
        if t is None:
            continue
        if t.dim() != 2 or t.shape[0] != rows or t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous() or top not in (0, t.shape[1]):
            _refuse(t, f"a contiguous {dtype} ({rows}, top) tensor")
        top = t.shape[1]
        if dtype is torch.int32:
            pid = t.data_ptr()
        else:
            ptl = t.data_ptr()
    _check(lib().nvfp4_logprob_fwd(logits.data_ptr(), logits.dtype is torch.float32, _matrix(logits, logits.shape, dev, _BF16_OR_FP32, 8), rows,
                                   vocab, pt, wide, scale, _vector(logprob, rows, dev), _vector(lse, rows, dev),
                                   _row_stats(stats, rows, dev), _vector(entropy, rows, dev), top, pid, ptl, _stream()), "nvfp4_logprob_fwd")


def nvfp4_logprob_bwd(logits: torch.Tensor, targets: Optional[torch.Tensor], stats: torch.Tensor, dlogits: torch.Tensor,
                      dlogprob: Optional[torch.Tensor] = None, entropy: Optional[torch.Tensor] = None,
                      dentropy: Optional[torch.Tensor] = None, scale: float = 1.0) -> None:
    """The gradient of sum(dlogprob * logprob + dentropy * entropy) by the logits.  dlogits may have more columns than logits, which are
    set to zero, and may be logits itself."""
    dev = _device()
    rows, vocab = logits.shape
    dcols = dlogits.shape[1]
    pt, wide = 0, False
    if targets is not None:
        pt, wide = _indices(targets, rows, dev, "targets")
    _check(lib().nvfp4_logprob_bwd(logits.data_ptr(), logits.dtype is torch.float32, _matrix(logits, logits.shape, dev, _BF16_OR_FP32, 8), rows,
                                   vocab, pt, wide, scale, _row_stats(stats, rows, dev), _vector(entropy, rows, dev),
                                   _vector(dlogprob, rows, dev), _vector(dentropy, rows, dev), dlogits.data_ptr(),
                                   dlogits.dtype is torch.float32, _matrix(dlogits, (rows, dcols), dev, _BF16_OR_FP32, 8), dcols, _stream()),
           "nvfp4_logprob_bwd")


_GRAD_FIELDS = struct.Struct("PPqii")  # nvfp4_grad


class GradList:
    """Gradients (and where their clipped values go) as the C calls take them; holds the tensors."""

    def __init__(self, grads, outs=None):
        self.grads, self.outs = list(grads), list(outs) if outs is not None else None
        assert self.grads and (self.outs is None or len(self.outs) == len(self.grads))
        self.device = self.grads[0].get_device()
        fields = []
        for g, o in zip(self.grads, self.outs if self.outs is not None else self.grads):
            for t in (g, o):
                if t.dtype not in _BF16_OR_FP32 or t.get_device() != self.device or t.device.type != "cuda" or not t.is_contiguous():
                    _refuse(t, "a contiguous bf16 or binary32 tensor, as the others,")
            assert o.numel() == g.numel()
            fields.append(_GRAD_FIELDS.pack(g.data_ptr(), o.data_ptr(), g.numel(), g.dtype is torch.float32, o.dtype is torch.float32))
        self.n, self.packed = len(fields), b"".join(fields)


def grad_list(grads, outs=None) -> GradList:
    """The list that nvfp4_grad_sq_norm and nvfp4_grad_clip take, to be kept while the tensors stay where they are."""
    return GradList(grads, outs)


def _total(t: torch.Tensor, device: int) -> int:
    if t.dtype is not torch.float64 or t.numel() != 1 or t.get_device() != device:
        _refuse(t, "one binary64 number")
    return t.data_ptr()


def nvfp4_grad_sq_norm_workspace_bytes() -> int:
    return int(lib().nvfp4_grad_sq_norm_workspace_bytes())


def nvfp4_grad_sq_norm(grads: GradList, total: torch.Tensor, workspace: torch.Tensor, accumulate: bool = False) -> None:
    """total (binary64, one number) (+)= the sum of the squares of all gradients."""
    dev = _device()
    assert grads.device == dev, "gradients on the current device are wanted"
    ws, nws = _scratch(workspace, dev)
    _check(lib().nvfp4_grad_sq_norm(grads.packed, grads.n, _total(total, dev), accumulate, ws, nws, _stream()), "nvfp4_grad_sq_norm")


def nvfp4_grad_clip(grads: GradList, total: torch.Tensor, max_norm: float, stats: Optional[torch.Tensor] = None) -> None:
    """Scales the gradients to a norm of max_norm where sqrt(total) is larger; stats: binary32 {norm, factor}."""
    dev = _device()
    assert grads.device == dev, "gradients on the current device are wanted"
    _check(lib().nvfp4_grad_clip(grads.packed, grads.n, _total(total, dev), max_norm, _vector(stats, 2, dev), _stream()), "nvfp4_grad_clip")


def nvfp4_rht16(x: torch.Tensor, colwise: bool, sign_mask: int) -> torch.Tensor:
    R, C = (x.shape[1], x.shape[0]) if colwise else tuple(x.shape)
    out = torch.empty((R, C), dtype=torch.float32, device=x.device)
    _check(lib().nvfp4_rht16(x.data_ptr(), x.shape[0], x.shape[1], x.stride(0), int(colwise), sign_mask,
                             out.data_ptr(), _stream()), "nvfp4_rht16")
    return out


def nvfp4_e2m1_sr(v: torch.Tensor, u: torch.Tensor) -> torch.Tensor:
    """E2M1 codes of the scaled fp32 values `v` under stochastic rounding with the uint8 draws `u` (test aid)."""
    assert v.dtype == torch.float32 and u.dtype == torch.uint8 and v.numel() == u.numel()
    v, u = v.contiguous(), u.contiguous()
    out = torch.empty(v.numel(), dtype=torch.uint8, device=v.device)
    _check(lib().nvfp4_e2m1_sr(v.data_ptr(), u.data_ptr(), v.numel(), out.data_ptr(), _stream()), "nvfp4_e2m1_sr")
    return out


def nvfp4_test_wait_timeout(limit_ns: int) -> None:
    """Enqueues the test kernel whose bounded wait runs out after `limit_ns` (the status word then holds 0x7E570001)."""
    _check(lib().nvfp4_test_wait_timeout(limit_ns, _stream()), "nvfp4_test_wait_timeout")


def nvfp4_test_cluster_leave(delay_ns: int, times: torch.Tensor) -> None:
    """Enqueues the test kernel that leaves a cluster in which one block has given up (see the header); times: int64[24]."""
    assert times.dtype == torch.int64 and times.is_contiguous() and times.numel() >= 24 and times.is_cuda
    _check(lib().nvfp4_test_cluster_leave(delay_ns, times.data_ptr(), _stream()), "nvfp4_test_cluster_leave")


def nvfp4_device_status() -> int:
    """Synchronises the current stream; raises if a bounded device-side wait expired."""
    detail = ctypes.c_uint32(0)
    st = lib().nvfp4_device_status(_stream(), ctypes.byref(detail))
    if st != OK:
        raise NVFP4Error(st, f"nvfp4_device_status (code 0x{detail.value:x})")
    return 0


def nvfp4_set_gemm_experiment(mode: int = 0, max_pairs: int = 0, probe: Optional[torch.Tensor] = None) -> None:
    """Measurement aid of the CTA-pair GEMM (see the header); probe: int64 device tensor of 8 words per pair."""
    assert probe is None or (probe.dtype == torch.int64 and probe.is_contiguous())
    if lib().nvfp4_set_gemm_experiment(mode, max_pairs, probe.data_ptr() if probe is not None else None) != 0:
        raise ValueError("nvfp4_set_gemm_experiment: value out of range")


def nvfp4_set_gemm_tile_n(tile_n: int) -> None:
    if lib().nvfp4_set_gemm_tile_n(tile_n) != 0:
        raise ValueError("tile_n must be 0, 128, 256, 512, 640, 642, 644 or 768")


def nvfp4_gemm_tile(bf16: bool, M: int, N: int, K: int, d_is_fp32: bool) -> int:
    """The tile that such a product takes on the current device (see the header); -1 for a size that is refused."""
    return int(lib().nvfp4_gemm_tile(int(bf16), M, N, K, int(d_is_fp32)))


def nvfp4_launch_count() -> int:
    return int(lib().nvfp4_launch_count())
