"""ctypes binding of libsparseffn.so: argument marshalling only.

Every function has the name of the C entry point it calls (see include/sparseffn.h) and takes
torch tensors (device memory, streams) or raw integers; no step of the method runs in Python.
The shared library must have been built (``python -m paper_2602_06183_b200.build``); loading
fails loudly otherwise and there is no fallback path.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsparseffn.so")

SF_OK = 0
SF_ERR_NULL, SF_ERR_SHAPE, SF_ERR_ALIGN, SF_ERR_WORKSPACE = -1, -2, -3, -4
SF_ERR_ARCH, SF_ERR_CUDA, SF_ERR_TIMEOUT, SF_ERR_UNSUPPORTED = -5, -6, -7, -8

SF_CTX_Y2_VALS, SF_CTX_RELU_VALS, SF_CTX_META, SF_CTX_COLIDX, SF_CTX_Y1, SF_CTX_DY1_VALS = range(6)
SF_CTX_Y2_VALS24, SF_CTX_Y2_META24, SF_CTX_DY1_VALS24, SF_CTX_RELU_VALS24 = 6, 7, 8, 9
SF_FFN_SAVE_Y1, SF_FFN_UNFUSED_ACT, SF_FFN_FUSED_ACT, SF_FFN_PACKED_GRAD_OPERANDS, SF_FFN_W2_FD = 1, 2, 4, 8, 16


class sf_ffn_desc(C.Structure):
    _fields_ = [("T", C.c_int64), ("D", C.c_int64), ("F", C.c_int64),
                ("V", C.c_int32), ("N", C.c_int32), ("M", C.c_int32),
                ("prune_mode", C.c_int32), ("flags", C.c_int32)]


class sf_ffn_plan(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("cta_pairs", "y1_selects", "y1_rows", "y1_cols", "dy1_rows", "dy1_cols",
                                         "weight_grad_launches", "weight_grad_cols", "y3_rows", "y3_cols")]


class sf_router_desc(C.Structure):
    _fields_ = [("T", C.c_int64), ("D", C.c_int64), ("F", C.c_int64), ("E", C.c_int32), ("prune_mode", C.c_int32),
                ("flags", C.c_int32), ("reserved", C.c_int32)]


(SF_RCTX_EXPERT, SF_RCTX_ROW_OF_TOKEN, SF_RCTX_SRC_OF_ROW, SF_RCTX_SEGMENTS, SF_RCTX_LOGITS, SF_RCTX_Y2_VALS,
 SF_RCTX_RELU_VALS, SF_RCTX_META, SF_RCTX_Y1, SF_RCTX_DY1_VALS) = range(10)


class sf_gated_ffn_desc(C.Structure):
    _fields_ = [("T", C.c_int64), ("D", C.c_int64), ("F", C.c_int64), ("act", C.c_int32), ("reserved", C.c_int32)]


class sf_gated_ffn_plan(C.Structure):
    _fields_ = [("form", C.c_int32 * 6), ("cols", C.c_int32 * 6), ("parts", C.c_int32 * 6)]


class sf_fp4_plan(C.Structure):
    _fields_ = [("form", C.c_int32), ("cols", C.c_int32), ("parts", C.c_int32)]


SF_GATED_H, SF_GATED_H_KEPT, SF_GATED_Y, SF_GATED_DH, SF_GATED_DX, SF_GATED_DW = range(6)
SF_GATED_NONE, SF_GATED_FEW, SF_GATED_TILES, SF_GATED_SPLIT = range(4)
SF_ACT_SILU, SF_ACT_GELU, SF_ACT_GELU_TANH, SF_ACT_RELU, SF_ACT_SQRELU = range(5)
SF_FP4_NV, SF_FP4_MX = range(2)
SF_BF16, SF_F32 = range(2)


class sf_schedule(C.Structure):
    _fields_ = [("warmup_steps", C.c_int64), ("sparse_steps", C.c_int64), ("total_steps", C.c_int64)]


SF_STEP_DENSE, SF_STEP_SPARSE = 0, 1


class SparseFFNError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (cuda error {last_cuda_error()})")


_lib = None

_vp, _i64, _i32, _sz = C.c_void_p, C.c_int64, C.c_int, C.c_size_t
_SIGNATURES = {
    "sf_status_string": (C.c_char_p, [_i32]),
    "sf_last_cuda_error": (_i32, []),
    "sf_prune24_sizes": (_i32, [_i64, _i64, _i32, C.POINTER(_sz), C.POINTER(_sz)]),
    "sf_prune24_compress": (_i32, [_vp, _i64, _i64, _i64, _i32, _i32, _vp, _vp, _vp, _vp]),
    "sf_vnm_sizes": (_i32, [_i64, _i64, _i32, _i32, _i32, C.POINTER(_sz), C.POINTER(_sz), C.POINTER(_sz)]),
    "sf_vnm_sparsify_act": (_i32, [_vp, _i64, _i64, _i64, _i32, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp]),
    "sf_gemm_workspace_size": (_i32, [_i64, _i64, C.POINTER(_sz)]),
    "sf_gemm_dense": (_i32, [_vp, _i32, _vp, _i32, _vp, _i64, _i64, _i64, _vp, _vp]),
    "sf_gemm_sparse24": (_i32, [_vp, _vp, _vp, _vp, _i64, _i64, _i64, _vp, _vp]),
    "sf_gemm_sparse24_rm": (_i32, [_vp, _vp, _vp, _i32, _vp, _i64, _i64, _i64, _vp, _vp]),
    "sf_gemm_sparse24_noalloc": (_i32, [_vp, _vp, _vp, _vp, _i64, _i64, _i64, _vp]),
    "sf_fp8_quantize": (_i32, [_vp, _i64, _i64, _i64, C.c_float, _vp, _vp]),
    "sf_prune24_fp8_sizes": (_i32, [_i64, _i64, _i32, C.POINTER(_sz), C.POINTER(_sz)]),
    "sf_prune24_compress_fp8": (_i32, [_vp, _i64, _i64, _i64, _i32, _i32, C.c_float, _vp, _vp, _vp, _vp]),
    "sf_gemm_fp8_workspace_size": (_i32, [_i64, _i64, C.POINTER(_sz)]),
    "sf_gemm_fp8_dense": (_i32, [_vp, _vp, _vp, _i64, _i64, _i64, C.c_float, _vp, _vp]),
    "sf_gemm_fp8_sparse24": (_i32, [_vp, _vp, _vp, _vp, _i64, _i64, _i64, C.c_float, _vp, _vp]),
    "sf_gemm_venom": (_i32, [_vp, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _i32, _i32, _vp, _vp]),
    "sf_ffn_workspace_size": (_i32, [C.POINTER(sf_ffn_desc), C.POINTER(_sz), C.POINTER(_sz)]),
    "sf_ffn_step_plan": (_i32, [C.POINTER(sf_ffn_desc), C.POINTER(sf_ffn_plan)]),
    "sf_sparse_ffn_fwd": (_i32, [C.POINTER(sf_ffn_desc), _vp, _vp, _vp, _vp, _vp, _sz, _vp, _sz, _vp]),
    "sf_sparse_ffn_bwd": (_i32, [C.POINTER(sf_ffn_desc), _vp, _vp, _vp, _vp, _vp, _sz, _vp, _vp, _vp, _vp, _sz, _vp]),
    "sf_dense_ffn_fwd": (_i32, [C.POINTER(sf_ffn_desc), _vp, _vp, _vp, _vp, _vp, _sz, _vp, _sz, _vp]),
    "sf_dense_ffn_bwd": (_i32, [C.POINTER(sf_ffn_desc), _vp, _vp, _vp, _vp, _vp, _sz, _vp, _vp, _vp, _vp, _sz, _vp]),
    "sf_ctx_view": (_i32, [C.POINTER(sf_ffn_desc), _vp, _i32, C.POINTER(_vp), C.POINTER(_sz)]),
    "sf_ffn_host_staging_size": (_i32, [C.POINTER(sf_ffn_desc), C.POINTER(_sz)]),
    "sf_ffn_step_host": (_i32, [C.POINTER(sf_ffn_desc), _i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp,
                                _sz, _vp]),
    "sf_gated_ffn_workspace_size": (_i32, [C.POINTER(sf_gated_ffn_desc), C.POINTER(_sz), C.POINTER(_sz)]),
    "sf_gated_ffn_step_plan": (_i32, [C.POINTER(sf_gated_ffn_desc), C.POINTER(sf_gated_ffn_plan)]),
    "sf_gated_ffn_fwd": (_i32, [C.POINTER(sf_gated_ffn_desc), _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp, _sz, _vp]),
    "sf_gated_ffn_bwd": (_i32, [C.POINTER(sf_gated_ffn_desc), _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp, _vp, _vp, _vp, _vp, _sz,
                                _vp]),
    "sf_fp4_sizes": (_i32, [_i64, _i64, _i32, C.POINTER(_sz), C.POINTER(_sz)]),
    "sf_fp4_quantize": (_i32, [_vp, _i64, _i64, _i64, _i32, C.c_float, _vp, _vp, _vp]),
    "sf_fp4_dequantize": (_i32, [_vp, _vp, _i64, _i64, _i32, C.c_float, _vp, _i64, _vp]),
    "sf_gemm_fp4_workspace_size": (_i32, [_i64, _i64, _i64, C.POINTER(_sz)]),
    "sf_gemm_fp4_plan": (_i32, [_i64, _i64, _i64, _i32, _i32, C.POINTER(sf_fp4_plan)]),
    "sf_gemm_fp4": (_i32, [_vp, _vp, _vp, _vp, _i32, _vp, _i64, _i64, _i64, C.c_float, _vp, _sz, _vp]),
    "sf_gemm_fp4_gated": (_i32, [_vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _vp, _i64, _i64, _i64, C.c_float, C.c_float, _vp,
                                 _sz, _vp]),
    "sf_rmsnorm_fwd": (_i32, [_vp, _i64, _vp, _vp, _i64, _i64, C.c_float, _vp, _vp, _vp, _vp, C.c_float, _vp, _vp]),
    "sf_rmsnorm_bwd_workspace_size": (_i32, [_i64, _i64, C.POINTER(_sz)]),
    "sf_rmsnorm_bwd": (_i32, [_vp, _vp, _vp, _vp, _vp, _i64, _i64, _vp, _vp, _vp, _sz, _vp]),
    "sf_gemm_fp8_rows_workspace_size": (_i32, [_i64, _i64, _i64, C.POINTER(_sz)]),
    "sf_gemm_fp8_rows": (_i32, [_vp, _vp, _vp, _vp, _i64, _i64, _i64, C.c_float, _vp, _sz, _vp]),
    "sf_router_balance_workspace_size": (_i32, [_i64, _i64, _i32, C.POINTER(_sz)]),
    "sf_router_balance_fwd": (_i32, [_vp, _vp, _i64, _i32, C.c_float, C.c_float, _vp, _vp, _vp, _sz, _vp]),
    "sf_router_balance_bwd": (_i32, [_vp, _vp, _vp, _vp, _vp, _vp, _i64, _i64, _i32, C.c_float, C.c_float, _vp, _vp, _vp, _vp, _sz, _vp]),
    "sf_orthogonalize_workspace_size": (_i32, [_i64, _i64, C.POINTER(_sz)]),
    "sf_orthogonalize": (_i32, [_vp, _i32, _i64, _i64, _i64, _i32, C.c_float, C.c_float, C.c_float, C.c_float, _vp, _i64, _vp, _sz, _vp]),
    "sf_schedule_step_kind": (_i32, [C.POINTER(sf_schedule), _i64, C.POINTER(_i32)]),
    "sf_schedule_speedup": (_i32, [C.POINTER(sf_schedule), C.c_double, C.POINTER(C.c_double)]),
    "sf_ffn_flop_fraction": (_i32, [_i64, _i64, _i64, _i64, _i64, C.POINTER(C.c_double)]),
    "sf_end_to_end_speedup": (_i32, [C.c_double, C.c_double, C.POINTER(C.c_double)]),
    "sf_ffn_fwd_scheduled": (_i32, [C.POINTER(sf_schedule), _i64, C.POINTER(sf_ffn_desc), _vp, _vp, _vp, _vp, _vp,
                                    _sz, _vp, _sz, _vp]),
    "sf_ffn_bwd_scheduled": (_i32, [C.POINTER(sf_schedule), _i64, C.POINTER(sf_ffn_desc), _vp, _vp, _vp, _vp, _vp,
                                    _sz, _vp, _vp, _vp, _vp, _sz, _vp]),
    "sf_router_fit_host": (_i32, [_vp, _i64, _i64, _i32, _i32, _vp, _vp, _vp]),
    "sf_router_route": (_i32, [_vp, _vp, _i64, _i64, _i32, _vp, _vp, _vp]),
    "sf_routed_ffn_workspace_size": (_i32, [C.POINTER(sf_router_desc), C.POINTER(_sz), C.POINTER(_sz)]),
    "sf_routed_ffn_fwd": (_i32, [C.POINTER(sf_router_desc), _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp, _sz, _vp]),
    "sf_routed_ffn_bwd": (_i32, [C.POINTER(sf_router_desc), _vp, _vp, _vp, _vp, _vp, _sz, _vp, _vp, _vp, _vp, _sz, _vp]),
    "sf_routed_ctx_view": (_i32, [C.POINTER(sf_router_desc), _vp, _i32, C.POINTER(_vp), C.POINTER(_sz)]),
    "sf_selftest_wait_expiry": (_i32, [_vp, _i64, _vp]),
    "sf_trace_set": (_i32, [C.POINTER(_vp), _i32]),
    "sf_trace_count": (_i32, []),
    "sf_check_status": (_i32, [_vp, _vp]),
}

EXPORTED_SYMBOLS = tuple(_SIGNATURES)


def lib() -> C.CDLL:
    """Load the shared library (once). Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2602_06183_b200.build` "
                "(there is no fallback implementation)")
        loaded = C.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(loaded, name)
            fn.restype, fn.argtypes = res, args
        _lib = loaded                    # complete: another thread may take it from here on
    return _lib


def status_string(status: int) -> str:
    return lib().sf_status_string(status).decode()


def last_cuda_error() -> int:
    return lib().sf_last_cuda_error()


def _check(status: int, where: str) -> None:
    if status != SF_OK:
        raise SparseFFNError(status, where)


# Plain integers: the argument types say what they are. A call on a small matrix is host-bound (back to back at
# 4096 x 4096 the pruning call took 10.7 us for a kernel of 7.6), and building ctypes objects and a torch stream object
# was half of its host time.
def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


# The raw handle of the current stream, without a torch.cuda.Stream object where this torch offers it (a private name).
try:
    from torch._C import _cuda_getCurrentRawStream, _cuda_getDevice

    def _current_stream() -> int:
        return _cuda_getCurrentRawStream(_cuda_getDevice())

    _current_device = _cuda_getDevice
except ImportError:
    def _current_stream() -> int:
        return torch.cuda.current_stream().cuda_stream

    _current_device = torch.cuda.current_device


def _stream(stream: Optional[torch.cuda.Stream] = None):
    return _current_stream() if stream is None else stream.cuda_stream


def make_desc(T, D, F, V, M, N=2, prune_mode=0, flags=0) -> sf_ffn_desc:
    return sf_ffn_desc(T, D, F, V, N, M, prune_mode, flags)


# ---- 2:4 pruning -----------------------------------------------------------------------------

def sf_prune24_sizes(rows: int, cols: int, group_dim: int):
    a, b = _sz(), _sz()
    _check(lib().sf_prune24_sizes(rows, cols, group_dim, C.byref(a), C.byref(b)), "sf_prune24_sizes")
    return a.value, b.value


def sf_prune24_compress(W: torch.Tensor, group_dim: int = 1, prune_mode: int = 0, want_dense: bool = False,
                        out=None, stream=None):
    """W: [rows, cols] 16-bit tensor on the device. Returns (vals, meta, dense_or_None)."""
    rows, cols = W.shape
    if out is None:
        R, K = (rows, cols) if group_dim == 1 else (cols, rows)
        sf_prune24_sizes(rows, cols, group_dim)
        vals = torch.empty((R, K // 2), dtype=W.dtype, device=W.device)
        meta = torch.empty((R, K // 16), dtype=torch.int16, device=W.device)
        dense = torch.empty((rows, cols), dtype=W.dtype, device=W.device) if want_dense else None
    else:
        vals, meta, dense = out
    st = lib().sf_prune24_compress(_ptr(W), rows, cols, W.stride(0), group_dim, prune_mode,
                                   _ptr(vals), _ptr(meta), _ptr(dense), _stream(stream))
    _check(st, "sf_prune24_compress")
    return vals, meta, dense


# ---- V:N:M activation sparsification ------------------------------------------------------------

def sf_vnm_sizes(T, F, V, N, M):
    a, b, c = _sz(), _sz(), _sz()
    _check(lib().sf_vnm_sizes(T, F, V, N, M, C.byref(a), C.byref(b), C.byref(c)), "sf_vnm_sizes")
    return a.value, b.value, c.value


def sf_vnm_sparsify_act(P: torch.Tensor, V: int, M: int, N: int = 2, apply_sqrelu: bool = True,
                        want_relu: bool = True, want_dense: bool = False, out=None, stream=None):
    """P: [T, F] 16-bit tensor. Returns (vals, meta, colidx, relu_vals_or_None, dense_or_None)."""
    T, F = P.shape
    if out is None:
        sf_vnm_sizes(T, F, V, N, M)
        G = F // M
        vals = torch.empty((T, 2 * G), dtype=P.dtype, device=P.device)
        meta = torch.empty((T, G // 4), dtype=torch.int16, device=P.device)
        colidx = torch.empty((T // V, G, 4), dtype=torch.uint8, device=P.device)
        relu = torch.empty((T, 2 * G), dtype=P.dtype, device=P.device) if (want_relu and apply_sqrelu) else None
        dense = torch.empty((T, F), dtype=P.dtype, device=P.device) if want_dense else None
    else:
        vals, meta, colidx, relu, dense = out
    st = lib().sf_vnm_sparsify_act(_ptr(P), T, F, P.stride(0), V, N, M, int(apply_sqrelu), _ptr(vals), _ptr(meta),
                                   _ptr(colidx), _ptr(relu), _ptr(dense), _stream(stream))
    _check(st, "sf_vnm_sparsify_act")
    return vals, meta, colidx, relu, dense


# ---- single products -----------------------------------------------------------------------------

def sf_gemm_workspace_size(Mr: int, K: int) -> int:
    a = _sz()
    _check(lib().sf_gemm_workspace_size(Mr, K, C.byref(a)), "sf_gemm_workspace_size")
    return a.value


def _workspace(nbytes: int, device) -> torch.Tensor:
    return torch.zeros((max(nbytes, 256),), dtype=torch.uint8, device=device)


def sf_gemm_dense(A: torch.Tensor, a_kmajor: bool, B: torch.Tensor, b_kmajor: bool, C_out=None,
                  workspace=None, stream=None):
    """C[Mr,Nc] = op(A) op(B)^T. A is [Mr,K] (a_kmajor) or [K,Mr]; B is [Nc,K] (b_kmajor) or [K,Nc]."""
    Mr, K = A.shape if a_kmajor else (A.shape[1], A.shape[0])
    Nc = B.shape[0] if b_kmajor else B.shape[1]
    if C_out is None:
        C_out = torch.empty((Mr, Nc), dtype=A.dtype, device=A.device)
    if workspace is None:
        workspace = _workspace(sf_gemm_workspace_size(Mr, K), A.device)
    st = lib().sf_gemm_dense(_ptr(A), int(a_kmajor), _ptr(B), int(b_kmajor), _ptr(C_out), Mr, Nc, K,
                             _ptr(workspace), _stream(stream))
    _check(st, "sf_gemm_dense")
    return C_out, workspace


def sf_gemm_sparse24(a_vals, a_meta, B, Ct_out=None, workspace=None, stream=None):
    """Ct[Nc,Mr] = (A_s[Mr,K] B[Nc,K]^T)^T with A_s packed (vals [Mr,K/2], meta [Mr,K/16])."""
    Mr, K = a_vals.shape[0], a_vals.shape[1] * 2
    Nc = B.shape[0]
    if Ct_out is None:
        Ct_out = torch.empty((Nc, Mr), dtype=B.dtype, device=B.device)
    if workspace is None:
        workspace = _workspace(sf_gemm_workspace_size(Mr, K), B.device)
    st = lib().sf_gemm_sparse24(_ptr(a_vals), _ptr(a_meta), _ptr(B), _ptr(Ct_out), Mr, Nc, K,
                                _ptr(workspace), _stream(stream))
    _check(st, "sf_gemm_sparse24")
    return Ct_out, workspace


def sf_gemm_sparse24_rm(a_vals, a_meta, B, b_kmajor: bool, C_out=None, workspace=None, stream=None):
    """C[Mr,Nc] = A_s[Mr,K] op(B)^T, row-major output; B is [Nc,K] (b_kmajor) or [K,Nc]."""
    Mr, K = a_vals.shape[0], a_vals.shape[1] * 2
    Nc = B.shape[0] if b_kmajor else B.shape[1]
    if C_out is None:
        C_out = torch.empty((Mr, Nc), dtype=B.dtype, device=B.device)
    if workspace is None:
        workspace = _workspace(sf_gemm_workspace_size(Mr, K), B.device)
    st = lib().sf_gemm_sparse24_rm(_ptr(a_vals), _ptr(a_meta), _ptr(B), int(b_kmajor), _ptr(C_out), Mr, Nc, K,
                                   _ptr(workspace), _stream(stream))
    _check(st, "sf_gemm_sparse24_rm")
    return C_out, workspace


def sf_fp8_quantize(X, scale: float, out=None, stream=None):
    """E4M3 codes (uint8 [rows, cols]) of float(X) * scale; X bf16, may be a strided row view."""
    rows, cols = X.shape
    if out is None:
        out = torch.empty((rows, cols), dtype=torch.uint8, device=X.device)
    _check(lib().sf_fp8_quantize(_ptr(X), rows, cols, X.stride(0) if rows > 1 else cols, float(scale), _ptr(out),
                                 _stream(stream)), "sf_fp8_quantize")
    return out


def sf_prune24_compress_fp8(W, prune_mode: int, scale: float, want_dense: bool = False, out=None, stream=None,
                            group_dim: int = 1):
    """2:4 with the kept values quantised to E4M3 in the same pass. group_dim as for sf_prune24_compress
    (1: groups along a row; 0: along a column, outputs K-major). Returns (vals uint8 [R, K/2], meta int16
    [R, K/16], dense uint8 [rows, cols] or None); ``out`` = a previous result to write into."""
    rows, cols = W.shape
    if out is not None:
        vals, meta, dense = out
    else:
        R, K = (rows, cols) if group_dim == 1 else (cols, rows)
        vb, mb = _sz(), _sz()
        _check(lib().sf_prune24_fp8_sizes(rows, cols, group_dim, C.byref(vb), C.byref(mb)), "sf_prune24_fp8_sizes")
        vals = torch.empty((R, K // 2), dtype=torch.uint8, device=W.device)
        meta = torch.empty((R, K // 16), dtype=torch.int16, device=W.device)
        dense = torch.empty((rows, cols), dtype=torch.uint8, device=W.device) if want_dense else None
    _check(lib().sf_prune24_compress_fp8(_ptr(W), rows, cols, W.stride(0) if rows > 1 else cols, group_dim, prune_mode,
                                         float(scale), _ptr(vals), _ptr(meta), _ptr(dense), _stream(stream)),
           "sf_prune24_compress_fp8")
    return vals, meta, dense


def sf_gemm_fp8_workspace_size(Mr: int, K: int) -> int:
    b = _sz()
    _check(lib().sf_gemm_fp8_workspace_size(Mr, K, C.byref(b)), "sf_gemm_fp8_workspace_size")
    return b.value


def sf_gemm_fp8_dense(A, B, alpha: float, C_out=None, workspace=None, stream=None):
    """C[Mr,Nc] = bf16(alpha * A B^T) on E4M3 codes A [Mr,K], B [Nc,K] (uint8)."""
    Mr, K = A.shape
    Nc = B.shape[0]
    if C_out is None:
        C_out = torch.empty((Mr, Nc), dtype=torch.bfloat16, device=B.device)
    if workspace is None:
        workspace = _workspace(sf_gemm_fp8_workspace_size(Mr, K), B.device)
    _check(lib().sf_gemm_fp8_dense(_ptr(A), _ptr(B), _ptr(C_out), Mr, Nc, K, float(alpha), _ptr(workspace),
                                   _stream(stream)), "sf_gemm_fp8_dense")
    return C_out, workspace


def sf_gemm_fp8_sparse24(a_vals, a_meta, B, alpha: float, C_out=None, workspace=None, stream=None):
    """The same product with A 2:4-packed: a_vals uint8 [Mr,K/2], a_meta canonical [Mr,K/16]."""
    Mr, K = a_vals.shape[0], a_vals.shape[1] * 2
    Nc = B.shape[0]
    if C_out is None:
        C_out = torch.empty((Mr, Nc), dtype=torch.bfloat16, device=B.device)
    if workspace is None:
        workspace = _workspace(sf_gemm_fp8_workspace_size(Mr, K), B.device)
    _check(lib().sf_gemm_fp8_sparse24(_ptr(a_vals), _ptr(a_meta), _ptr(B), _ptr(C_out), Mr, Nc, K, float(alpha),
                                      _ptr(workspace), _stream(stream)), "sf_gemm_fp8_sparse24")
    return C_out, workspace


def sf_gemm_sparse24_noalloc(a_vals, a_meta, B, Ct_out, stream=None):
    """Same product as sf_gemm_sparse24 without a workspace: for callers that cannot allocate device
    memory. ``Ct_out`` [Nc, Mr] must be supplied by the caller; nothing is allocated here either.
    Limit: Mr * K / 8 <= 4 MiB. Calls share one built-in scratch array: keep them on one stream."""
    Mr, K = a_vals.shape[0], a_vals.shape[1] * 2
    Nc = B.shape[0]
    st = lib().sf_gemm_sparse24_noalloc(_ptr(a_vals), _ptr(a_meta), _ptr(B), _ptr(Ct_out), Mr, Nc, K, _stream(stream))
    _check(st, "sf_gemm_sparse24_noalloc")
    return Ct_out


def sf_gemm_venom(a_vals, a_meta, colidx, Bt, V: int, M: int, C_out=None, workspace=None, stream=None):
    """C[T,Nc] = A_vnm[T,F] Bt[F,Nc] with A_vnm in packed V:N:M form."""
    T = a_vals.shape[0]
    F, Nc = Bt.shape
    if C_out is None:
        C_out = torch.empty((T, Nc), dtype=Bt.dtype, device=Bt.device)
    if workspace is None:
        workspace = _workspace(sf_gemm_workspace_size(T, 4 * F // M), Bt.device)
    st = lib().sf_gemm_venom(_ptr(a_vals), _ptr(a_meta), _ptr(colidx), _ptr(Bt), _ptr(C_out), T, F, Nc, V, M,
                             _ptr(workspace), _stream(stream))
    _check(st, "sf_gemm_venom")
    return C_out, workspace


# ---- FFN step --------------------------------------------------------------------------------------

def sf_ffn_workspace_size(desc: sf_ffn_desc):
    a, b = _sz(), _sz()
    _check(lib().sf_ffn_workspace_size(C.byref(desc), C.byref(a), C.byref(b)), "sf_ffn_workspace_size")
    return a.value, b.value


def sf_ffn_step_plan(desc: sf_ffn_desc) -> sf_ffn_plan:
    plan = sf_ffn_plan()
    _check(lib().sf_ffn_step_plan(C.byref(desc), C.byref(plan)), "sf_ffn_step_plan")
    return plan


def alloc_ffn_buffers(desc: sf_ffn_desc, device="cuda"):
    """(fwd_ctx, workspace) as zero-initialised uint8 tensors of the sizes the library asks for."""
    c, w = sf_ffn_workspace_size(desc)
    return _workspace(c, device), _workspace(w, device)


def _nbytes(t: torch.Tensor) -> int:
    return t.numel() * t.element_size()


def sf_sparse_ffn_fwd(desc, X, W1, W2, Y, fwd_ctx, workspace, stream=None):
    _check(lib().sf_sparse_ffn_fwd(C.byref(desc), _ptr(X), _ptr(W1), _ptr(W2), _ptr(Y), _ptr(fwd_ctx),
                                   _nbytes(fwd_ctx), _ptr(workspace), _nbytes(workspace), _stream(stream)),
           "sf_sparse_ffn_fwd")


def sf_sparse_ffn_bwd(desc, dY, X, W1, W2, fwd_ctx, dX, dW1, dW2, workspace, stream=None):
    _check(lib().sf_sparse_ffn_bwd(C.byref(desc), _ptr(dY), _ptr(X), _ptr(W1), _ptr(W2), _ptr(fwd_ctx),
                                   _nbytes(fwd_ctx), _ptr(dX), _ptr(dW1), _ptr(dW2), _ptr(workspace),
                                   _nbytes(workspace), _stream(stream)), "sf_sparse_ffn_bwd")


def sf_dense_ffn_fwd(desc, X, W1, W2, Y, fwd_ctx, workspace, stream=None):
    _check(lib().sf_dense_ffn_fwd(C.byref(desc), _ptr(X), _ptr(W1), _ptr(W2), _ptr(Y), _ptr(fwd_ctx),
                                  _nbytes(fwd_ctx), _ptr(workspace), _nbytes(workspace), _stream(stream)),
           "sf_dense_ffn_fwd")


def sf_dense_ffn_bwd(desc, dY, X, W1, W2, fwd_ctx, dX, dW1, dW2, workspace, stream=None):
    _check(lib().sf_dense_ffn_bwd(C.byref(desc), _ptr(dY), _ptr(X), _ptr(W1), _ptr(W2), _ptr(fwd_ctx),
                                  _nbytes(fwd_ctx), _ptr(dX), _ptr(dW1), _ptr(dW2), _ptr(workspace),
                                  _nbytes(workspace), _stream(stream)), "sf_dense_ffn_bwd")


_CTX_DTYPES = {SF_CTX_Y2_VALS: torch.bfloat16, SF_CTX_RELU_VALS: torch.bfloat16, SF_CTX_META: torch.int16,
               SF_CTX_COLIDX: torch.uint8, SF_CTX_Y1: torch.bfloat16, SF_CTX_DY1_VALS: torch.bfloat16,
               SF_CTX_Y2_VALS24: torch.bfloat16, SF_CTX_Y2_META24: torch.int16, SF_CTX_DY1_VALS24: torch.bfloat16,
               SF_CTX_RELU_VALS24: torch.bfloat16}


def sf_ctx_view(desc, buf: torch.Tensor, field: int) -> torch.Tensor:
    """A flat tensor aliasing one field of the forward context (or workspace for DY1_VALS)."""
    p, n = _vp(), _sz()
    _check(lib().sf_ctx_view(C.byref(desc), _ptr(buf), field, C.byref(p), C.byref(n)), "sf_ctx_view")
    off = p.value - buf.data_ptr()
    return buf[off:off + n.value].view(_CTX_DTYPES[field])


def sf_ffn_host_staging_size(desc) -> int:
    a = _sz()
    _check(lib().sf_ffn_host_staging_size(C.byref(desc), C.byref(a)), "sf_ffn_host_staging_size")
    return a.value


def sf_ffn_step_host(desc, dense: bool, hX, hW1, hW2, hdY, hY, hdX, hdW1, hdW2, staging, fwd_ctx, workspace,
                     stream=None):
    """Host tensors in, host tensors out (pinned memory recommended); does not synchronise."""
    _check(lib().sf_ffn_step_host(C.byref(desc), int(dense), _ptr(hX), _ptr(hW1), _ptr(hW2), _ptr(hdY), _ptr(hY),
                                  _ptr(hdX), _ptr(hdW1), _ptr(hdW2), _ptr(staging), _ptr(fwd_ctx), _nbytes(fwd_ctx),
                                  _ptr(workspace), _nbytes(workspace), _stream(stream)), "sf_ffn_step_host")


# ---- routed step (neuron-level experts) ------------------------------------------------------------

def make_router_desc(T, D, F, E, prune_mode=0, flags=0) -> sf_router_desc:
    return sf_router_desc(T, D, F, E, prune_mode, flags, 0)


def sf_router_fit_host(W1_bits, E: int, iters: int = 8):
    """Offline balanced clustering on the host. W1_bits: numpy uint16 [F, D] (bf16 patterns).
    Returns numpy arrays (expert int32 [F], perm int32 [F], means uint16 [E, D])."""
    import numpy as np
    W = np.ascontiguousarray(W1_bits, dtype=np.uint16)
    F, D = W.shape
    expert, perm = np.empty(F, dtype=np.int32), np.empty(F, dtype=np.int32)
    means = np.empty((E, D), dtype=np.uint16)
    _check(lib().sf_router_fit_host(W.ctypes.data_as(_vp), F, D, E, iters, expert.ctypes.data_as(_vp),
                                    perm.ctypes.data_as(_vp), means.ctypes.data_as(_vp)), "sf_router_fit_host")
    return expert, perm, means


def sf_router_route(X: torch.Tensor, means: torch.Tensor, want_logits: bool = True, stream=None):
    """X [T, D], means [E, D] (16-bit tensors). Returns (expert int32 [T], logits float32 [T, E] or None)."""
    T, D = X.shape
    E = means.shape[0]
    expert = torch.empty((T,), dtype=torch.int32, device=X.device)
    logits = torch.empty((T, E), dtype=torch.float32, device=X.device) if want_logits else None
    _check(lib().sf_router_route(_ptr(X), _ptr(means), T, D, E, _ptr(expert), _ptr(logits), _stream(stream)),
           "sf_router_route")
    return expert, logits


def sf_routed_ffn_workspace_size(desc: sf_router_desc):
    a, b = _sz(), _sz()
    _check(lib().sf_routed_ffn_workspace_size(C.byref(desc), C.byref(a), C.byref(b)), "sf_routed_ffn_workspace_size")
    return a.value, b.value


def sf_routed_ffn_fwd(desc, X, W1, W2, means, Y, fwd_ctx, workspace, forced_expert=None, stream=None):
    _check(lib().sf_routed_ffn_fwd(C.byref(desc), _ptr(X), _ptr(W1), _ptr(W2), _ptr(means), _ptr(forced_expert), _ptr(Y),
                                   _ptr(fwd_ctx), _nbytes(fwd_ctx), _ptr(workspace), _nbytes(workspace),
                                   _stream(stream)), "sf_routed_ffn_fwd")


def sf_routed_ffn_bwd(desc, dY, X, W1, W2, fwd_ctx, dX, dW1, dW2, workspace, stream=None):
    _check(lib().sf_routed_ffn_bwd(C.byref(desc), _ptr(dY), _ptr(X), _ptr(W1), _ptr(W2), _ptr(fwd_ctx),
                                   _nbytes(fwd_ctx), _ptr(dX), _ptr(dW1), _ptr(dW2), _ptr(workspace),
                                   _nbytes(workspace), _stream(stream)), "sf_routed_ffn_bwd")


_RCTX_DTYPES = {SF_RCTX_EXPERT: torch.int32, SF_RCTX_ROW_OF_TOKEN: torch.int32, SF_RCTX_SRC_OF_ROW: torch.int32,
                SF_RCTX_SEGMENTS: torch.int32, SF_RCTX_LOGITS: torch.float32, SF_RCTX_Y2_VALS: torch.bfloat16,
                SF_RCTX_RELU_VALS: torch.bfloat16, SF_RCTX_META: torch.int16, SF_RCTX_Y1: torch.bfloat16,
                SF_RCTX_DY1_VALS: torch.bfloat16}


def sf_routed_ctx_view(desc, buf: torch.Tensor, field: int) -> torch.Tensor:
    p, n = _vp(), _sz()
    _check(lib().sf_routed_ctx_view(C.byref(desc), _ptr(buf), field, C.byref(p), C.byref(n)), "sf_routed_ctx_view")
    off = p.value - buf.data_ptr()
    return buf[off:off + n.value].view(_RCTX_DTYPES[field])


# ---- gated feed-forward block and 4-bit operands -------------------------------------------------------
# These calls take any number of tokens, so a tensor of another shape, type, layout or device would be read as something else
# without a trace: they are checked here, where the sizes are still known. A call on a single token is host-bound, so what passes is found
# in one expression (0.4 us a tensor) and only what does not is looked at closely. `dev` is the device of the call's first tensor;
# _launch_stream, the last argument of every call, refuses it unless it is the current one.

def _refused(where: str, name: str, t, dtype, shape):
    if t.dtype is not dtype or tuple(t.shape) != shape:
        return SparseFFNError(SF_ERR_SHAPE, f"{where}: {name} is {t.dtype} {tuple(t.shape)}, wanted {dtype} {shape}")
    if not t.is_contiguous():
        return SparseFFNError(SF_ERR_ALIGN, f"{where}: {name} is not contiguous")
    return SparseFFNError(SF_ERR_UNSUPPORTED, f"{where}: {name} is on {t.device}, another device than the first tensor")


def _tensor(where: str, name: str, t, dtype, shape, dev: int):
    """The address of a contiguous tensor of that type and shape on device `dev`."""
    if t.dtype is dtype and t.shape == shape and t.is_contiguous() and t.get_device() == dev:
        return t.data_ptr()
    raise _refused(where, name, t, dtype, shape)


def _buffer(where: str, name: str, t, dev: int):
    """(address, bytes) of a context or workspace; (None, 0) of None."""
    if t is None:
        return None, 0
    if t.is_contiguous() and t.get_device() == dev:
        return t.data_ptr(), t.nbytes
    raise _refused(where, name, t, t.dtype, tuple(t.shape))


def _launch_stream(where: str, dev: int, stream):
    if dev < 0 or dev != _current_device():
        raise SparseFFNError(SF_ERR_UNSUPPORTED, f"{where}: the tensors are on {'the CPU' if dev < 0 else f'device {dev}'}, not on the current device")
    return _current_stream() if stream is None else stream.cuda_stream


def _allocating(stream):
    """Where a call makes its own result, it belongs to the stream that the call runs on."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def make_gated_desc(T, D, F, act=SF_ACT_SILU) -> sf_gated_ffn_desc:
    return sf_gated_ffn_desc(T, D, F, act, 0)


def sf_gated_ffn_workspace_size(desc: sf_gated_ffn_desc):
    a, b = _sz(), _sz()
    _check(lib().sf_gated_ffn_workspace_size(C.byref(desc), C.byref(a), C.byref(b)), "sf_gated_ffn_workspace_size")
    return a.value, b.value


def sf_gated_ffn_step_plan(desc: sf_gated_ffn_desc) -> sf_gated_ffn_plan:
    plan = sf_gated_ffn_plan()
    _check(lib().sf_gated_ffn_step_plan(C.byref(desc), C.byref(plan)), "sf_gated_ffn_step_plan")
    return plan


def alloc_gated_ffn_buffers(desc: sf_gated_ffn_desc, device="cuda", training: bool = True):
    """(fwd_ctx, workspace); without training the context is None. The context is not initialised, the workspace is zero."""
    c, w = sf_gated_ffn_workspace_size(desc)
    return torch.empty((c,), dtype=torch.uint8, device=device) if training else None, _workspace(w, device)


def sf_gated_ffn_fwd(desc, X, Wg, Wu, Wd, Y, fwd_ctx, workspace, stream=None):
    """Y = (act(X Wg^T) * (X Wu^T)) Wd^T. fwd_ctx None: nothing is kept for a backward pass."""
    w, bf, dev = "sf_gated_ffn_fwd", _BF16, X.get_device()
    td, fd, df = (desc.T, desc.D), (desc.F, desc.D), (desc.D, desc.F)
    _check(lib().sf_gated_ffn_fwd(
        C.byref(desc), _tensor(w, "X", X, bf, td, dev), _tensor(w, "Wg", Wg, bf, fd, dev), _tensor(w, "Wu", Wu, bf, fd, dev),
        _tensor(w, "Wd", Wd, bf, df, dev), _tensor(w, "Y", Y, bf, td, dev), *_buffer(w, "fwd_ctx", fwd_ctx, dev),
        *_buffer(w, "workspace", workspace, dev), _launch_stream(w, dev, stream)), w)


def sf_gated_ffn_bwd(desc, dY, X, Wg, Wu, Wd, fwd_ctx, dX, dWg, dWu, dWd, workspace, stream=None):
    """Gradients of sf_gated_ffn_fwd with the context that it filled. An output of None is left out."""
    w, bf, dev = "sf_gated_ffn_bwd", _BF16, X.get_device()
    td, fd, df = (desc.T, desc.D), (desc.F, desc.D), (desc.D, desc.F)
    _check(lib().sf_gated_ffn_bwd(
        C.byref(desc), _tensor(w, "dY", dY, bf, td, dev), _tensor(w, "X", X, bf, td, dev), _tensor(w, "Wg", Wg, bf, fd, dev),
        _tensor(w, "Wu", Wu, bf, fd, dev), _tensor(w, "Wd", Wd, bf, df, dev), *_buffer(w, "fwd_ctx", fwd_ctx, dev),
        None if dX is None else _tensor(w, "dX", dX, bf, td, dev), None if dWg is None else _tensor(w, "dWg", dWg, bf, fd, dev),
        None if dWu is None else _tensor(w, "dWu", dWu, bf, fd, dev), None if dWd is None else _tensor(w, "dWd", dWd, bf, df, dev),
        *_buffer(w, "workspace", workspace, dev), _launch_stream(w, dev, stream)), w)


def sf_fp4_sizes(rows: int, cols: int, fmt: int):
    a, b = _sz(), _sz()
    _check(lib().sf_fp4_sizes(rows, cols, fmt, C.byref(a), C.byref(b)), "sf_fp4_sizes")
    return a.value, b.value


_BF16, _U8 = torch.bfloat16, torch.uint8
_SCALE_TILE = {SF_FP4_NV: 6, SF_FP4_MX: 7}          # log2 of the columns of a tile of scales


def _scale_bytes(rows: int, cols: int, fmt: int) -> int:
    """Bytes of the scale tiles, as sf_fp4_sizes has them."""
    lg = _SCALE_TILE.get(fmt)
    if lg is None or cols & 31:
        return sf_fp4_sizes(rows, cols, fmt)[1]                  # refuses
    return ((rows + 127 >> 7) * (cols + (1 << lg) - 1 >> lg)) << 9


def _matrix_shape(where: str, t, name: str = "codes"):
    if t.dim() != 2:
        raise SparseFFNError(SF_ERR_SHAPE, f"{where}: {name} must be a matrix")
    return t.shape


def _row_stride(where: str, name: str, t) -> int:
    """Leading dimension of a bfloat16 matrix with contiguous rows."""
    if t.dtype is not torch.bfloat16 or t.dim() != 2:
        raise SparseFFNError(SF_ERR_SHAPE, f"{where}: {name} must be a bfloat16 matrix")
    if t.stride(1) != 1 and t.size(1) > 1:
        raise SparseFFNError(SF_ERR_ALIGN, f"{where}: {name}'s rows are not contiguous")
    return t.stride(0) if t.size(0) > 1 else t.size(1)


def sf_fp4_quantize(X, fmt: int, scale: float, out=None, stream=None):
    """(codes uint8 [rows, cols/2], scales uint8 tiles) of bf16 X, which may be a strided row view; ``out`` = a previous result
    to write into."""
    w, u8, dev = "sf_fp4_quantize", _U8, X.get_device()
    ld = _row_stride(w, "X", X)
    rows, cols = X.shape
    n = _scale_bytes(rows, cols, fmt)
    if out is None:
        with _allocating(stream):
            out = torch.empty((rows, cols // 2), dtype=u8, device=X.device), torch.empty((n,), dtype=u8, device=X.device)
    codes, scales = out
    _check(lib().sf_fp4_quantize(X.data_ptr(), rows, cols, ld, fmt, scale, _tensor(w, "codes", codes, u8, (rows, cols // 2), dev),
                                 _tensor(w, "scales", scales, u8, (n,), dev), _launch_stream(w, dev, stream)), w)
    return out


def sf_fp4_dequantize(codes, scales, fmt: int, alpha: float, out=None, stream=None):
    """bf16 [rows, cols] = code * sf * alpha; ``out`` may be a strided row view."""
    w, u8, dev = "sf_fp4_dequantize", _U8, codes.get_device()
    rows, half = _matrix_shape(w, codes)
    cols = 2 * half
    if out is None:
        with _allocating(stream):
            out = torch.empty((rows, cols), dtype=torch.bfloat16, device=codes.device)
    ld = _row_stride(w, "out", out)
    if out.shape != (rows, cols) or out.get_device() != dev:
        raise _refused(w, "out", out, torch.bfloat16, (rows, cols))
    _check(lib().sf_fp4_dequantize(_tensor(w, "codes", codes, u8, (rows, half), dev),
                                   _tensor(w, "scales", scales, u8, (_scale_bytes(rows, cols, fmt),), dev), rows, cols, fmt, alpha,
                                   out.data_ptr(), ld, _launch_stream(w, dev, stream)), w)
    return out


def sf_gemm_fp4_workspace_size(Mr: int, Nc: int, K: int) -> int:
    a = _sz()
    _check(lib().sf_gemm_fp4_workspace_size(Mr, Nc, K, C.byref(a)), "sf_gemm_fp4_workspace_size")
    return a.value


def sf_gemm_fp4_plan(Mr: int, Nc: int, K: int, fmt: int, gated: bool = False) -> sf_fp4_plan:
    plan = sf_fp4_plan()
    _check(lib().sf_gemm_fp4_plan(Mr, Nc, K, fmt, gated, C.byref(plan)), "sf_gemm_fp4_plan")
    return plan


def sf_gemm_fp4(A, a_scales, B, b_scales, fmt: int, alpha: float, C_out=None, workspace=None, stream=None):
    """C[Mr,Nc] = bf16(alpha * A B^T) of two 4-bit operands, codes [Mr,K/2] and [Nc,K/2] with their scales."""
    w, u8, dev = "sf_gemm_fp4", _U8, A.get_device()
    Mr, half = _matrix_shape(w, A)
    Nc, K = _matrix_shape(w, B)[0], 2 * half
    a, a_s = _tensor(w, "A", A, u8, (Mr, half), dev), _tensor(w, "a_scales", a_scales, u8, (_scale_bytes(Mr, K, fmt),), dev)
    b, b_s = _tensor(w, "B", B, u8, (Nc, half), dev), _tensor(w, "b_scales", b_scales, u8, (_scale_bytes(Nc, K, fmt),), dev)
    if C_out is None or workspace is None:
        with _allocating(stream):
            C_out = torch.empty((Mr, Nc), dtype=_BF16, device=A.device) if C_out is None else C_out
            workspace = _workspace(sf_gemm_fp4_workspace_size(Mr, Nc, K), A.device) if workspace is None else workspace
    _check(lib().sf_gemm_fp4(a, a_s, b, b_s, fmt, _tensor(w, "C_out", C_out, _BF16, (Mr, Nc), dev), Mr, Nc, K, alpha,
                             *_buffer(w, "workspace", workspace, dev), _launch_stream(w, dev, stream)), w)
    return C_out


def sf_gemm_fp4_gated(A, a_scales, Bg, bg_scales, Bu, bu_scales, fmt: int, act: int, alpha_g: float, alpha_u: float, H_out=None,
                      workspace=None, stream=None):
    """H[Mr,Nc] = bf16(act(alpha_g * A Bg^T) * (alpha_u * A Bu^T)) of 4-bit operands."""
    w, u8, dev = "sf_gemm_fp4_gated", _U8, A.get_device()
    Mr, half = _matrix_shape(w, A)
    Nc, K = _matrix_shape(w, Bg)[0], 2 * half
    shape, tiles = (Nc, half), (_scale_bytes(Nc, K, fmt),)
    a, a_s = _tensor(w, "A", A, u8, (Mr, half), dev), _tensor(w, "a_scales", a_scales, u8, (_scale_bytes(Mr, K, fmt),), dev)
    g, g_s = _tensor(w, "Bg", Bg, u8, shape, dev), _tensor(w, "bg_scales", bg_scales, u8, tiles, dev)
    u, u_s = _tensor(w, "Bu", Bu, u8, shape, dev), _tensor(w, "bu_scales", bu_scales, u8, tiles, dev)
    if H_out is None or workspace is None:
        with _allocating(stream):
            H_out = torch.empty((Mr, Nc), dtype=_BF16, device=A.device) if H_out is None else H_out
            workspace = _workspace(sf_gemm_fp4_workspace_size(Mr, Nc, K), A.device) if workspace is None else workspace
    _check(lib().sf_gemm_fp4_gated(a, a_s, g, g_s, u, u_s, fmt, act, _tensor(w, "H_out", H_out, _BF16, (Mr, Nc), dev), Mr, Nc, K,
                                   alpha_g, alpha_u, *_buffer(w, "workspace", workspace, dev), _launch_stream(w, dev, stream)), w)
    return H_out


# ---- around the layer: norm, E4M3 rows, balance loss, orthogonalised update --------------------------------
# Checked like the calls above. What a call makes for itself (outputs, workspace) belongs to the stream that it runs on.

_F32, _I32 = torch.float32, torch.int32


def _sized(call: str, *args) -> int:
    n = _sz()
    _check(getattr(lib(), call)(*args, C.byref(n)), call)
    return n.value


def sf_rmsnorm_fwd(X, gamma, eps: float, residual=None, sum=None, Y=None, codes=None, scales=None, scale: float = 1.0, rstd=None, stream=None):
    """S = bf16(X + residual), y = S gamma / rms(S) of every row: S to ``sum``, y as bf16 to ``Y`` or as E4M3 to ``codes`` (with a
    scale to every row in ``scales``, or the given ``scale``), 1 / rms to ``rstd``. What is None is not written; without Y and codes a Y is made.
    X may be a strided row view. Returns Y (or the codes)."""
    w, dev = "sf_rmsnorm_fwd", X.get_device()
    T, D = shape = _matrix_shape(w, X, "X")
    ld = D if X.dtype is _BF16 and X.is_contiguous() else _row_stride(w, "X", X)
    if Y is None and codes is None:
        with _allocating(stream):
            Y = torch.empty((T, D), dtype=_BF16, device=X.device)
    _check(lib().sf_rmsnorm_fwd(X.data_ptr(), ld, None if residual is None else _tensor(w, "residual", residual, _BF16, shape, dev),
                                _tensor(w, "gamma", gamma, _BF16, (D,), dev), T, D, eps,
                                None if sum is None else _tensor(w, "sum", sum, _BF16, shape, dev),
                                None if Y is None else _tensor(w, "Y", Y, _BF16, shape, dev),
                                None if codes is None else _tensor(w, "codes", codes, _U8, shape, dev),
                                None if scales is None else _tensor(w, "scales", scales, _F32, (T,), dev), scale,
                                None if rstd is None else _tensor(w, "rstd", rstd, _F32, (T,), dev), _launch_stream(w, dev, stream)), w)
    return codes if Y is None else Y


def sf_rmsnorm_bwd_workspace_size(T: int, D: int) -> int:
    return _sized("sf_rmsnorm_bwd_workspace_size", T, D)


def sf_rmsnorm_bwd(dY, S, gamma, rstd, dS=None, dX=None, dgamma=None, workspace=None, stream=None):
    """Gradients of sf_rmsnorm_fwd from dY, its sum S and its rstd, dS added: into ``dX`` and ``dgamma``, of which a None is left out (both
    None: both are made). Returns (dX, dgamma)."""
    w, dev = "sf_rmsnorm_bwd", dY.get_device()
    T, D = shape = _matrix_shape(w, dY, "dY")
    both = dX is None and dgamma is None
    if both or (dgamma is not None and workspace is None):
        with _allocating(stream):
            if both:
                dX, dgamma = torch.empty((T, D), dtype=_BF16, device=dY.device), torch.empty((D,), dtype=_BF16, device=dY.device)
            if workspace is None:
                workspace = torch.empty((sf_rmsnorm_bwd_workspace_size(T, D),), dtype=_U8, device=dY.device)
    _check(lib().sf_rmsnorm_bwd(_tensor(w, "dY", dY, _BF16, shape, dev), _tensor(w, "S", S, _BF16, shape, dev), _tensor(w, "gamma", gamma, _BF16, (D,), dev),
                                _tensor(w, "rstd", rstd, _F32, (T,), dev), None if dS is None else _tensor(w, "dS", dS, _BF16, shape, dev), T, D,
                                None if dX is None else _tensor(w, "dX", dX, _BF16, shape, dev), None if dgamma is None else _tensor(w, "dgamma", dgamma, _BF16, (D,), dev),
                                *_buffer(w, "workspace", workspace, dev), _launch_stream(w, dev, stream)), w)
    return dX, dgamma


def sf_gemm_fp8_rows_workspace_size(Mr: int, Nc: int, K: int) -> int:
    return _sized("sf_gemm_fp8_rows_workspace_size", Mr, Nc, K)


def sf_gemm_fp8_rows(A, a_scales, B, alpha: float, C_out=None, workspace=None, stream=None):
    """C[Mr,Nc] = bf16(alpha * a_scales[m] * A B^T) of E4M3 codes A [Mr,K] and B [Nc,K], a float32 scale to every row of A."""
    w, u8, dev = "sf_gemm_fp8_rows", _U8, A.get_device()
    Mr, K = _matrix_shape(w, A)
    Nc = _matrix_shape(w, B)[0]
    if C_out is None or workspace is None:
        with _allocating(stream):
            C_out = torch.empty((Mr, Nc), dtype=_BF16, device=A.device) if C_out is None else C_out
            workspace = _workspace(sf_gemm_fp8_rows_workspace_size(Mr, Nc, K), A.device) if workspace is None else workspace
    _check(lib().sf_gemm_fp8_rows(_tensor(w, "A", A, u8, (Mr, K), dev), _tensor(w, "a_scales", a_scales, _F32, (Mr,), dev),
                                  _tensor(w, "B", B, u8, (Nc, K), dev), _tensor(w, "C_out", C_out, _BF16, (Mr, Nc), dev), Mr, Nc, K, alpha,
                                  *_buffer(w, "workspace", workspace, dev), _launch_stream(w, dev, stream)), w)
    return C_out


def sf_router_balance_workspace_size(T: int, D: int, E: int) -> int:
    return _sized("sf_router_balance_workspace_size", T, D, E)


def sf_router_balance_fwd(logits, expert, balance_coef: float, z_coef: float = 0.0, loss=None, counts=None, workspace=None, stream=None):
    """(loss float32 [3], counts int32 [E]) of logits float32 [T,E] and expert int32 [T] (tokens outside [0,E) are left out): the loss with its
    coefficients, the balance and the z term, and the tokens of every expert."""
    w, dev = "sf_router_balance_fwd", logits.get_device()
    T, E = _matrix_shape(w, logits, "logits")
    if loss is None or counts is None or workspace is None:
        with _allocating(stream):
            loss = torch.empty((3,), dtype=_F32, device=logits.device) if loss is None else loss
            counts = torch.empty((E,), dtype=_I32, device=logits.device) if counts is None else counts
            workspace = _workspace(sf_router_balance_workspace_size(T, 8, E), logits.device) if workspace is None else workspace
    _check(lib().sf_router_balance_fwd(_tensor(w, "logits", logits, _F32, (T, E), dev), _tensor(w, "expert", expert, _I32, (T,), dev), T, E, balance_coef,
                                       z_coef, _tensor(w, "loss", loss, _F32, (3,), dev), _tensor(w, "counts", counts, _I32, (E,), dev),
                                       *_buffer(w, "workspace", workspace, dev), _launch_stream(w, dev, stream)), w)
    return loss, counts


def sf_router_balance_bwd(logits, expert, counts, balance_coef: float, z_coef: float, X, means, dloss=None, dX_in=None, dX=None, dmeans=None,
                          workspace=None, stream=None):
    """Gradients of sf_router_balance_fwd's loss (times ``dloss`` float32 [1], or 1): dX = dX_in + dl means and dmeans = dl^T X, of which a None is
    left out (both None: both are made). Returns (dX, dmeans)."""
    w, dev = "sf_router_balance_bwd", logits.get_device()
    T, E = _matrix_shape(w, logits, "logits")
    D = _matrix_shape(w, X, "X")[1]
    both = dX is None and dmeans is None
    if both or workspace is None:
        with _allocating(stream):
            if both:
                dX, dmeans = torch.empty((T, D), dtype=_BF16, device=X.device), torch.empty((E, D), dtype=_BF16, device=X.device)
            if workspace is None:
                workspace = _workspace(sf_router_balance_workspace_size(T, D, E), X.device)
    _check(lib().sf_router_balance_bwd(_tensor(w, "logits", logits, _F32, (T, E), dev), _tensor(w, "expert", expert, _I32, (T,), dev),
                                       _tensor(w, "counts", counts, _I32, (E,), dev), None if dloss is None else _tensor(w, "dloss", dloss, _F32, (1,), dev),
                                       _tensor(w, "X", X, _BF16, (T, D), dev), _tensor(w, "means", means, _BF16, (E, D), dev), T, D, E, balance_coef, z_coef,
                                       None if dX_in is None else _tensor(w, "dX_in", dX_in, _BF16, (T, D), dev), None if dX is None else _tensor(w, "dX", dX, _BF16, (T, D), dev),
                                       None if dmeans is None else _tensor(w, "dmeans", dmeans, _BF16, (E, D), dev), *_buffer(w, "workspace", workspace, dev),
                                       _launch_stream(w, dev, stream)), w)
    return dX, dmeans


def sf_orthogonalize_workspace_size(rows: int, cols: int) -> int:
    return _sized("sf_orthogonalize_workspace_size", rows, cols)


def _rows_of(where: str, name: str, t, dtypes, shape, dev: int) -> int:
    """Leading dimension of a matrix of contiguous rows, of one of these types, that shape and device."""
    if t.dtype not in dtypes or tuple(t.shape) != shape:
        raise SparseFFNError(SF_ERR_SHAPE, f"{where}: {name} is {t.dtype} {tuple(t.shape)}, wanted {' or '.join(map(str, dtypes))} {shape}")
    if (t.size(1) > 1 and t.stride(1) != 1) or (t.size(0) > 1 and t.stride(0) < t.size(1)):
        raise SparseFFNError(SF_ERR_ALIGN, f"{where}: {name}'s rows are not contiguous, or share elements")
    if t.get_device() != dev:
        raise SparseFFNError(SF_ERR_UNSUPPORTED, f"{where}: {name} is on {t.device}, another device than the first tensor")
    return t.stride(0) if t.size(0) > 1 else t.size(1)


def sf_orthogonalize(G, steps: int = 5, coefficients=(3.4445, -4.7750, 2.0315), scale: float = 1.0, out=None, workspace=None, stream=None):
    """O = bf16(scale * X) after ``steps`` of X <- a X + (b A + c A^2) X, A = X X^T, from X = G / |G|; G bf16 or float32. G and ``out`` may be
    strided row views."""
    w, dev = "sf_orthogonalize", G.get_device()
    if G.dim() != 2:
        raise SparseFFNError(SF_ERR_SHAPE, f"{w}: G must be a matrix")
    rows, cols = G.shape
    ldg = _rows_of(w, "G", G, (_BF16, _F32), (rows, cols), dev)
    if out is None or workspace is None:
        with _allocating(stream):
            out = torch.empty((rows, cols), dtype=_BF16, device=G.device) if out is None else out
            workspace = _workspace(sf_orthogonalize_workspace_size(rows, cols), G.device) if workspace is None else workspace
    a, b, c = coefficients
    _check(lib().sf_orthogonalize(G.data_ptr(), SF_F32 if G.dtype is _F32 else SF_BF16, rows, cols, ldg, steps, a, b, c, scale, out.data_ptr(),
                                  _rows_of(w, "out", out, (_BF16,), (rows, cols), dev), *_buffer(w, "workspace", workspace, dev),
                                  _launch_stream(w, dev, stream)), w)
    return out


def make_schedule(warmup_steps: int, sparse_steps: int, total_steps: int) -> sf_schedule:
    return sf_schedule(warmup_steps, sparse_steps, total_steps)


def sf_schedule_step_kind(schedule, step: int) -> int:
    kind = _i32(0)
    _check(lib().sf_schedule_step_kind(C.byref(schedule), step, C.byref(kind)), "sf_schedule_step_kind")
    return kind.value


def sf_schedule_speedup(schedule, sparse_step_speedup: float) -> float:
    out = C.c_double(0)
    _check(lib().sf_schedule_speedup(C.byref(schedule), sparse_step_speedup, C.byref(out)), "sf_schedule_speedup")
    return out.value


def sf_ffn_flop_fraction(D: int, F: int, n_q_heads: int, n_kv_heads: int, head_dim: int) -> float:
    out = C.c_double(0)
    _check(lib().sf_ffn_flop_fraction(D, F, n_q_heads, n_kv_heads, head_dim, C.byref(out)), "sf_ffn_flop_fraction")
    return out.value


def sf_end_to_end_speedup(ffn_fraction: float, ffn_speedup: float) -> float:
    out = C.c_double(0)
    _check(lib().sf_end_to_end_speedup(ffn_fraction, ffn_speedup, C.byref(out)), "sf_end_to_end_speedup")
    return out.value


def sf_ffn_fwd_scheduled(schedule, step: int, desc, X, W1, W2, Y, fwd_ctx, workspace, stream=None):
    _check(lib().sf_ffn_fwd_scheduled(C.byref(schedule), step, C.byref(desc), _ptr(X), _ptr(W1), _ptr(W2), _ptr(Y),
                                      _ptr(fwd_ctx), _nbytes(fwd_ctx), _ptr(workspace), _nbytes(workspace),
                                      _stream(stream)), "sf_ffn_fwd_scheduled")


def sf_ffn_bwd_scheduled(schedule, step: int, desc, dY, X, W1, W2, fwd_ctx, dX, dW1, dW2, workspace, stream=None):
    _check(lib().sf_ffn_bwd_scheduled(C.byref(schedule), step, C.byref(desc), _ptr(dY), _ptr(X), _ptr(W1), _ptr(W2),
                                      _ptr(fwd_ctx), _nbytes(fwd_ctx), _ptr(dX), _ptr(dW1), _ptr(dW2), _ptr(workspace),
                                      _nbytes(workspace), _stream(stream)), "sf_ffn_bwd_scheduled")


def sf_selftest_wait_expiry(workspace, budget_clocks: int = 1_000_000, stream=None) -> None:
    """One bounded wait on a barrier nothing completes: sets the status word of ``workspace``."""
    _check(lib().sf_selftest_wait_expiry(_ptr(workspace), budget_clocks, _stream(stream)), "sf_selftest_wait_expiry")


def sf_check_status(workspace, stream=None) -> int:
    return lib().sf_check_status(_ptr(workspace), _stream(stream))


class StageTrace:
    """Records CUDA events between the kernels of the FFN step calls made inside the `with` block.

    After the block, ``durations_ms()`` returns the time between consecutive events (the caller
    knows the stage order of the calls it made; see sf_trace_set in the header)."""

    def __init__(self, capacity: int):
        self.events = [torch.cuda.Event(enable_timing=True) for _ in range(capacity)]
        for e in self.events:          # torch creates the CUDA event lazily on first record
            e.record()
        torch.cuda.synchronize()
        self._arr = (C.c_void_p * capacity)(*[C.c_void_p(e.cuda_event) for e in self.events])
        self.count = 0

    def __enter__(self):
        _check(lib().sf_trace_set(self._arr, len(self.events)), "sf_trace_set")
        return self

    def __exit__(self, *exc):
        self.count = lib().sf_trace_count()
        lib().sf_trace_set(None, 0)
        return False

    def durations_ms(self):
        torch.cuda.synchronize()
        return [self.events[i].elapsed_time(self.events[i + 1]) for i in range(self.count - 1)]
