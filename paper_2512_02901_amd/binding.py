"""Thin ctypes binding of libfairy2i.so (declared in include/fairy2i.h).

Argument marshalling only: torch tensors supply device pointers and the
current HIP stream; every step of the computation runs in the library's
kernels.  There is no fallback: if the library is missing, ``load()`` raises.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libfairy2i.so")
_lib = None

OK, ERR_NULL, ERR_SHAPE, ERR_STAGES, ERR_DTYPE, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP = range(8)
ACT_F32, ACT_BF16, ACT_I8 = 0, 1, 2
LAYOUT_D3, LAYOUT_TILED, LAYOUT_TILED_FP4 = 0, 1, 2
MAX_STAGES = 4
MAX_DECODE_BATCH = 16

_c_i32, _c_i64, _c_size, _c_p = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_void_p

_SIGNATURES = {
    "fairy2i_status_string": (ctypes.c_char_p, [_c_i32]),
    "fairy2i_abi_version": (_c_i32, []),
    "fairy2i_to_widely_linear": (_c_i32, [_c_p, _c_i64, _c_i64, _c_p, _c_p, _c_p]),
    "fairy2i_quantize_workspace_bytes": (_c_size, [_c_i64, _c_i64, _c_i32]),
    "fairy2i_quantize": (_c_i32, [_c_p, _c_i64, _c_i64, _c_i32, _c_p, _c_p, _c_p, _c_size, _c_p]),
    "fairy2i_quantize_grouped": (_c_i32, [_c_p, _c_i64, _c_i64, _c_i32, _c_i64, _c_p, _c_p, _c_p]),
    "fairy2i_repack_tiled_bytes": (_c_size, [_c_i64, _c_i64, _c_i32]),
    "fairy2i_repack_tiled": (_c_i32, [_c_p, _c_i64, _c_i64, _c_i32, _c_p, _c_size, _c_p]),
    "fairy2i_repack_tiled_fp4": (_c_i32, [_c_p, _c_i64, _c_i64, _c_i32, _c_p, _c_size, _c_p]),
    "fairy2i_quantize_act_int8": (_c_i32, [_c_p, _c_i32, _c_i64, _c_i64, _c_p, _c_p, _c_p]),
    "fairy2i_wl_matmul_workspace_bytes": (_c_size, [_c_i64, _c_i64, _c_i32, _c_i64, _c_i32]),
    "fairy2i_wl_matmul": (_c_i32, [_c_p, _c_p, _c_p, _c_p, _c_i32, _c_i64, _c_i64, _c_p, _c_p,
                                   _c_i32, _c_i64, _c_p, _c_p, _c_size, _c_p]),
    "fairy2i_wl_matmul_noalloc": (_c_i32, [_c_p, _c_p, _c_p, _c_p, _c_i32, _c_i64, _c_i64, _c_p, _c_p,
                                           _c_i32, _c_i64, _c_p, _c_p]),
    "fairy2i_wl_int8_accumulators": (_c_i32, [_c_p, _c_p, _c_i32, _c_i64, _c_i64, _c_p, _c_i64,
                                              _c_p, _c_p, _c_size, _c_p]),
    "fairy2i_host_exact_mean_f32": (_c_i32, [_c_p, _c_i64, _c_p]),
    "fairy2i_wl_group_workspace_bytes": (_c_size, [_c_p, _c_i32, _c_i32, _c_i32, _c_i64]),
    "fairy2i_wl_group_table_bytes": (_c_size, [_c_i32]),
    "fairy2i_wl_group_build_table": (_c_i32, [_c_p, _c_i32, _c_i32, _c_i32, _c_i64, _c_p, _c_size,
                                              _c_p, _c_size]),
    "fairy2i_wl_matmul_group": (_c_i32, [_c_p, _c_p, _c_p]),
    "fairy2i_wl_matmul_group_timed": (_c_i32, [_c_p, _c_p, _c_p, _c_p]),
    "fairy2i_block_workspace_bytes": (_c_size, [_c_p]),
    "fairy2i_block_plan_bytes": (_c_size, [_c_p]),
    "fairy2i_block_build_plan": (_c_i32, [_c_p, _c_p, _c_size, _c_p, _c_size]),
    "fairy2i_block_decode": (_c_i32, [_c_p, _c_p, _c_p, _c_p, _c_p, _c_i64, _c_p, _c_p]),
    "fairy2i_block_intermediates": (_c_i32, [_c_p, _c_p]),
    "fairy2i_qat_fake_quant": (_c_i32, [_c_p, _c_i64, _c_i64, _c_i32, _c_p, _c_p, _c_p, _c_i32, _c_p, _c_size,
                                        _c_p]),
    "fairy2i_qat_ste_workspace_bytes": (_c_size, [_c_i64, _c_i64]),
    "fairy2i_qat_ste_backward": (_c_i32, [_c_p, _c_p, _c_i32, _c_i64, _c_i64, _c_p, _c_p, _c_p, _c_size, _c_p]),
    "fairy2i_cgemm_gauss": (_c_i32, [_c_p, _c_p, _c_p, _c_i32, _c_i64, _c_i64, _c_p, _c_i64, _c_i32, _c_p]),
    "fairy2i_cgemm_gauss_planar_workspace_bytes": (_c_size, [_c_p, _c_i32, _c_i64, _c_i64]),
    "fairy2i_cgemm_gauss_planar": (_c_i32, [_c_p, _c_p, _c_p, _c_i32, _c_i64, _c_i64, _c_p, _c_i64, _c_i32, _c_p,
                                            _c_size, _c_p]),
    "fairy2i_probe_mfma": (_c_i32, [_c_i32, _c_i32, _c_i32, _c_p, _c_p, _c_p]),
    "fairy2i_wl_realify": (_c_i32, [_c_p, _c_p, _c_i32, _c_i64, _c_i64, _c_p, _c_p]),
    "fairy2i_wl_realify_codes": (_c_i32, [_c_p, _c_p, _c_p, _c_p, _c_i32, _c_i64, _c_i64, _c_p, _c_p]),
    "fairy2i_wl_unrealify_grad": (_c_i32, [_c_p, _c_i64, _c_i64, _c_p, _c_p, _c_p]),
    "fairy2i_f32_to_bf16": (_c_i32, [_c_p, _c_i64, _c_p, _c_p]),
    "fairy2i_gemm_bf16_workspace_bytes": (_c_size, []),
    "fairy2i_gemm_bf16_tune": (_c_i32, [_c_p, _c_i64, _c_i32, _c_p, _c_i64, _c_i32, _c_i64, _c_i64, _c_i64, _c_p,
                                        _c_i64, _c_p, _c_size, _c_p, _c_p]),
    "fairy2i_gemm_bf16": (_c_i32, [_c_p, _c_i64, _c_i32, _c_p, _c_i64, _c_i32, _c_i64, _c_i64, _c_i64, _c_p, _c_i64,
                                   _c_p, _c_size, _c_p]),
    "fairy2i_add_rmsnorm_i8": (_c_i32, [_c_p, _c_p, _c_p, ctypes.c_float, _c_i64, _c_i64, _c_p, _c_p, _c_p, _c_p]),
    "fairy2i_kv_cache_bytes": (_c_size, [_c_i64, _c_i32, _c_i32, _c_i32]),
    "fairy2i_rope_table": (_c_i32, [_c_i64, _c_i32, ctypes.c_double, _c_p, _c_p]),
    "fairy2i_kv_append": (_c_i32, [_c_p, _c_p, _c_p, _c_i64, _c_i32, _c_p, _c_i64, _c_p, _c_i64, _c_p, _c_i64, _c_p,
                                   _c_p]),
    "fairy2i_kv_read": (_c_i32, [_c_p, _c_p, _c_p, _c_p, _c_p]),
    "fairy2i_kv_attend_workspace_bytes": (_c_size, [_c_p, _c_i64, _c_i64, _c_i32]),
    "fairy2i_kv_attend": (_c_i32, [_c_p, _c_p, _c_p, _c_i32, ctypes.c_float, _c_p, _c_p, _c_size, _c_p]),
    "fairy2i_fp8_codes_bytes": (_c_size, [_c_i64, _c_i64]),
    "fairy2i_fp8_scales_bytes": (_c_size, [_c_i64, _c_i64]),
    "fairy2i_fp8_quantize": (_c_i32, [_c_p, _c_i32, _c_i64, _c_p, _c_p, _c_p]),
    "fairy2i_fp8_transpose": (_c_i32, [_c_p, _c_p, _c_p]),
    "fairy2i_fp8_dequantize": (_c_i32, [_c_p, _c_p, _c_p]),
    "fairy2i_gemm_fp8_workspace_bytes": (_c_size, [_c_i64, _c_i64, _c_i64]),
    "fairy2i_gemm_fp8": (_c_i32, [_c_p, _c_p, _c_p, _c_i32, _c_i64, _c_i32, _c_p, _c_size, _c_p]),
    "fairy2i_add_layernorm": (_c_i32, [_c_p, _c_p, _c_p, _c_p, ctypes.c_float, _c_i32, _c_i64, _c_i64, _c_p, _c_p,
                                       _c_p, _c_p, _c_p]),
    "fairy2i_layernorm_backward_workspace_bytes": (_c_size, [_c_i64, _c_i64]),
    "fairy2i_layernorm_backward": (_c_i32, [_c_p, _c_i32, _c_p, _c_p, _c_p, _c_p, _c_i32, _c_i64, _c_i64, _c_p, _c_p,
                                            _c_p, _c_p, _c_size, _c_p]),
    "fairy2i_cpu_lut_workspace_bytes": (_c_size, [_c_i32, _c_i64, _c_i64, _c_i32]),
    "fairy2i_cpu_lut_wl_matmul": (_c_i32, [_c_p, _c_p, _c_p, _c_p, _c_i32, _c_i64, _c_i64, _c_p, _c_p, _c_i64,
                                           _c_p, _c_p, _c_p, _c_size, _c_i32]),
}


class WlLayer(ctypes.Structure):
    """fairy2i_wl_layer of include/fairy2i.h."""
    _fields_ = [("codes_U", _c_p), ("scales_U", _c_p), ("codes_W", _c_p), ("scales_W", _c_p),
                ("x", _c_p), ("x_scale", _c_p), ("y", _c_p), ("N", _c_i64), ("K", _c_i64),
                ("layout", _c_i32), ("group_size", _c_i32)]


class CgemmOperand(ctypes.Structure):
    """fairy2i_cgemm_operand of include/fairy2i.h."""
    _fields_ = [("data", _c_p), ("ld", _c_i64), ("dtype", _c_i32), ("trans", _c_i32), ("conj", _c_i32),
                ("reserved", _c_i32)]


class BlockDesc(ctypes.Structure):
    """fairy2i_block_desc of include/fairy2i.h."""
    _fields_ = [("n", _c_i64), ("n_ff", _c_i64), ("n_heads", _c_i32), ("T", _c_i32), ("max_ctx", _c_i64),
                ("eps", ctypes.c_float), ("reserved", _c_i32), ("rope_base", ctypes.c_double),
                ("codes_U", _c_p * 7), ("scales_U", _c_p * 7), ("codes_W", _c_p * 7), ("scales_W", _c_p * 7),
                ("norm_attn", _c_p), ("norm_mlp", _c_p)]


class KvCacheDesc(ctypes.Structure):
    """fairy2i_kv_cache of include/fairy2i.h."""
    _fields_ = [("data", _c_p), ("n_pages", _c_i64), ("page_size", _c_i32), ("n_kv_heads", _c_i32), ("dc", _c_i32),
                ("reserved", _c_i32)]


class KvBatchDesc(ctypes.Structure):
    """fairy2i_kv_batch of include/fairy2i.h."""
    _fields_ = [("pages", _c_p), ("cu_new", _c_p), ("lens", _c_p), ("n_new", _c_i64), ("n_seqs", _c_i32),
                ("max_pages", _c_i32)]


class Fp8Desc(ctypes.Structure):
    """fairy2i_fp8_matrix of include/fairy2i.h."""
    _fields_ = [("codes", _c_p), ("scales", _c_p), ("rows", _c_i64), ("cols", _c_i64)]


class Fairy2iError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = _lib.fairy2i_status_string(status).decode() if _lib is not None else str(status)
        super().__init__(f"{where}: status {status} ({msg})")


def lib_path() -> str:
    return _LIB_PATH


def load():
    """Load libfairy2i.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with "
                               "`python -m paper_2512_02901_amd.build`")
        lib = ctypes.CDLL(_LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def _check(status: int, where: str):
    if status != OK:
        raise Fairy2iError(status, where)


# --------------------------------------------------------------- helpers ---

_torch_module = None
_raw_stream = None  # device index -> handle of torch's current stream there


def _torch():
    global _torch_module, _raw_stream
    if _torch_module is None:
        import torch
        # the handle alone (0.07 us); torch.cuda.current_stream builds a Stream object for it (1.9 us)
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
            (lambda index: torch.cuda.current_stream(index).cuda_stream)
        _torch_module = torch  # last: another thread that sees the module calls _raw_stream
    return _torch_module


def _stream_ptr(tensor) -> int:
    _torch()
    return _raw_stream(tensor.get_device())


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _require(t, dtype, name, device=None):
    torch = _torch_module or _torch()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")


# ------------------------------------------------------------------ API ---

def wl_realify(U, W, out=None):
    """U, W: [N, K] complex64 or bf16 [N, K, 2] device tensors -> R: bf16
    [2N, 2K], the layer's real map with (re, im) rows and columns
    interleaved (fairy2i_wl_realify; out: such a tensor to write)."""
    torch = _torch()
    lib = load()
    if U.dtype == torch.complex64:
        dt = ACT_F32
        N, K = U.shape
    else:
        dt = ACT_BF16
        N, K = U.shape[0], U.shape[1]
    for t, n in ((U, "U"), (W, "W")):
        _require(t, U.dtype, n, U.device)
        if t.shape != U.shape or (dt == ACT_BF16 and (t.dim() != 3 or t.shape[2] != 2 or t.dtype != torch.bfloat16)):
            raise ValueError(f"{n} must be [N, K] complex64 or [N, K, 2] bf16")
    R = torch.empty((2 * N, 2 * K), dtype=torch.bfloat16, device=U.device) if out is None else out
    _require(R, torch.bfloat16, "out", U.device)
    if tuple(R.shape) != (2 * N, 2 * K):
        raise ValueError("out must be [2N, 2K]")
    _check(lib.fairy2i_wl_realify(_ptr(U), _ptr(W), dt, N, K, _ptr(R), _stream_ptr(U)), "fairy2i_wl_realify")
    return R


def wl_realify_codes(codes_U, scales_U, codes_W, scales_W, out=None):
    """The layer's real map R (bf16 [2N, 2K]) straight from the quantised
    pair: canonical codes uint8 [T, N, K/4] and scales float32 [T, 2] of U
    and of W (fairy2i_wl_realify_codes)."""
    torch = _torch()
    lib = load()
    _require(codes_U, torch.uint8, "codes_U")
    T, N, K4 = codes_U.shape
    d = codes_U.device
    _require(codes_W, torch.uint8, "codes_W", d)
    for t, n in ((scales_U, "scales_U"), (scales_W, "scales_W")):
        _require(t, torch.float32, n, d)
        if tuple(t.shape) != (T, 2):
            raise ValueError(f"{n} must be [T, 2]")
    if tuple(codes_W.shape) != (T, N, K4):
        raise ValueError("codes_W must match codes_U")
    K = 4 * K4
    R = torch.empty((2 * N, 2 * K), dtype=torch.bfloat16, device=d) if out is None else out
    _require(R, torch.bfloat16, "out", d)
    if tuple(R.shape) != (2 * N, 2 * K):
        raise ValueError("out must be [2N, 2K]")
    _check(lib.fairy2i_wl_realify_codes(_ptr(codes_U), _ptr(scales_U), _ptr(codes_W), _ptr(scales_W), T, N, K,
                                        _ptr(R), _stream_ptr(codes_U)), "fairy2i_wl_realify_codes")
    return R


def wl_unrealify_grad(G_R, N, K, out=None):
    """G_R: float32 [2N, 2K] -> (G_U, G_W) complex64 [N, K] (out: a pair
    of such tensors to write)."""
    torch = _torch()
    lib = load()
    _require(G_R, torch.float32, "G_R")
    if tuple(G_R.shape) != (2 * N, 2 * K):
        raise ValueError("G_R must be [2N, 2K]")
    if out is None:
        G_U = torch.empty((N, K), dtype=torch.complex64, device=G_R.device)
        G_W = torch.empty_like(G_U)
    else:
        G_U, G_W = out
        for t, n in ((G_U, "G_U"), (G_W, "G_W")):
            _require(t, torch.complex64, n, G_R.device)
            if tuple(t.shape) != (N, K):
                raise ValueError(f"{n} must be [N, K]")
    _check(lib.fairy2i_wl_unrealify_grad(_ptr(G_R), N, K, _ptr(G_U), _ptr(G_W), _stream_ptr(G_R)),
           "fairy2i_wl_unrealify_grad")
    return G_U, G_W


def f32_to_bf16(x, out=None):
    """float32 (or complex64, as its float pairs) device tensor -> bf16 of
    the same number of values, nearest even; complex input gives [..., 2]."""
    torch = _torch()
    lib = load()
    _require(x, None, "x")
    xf = torch.view_as_real(x) if x.dtype == torch.complex64 else x
    if xf.dtype != torch.float32:
        raise TypeError("x must be float32 or complex64")
    if out is None:
        out = torch.empty(xf.shape, dtype=torch.bfloat16, device=x.device)
    _require(out, torch.bfloat16, "out", x.device)
    if out.numel() != xf.numel():
        raise ValueError("out must hold as many values as x")
    _check(lib.fairy2i_f32_to_bf16(ctypes.c_void_p(xf.data_ptr()), xf.numel(), _ptr(out), _stream_ptr(x)),
           "fairy2i_f32_to_bf16")
    return out


def gemm_bf16(A, B, transA=False, transB=False, out=None, workspace=None, tune=False):
    """C (float32 M x N) = op(A) op(B) for bf16 row-major 2-D device tensors
    (fairy2i_gemm_bf16); op(X) is X or X^T.  tune=True first times the
    library's candidate algorithms for this problem (fairy2i_gemm_bf16_tune,
    which synchronises) and keeps the fastest."""
    torch = _torch()
    lib = load()
    _require(A, torch.bfloat16, "A")
    _require(B, torch.bfloat16, "B", A.device)
    if A.dim() != 2 or B.dim() != 2:
        raise ValueError("A and B must be 2-D")
    M, K = (A.shape[1], A.shape[0]) if transA else (A.shape[0], A.shape[1])
    Kb, N = (B.shape[1], B.shape[0]) if transB else (B.shape[0], B.shape[1])
    if Kb != K:
        raise ValueError("inner dimensions differ")
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=A.device)
    _require(out, torch.float32, "out", A.device)
    if tuple(out.shape) != (M, N):
        raise ValueError("out must be M x N")
    ws, wsb = _workspace(lib.fairy2i_gemm_bf16_workspace_bytes(), workspace, A.device)
    if tune:
        _check(lib.fairy2i_gemm_bf16_tune(_ptr(A), A.shape[1], int(transA), _ptr(B), B.shape[1], int(transB), M, N,
                                          K, _ptr(out), N, _ptr(ws), wsb, None, _stream_ptr(A)),
               "fairy2i_gemm_bf16_tune")
    _check(lib.fairy2i_gemm_bf16(_ptr(A), A.shape[1], int(transA), _ptr(B), B.shape[1], int(transB), M, N, K,
                                 _ptr(out), N, _ptr(ws), wsb, _stream_ptr(A)), "fairy2i_gemm_bf16")
    return out


PROBE_MFMA_I8 = 0    # v_mfma_i32_16x16x64_i8 (the prefill GEMM's instruction)
PROBE_MFMA_F8F4 = 1  # v_mfma_scale_f32_16x16x128_f8f6f4, e4m3 x e2m1 (the decode product's)
PROBE_MFMA_I8_32X32 = 2  # v_mfma_i32_32x32x32_i8


def probe_mfma(kind: int, blocks: int, iters: int, sink) -> float:
    """Launch the matrix-core rate probe on the current stream of sink's
    device (sink: int32 device tensor of at least blocks * 256 words);
    returns the operations of the launch, for the caller to time."""
    torch = _torch()
    lib = load()
    _require(sink, torch.int32, "sink")
    if sink.numel() < blocks * 256:
        raise ValueError("sink needs blocks * 256 words")
    ops = ctypes.c_double()
    _check(lib.fairy2i_probe_mfma(kind, blocks, iters, _ptr(sink), ctypes.byref(ops), _stream_ptr(sink)),
           "fairy2i_probe_mfma")
    return ops.value


def to_widely_linear(A):
    """A: float32 [2N, 2K] device tensor -> (U, W) complex64 [N, K]."""
    torch = _torch()
    lib = load()
    _require(A, torch.float32, "A")
    rows, cols = A.shape
    U = torch.empty((rows // 2, cols // 2), dtype=torch.complex64, device=A.device)
    W = torch.empty_like(U)
    _check(lib.fairy2i_to_widely_linear(_ptr(A), rows, cols, _ptr(U), _ptr(W), _stream_ptr(A)),
           "fairy2i_to_widely_linear")
    return U, W


def quantize(M, T: int):
    """M: complex64 [N, K] -> (codes uint8 [T, N, K/4], scales float32 [T, 2])."""
    torch = _torch()
    lib = load()
    _require(M, torch.complex64, "M")
    N, K = M.shape
    codes = torch.empty((T, N, K // 4), dtype=torch.uint8, device=M.device)
    scales = torch.empty((T, 2), dtype=torch.float32, device=M.device)
    wsb = lib.fairy2i_quantize_workspace_bytes(N, K, T)
    ws = torch.empty(max(int(wsb), 1), dtype=torch.uint8, device=M.device)
    _check(lib.fairy2i_quantize(_ptr(M), N, K, T, _ptr(codes), _ptr(scales), _ptr(ws), wsb,
                                _stream_ptr(M)), "fairy2i_quantize")
    return codes, scales


def quantize_grouped(M, T: int, G: int):
    """M: complex64 [N, K] -> (codes uint8 [T, N, K/4], scales float32
    [T, N, ceil(K/G), 2]): one pair of axis scales per group of G input
    columns of a row."""
    torch = _torch()
    lib = load()
    _require(M, torch.complex64, "M")
    N, K = M.shape
    ng = -(-K // G) if G > 0 else 0
    codes = torch.empty((T, N, K // 4), dtype=torch.uint8, device=M.device)
    scales = torch.empty((T, N, max(ng, 1), 2), dtype=torch.float32, device=M.device)
    _check(lib.fairy2i_quantize_grouped(_ptr(M), N, K, T, G, _ptr(codes), _ptr(scales), _stream_ptr(M)),
           "fairy2i_quantize_grouped")
    return codes, scales


def _act_dtype(x):
    torch = _torch_module or _torch()
    dtype = x.dtype
    if dtype is torch.complex64:
        return ACT_F32
    if dtype is torch.bfloat16:
        return ACT_BF16
    if dtype is torch.int8:
        return ACT_I8
    raise TypeError(f"unsupported activation dtype {dtype}")


def _act_shape(x):
    """(B, K) of an activation tensor: complex64 [B, K] or bf16/int8 [B, K, 2]."""
    shape = x.shape
    if len(shape) == 2 or (len(shape) == 3 and shape[2] == 2):
        return shape[0], shape[1]
    raise ValueError("activations must be complex64 [B, K] or bf16/int8 [B, K, 2]")


def quantize_act_int8(x):
    """x: complex64 [B, K] or bf16 [B, K, 2] -> (q int8 [B, K, 2], x_scale float32 [B])."""
    torch = _torch_module or _torch()
    lib = _lib or load()
    _require(x, None, "x")
    dt = _act_dtype(x)
    B, K = _act_shape(x)
    q = torch.empty((B, K, 2), dtype=torch.int8, device=x.device)
    xs = torch.empty((B,), dtype=torch.float32, device=x.device)
    _check(lib.fairy2i_quantize_act_int8(x.data_ptr(), dt, B, K, q.data_ptr(), xs.data_ptr(), _stream_ptr(x)),
           "fairy2i_quantize_act_int8")
    return q, xs


def wl_matmul_workspace_bytes(N, K, T, B, dtype) -> int:
    return int(load().fairy2i_wl_matmul_workspace_bytes(N, K, T, B, dtype))


def wl_matmul(codes_U, scales_U, codes_W, scales_W, x, x_scale=None, out=None, workspace=None):
    """y = sum_t U^(t) x + W^(t) conj(x) for each token; complex64 [B, N]."""
    torch = _torch_module or _torch()
    lib = _lib or load()
    # Launch latency counts here (a small layer's kernel runs 4 us), so all
    # operands are first looked over in one expression; _check_wl names what is wrong.
    try:
        index = x.get_device()
        ok = (index >= 0
              and codes_U.dtype is torch.uint8 and codes_U.get_device() == index and codes_U.is_contiguous()
              and codes_W.dtype is torch.uint8 and codes_W.get_device() == index and codes_W.is_contiguous()
              and scales_U.dtype is torch.float32 and scales_U.get_device() == index and scales_U.is_contiguous()
              and scales_W.dtype is torch.float32 and scales_W.get_device() == index and scales_W.is_contiguous()
              and x.is_contiguous())
    except (AttributeError, TypeError):
        ok = False
    if not ok:
        _check_wl(codes_U, scales_U, codes_W, scales_W, x)
    T, N, KB = codes_U.shape
    if codes_W.shape != codes_U.shape or scales_U.shape != (T, 2) or scales_W.shape != (T, 2):
        raise ValueError("codes/scales shapes disagree")
    dt = _act_dtype(x)
    B, K = _act_shape(x)
    if K != 4 * KB:
        raise ValueError(f"activations have K={K}, codes have K={4 * KB}")
    dev_ = x.device
    if x_scale is not None:
        _require(x_scale, torch.float32, "x_scale", dev_)
        if x_scale.shape != (B,):
            raise ValueError(f"x_scale must have shape ({B},), got {tuple(x_scale.shape)}")
    if out is None:
        out = torch.empty((B, N), dtype=torch.complex64, device=dev_)
    else:
        _require(out, torch.complex64, "out", dev_)
        if out.shape != (B, N):
            raise ValueError(f"out must have shape ({B}, {N}), got {tuple(out.shape)}")
    if workspace is None:
        workspace, wsb = _workspace(lib.fairy2i_wl_matmul_workspace_bytes(N, K, T, B, dt), None, dev_)
    else:  # its size is the library's to check
        _require(workspace, torch.uint8, "workspace", dev_)
        wsb = workspace.numel()
    _check(lib.fairy2i_wl_matmul(codes_U.data_ptr(), scales_U.data_ptr(), codes_W.data_ptr(), scales_W.data_ptr(),
                                 T, N, K, x.data_ptr(), None if x_scale is None else x_scale.data_ptr(), dt, B,
                                 out.data_ptr(), None if workspace is None else workspace.data_ptr(), wsb,
                                 _raw_stream(x.get_device())), "fairy2i_wl_matmul")
    return out


def _check_wl(codes_U, scales_U, codes_W, scales_W, x):
    torch = _torch()
    for t, n in ((codes_U, "codes_U"), (codes_W, "codes_W")):
        _require(t, torch.uint8, n)
    for t, n in ((scales_U, "scales_U"), (scales_W, "scales_W")):
        _require(t, torch.float32, n)
    _require(x, None, "x")
    for t, n in ((codes_U, "codes_U"), (codes_W, "codes_W"), (scales_U, "scales_U"), (scales_W, "scales_W")):
        _require(t, None, n, x.device)


NOALLOC_SCRATCH_BYTES = 32 << 20


def wl_matmul_noalloc(codes_U, scales_U, codes_W, scales_W, x, x_scale=None, out=None):
    """wl_matmul without a workspace: the library's fixed device array
    (NOALLOC_SCRATCH_BYTES per GPU) serves as one; allocates nothing when
    ``out`` is given.  Calls that overlap on one GPU race."""
    torch = _torch()
    lib = load()
    for t, n in ((codes_U, "codes_U"), (codes_W, "codes_W")):
        _require(t, torch.uint8, n, x.device)
    for t, n in ((scales_U, "scales_U"), (scales_W, "scales_W")):
        _require(t, torch.float32, n, x.device)
    _require(x, None, "x")
    T, N, KB = codes_U.shape
    if codes_W.shape != codes_U.shape or scales_U.shape != (T, 2) or scales_W.shape != (T, 2):
        raise ValueError("codes/scales shapes disagree")
    dt = _act_dtype(x)
    B, K = _act_shape(x)
    if K != 4 * KB:
        raise ValueError(f"activations have K={K}, codes have K={4 * KB}")
    if x_scale is not None:
        _require(x_scale, torch.float32, "x_scale", x.device)
        if tuple(x_scale.shape) != (B,):
            raise ValueError(f"x_scale must have shape ({B},), got {tuple(x_scale.shape)}")
    if out is None:
        out = torch.empty((B, N), dtype=torch.complex64, device=x.device)
    else:
        _require(out, torch.complex64, "out", x.device)
        if tuple(out.shape) != (B, N):
            raise ValueError(f"out must have shape ({B}, {N}), got {tuple(out.shape)}")
    _check(lib.fairy2i_wl_matmul_noalloc(_ptr(codes_U), _ptr(scales_U), _ptr(codes_W), _ptr(scales_W), T, N, K,
                                         _ptr(x), _ptr(x_scale), dt, B, _ptr(out), _stream_ptr(x)),
           "fairy2i_wl_matmul_noalloc")
    return out


def _workspace(need, workspace, device):
    """(workspace tensor or None, its size in bytes): a fresh uint8 device
    buffer of `need` bytes when none is given, else the caller's, checked."""
    torch = _torch()
    need = int(need)
    if workspace is None:
        if need == 0:
            return None, 0
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    _require(workspace, torch.uint8, "workspace", device)
    return workspace, workspace.numel()


def repack_tiled_bytes(N, K, T) -> int:
    return int(load().fairy2i_repack_tiled_bytes(N, K, T))


def _repack(fn, codes, out):
    torch = _torch()
    lib = load()
    _require(codes, torch.uint8, "codes")
    T, N, KB = codes.shape
    nb = repack_tiled_bytes(N, 4 * KB, T)
    if out is None:
        out = torch.empty(nb, dtype=torch.uint8, device=codes.device)
    else:
        _require(out, torch.uint8, "out")
    _check(getattr(lib, fn)(_ptr(codes), N, 4 * KB, T, _ptr(out), out.numel(), _stream_ptr(codes)), fn)
    return out


def repack_tiled(codes, out=None):
    """D3 codes [T, N, K/4] -> the tiled decode layout (1-D uint8 tensor of
    fairy2i_repack_tiled_bytes bytes)."""
    return _repack("fairy2i_repack_tiled", codes, out)


def repack_tiled_fp4(codes, out=None):
    """D3 codes [T, N, K/4] -> the fp4 tiled decode layout (1-D uint8 tensor
    of fairy2i_repack_tiled_bytes bytes)."""
    return _repack("fairy2i_repack_tiled_fp4", codes, out)


def int8_accumulators(codes_U, codes_W, q, workspace=None):
    """Exact int32 products acc[M][t][p][b][i][c] behind the int8 path."""
    torch = _torch()
    lib = load()
    _require(codes_U, torch.uint8, "codes_U")
    _require(codes_W, torch.uint8, "codes_W")
    _require(q, torch.int8, "q")
    T, N, KB = codes_U.shape
    B, K = _act_shape(q)
    if K != 4 * KB:
        raise ValueError("K mismatch")
    _require(codes_W, None, "codes_W", q.device)
    _require(codes_U, None, "codes_U", q.device)
    if codes_W.shape != codes_U.shape:
        raise ValueError("codes_U and codes_W shapes disagree")
    acc = torch.empty((2, T, 2, B, N, 2), dtype=torch.int32, device=q.device)
    workspace, wsb = _workspace(lib.fairy2i_wl_matmul_workspace_bytes(N, K, T, B, ACT_I8), workspace, q.device)
    _check(lib.fairy2i_wl_int8_accumulators(_ptr(codes_U), _ptr(codes_W), T, N, K, _ptr(q), B,
                                            _ptr(acc), _ptr(workspace), wsb, _stream_ptr(q)),
           "fairy2i_wl_int8_accumulators")
    return acc


def host_exact_mean_f32(values) -> np.float32:
    """Host-side self-check of the scale rounding (no GPU involved)."""
    lib = load()
    v = np.ascontiguousarray(values, dtype=np.float64)
    out = ctypes.c_float(0.0)
    _check(lib.fairy2i_host_exact_mean_f32(v.ctypes.data_as(ctypes.c_void_p), v.size,
                                           ctypes.byref(out)), "fairy2i_host_exact_mean_f32")
    return np.float32(out.value)


def qat_fake_quant(M, T: int, out_dtype: int = ACT_BF16):
    """Fake-quant forward of a complex64 master [N, K]: (W^, codes, scales);
    W^ is bf16 pairs [N, K, 2] (ACT_BF16) or complex64 [N, K] (ACT_F32)."""
    torch = _torch()
    lib = load()
    _require(M, torch.complex64, "M")
    N, K = M.shape
    codes = torch.empty((T, N, K // 4), dtype=torch.uint8, device=M.device)
    scales = torch.empty((T, 2), dtype=torch.float32, device=M.device)
    if out_dtype == ACT_BF16:
        w_hat = torch.empty((N, K, 2), dtype=torch.bfloat16, device=M.device)
    else:
        w_hat = torch.empty((N, K), dtype=torch.complex64, device=M.device)
    wsb = lib.fairy2i_quantize_workspace_bytes(N, K, T)
    ws = torch.empty(max(int(wsb), 1), dtype=torch.uint8, device=M.device)
    _check(lib.fairy2i_qat_fake_quant(_ptr(M), N, K, T, _ptr(codes), _ptr(scales), _ptr(w_hat), out_dtype, _ptr(ws),
                                      wsb, _stream_ptr(M)), "fairy2i_qat_fake_quant")
    return w_hat, codes, scales


def qat_ste_backward(codes, scales, g_hat):
    """dL/dM from dL/dW^ (complex64 [N, K]) through the fake quantiser."""
    torch = _torch()
    lib = load()
    _require(g_hat, torch.complex64, "g_hat")
    N, K = g_hat.shape
    T = codes.shape[0]
    _require(codes, torch.uint8, "codes", g_hat.device)
    _require(scales, torch.float32, "scales", g_hat.device)
    if tuple(codes.shape) != (T, N, K // 4) or tuple(scales.shape) != (T, 2):
        raise ValueError("codes [T, N, K/4] and scales [T, 2] must match g_hat")
    out = torch.empty_like(g_hat)
    wsb = lib.fairy2i_qat_ste_workspace_bytes(N, K)
    ws = torch.empty(max(int(wsb), 1), dtype=torch.uint8, device=g_hat.device)
    _check(lib.fairy2i_qat_ste_backward(_ptr(codes), _ptr(scales), T, N, K, _ptr(g_hat), _ptr(out), _ptr(ws), wsb,
                                        _stream_ptr(g_hat)), "fairy2i_qat_ste_backward")
    return out


def _cgemm_operand(t, trans, conj, rows, K, name):
    """A complex operand tensor: complex64 [a, b] or bf16 pairs [a, b, 2],
    contiguous; [rows, K] when trans == 0, [K, rows] when trans == 1."""
    torch = _torch()
    _require(t, None, name)
    if t.dtype == torch.complex64 and t.dim() == 2:
        dt = ACT_F32
    elif t.dtype == torch.bfloat16 and t.dim() == 3 and t.shape[2] == 2:
        dt = ACT_BF16
    else:
        raise TypeError(f"{name} must be complex64 [a, b] or bf16 [a, b, 2]")
    want = (K, rows) if trans else (rows, K)
    if tuple(t.shape[:2]) != want:
        raise ValueError(f"{name} has shape {tuple(t.shape[:2])}, expected {want}")
    return CgemmOperand(t.data_ptr(), t.shape[1], dt, int(trans), int(conj), 0)


def cgemm_gauss_planar_workspace_bytes(Ks, M: int, N: int) -> int:
    k = (ctypes.c_int64 * 2)(*(list(Ks) + [0] * (2 - len(Ks))))
    return int(load().fairy2i_cgemm_gauss_planar_workspace_bytes(ctypes.byref(k), len(Ks), M, N))


def cgemm_gauss(segments, M: int, N: int, out=None, accumulate: bool = False, planar: bool = False,
                workspace=None):
    """C [M, N] complex64 (+)= sum over segments of op(A) op(B)^T with
    Gauss's three real products.  segments: up to two tuples
    (A, a_trans, a_conj, B, b_trans, b_conj, K); see _cgemm_operand.
    planar: bf16 planes and one batched library GEMM
    (fairy2i_cgemm_gauss_planar, with a uint8 device workspace of
    cgemm_gauss_planar_workspace_bytes, allocated here when not given);
    else the single-kernel fairy2i_cgemm_gauss."""
    torch = _torch()
    lib = load()
    if not 1 <= len(segments) <= 2:
        raise ValueError("one or two segments")
    dev = segments[0][0].device
    A = (CgemmOperand * 2)()
    Bo = (CgemmOperand * 2)()
    Ks = (ctypes.c_int64 * 2)()
    for i, (a, at, ac, b, bt, bc, K) in enumerate(segments):
        A[i] = _cgemm_operand(a, at, ac, M, K, f"segments[{i}].A")
        Bo[i] = _cgemm_operand(b, bt, bc, N, K, f"segments[{i}].B")
        Ks[i] = K
    if out is None:
        out = torch.zeros((M, N), dtype=torch.complex64, device=dev) if accumulate else \
            torch.empty((M, N), dtype=torch.complex64, device=dev)
    _require(out, torch.complex64, "out", dev)
    if tuple(out.shape) != (M, N):
        raise ValueError(f"out must have shape ({M}, {N})")
    if not planar:
        _check(lib.fairy2i_cgemm_gauss(ctypes.byref(A), ctypes.byref(Bo), ctypes.byref(Ks), len(segments), M, N,
                                       _ptr(out), N, int(accumulate), _stream_ptr(out)), "fairy2i_cgemm_gauss")
        return out
    need = int(lib.fairy2i_cgemm_gauss_planar_workspace_bytes(ctypes.byref(Ks), len(segments), M, N))
    if workspace is None:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    _require(workspace, torch.uint8, "workspace", dev)
    _check(lib.fairy2i_cgemm_gauss_planar(ctypes.byref(A), ctypes.byref(Bo), ctypes.byref(Ks), len(segments), M, N,
                                          _ptr(out), N, int(accumulate), _ptr(workspace),
                                          workspace.numel(), _stream_ptr(out)), "fairy2i_cgemm_gauss_planar")
    return out


def _host(a, dtype, name, shape=None):
    """A C-contiguous numpy view of a host array or CPU tensor, checked."""
    if hasattr(a, "is_cuda"):
        if a.is_cuda:
            raise ValueError(f"{name} must be host memory")
        a = a.numpy()
    if not isinstance(a, np.ndarray) or a.dtype != dtype or not a.flags.c_contiguous:
        raise TypeError(f"{name} must be a C-contiguous {np.dtype(dtype).name} array")
    if shape is not None and a.shape != tuple(shape):
        raise ValueError(f"{name} has shape {a.shape}, expected {tuple(shape)}")
    return a


def _hp(a):
    return None if a is None else a.ctypes.data_as(ctypes.c_void_p)


def cpu_lut_workspace_bytes(T: int, K: int, B: int, threads: int = 0) -> int:
    return int(load().fairy2i_cpu_lut_workspace_bytes(T, K, B, threads))


def cpu_lut_wl_matmul(codes_U, scales_U, codes_W, scales_W, q, x_scale, want_y=True, want_acc=False,
                      threads: int = 0, workspace=None):
    """The CPU table-lookup product (host arrays only): codes uint8 [T, N,
    K/4], scales float32 [T, 2], q int8 [B, K, 2], x_scale float32 [B].
    Returns (y complex64 [B, N] or None, acc int32 [2, T, 2, B, N, 2] or
    None).  ``workspace``: optional uint8 host array to reuse across calls."""
    lib = load()
    codes_U = _host(codes_U, np.uint8, "codes_U")
    if codes_U.ndim != 3:
        raise ValueError("codes_U must be [T, N, K/4]")
    T, N, K4 = codes_U.shape
    K = 4 * K4
    codes_W = _host(codes_W, np.uint8, "codes_W", (T, N, K4))
    q = _host(q, np.int8, "q")
    if q.ndim != 3 or q.shape[1:] != (K, 2):
        raise ValueError(f"q must be [B, {K}, 2], got {q.shape}")
    B = q.shape[0]
    su = sw = xs = None
    y = acc = None
    if want_y:
        su = _host(scales_U, np.float32, "scales_U", (T, 2))
        sw = _host(scales_W, np.float32, "scales_W", (T, 2))
        xs = _host(x_scale, np.float32, "x_scale", (B,))
        y = np.empty((B, N), dtype=np.complex64)
    if want_acc:
        acc = np.empty((2, T, 2, B, N, 2), dtype=np.int32)
    need = cpu_lut_workspace_bytes(T, K, B, threads)
    if need == 0:
        raise ValueError(f"unsupported shape T={T} K={K} B={B}")
    if workspace is None or workspace.nbytes < need:
        workspace = np.empty(need, dtype=np.uint8)
    _host(workspace, np.uint8, "workspace")
    _check(lib.fairy2i_cpu_lut_wl_matmul(_hp(codes_U), _hp(su), _hp(codes_W), _hp(sw), T, N, K, _hp(q), _hp(xs), B,
                                         _hp(y), _hp(acc), _hp(workspace), workspace.nbytes, threads),
           "fairy2i_cpu_lut_wl_matmul")
    return y, acc


class WlGroup:
    """A table of independent layers decoded by one fairy2i_wl_matmul_group
    call.  ``layers`` is a list of (codes_U, scales_U, codes_W, scales_W, x,
    x_scale, y) device tensors (x_scale None for bf16); the object keeps them,
    the workspace and both copies of the table alive.  ``layout``: LAYOUT_D3
    (codes [T, N, K/4]), LAYOUT_TILED or LAYOUT_TILED_FP4 (repacked copies,
    a 1-D uint8 tensor per matrix; N is then taken from y); ``tiled=True``
    is LAYOUT_TILED.  ``group_size`` G > 0: every layer has per-group scales
    [T, N, ceil(K/G), 2] (fairy2i_quantize_grouped; LAYOUT_TILED_FP4 only)."""

    def __init__(self, layers, T: int, B: int, tiled: bool = False, layout=None, group_size: int = 0):
        if layout is None:
            layout = LAYOUT_TILED if tiled else LAYOUT_D3
        tiled = layout != LAYOUT_D3
        torch = _torch()
        lib = load()
        if not layers:
            raise ValueError("empty group")
        dt = _act_dtype(layers[0][4])
        dev = layers[0][4].device
        self._keep = [t for layer in layers for t in layer if t is not None]
        arr = (WlLayer * len(layers))()
        for i, (cu, su, cw, sw, x, xs, y) in enumerate(layers):
            _require(x, None, f"layers[{i}].x", dev)
            Bx, K = _act_shape(x)
            if Bx != B or _act_dtype(x) != dt:
                raise ValueError("all layers of a group share B and the activation dtype")
            for t, n in ((cu, "codes_U"), (cw, "codes_W")):
                _require(t, torch.uint8, f"layers[{i}].{n}", dev)
            _require(y, torch.complex64, f"layers[{i}].y", dev)
            if y.dim() != 2 or y.shape[0] != B:
                raise ValueError(f"layers[{i}].y must have shape ({B}, N)")
            N = y.shape[1]
            sshape = (T, 2) if group_size == 0 else (T, N, -(-K // group_size) if group_size > 0 else 0, 2)
            for t, n in ((su, "scales_U"), (sw, "scales_W")):
                _require(t, torch.float32, f"layers[{i}].{n}", dev)
                if tuple(t.shape) != sshape:
                    raise ValueError(f"layers[{i}].{n} must have shape {sshape}")
            if xs is not None:
                _require(xs, torch.float32, f"layers[{i}].x_scale", dev)
                if tuple(xs.shape) != (B,):
                    raise ValueError(f"layers[{i}].x_scale must have shape ({B},)")
            if tiled:
                need = repack_tiled_bytes(N, K, T)
                if cu.numel() < need or cw.numel() < need:
                    raise ValueError("tiled codes smaller than fairy2i_repack_tiled_bytes")
            elif tuple(cu.shape) != (T, N, K // 4) or tuple(cw.shape) != (T, N, K // 4):
                raise ValueError(f"layers[{i}] codes must have shape ({T}, {N}, {K // 4})")
            arr[i] = WlLayer(cu.data_ptr(), su.data_ptr(), cw.data_ptr(), sw.data_ptr(), x.data_ptr(),
                             None if xs is None else xs.data_ptr(), y.data_ptr(), N, K,
                             layout, group_size)
        self.n = len(layers)
        wsb = int(lib.fairy2i_wl_group_workspace_bytes(ctypes.byref(arr), self.n, T, dt, B))
        self.workspace = torch.empty(max(wsb, 1), dtype=torch.uint8, device=dev)
        tb = int(lib.fairy2i_wl_group_table_bytes(self.n))
        self._table = (ctypes.c_uint8 * tb)()
        _check(lib.fairy2i_wl_group_build_table(ctypes.byref(arr), self.n, T, dt, B,
                                                _ptr(self.workspace), wsb, ctypes.byref(self._table), tb),
               "fairy2i_wl_group_build_table")
        host = torch.frombuffer(bytearray(bytes(self._table)), dtype=torch.uint8)
        self.table_device = host.to(dev)
        torch.cuda.synchronize(dev)
        self._layers = arr

    def run(self, events=None):
        """One grouped call.  ``events``: optional 4 torch.cuda.Event already
        recorded once (so they exist); the library re-records them around its
        three kernels on the current stream."""
        lib = load()
        stream = _stream_ptr(self.table_device)
        if events is None:
            _check(lib.fairy2i_wl_matmul_group(ctypes.byref(self._table), _ptr(self.table_device), stream),
                   "fairy2i_wl_matmul_group")
            return
        handles = (_c_p * 4)(*[e.cuda_event for e in events])
        _check(lib.fairy2i_wl_matmul_group_timed(ctypes.byref(self._table), _ptr(self.table_device), stream,
                                                 handles), "fairy2i_wl_matmul_group_timed")


BLOCK_PROJ = ("q", "k", "v", "o", "gate", "up", "down")


class WlBlock:
    """One widely-linear decoder block for one decode token
    (fairy2i_block_decode).  ``layers``: {name: (codes_U, scales_U, codes_W,
    scales_W)} for q, k, v, o, gate, up, down, codes in the fp4 tiled layout
    (repack_tiled_fp4); ``norm_attn``, ``norm_mlp``: float32 [2n] device
    tensors.  Keeps the weights, the workspace and both plan copies alive."""

    def __init__(self, layers, norm_attn, norm_mlp, n, n_ff, n_heads, T, max_ctx, eps=1e-5, rope_base=10000.0):
        torch = _torch()
        lib = load()
        dev = norm_attn.device
        d = BlockDesc()
        d.n, d.n_ff, d.n_heads, d.T, d.max_ctx = n, n_ff, n_heads, T, max_ctx
        d.eps, d.reserved, d.rope_base = eps, 0, rope_base
        self._keep = []
        for i, name in enumerate(BLOCK_PROJ):
            cu, su, cw, sw = layers[name]
            for t, nm, dt in ((cu, "codes_U", torch.uint8), (cw, "codes_W", torch.uint8),
                              (su, "scales_U", torch.float32), (sw, "scales_W", torch.float32)):
                _require(t, dt, f"{name}.{nm}", dev)
            N = n_ff if name in ("gate", "up") else n
            K = n_ff if name == "down" else n
            need = repack_tiled_bytes(N, K, T)
            if cu.numel() < need or cw.numel() < need or tuple(su.shape) != (T, 2) or tuple(sw.shape) != (T, 2):
                raise ValueError(f"{name}: codes or scales do not match a {N}x{K} layer with T={T}")
            d.codes_U[i], d.scales_U[i] = cu.data_ptr(), su.data_ptr()
            d.codes_W[i], d.scales_W[i] = cw.data_ptr(), sw.data_ptr()
            self._keep += [cu, su, cw, sw]
        for t, nm in ((norm_attn, "norm_attn"), (norm_mlp, "norm_mlp")):
            _require(t, torch.float32, nm, dev)
            if t.numel() != 2 * n:
                raise ValueError(f"{nm} must hold 2n = {2 * n} gains")
        d.norm_attn, d.norm_mlp = norm_attn.data_ptr(), norm_mlp.data_ptr()
        self._keep += [norm_attn, norm_mlp]
        self.n, self.n_ff, self.n_heads, self.max_ctx = n, n_ff, n_heads, max_ctx
        self._desc = d
        wsb = int(lib.fairy2i_block_workspace_bytes(ctypes.byref(d)))
        pb = int(lib.fairy2i_block_plan_bytes(ctypes.byref(d)))
        if wsb == 0 or pb == 0:
            raise Fairy2iError(ERR_SHAPE, "fairy2i_block_workspace_bytes")
        self.workspace = torch.empty(wsb, dtype=torch.uint8, device=dev)
        self._plan = (ctypes.c_uint8 * pb)()
        _check(lib.fairy2i_block_build_plan(ctypes.byref(d), _ptr(self.workspace), wsb, ctypes.byref(self._plan), pb),
               "fairy2i_block_build_plan")
        self.plan_device = torch.frombuffer(bytearray(bytes(self._plan)), dtype=torch.uint8).to(dev)
        torch.cuda.synchronize(dev)

    BLOCK_INTERMEDIATES = (("z", "bf16", "n"), ("q_rot", "c64", "n"), ("v", "c64", "n"), ("o", "bf16", "n"),
                           ("a", "c64", "n"), ("h1", "c64", "n"), ("z2", "bf16", "n"), ("g", "c64", "f"),
                           ("u", "c64", "f"), ("act", "bf16", "f"), ("d", "c64", "n"), ("k", "c64", "n"))

    def intermediates(self):
        """Views of the workspace buffers that the last decode left
        (fairy2i_block_intermediates): {name: tensor}, complex64 [len] or
        bf16 [len, 2]."""
        torch = _torch()
        lib = load()
        ptrs = (_c_p * 12)()
        _check(lib.fairy2i_block_intermediates(ctypes.byref(self._plan), ptrs), "fairy2i_block_intermediates")
        base = self.workspace.data_ptr()
        out = {}
        for (name, kind, ln), p in zip(self.BLOCK_INTERMEDIATES, ptrs):
            count = self.n if ln == "n" else self.n_ff
            off = int(p) - base
            if kind == "c64":
                out[name] = self.workspace[off:off + 8 * count].view(torch.complex64)
            else:
                out[name] = self.workspace[off:off + 4 * count].view(torch.bfloat16).view(count, 2)
        return out

    def decode(self, x, k_cache, v_cache, pos, out=None):
        """x: complex64 [1, n]; caches complex64 [n_heads, max_ctx, n / n_heads];
        returns out complex64 [1, n]."""
        torch = _torch()
        lib = load()
        dev = self.plan_device.device
        dc = self.n // self.n_heads
        _require(x, torch.complex64, "x", dev)
        if x.numel() != self.n:
            raise ValueError(f"x must hold {self.n} complex entries")
        for t, nm in ((k_cache, "k_cache"), (v_cache, "v_cache")):
            _require(t, torch.complex64, nm, dev)
            if tuple(t.shape) != (self.n_heads, self.max_ctx, dc):
                raise ValueError(f"{nm} must have shape ({self.n_heads}, {self.max_ctx}, {dc})")
        if out is None:
            out = torch.empty((1, self.n), dtype=torch.complex64, device=dev)
        else:
            _require(out, torch.complex64, "out", dev)
            if out.numel() != self.n:
                raise ValueError(f"out must hold {self.n} complex entries")
        _check(lib.fairy2i_block_decode(ctypes.byref(self._plan), _ptr(self.plan_device), _ptr(x), _ptr(k_cache),
                                        _ptr(v_cache), int(pos), _ptr(out), _stream_ptr(x)), "fairy2i_block_decode")
        return out


# -------------------------------------------------------------- serving ---

def add_rmsnorm_i8(x, gain, delta=None, eps=1e-5, h_out=None, out=None):
    """h = x + delta and RMSNorm(h) as int8 activations in one pass
    (fairy2i_add_rmsnorm_i8).

    x, delta: complex64 [B, n] (delta may be None: h is x); gain: float32
    [2n], the real parts' gains, then the imaginary parts'.  Returns (h,
    q int8 [B, n, 2], x_scale float32 [B]); (q, x_scale) is what wl_matmul
    takes.  h_out: where h goes (x and delta themselves are allowed; by
    default a new tensor, and x as it is where there is no delta); out: a pair
    (q, x_scale) to write."""
    torch = _torch_module or _torch()
    lib = _lib or load()
    # launch latency counts: everything is looked over in one expression, _check_norm names what is wrong
    try:
        index = x.get_device()
        ok = (index >= 0 and x.dtype is torch.complex64 and x.is_contiguous() and not x.is_conj()
              and gain.dtype is torch.float32 and gain.get_device() == index and gain.is_contiguous()
              and (delta is None or (delta.dtype is torch.complex64 and delta.get_device() == index
                                     and delta.is_contiguous() and not delta.is_conj() and delta.shape == x.shape)))
        B, n = x.shape
        ok = ok and gain.shape == (2 * n,)
    except (AttributeError, TypeError, ValueError):
        ok = False
    if not ok:
        _check_norm(x, gain, delta)
    if h_out is not None:
        _require(h_out, torch.complex64, "h_out", x.device)
        if h_out.shape != x.shape or h_out.is_conj():
            raise ValueError("h_out must have x's shape, and not be a conjugated view")
    elif delta is not None:
        h_out = torch.empty_like(x)
    if out is None:
        q = torch.empty((B, n, 2), dtype=torch.int8, device=x.device)
        scale = torch.empty(B, dtype=torch.float32, device=x.device)
    else:
        q, scale = out
        _require(q, torch.int8, "out[0]", x.device)
        _require(scale, torch.float32, "out[1]", x.device)
        if q.shape != (B, n, 2) or scale.shape != (B,):
            raise ValueError("out must be (int8 [B, n, 2], float32 [B])")
    _check(lib.fairy2i_add_rmsnorm_i8(x.data_ptr(), None if delta is None else delta.data_ptr(), gain.data_ptr(), eps,
                                      B, n, None if h_out is None else h_out.data_ptr(), q.data_ptr(),
                                      scale.data_ptr(), _raw_stream(index)), "fairy2i_add_rmsnorm_i8")
    return x if h_out is None else h_out, q, scale


def _check_norm(x, gain, delta):
    torch = _torch()
    _require(x, torch.complex64, "x")
    if x.dim() != 2:
        raise ValueError("x must be [B, n]")
    _require(gain, torch.float32, "gain", x.device)
    if gain.shape != (2 * x.shape[1],):
        raise ValueError(f"gain must have shape ({2 * x.shape[1]},), got {tuple(gain.shape)}")
    if delta is not None:
        _require(delta, torch.complex64, "delta", x.device)
        if delta.shape != x.shape:
            raise ValueError("delta must have x's shape")
    for t, name in ((x, "x"), (delta, "delta")):
        if t is not None and t.is_conj():
            raise ValueError(f"{name} is a conjugated view: resolve_conj() it first")


def rope_table(n_pos, dc, base=10000.0, device="cuda"):
    """float32 [n_pos, dc, 2]: (cos, sin) of p * base^(-j / dc) for position p
    and entry j of a head (fairy2i_rope_table)."""
    torch = _torch()
    lib = load()
    if n_pos < 1 or dc < 1:
        raise ValueError("n_pos and dc must be positive")
    out = torch.empty((n_pos, dc, 2), dtype=torch.float32, device=device)
    _require(out, None, "device")
    with torch.cuda.device(out.device):
        _check(lib.fairy2i_rope_table(n_pos, dc, base, out.data_ptr(), _stream_ptr(out)), "fairy2i_rope_table")
    return out


class PagedKv:
    """Paged cache of keys and values in microscaled 4-bit floating point, for
    any number of sequences (fairy2i_kv_cache; the format and its layout are in
    include/fairy2i.h).

    n_pages pages of page_size positions (a multiple of 32), n_kv_heads heads
    of dc complex entries (a multiple of 16, up to 128).  ``data``: a uint8
    device tensor of PagedKv.bytes(...) bytes to use; a new one otherwise.

    Every call takes the batch as three int32 device tensors: ``pages``
    [n_seqs, max_pages] (the page of each run of page_size positions),
    ``cu_new`` [n_seqs + 1] (sequence i's rows are cu_new[i] ..
    cu_new[i + 1] - 1) and ``lens`` [n_seqs] (positions of the sequence, its
    rows included).  They stay on the device: a captured graph follows what
    they hold."""

    def __init__(self, n_pages, page_size, n_kv_heads, dc, data=None, device="cuda"):
        torch = _torch()
        need = self.bytes(n_pages, page_size, n_kv_heads, dc)
        if data is None:
            data = torch.empty(need, dtype=torch.uint8, device=device)
        _require(data, torch.uint8, "data")
        if data.numel() < need:
            raise ValueError(f"data must hold {need} bytes, got {data.numel()}")
        self.data = data
        self._index = data.get_device()
        self.n_pages, self.page_size, self.n_kv_heads, self.dc = n_pages, page_size, n_kv_heads, dc
        self._desc = KvCacheDesc(data.data_ptr(), n_pages, page_size, n_kv_heads, dc, 0)
        self._ref = ctypes.byref(self._desc)

    @staticmethod
    def bytes(n_pages, page_size, n_kv_heads, dc) -> int:
        """Bytes of such a cache."""
        need = int(load().fairy2i_kv_cache_bytes(n_pages, page_size, n_kv_heads, dc))
        if need == 0:
            raise ValueError("a cache has n_pages >= 1, page_size a multiple of 32 up to 65536, n_kv_heads in "
                             "[1, 65535] and dc a multiple of 16 up to 128")
        return need

    def _batch(self, pages, cu_new, lens, n_new):
        torch = _torch_module
        index = self._index
        int32 = torch.int32
        try:
            n_seqs, max_pages = pages.shape
            if (pages.dtype is int32 and pages.get_device() == index and pages.is_contiguous()
                    and cu_new.dtype is int32 and cu_new.get_device() == index and cu_new.is_contiguous()
                    and lens.dtype is int32 and lens.get_device() == index and lens.is_contiguous()
                    and lens.shape == (n_seqs,) and cu_new.shape == (n_seqs + 1,)):
                return KvBatchDesc(pages.data_ptr(), cu_new.data_ptr(), lens.data_ptr(), n_new, n_seqs, max_pages)
        except (AttributeError, TypeError, ValueError):
            pass
        for t, name in ((pages, "pages"), (cu_new, "cu_new"), (lens, "lens")):
            _require(t, int32, name, self.data.device)
        raise ValueError("pages must be [n_seqs, max_pages], cu_new [n_seqs + 1] and lens [n_seqs]")

    def _rows(self, x, heads, name):
        """(rows, heads, row stride) of complex64 [N, heads * dc] or [N, heads, dc] whose rows are whole."""
        torch = _torch_module
        if not isinstance(x, torch.Tensor):
            raise TypeError(f"{name} must be a torch.Tensor")
        if x.get_device() != self._index:
            raise ValueError(f"{name} is on {x.device}, expected {self.data.device}")
        if x.dtype is not torch.complex64:
            raise TypeError(f"{name} must be {torch.complex64}, got {x.dtype}")
        if x.is_conj():
            raise ValueError(f"{name} is a conjugated view: resolve_conj() it first")
        dc, shape, stride = self.dc, x.shape, x.stride()
        if len(shape) == 3:
            n = shape[1]
            whole = shape[2] == dc and stride[2] == 1 and (n == 1 or stride[1] == dc)
        else:
            whole = len(shape) == 2 and shape[1] % dc == 0 and stride[1] == 1
            n = shape[1] // dc if whole else 0
        if not whole or n == 0 or (heads is not None and n != heads):
            raise ValueError(f"{name} must be [N, heads * {dc}] or [N, heads, {dc}]"
                             + ("" if heads is None else f" with {heads} heads") + ", each row contiguous")
        ld = stride[0] if shape[0] > 1 else n * dc
        if ld < n * dc:
            raise ValueError(f"{name}'s rows overlap")
        return shape[0], n, ld

    def append(self, k, v, pages, cu_new, lens, rope, q=None, q_out=None):
        """Append the rows of k and v, k turned by its position, and turn q
        alike (fairy2i_kv_append).

        k, v: complex64 [N, n_kv_heads * dc]; q: complex64 [N, heads * dc] or
        None (also [N, heads, dc]; rows may be columns of one wider product);
        rope: float32 [positions, dc, 2] (rope_table).  Returns q in bf16,
        [N, heads, dc, 2] (q_out: such a tensor to write), or None."""
        torch = _torch_module or _torch()
        lib = _lib or load()
        N, _, k_ld = self._rows(k, self.n_kv_heads, "k")
        Nv, _, v_ld = self._rows(v, self.n_kv_heads, "v")
        heads = q_ld = 0
        if q is not None:
            Nq, heads, q_ld = self._rows(q, None, "q")
            if Nq != N:
                raise ValueError("q, k and v must have as many rows")
            if q_out is None:
                q_out = torch.empty((N, heads, self.dc, 2), dtype=torch.bfloat16, device=k.device)
            else:
                _require(q_out, torch.bfloat16, "q_out", k.device)
                if q_out.shape != (N, heads, self.dc, 2):
                    raise ValueError(f"q_out must have shape {(N, heads, self.dc, 2)}")
        elif q_out is not None:
            raise ValueError("q_out without q")
        if Nv != N:
            raise ValueError("q, k and v must have as many rows")
        _require(rope, torch.float32, "rope", k.device)
        if rope.dim() != 3 or rope.shape[1:] != (self.dc, 2):
            raise ValueError(f"rope must be [positions, {self.dc}, 2]")
        batch = self._batch(pages, cu_new, lens, N)
        _check(lib.fairy2i_kv_append(self._ref, ctypes.byref(batch), None if q is None else q.data_ptr(), q_ld, heads,
                                     k.data_ptr(), k_ld, v.data_ptr(), v_ld, rope.data_ptr(), rope.shape[0],
                                     None if q is None else q_out.data_ptr(), _raw_stream(self._index)),
               "fairy2i_kv_append")
        return q_out

    def read(self, pages, cu_new, lens, n_new, out=None):
        """(k, v) bf16 [n_new, n_kv_heads, dc, 2]: what the cache stands for
        at the positions of the batch's n_new rows, exact (fairy2i_kv_read);
        cu_new over whole sequences reads them all."""
        torch = _torch_module or _torch()
        lib = _lib or load()
        dev = self.data.device
        shape = (n_new, self.n_kv_heads, self.dc, 2)
        if out is None:
            out = (torch.empty(shape, dtype=torch.bfloat16, device=dev),
                   torch.empty(shape, dtype=torch.bfloat16, device=dev))
        else:
            for t in out:
                _require(t, torch.bfloat16, "out", dev)
                if t.shape != shape:
                    raise ValueError(f"out must be a pair of shape {shape}")
        batch = self._batch(pages, cu_new, lens, n_new)
        _check(lib.fairy2i_kv_read(self._ref, ctypes.byref(batch), out[0].data_ptr(), out[1].data_ptr(),
                                   _raw_stream(self._index)), "fairy2i_kv_read")
        return tuple(out)

    def attend_workspace_bytes(self, n_new, n_seqs, heads) -> int:
        """Bytes of workspace that attend takes for such a batch."""
        return int(load().fairy2i_kv_attend_workspace_bytes(self._ref, n_new, n_seqs, heads))

    def attend(self, q, pages, cu_new, lens, scale=None, out=None, workspace=None):
        """Causal Hermitian-score attention of the batch's rows over the cache
        (fairy2i_kv_attend).

        q: bf16 [N, heads, dc, 2], turned by its positions (append's result);
        heads a multiple of n_kv_heads, neighbours sharing a key head; scale:
        1 / sqrt(2 dc) by default.  Returns bf16 [N, heads, dc, 2] (out: such a
        tensor to write); seen as [N, heads * dc, 2] it is what wl_matmul
        takes."""
        torch = _torch_module or _torch()
        lib = _lib or load()
        index = self._index
        try:
            ok = q.dtype is torch.bfloat16 and q.get_device() == index and q.is_contiguous()
            N, heads, dc, two = q.shape
            ok = ok and dc == self.dc and two == 2
        except (AttributeError, ValueError):
            ok = False
        if not ok:
            _require(q, torch.bfloat16, "q", self.data.device)
            raise ValueError(f"q must be [N, heads, {self.dc}, 2]")
        if heads == 0 or heads % self.n_kv_heads != 0:
            raise ValueError(f"q's heads must be a multiple of {self.n_kv_heads}")
        if out is None:
            out = torch.empty_like(q)
        else:
            _require(out, torch.bfloat16, "out", q.device)
            if out.shape != q.shape:
                raise ValueError("out must have q's shape")
        batch = self._batch(pages, cu_new, lens, N)
        if workspace is None:
            need = lib.fairy2i_kv_attend_workspace_bytes(self._ref, N, pages.shape[0], heads)
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
        else:  # its size is the library's to check
            _require(workspace, torch.uint8, "workspace", q.device)
        _check(lib.fairy2i_kv_attend(self._ref, ctypes.byref(batch), q.data_ptr(), heads,
                                     (2 * self.dc) ** -0.5 if scale is None else scale, out.data_ptr(),
                                     workspace.data_ptr(), workspace.numel(), _raw_stream(index)),
               "fairy2i_kv_attend")
        return out


# ------------------------------------------------------------- training ---

def _call(name, index, *args):
    """A library call on the current stream of device `index`, which is made the current one for it."""
    fn = getattr(_lib, name)
    if _torch_module._C._cuda_getDevice() == index:  # torch.cuda.current_device less its own look whether CUDA is there
        status = fn(*args, _raw_stream(index))
    else:
        with _torch_module.cuda.device(index):
            status = fn(*args, _raw_stream(index))
    if status != OK:
        raise Fairy2iError(status, name)


class Fp8Matrix:
    """rows x cols reals in e4m3 with a power-of-two scale for 128 neighbours of
    a row (fairy2i_fp8_matrix; the format is in include/fairy2i.h).

    ``codes``: float8_e4m3fn [rows, cols rounded up to 128], zeros past cols;
    ``scales``: uint8 [ceil(cols / 512), rows, 4]; both device tensors, new ones
    (their contents undefined) where they are not given.  rows and cols up to
    2^22."""

    def __init__(self, rows, cols, codes=None, scales=None, device="cuda"):
        torch = _torch_module or _torch()
        if _lib is None:
            load()
        if not (1 <= rows <= 1 << 22 and 1 <= cols <= 1 << 22):
            raise ValueError("rows and cols must be in [1, 2^22]")
        self.rows, self.cols = rows, cols
        ld, groups = -(-cols // 128) * 128, -(-cols // 512)
        if codes is None and scales is None:  # one piece of memory, seen as codes and scales when they are asked for
            self._data = torch.empty(rows * (ld + 4 * groups), dtype=torch.uint8, device=device)
            self._codes = self._scales = None
            at = self._data.data_ptr()
            self._set(self._data, at, at + rows * ld)
            return
        if codes is None:
            codes = torch.empty((rows, ld), dtype=torch.float8_e4m3fn, device=scales.device)
        if scales is None:
            scales = torch.empty((groups, rows, 4), dtype=torch.uint8, device=codes.device)
        _require(codes, torch.float8_e4m3fn, "codes")
        _require(scales, torch.uint8, "scales", codes.device)
        if codes.shape != (rows, ld) or scales.shape != (groups, rows, 4):
            raise ValueError(f"codes must be {(rows, ld)} and scales {(groups, rows, 4)}")
        self._codes, self._scales = codes, scales
        self._set(codes, codes.data_ptr(), scales.data_ptr())

    def _set(self, data, codes, scales):
        self.device, self._index = data.device, data.get_device()
        if self._index < 0:
            raise ValueError("a Fp8Matrix lives on a GPU")
        self._desc = Fp8Desc(codes, scales, self.rows, self.cols)
        self._ref = ctypes.byref(self._desc)

    @property
    def codes(self):
        if self._codes is None:
            n = self.rows * (-(-self.cols // 128) * 128)
            self._codes = self._data[:n].view(_torch_module.float8_e4m3fn).view(self.rows, -1)
        return self._codes

    @property
    def scales(self):
        if self._scales is None:
            n = self.rows * (-(-self.cols // 128) * 128)
            self._scales = self._data[n:].view(-1, self.rows, 4)
        return self._scales

    def dequantize(self, out=None):
        """What the matrix stands for: bf16 [rows, cols], exact (out: such a tensor to write)."""
        torch = _torch_module
        if out is None:
            out = torch.empty((self.rows, self.cols), dtype=torch.bfloat16, device=self.device)
        else:
            _require(out, torch.bfloat16, "out", self.device)
            if out.shape != (self.rows, self.cols):
                raise ValueError(f"out must have shape {(self.rows, self.cols)}")
        _call("fairy2i_fp8_dequantize", self._index, self._ref, out.data_ptr())
        return out

    def transpose(self, out=None):
        """The transposed matrix, scales along the other axis (fairy2i_fp8_transpose;
        out: a Fp8Matrix to write)."""
        out = _fp8_out(out, self.cols, self.rows, self.device, "out")
        if out._desc.codes == self._desc.codes or out._desc.scales == self._desc.scales:
            raise ValueError("out must be other memory than the matrix itself")
        _call("fairy2i_fp8_transpose", self._index, self._ref, out._ref)
        return out


def _fp8_out(out, rows, cols, device, name):
    if out is None:
        return Fp8Matrix(rows, cols, device=device)
    if not isinstance(out, Fp8Matrix):
        raise TypeError(f"{name} must be a Fp8Matrix")
    if out.device != device:
        raise ValueError(f"{name} is on {out.device}, expected {device}")
    if (out.rows, out.cols) != (rows, cols):
        raise ValueError(f"{name} must be {rows} x {cols}, got {out.rows} x {out.cols}")
    return out


def _real_rows(x, name):
    """(dtype, rows, cols, row stride) of a matrix of reals: float32 or bf16 [rows, cols], its pairs [rows, n, 2], or
    complex64 [rows, n]; each row contiguous."""
    torch = _torch_module or _torch()
    if not isinstance(x, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not x.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if x.dtype is torch.complex64:
        if x.is_conj():
            raise ValueError(f"{name} is a conjugated view: resolve_conj() it first")
        if x.dim() != 2:
            raise ValueError(f"{name} must be [rows, n] where it is complex")
        dt, per = ACT_F32, 2
    elif x.dtype is torch.float32 or x.dtype is torch.bfloat16:
        if x.is_neg():
            raise ValueError(f"{name} is a negated view: resolve_neg() it first")
        dt, per = (ACT_F32 if x.dtype is torch.float32 else ACT_BF16), 1
    else:
        raise TypeError(f"{name} must be float32, bfloat16 or complex64, got {x.dtype}")
    shape, stride = x.shape, x.stride()
    if len(shape) == 3 and shape[2] == 2:
        cols, whole = 2 * shape[1], stride[2] == 1 and (shape[1] == 1 or stride[1] == 2)
    elif len(shape) == 2:
        cols, whole = per * shape[1], shape[1] == 1 or stride[1] == 1
    else:
        raise ValueError(f"{name} must be [rows, cols] or [rows, n, 2]")
    if not whole:
        raise ValueError(f"{name}'s rows must be contiguous")
    ld = per * stride[0] if shape[0] > 1 else cols
    if ld < cols:
        raise ValueError(f"{name}'s rows overlap")
    return dt, shape[0], cols, ld


def quantize_fp8(x, transposed=False, out=None):
    """The 8-bit form of a matrix of reals (fairy2i_fp8_quantize).

    x: float32 or bf16 [rows, cols], the pairs [rows, n, 2] or complex64 [rows,
    n] (cols = 2n); rows may be columns of a wider tensor.  Returns a Fp8Matrix
    rows x cols with blocks along the rows; with transposed=True the transposed
    matrix, cols x rows, with blocks along the columns of x; with
    transposed="both" the pair of them from one pass.  out: such a Fp8Matrix (or
    pair) to write."""
    dt, rows, cols, ld = _real_rows(x, "x")
    if _lib is None:
        load()
    if transposed not in (False, True, "both"):
        raise ValueError('transposed must be False, True or "both"')
    both = transposed == "both"
    a, b = out if both and out is not None else (out, out)
    direct = turned = None
    if both or not transposed:
        direct = _fp8_out(a, rows, cols, x.device, "out")
    if transposed:
        turned = _fp8_out(b, cols, rows, x.device, "out")
    _call("fairy2i_fp8_quantize", x.get_device(), x.data_ptr(), dt, ld, None if direct is None else direct._ref,
          None if turned is None else turned._ref)
    if both:
        return direct, turned
    return turned if transposed else direct


def gemm_fp8(A, B, out=None, dtype=None, accumulate=False, workspace=None):
    """C = A B^T of two Fp8Matrix, A [M, K] and B [N, K] (fairy2i_gemm_fp8).

    Returns C [M, N] in dtype (bfloat16 by default, or float32); out: such a
    tensor to write, whose rows may be columns of a wider one; accumulate=True
    adds to it.  With tokens in rows a layer of real form R (wl_realify) has
    Y = gemm_fp8(X, R), G_X = gemm_fp8(G_Y, R transposed) and
    G_R = gemm_fp8(G_Y transposed, X transposed)."""
    torch = _torch_module or _torch()
    for m, name in ((A, "A"), (B, "B")):
        if not isinstance(m, Fp8Matrix):
            raise TypeError(f"{name} must be a Fp8Matrix")
    if A.cols != B.cols:
        raise ValueError(f"A has {A.cols} columns, B {B.cols}")
    index = A._index
    if B._index != index:
        raise ValueError(f"B is on {B.device}, expected {A.device}")
    M, N = A.rows, B.rows
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs out")
        out = torch.empty((M, N), dtype=torch.bfloat16 if dtype is None else dtype, device=A.device)
        ldc = N
    else:
        if not isinstance(out, torch.Tensor):
            raise TypeError("out must be a torch.Tensor")
        if out.get_device() != index:
            raise ValueError(f"out is on {out.device}, expected {A.device}")
        if dtype is not None and out.dtype is not dtype:
            raise TypeError(f"out must be {dtype}, got {out.dtype}")
        if out.is_neg():
            raise ValueError("out is a negated view")
        if out.shape != (M, N) or (N > 1 and out.stride(1) != 1):
            raise ValueError(f"out must have shape ({M}, {N}), each row contiguous")
        ldc = out.stride(0) if M > 1 else N
        if ldc < N:
            raise ValueError("out's rows overlap")
    if out.dtype is torch.bfloat16:
        dt = ACT_BF16
    elif out.dtype is torch.float32:
        dt = ACT_F32
    else:
        raise TypeError(f"the product is bfloat16 or float32, not {out.dtype}")
    if workspace is None:
        need = _lib.fairy2i_gemm_fp8_workspace_bytes(M, N, A.cols)
        if need:
            workspace = torch.empty(need, dtype=torch.uint8, device=out.device)
    else:  # its size is the library's to check
        _require(workspace, torch.uint8, "workspace", out.device)
    _call("fairy2i_gemm_fp8", index, A._ref, B._ref, out.data_ptr(), dt, ldc, int(bool(accumulate)),
          None if workspace is None else workspace.data_ptr(), 0 if workspace is None else workspace.numel())
    return out


def add_layernorm(x, gain, bias=None, delta=None, eps=1e-5, center=True, h_out=None, out=None, fp8=False):
    """h = x + delta and its layer norm, or RMSNorm for center=False
    (fairy2i_add_layernorm).

    x, delta: complex64 [B, n] (delta may be None: h is x); gain, bias: float32
    [2n], the real parts' values, then the imaginary parts' (bias may be None).
    Returns (h, z, stats): z in bf16 [B, n, 2], or with fp8=True a Fp8Matrix B x
    2n, what gemm_fp8 takes; stats float32 [B, 2], for layernorm_backward.
    h_out: where h goes (x and delta themselves are allowed; by default a new
    tensor, and x as it is where there is no delta); out: the z to write."""
    torch = _torch_module or _torch()
    lib = _lib or load()
    # launch latency counts: everything is looked over in one expression, _check_layernorm names what is wrong
    try:
        index = x.get_device()
        ok = (index >= 0 and x.dtype is torch.complex64 and x.is_contiguous() and not x.is_conj()
              and gain.dtype is torch.float32 and gain.get_device() == index and gain.is_contiguous()
              and (bias is None or (bias.dtype is torch.float32 and bias.get_device() == index
                                    and bias.is_contiguous() and bias.shape == gain.shape))
              and (delta is None or (delta.dtype is torch.complex64 and delta.get_device() == index
                                     and delta.is_contiguous() and not delta.is_conj() and delta.shape == x.shape)))
        B, n = x.shape
        ok = ok and gain.shape == (2 * n,)
    except (AttributeError, TypeError, ValueError):
        ok = False
    if not ok:
        _check_layernorm(x, gain, bias, delta)
    if h_out is not None:
        _require(h_out, torch.complex64, "h_out", x.device)
        if h_out.shape != x.shape or h_out.is_conj():
            raise ValueError("h_out must have x's shape, and not be a conjugated view")
    elif delta is not None:
        h_out = torch.empty_like(x)
    if fp8:
        out = _fp8_out(out, B, 2 * n, x.device, "out")
    elif out is None:
        out = torch.empty((B, n, 2), dtype=torch.bfloat16, device=x.device)
    else:
        _require(out, torch.bfloat16, "out", x.device)
        if out.shape != (B, n, 2):
            raise ValueError(f"out must have shape ({B}, {n}, 2)")
    stats = gain.new_empty((B, 2))  # 0.3 us less than torch.empty with type and device
    _call("fairy2i_add_layernorm", index, x.data_ptr(), None if delta is None else delta.data_ptr(), gain.data_ptr(),
          None if bias is None else bias.data_ptr(), eps, int(bool(center)), B, n,
          None if h_out is None else h_out.data_ptr(), None if fp8 else out.data_ptr(), out._ref if fp8 else None,
          stats.data_ptr())
    return x if h_out is None else h_out, out, stats


def _check_layernorm(x, gain, bias, delta):
    _check_norm(x, gain, delta)
    if bias is not None:
        _require(bias, _torch().float32, "bias", x.device)
        if bias.shape != gain.shape:
            raise ValueError("bias must have gain's shape")


def layernorm_backward(dz, h, stats, gain, dh=None, center=True, bias=True, out=None, workspace=None):
    """The gradient of add_layernorm (fairy2i_layernorm_backward).

    dz: the gradient of z, bf16 [B, n, 2] or complex64 [B, n]; h, stats: what
    add_layernorm returned; dh: complex64 [B, n], the gradient that reaches h by
    the residual, or None; center: as there.  Returns (dx, dgain, dbias): dx
    complex64 [B, n], of x and of delta alike (out: such a tensor to write, dh
    and h themselves are allowed); dgain, dbias float32 [2n], dbias None for
    bias=False."""
    torch = _torch_module or _torch()
    lib = _lib or load()
    # launch latency counts: everything is looked over in one expression, _check_backward names what is wrong
    try:
        index = h.get_device()
        B, n = h.shape
        c64, f32 = torch.complex64, torch.float32
        dt = ACT_BF16 if dz.dtype is torch.bfloat16 else ACT_F32
        ok = (index >= 0 and h.dtype is c64 and h.is_contiguous() and not h.is_conj()
              and dz.get_device() == index and dz.is_contiguous()
              and (dz.shape == (B, n, 2) if dt == ACT_BF16 else
                   dz.dtype is c64 and dz.shape == (B, n) and not dz.is_conj())
              and stats.dtype is f32 and stats.get_device() == index and stats.is_contiguous() and stats.shape == (B, 2)
              and gain.dtype is f32 and gain.get_device() == index and gain.is_contiguous() and gain.shape == (2 * n,))
        for t in (dh, out):
            ok = ok and (t is None or (t.dtype is c64 and t.get_device() == index and t.is_contiguous()
                                       and not t.is_conj() and t.shape == h.shape))
    except (AttributeError, TypeError, ValueError):
        ok = False
    if not ok:
        _check_backward(dz, h, stats, gain, dh, out)
    dev = h.device
    dx = torch.empty_like(h) if out is None else out
    sums = torch.empty(4 * n if bias else 2 * n, dtype=torch.float32, device=dev)
    dgain, dbias = sums[:2 * n], sums[2 * n:] if bias else None
    if workspace is None:
        need = lib.fairy2i_layernorm_backward_workspace_bytes(B, n)
        if need:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    else:  # its size is the library's to check
        _require(workspace, torch.uint8, "workspace", dev)
    _call("fairy2i_layernorm_backward", index, dz.data_ptr(), dt, h.data_ptr(), stats.data_ptr(), gain.data_ptr(),
          None if dh is None else dh.data_ptr(), int(bool(center)), B, n, dx.data_ptr(), dgain.data_ptr(),
          dbias.data_ptr() if bias else None, None if workspace is None else workspace.data_ptr(),
          0 if workspace is None else workspace.numel())
    return dx, dgain, dbias


def _check_backward(dz, h, stats, gain, dh, out):
    torch = _torch()
    _require(h, torch.complex64, "h")
    if h.dim() != 2:
        raise ValueError("h must be [B, n]")
    (B, n), dev = h.shape, h.device
    _require(dz, None, "dz", dev)
    if dz.dtype not in (torch.bfloat16, torch.complex64):
        raise TypeError(f"dz must be bfloat16 or complex64, got {dz.dtype}")
    shape = (B, n, 2) if dz.dtype is torch.bfloat16 else (B, n)
    if dz.shape != shape:
        raise ValueError(f"dz must have shape {shape}, got {tuple(dz.shape)}")
    _require(stats, torch.float32, "stats", dev)
    if stats.shape != (B, 2):
        raise ValueError(f"stats must have shape ({B}, 2)")
    _require(gain, torch.float32, "gain", dev)
    if gain.shape != (2 * n,):
        raise ValueError(f"gain must have shape ({2 * n},), got {tuple(gain.shape)}")
    for t, name in ((dh, "dh"), (out, "out")):
        if t is not None:
            _require(t, torch.complex64, name, dev)
            if t.shape != h.shape:
                raise ValueError(f"{name} must have h's shape")
    for t, name in ((dz, "dz"), (h, "h"), (dh, "dh"), (out, "out")):
        if t is not None and t.is_conj():
            raise ValueError(f"{name} is a conjugated view: resolve_conj() it first")
