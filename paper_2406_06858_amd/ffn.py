"""ctypes binding of libflux_ffn_mi355.so (include/flux_ffn.h): the gated feed-forward block, forward and backward, and
4-bit microscaled matrices with their products.  Argument marshalling only, as in `binding`: every function has the name
of the C entry point it calls, tensors are device buffers, nothing is computed in Python.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

from . import binding
from .binding import FLUX_BF16, FLUX_ERR_HIP, FLUX_F32, FLUX_OK, FluxError

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libflux_ffn_mi355.so")
_lib = None

FLUX_ACT_SILU, FLUX_ACT_GELU, FLUX_ACT_GELU_TANH = 0, 1, 2
FLUX_GLU_FORWARD, FLUX_GLU_BACKWARD = 0, 1
FLUX_MX4_GEMM, FLUX_MX4_GLU = 0, 1

EXPORTS = [
    "flux_glu", "flux_glu_backward", "flux_glu_workspace_bytes", "flux_ffn_init", "flux_mx4_row_bytes",
    "flux_mx4_scale_row_bytes", "flux_mx4_quantize", "flux_mx4_dequantize", "flux_mx4_workspace_bytes", "flux_mx4_gemm",
    "flux_mx4_glu", "flux_ffn_tile_config_count", "flux_ffn_tile_config_info", "flux_ffn_last_hip_error",
]


class flux_glu_t(C.Structure):
    _fields_ = [
        ("M", C.c_int32), ("N", C.c_int32), ("K", C.c_int32),
        ("act", C.c_int32), ("w_is_nk", C.c_int32),
        ("out_dtype", C.c_int32), ("dw_dtype", C.c_int32), ("dw_accumulate", C.c_int32),
        ("ldx", C.c_int64), ("ldw", C.c_int64), ("ldh", C.c_int64),
        ("tile_config", C.c_int32), ("split_k", C.c_int32),
    ]


class flux_mx4_t(C.Structure):
    _fields_ = [
        ("M", C.c_int32), ("N", C.c_int32), ("K", C.c_int32),
        ("out_dtype", C.c_int32), ("act", C.c_int32), ("reserved", C.c_int32),
        ("ldc", C.c_int64), ("tile_config", C.c_int32), ("split_k", C.c_int32),
    ]


def lib():
    """Loads the shared library on first use."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with `python -m paper_2406_06858_amd.build`")
        L = C.CDLL(_LIB_PATH)
        vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
        pg, pm = C.POINTER(flux_glu_t), C.POINTER(flux_mx4_t)
        L.flux_glu.argtypes = [pg, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.flux_glu_backward.argtypes = [pg, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.flux_glu_workspace_bytes.argtypes = [C.c_int, pg]
        L.flux_mx4_workspace_bytes.argtypes = [C.c_int, pm]
        L.flux_ffn_init.argtypes = [vp, sz, vp]
        L.flux_mx4_row_bytes.argtypes = [i32]
        L.flux_mx4_scale_row_bytes.argtypes = [i32]
        L.flux_mx4_quantize.argtypes = [i32, i32, i32, vp, i64, vp, vp, vp]
        L.flux_mx4_dequantize.argtypes = [i32, i32, vp, vp, i32, vp, i64, vp]
        L.flux_mx4_gemm.argtypes = [pm, vp, vp, vp, vp, vp, vp, sz, vp]
        L.flux_mx4_glu.argtypes = [pm, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.flux_ffn_tile_config_info.argtypes = [i32, C.POINTER(i32), C.POINTER(i32)]
        for name in EXPORTS:
            getattr(L, name).restype = sz if name.endswith("_bytes") else C.c_int
        _lib = L
    return _lib


_DT = {"bf16": FLUX_BF16, "f32": FLUX_F32, torch.bfloat16: FLUX_BF16, torch.float32: FLUX_F32}
_ACT = {"silu": FLUX_ACT_SILU, "gelu": FLUX_ACT_GELU, "gelu_tanh": FLUX_ACT_GELU_TANH}
_ptr = binding._ptr


def _stream(s) -> int:
    # (the current stream's handle without a torch.cuda.Stream around it: 0.1 us where that takes 2.9, as long as a launch)
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()) if s is None else s.cuda_stream


def _check(status: int, where: str):
    if status != FLUX_OK:
        raise FluxError(status, where, lib().flux_ffn_last_hip_error() if status == FLUX_ERR_HIP else None)


def _ws(workspace):
    return (0, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())


def glu_problem(M, N, K, act="silu", w_is_nk=0, out_dtype="bf16", dw_dtype="bf16", dw_accumulate=0, ldx=0, ldw=0, ldh=0,
                tile_config=0, split_k=0) -> flux_glu_t:
    return flux_glu_t(M, N, K, _ACT.get(act, act), w_is_nk, _DT[out_dtype], _DT[dw_dtype], dw_accumulate, ldx, ldw, ldh,
                      tile_config, split_k)


def mx4_problem(M, N, K, out_dtype="bf16", act="silu", ldc=0, tile_config=0, split_k=0) -> flux_mx4_t:
    return flux_mx4_t(M, N, K, _DT[out_dtype], _ACT.get(act, act), 0, ldc, tile_config, split_k)


def flux_glu_workspace_bytes(op: int, p: flux_glu_t) -> int:
    return int(lib().flux_glu_workspace_bytes(op, C.byref(p)))


def flux_mx4_workspace_bytes(op: int, p: flux_mx4_t) -> int:
    return int(lib().flux_mx4_workspace_bytes(op, C.byref(p)))


def flux_mx4_row_bytes(K: int) -> int:
    return int(lib().flux_mx4_row_bytes(K))


def flux_mx4_scale_row_bytes(K: int) -> int:
    return int(lib().flux_mx4_scale_row_bytes(K))


def flux_ffn_tile_config_count() -> int:
    return lib().flux_ffn_tile_config_count()


def flux_ffn_tile_config_info(cfg_id: int):
    v = [C.c_int32(0) for _ in range(2)]
    _check(lib().flux_ffn_tile_config_info(cfg_id, *[C.byref(x) for x in v]), "flux_ffn_tile_config_info")
    return tuple(x.value for x in v)


def flux_ffn_init(workspace, stream=None):
    _check(lib().flux_ffn_init(*_ws(workspace), _stream(stream)), "flux_ffn_init")


def flux_glu(p, X, Wg, Wu, H, G=None, U=None, workspace=None, stream=None):
    _check(lib().flux_glu(C.byref(p), _ptr(X), _ptr(Wg), _ptr(Wu), _ptr(H), _ptr(G), _ptr(U), *_ws(workspace), _stream(stream)),
           "flux_glu")


def flux_glu_backward(p, X, Wg, Wu, G, U, dH, dX, dWg, dWu, workspace, stream=None):
    _check(lib().flux_glu_backward(C.byref(p), _ptr(X), _ptr(Wg), _ptr(Wu), _ptr(G), _ptr(U), _ptr(dH), _ptr(dX), _ptr(dWg),
                                   _ptr(dWu), *_ws(workspace), _stream(stream)), "flux_glu_backward")


def _rows(t):
    """(rows, K, dtype, pitch) of a matrix whose rows are runs of memory, one behind the other.  (A pitch of 0 would say "packed" to the
    library, so an expanded row must not get there.)"""
    rows, K = t.shape
    step, one = t.stride()
    if K > 1 and one != 1:
        raise ValueError("the rows of the matrix have to be contiguous")
    if rows > 1 and step < K:
        raise ValueError("the rows of the matrix overlap")
    return rows, K, _DT[t.dtype], step if rows > 1 else 0


def _whole(t, nbytes, what):
    """Blocks have no pitch: row r lies r rows behind the first."""
    if t is not None and not (t.is_contiguous() and t.nbytes >= nbytes):
        raise ValueError(f"{what} has to be contiguous and hold {nbytes} bytes")


def _packed(q, scales, rows, K):
    blocks = (K + 31) // 32
    _whole(q, rows * blocks * 16, "q")
    _whole(scales, rows * ((blocks + 15) // 16 * 16), "scales")


def flux_mx4_quantize(src, q, scales, stream=None):
    rows, K, dtype, ld = _rows(src)
    _packed(q, scales, rows, K)
    _check(lib().flux_mx4_quantize(rows, K, dtype, _ptr(src), ld, _ptr(q), _ptr(scales), _stream(stream)), "flux_mx4_quantize")


def flux_mx4_dequantize(q, scales, dst, stream=None):
    rows, K, dtype, ld = _rows(dst)
    _packed(q, scales, rows, K)
    _check(lib().flux_mx4_dequantize(rows, K, _ptr(q), _ptr(scales), dtype, _ptr(dst), ld, _stream(stream)), "flux_mx4_dequantize")


def flux_mx4_gemm(p, Aq, As, Bq, Bs, Cout, workspace=None, stream=None):
    _check(lib().flux_mx4_gemm(C.byref(p), _ptr(Aq), _ptr(As), _ptr(Bq), _ptr(Bs), _ptr(Cout), *_ws(workspace), _stream(stream)),
           "flux_mx4_gemm")


def flux_mx4_glu(p, Xq, Xs, Wgq, Wgs, Wuq, Wus, H, workspace=None, stream=None):
    _check(lib().flux_mx4_glu(C.byref(p), _ptr(Xq), _ptr(Xs), _ptr(Wgq), _ptr(Wgs), _ptr(Wuq), _ptr(Wus), _ptr(H), *_ws(workspace),
                              _stream(stream)), "flux_mx4_glu")
