"""ctypes binding of include/flux_norm.h (in libflux_ffn_mi355.so): the root-mean-square norm with the residual's addition, its backward pass,
and 8-bit blocks read back.  Argument marshalling only, as in `ffn`; a tensor of another type than the problem's, of another device than the
current one, or whose numbers do not lie where the problem says, raises ValueError.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import ffn
from .binding import FLUX_BF16, FLUX_F32
from .ffn import _check, _packed, _rows, _stream, _ws

FLUX_NORM_BF16, FLUX_NORM_F32, FLUX_NORM_MX4, FLUX_NORM_MX8 = range(4)

EXPORTS = ["flux_norm", "flux_norm_backward", "flux_norm_workspace_bytes", "flux_mx8_row_bytes", "flux_mx8_dequantize"]


class flux_norm_t(C.Structure):
    _fields_ = [
        ("M", C.c_int32), ("K", C.c_int32), ("x_dtype", C.c_int32), ("s_dtype", C.c_int32), ("w_dtype", C.c_int32),
        ("out", C.c_int32), ("dw_dtype", C.c_int32), ("dw_accumulate", C.c_int32), ("eps", C.c_float), ("reserved", C.c_int32),
        ("ldx", C.c_int64), ("lds", C.c_int64), ("ldy", C.c_int64),
    ]


_lib = None


def lib():
    """The shared library, with this header's functions declared."""
    global _lib
    if _lib is None:
        L = ffn.lib()
        vp, i32, i64, sz, pn = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t, C.POINTER(flux_norm_t)
        L.flux_norm.argtypes = [pn, vp, vp, vp, vp, vp, vp, vp, vp]
        L.flux_norm_backward.argtypes = [pn, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.flux_norm_workspace_bytes.argtypes = [pn]
        L.flux_mx8_row_bytes.argtypes = [i32]
        L.flux_mx8_dequantize.argtypes = [i32, i32, vp, vp, i32, vp, i64, vp]
        for name in EXPORTS:
            getattr(L, name).restype = sz if name.endswith("_bytes") else C.c_int
        _lib = L
    return _lib


_DT = {"bf16": FLUX_BF16, "f32": FLUX_F32, torch.bfloat16: FLUX_BF16, torch.float32: FLUX_F32}
_OUT = {"bf16": FLUX_NORM_BF16, "f32": FLUX_NORM_F32, "mx4": FLUX_NORM_MX4, "mx8": FLUX_NORM_MX8, torch.bfloat16: FLUX_NORM_BF16, torch.float32: FLUX_NORM_F32}
_TYPES = (torch.bfloat16, torch.float32, torch.uint8, torch.uint8)          # by flux_dtype_t and flux_norm_out_t
_U8, _F32 = torch.uint8, torch.float32
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)          # (a torch without GPU has no such function, and an error for every call)


def _buf(t, dtype, device, what):
    """The address of a tensor of `dtype` on the current device; 0 for None."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.get_device() != device:
        raise ValueError(f"{what} has to be {dtype} on device {device}, not {t.dtype} on {t.device}")
    return t.data_ptr()


def _lies(t, what, rows, cols=None, pitch=0):
    """Raises if t has not `rows` numbers side by side; with `cols`, rows of so many, `pitch` apart (0: side by side).  A matrix may be of any shape if it is side by side as
    a whole; rows behind the last one are nobody's business."""
    if cols is None:
        ok, wanted = t.is_contiguous() and t.numel() >= rows, f"{rows} numbers side by side"
    else:
        pitch = pitch or cols
        if t.dim() != 2 and t.is_contiguous():
            t = t.view(-1, t.shape[-1]) if t.dim() > 2 else t.view(-1)
        if t.dim() == 1:
            ok = t.numel() >= (rows - 1) * pitch + cols
        else:
            ok = t.dim() == 2 and t.shape[0] >= rows and t.shape[1] >= cols and (cols == 1 or t.stride(1) == 1) and (rows == 1 or t.stride(0) == pitch)
        wanted = f"{rows} rows of {cols} numbers, {pitch} apart"
    if not ok:
        raise ValueError(f"{what} has to be {wanted}, not {tuple(t.shape)} with strides {t.stride()}")


def _space(workspace, device):
    if workspace is None:
        return 0, 0
    if workspace.get_device() != device or not workspace.is_contiguous():
        raise ValueError(f"the workspace has to be in one piece on device {device}, not {tuple(workspace.shape)} with strides {workspace.stride()} on {workspace.device}")
    return _ws(workspace)


def norm_problem(M, K, x_dtype="bf16", s_dtype="bf16", out="bf16", w_dtype="bf16", eps=1e-5, dw_dtype="f32", dw_accumulate=0, ldx=0, lds=0,
                 ldy=0) -> flux_norm_t:
    return flux_norm_t(M, K, _DT[x_dtype], _DT[s_dtype], _DT[w_dtype], _OUT[out], _DT[dw_dtype], dw_accumulate, eps, 0, ldx, lds, ldy)


def flux_norm_workspace_bytes(p: flux_norm_t) -> int:
    return int(lib().flux_norm_workspace_bytes(C.byref(p)))


def _in_blocks(M, K, out):
    """Bytes of M rows of K numbers in blocks, and of their scales."""
    blocks = (K + 31) // 32
    return M * blocks * (16 if out == FLUX_NORM_MX4 else 32), M * ((blocks + 15) // 16 * 16)


def _fit(device, **tensors):
    """Raises for the first (tensor or None, dtype, where its numbers lie: see _lies) that does not fit.  (The calls look at all tensors at once and come here if one is not as
    it usually is: as long as a launch is a microsecond or two, so is a function call a tensor.)"""
    for what, (t, dtype, *place) in tensors.items():
        _buf(t, dtype, device, what)
        if t is not None:
            _lies(t, what, *place)


def flux_norm(p, X, R, W, S, Y, scales=None, rstd=None, stream=None):
    d, x, s, w, y = _device(), _TYPES[p.x_dtype & 1], _TYPES[p.s_dtype & 1], _TYPES[p.w_dtype & 1], _TYPES[p.out & 3]
    M, K = p.M, p.K
    held = n = M * K
    if y is _U8:
        held, scaled = _in_blocks(M, K, p.out)
    side = not (p.ldx or p.lds or p.ldy)                                        # (rows side by side)
    if not (X.dtype is x and W.dtype is w and Y.dtype is y and d == X.get_device() == W.get_device() == Y.get_device() and W.numel() == K and W.is_contiguous()
            and (X.numel() == n and X.is_contiguous() if side else X.shape == (M, K) and X.stride() == (p.ldx or K, 1))
            and (Y.numel() == held and Y.is_contiguous() if side or y is _U8 else Y.shape == (M, K) and Y.stride() == (p.ldy or K, 1))
            and (R is None or (R.dtype is s and R.get_device() == d and (R.numel() == n and R.is_contiguous() if side else R.shape == (M, K) and R.stride() == (p.lds or K, 1))))
            and (S is None or (S.dtype is s and S.get_device() == d and (S.numel() == n and S.is_contiguous() if side else S.shape == (M, K) and S.stride() == (p.lds or K, 1))))
            and (scales is None or (y is _U8 and scales.dtype is _U8 and scales.get_device() == d and scales.numel() == scaled and scales.is_contiguous()))
            and (rstd is None or (rstd.dtype is _F32 and rstd.get_device() == d and rstd.numel() >= M and rstd.is_contiguous()))):
        _fit(d, X=(X, x, M, K, p.ldx), R=(R, s, M, K, p.lds), W=(W, w, K), S=(S, s, M, K, p.lds), Y=(Y, y, held) if y is _U8 else (Y, y, M, K, p.ldy),
             scales=(scales, _U8, scaled if y is _U8 else 0), rstd=(rstd, _F32, M))
    status = lib().flux_norm(p, X.data_ptr(), 0 if R is None else R.data_ptr(), W.data_ptr(), 0 if S is None else S.data_ptr(), Y.data_ptr(),
                             0 if scales is None else scales.data_ptr(), 0 if rstd is None else rstd.data_ptr(), _stream(stream))
    if status:
        _check(status, "flux_norm")


def flux_norm_backward(p, dY, S, W, rstd, dS=None, dR=None, dX=None, dW=None, workspace=None, stream=None):
    d, x, s, w, y, dw = _device(), _TYPES[p.x_dtype & 1], _TYPES[p.s_dtype & 1], _TYPES[p.w_dtype & 1], _TYPES[p.out & 1], _TYPES[p.dw_dtype & 1]
    M, K = p.M, p.K
    n = M * K
    side = not (p.ldx or p.lds or p.ldy)
    if not (dY.dtype is y and S.dtype is s and W.dtype is w and rstd.dtype is _F32 and d == dY.get_device() == S.get_device() == W.get_device() == rstd.get_device()
            and W.numel() == K and W.is_contiguous() and rstd.numel() >= M and rstd.is_contiguous()
            and (dY.numel() == n and dY.is_contiguous() if side else dY.shape == (M, K) and dY.stride() == (p.ldy or K, 1))
            and (S.numel() == n and S.is_contiguous() if side else S.shape == (M, K) and S.stride() == (p.lds or K, 1))
            and (dS is None or (dS.dtype is s and dS.get_device() == d and (dS.numel() == n and dS.is_contiguous() if side else dS.shape == (M, K) and dS.stride() == (p.lds or K, 1))))
            and (dR is None or (dR.dtype is s and dR.get_device() == d and (dR.numel() == n and dR.is_contiguous() if side else dR.shape == (M, K) and dR.stride() == (p.lds or K, 1))))
            and (dX is None or (dX.dtype is x and dX.get_device() == d and (dX.numel() == n and dX.is_contiguous() if side else dX.shape == (M, K) and dX.stride() == (p.ldx or K, 1))))
            and (dW is None or (dW.dtype is dw and dW.get_device() == d and dW.numel() == K and dW.is_contiguous()))):
        _fit(d, dY=(dY, y, M, K, p.ldy), S=(S, s, M, K, p.lds), W=(W, w, K), rstd=(rstd, _F32, M), dS=(dS, s, M, K, p.lds), dR=(dR, s, M, K, p.lds),
             dX=(dX, x, M, K, p.ldx), dW=(dW, dw, K))
    status = lib().flux_norm_backward(p, dY.data_ptr(), S.data_ptr(), W.data_ptr(), rstd.data_ptr(), 0 if dS is None else dS.data_ptr(), 0 if dR is None else dR.data_ptr(),
                                      0 if dX is None else dX.data_ptr(), 0 if dW is None else dW.data_ptr(), *_space(workspace, d), _stream(stream))
    if status:
        _check(status, "flux_norm_backward")


def flux_mx8_row_bytes(K: int) -> int:
    return int(lib().flux_mx8_row_bytes(K))


def flux_mx8_dequantize(q, scales, dst, stream=None):
    rows, K, dtype, ld = _rows(dst)
    _packed(q, scales, rows, K, 32)
    d = _device()
    _check(lib().flux_mx8_dequantize(rows, K, _buf(q, torch.uint8, d, "q"), _buf(scales, torch.uint8, d, "scales"), dtype, _buf(dst, dst.dtype, d, "dst"), ld,
                                     _stream(stream)), "flux_mx8_dequantize")
