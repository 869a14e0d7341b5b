"""ctypes binding of include/flux_loss.h (in libflux_ffn_mi355.so): the softmax cross entropy of a vocabulary projection, its join over ranks and its
backward pass.  Argument marshalling only, as in `ffn`; a tensor of another type than the problem's, of another device than the current
one, or whose numbers do not lie where the problem says, raises ValueError.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import ffn
from .binding import _ptr, _ptr_list
from .ffn import _check, _stream
from .norm import _DT, _F32, _TYPES, _device, _fit, _space

FLUX_LOSS_FORWARD, FLUX_LOSS_BACKWARD = 0, 1
FLUX_TARGET_I32, FLUX_TARGET_I64 = 0, 1

EXPORTS = ["flux_loss", "flux_loss_join", "flux_loss_backward", "flux_loss_workspace_bytes"]


class flux_loss_t(C.Structure):
    _fields_ = [
        ("M", C.c_int32), ("V", C.c_int32), ("K", C.c_int32), ("target_dtype", C.c_int32), ("v0", C.c_int64), ("vocab", C.c_int64),
        ("dloss_one", C.c_int32), ("dx_dtype", C.c_int32), ("dw_dtype", C.c_int32), ("dw_accumulate", C.c_int32),
        ("ldx", C.c_int64), ("ldw", C.c_int64), ("piece", C.c_int32), ("tile_config", C.c_int32), ("split_k", C.c_int32), ("reserved", C.c_int32),
    ]


_lib = None


def lib():
    """The shared library, with this header's functions declared."""
    global _lib
    if _lib is None:
        L = ffn.lib()
        vp, sz, pl, lists = C.c_void_p, C.c_size_t, C.POINTER(flux_loss_t), C.POINTER(C.c_void_p)
        L.flux_loss.argtypes = [pl, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.flux_loss_join.argtypes = [pl, C.c_int32, lists, lists, vp, vp, vp, vp, vp]
        L.flux_loss_backward.argtypes = [pl, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.flux_loss_workspace_bytes.argtypes = [C.c_int, pl]
        for name in EXPORTS:
            getattr(L, name).restype = sz if name.endswith("_bytes") else C.c_int
        _lib = L
    return _lib


_TARGET = {"i32": FLUX_TARGET_I32, "i64": FLUX_TARGET_I64, torch.int32: FLUX_TARGET_I32, torch.int64: FLUX_TARGET_I64}
_TARGETS = (torch.int32, torch.int64)
_BF16 = torch.bfloat16


def loss_problem(M, V, K, v0=0, vocab=0, target_dtype="i64", dloss_one=0, dx_dtype="bf16", dw_dtype="bf16", dw_accumulate=0, ldx=0, ldw=0,
                 piece=0, tile_config=0, split_k=0) -> flux_loss_t:
    return flux_loss_t(M, V, K, _TARGET[target_dtype], v0, vocab, dloss_one, _DT[dx_dtype], _DT[dw_dtype], dw_accumulate, ldx, ldw, piece,
                       tile_config, split_k, 0)


def flux_loss_workspace_bytes(op: int, p: flux_loss_t) -> int:
    return int(lib().flux_loss_workspace_bytes(op, C.byref(p)))


def flux_loss(p, X, W, target, lse, logit, loss=None, workspace=None, stream=None):
    d, t, M, K = _device(), _TARGETS[p.target_dtype & 1], p.M, p.K
    if not (X.dtype is _BF16 and W.dtype is _BF16 and target.dtype is t and lse.dtype is _F32 and logit.dtype is _F32
            and d == X.get_device() == W.get_device() == target.get_device() == lse.get_device() == logit.get_device()
            and (X.numel() == M * K and W.numel() == p.V * K and X.is_contiguous() and W.is_contiguous() if not (p.ldx or p.ldw) else
                 X.shape == (M, K) and W.shape == (p.V, K) and X.stride() == (p.ldx or K, 1) and W.stride() == (p.ldw or K, 1))
            and target.numel() >= M and lse.numel() >= M and logit.numel() >= M and target.is_contiguous() and lse.is_contiguous() and logit.is_contiguous()
            and (loss is None or (loss.dtype is _F32 and loss.get_device() == d and loss.numel() >= M and loss.is_contiguous()))):
        _fit(d, X=(X, _BF16, M, K, p.ldx), W=(W, _BF16, p.V, K, p.ldw), target=(target, t, M), lse=(lse, _F32, M), logit=(logit, _F32, M), loss=(loss, _F32, M))
    status = lib().flux_loss(p, X.data_ptr(), W.data_ptr(), target.data_ptr(), lse.data_ptr(), logit.data_ptr(), 0 if loss is None else loss.data_ptr(),
                             *_space(workspace, d), _stream(stream))
    if status:
        _check(status, "flux_loss")


def flux_loss_join(p, lses, logits, target, lse=None, logit=None, loss=None, stream=None):
    d, M = _device(), p.M
    if len(lses) != len(logits):
        raise ValueError("as many lses as logits")
    for r, (a, b) in enumerate(zip(lses, logits)):
        _fit(d, **{f"lses[{r}]": (a, _F32, M), f"logits[{r}]": (b, _F32, M)})
    _fit(d, target=(target, _TARGETS[p.target_dtype & 1], M), lse=(lse, _F32, M), logit=(logit, _F32, M), loss=(loss, _F32, M))
    _check(lib().flux_loss_join(p, len(lses), _ptr_list(lses), _ptr_list(logits), *map(_ptr, (target, lse, logit, loss)), _stream(stream)), "flux_loss_join")


def flux_loss_backward(p, X, W, target, lse, dloss, dX, dW, workspace, stream=None):
    d, t, x, w, M, K = _device(), _TARGETS[p.target_dtype & 1], _TYPES[p.dx_dtype & 1], _TYPES[p.dw_dtype & 1], p.M, p.K
    n, m, rows, side = M * K, p.V * K, 1 if p.dloss_one else M, not (p.ldx or p.ldw)
    if not (X.dtype is _BF16 and W.dtype is _BF16 and target.dtype is t and lse.dtype is _F32 and dloss.dtype is _F32
            and d == X.get_device() == W.get_device() == target.get_device() == lse.get_device() == dloss.get_device()
            and (X.numel() == n and W.numel() == m and X.is_contiguous() and W.is_contiguous() if side else
                 X.shape == (M, K) and W.shape == (p.V, K) and X.stride() == (p.ldx or K, 1) and W.stride() == (p.ldw or K, 1))
            and target.numel() >= M and lse.numel() >= M and dloss.numel() >= rows and target.is_contiguous() and lse.is_contiguous() and dloss.is_contiguous()
            and (dX is None or (dX.dtype is x and dX.get_device() == d and (dX.numel() == n and dX.is_contiguous() if side else dX.shape == (M, K) and dX.stride() == (p.ldx or K, 1))))
            and (dW is None or (dW.dtype is w and dW.get_device() == d and (dW.numel() == m and dW.is_contiguous() if side else dW.shape == (p.V, K) and dW.stride() == (p.ldw or K, 1))))):
        _fit(d, X=(X, _BF16, M, K, p.ldx), W=(W, _BF16, p.V, K, p.ldw), target=(target, t, M), lse=(lse, _F32, M), dloss=(dloss, _F32, rows),
             dX=(dX, x, M, K, p.ldx), dW=(dW, w, p.V, K, p.ldw))
    status = lib().flux_loss_backward(p, X.data_ptr(), W.data_ptr(), target.data_ptr(), lse.data_ptr(), dloss.data_ptr(), 0 if dX is None else dX.data_ptr(),
                                      0 if dW is None else dW.data_ptr(), *_space(workspace, d), _stream(stream))
    if status:
        _check(status, "flux_loss_backward")
