"""Oracle of the root-mean-square norm, of 8-bit microscaled blocks and of the cross entropy of a vocabulary projection: numpy, 64 bits, from
the formulas.  Test infrastructure only; shares no code with the library."""
from __future__ import annotations

import numpy as np


def norm(s, w, eps):
    """(Y, 1 / rms)"""
    r = 1.0 / np.sqrt((s * s).mean(axis=1) + eps)
    return s * r[:, None] * w, r


def norm_backward(dy, s, w, r, ds):
    """(dR, dW), r as the forward pass kept it."""
    h, g = s * r[:, None], dy * w
    return r[:, None] * (g - h * (g * h).mean(axis=1, keepdims=True)) + ds, (dy * h).sum(axis=0)


def _e4m3():
    """The non-negative numbers of E4M3 by code, 0 .. 126: four bits of exponent, three of mantissa, no infinity, code 127 NaN."""
    codes = np.arange(127)
    e, m = codes >> 3, codes & 7
    return np.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * 2.0 ** (e - 7.0))


E4M3 = _e4m3()
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
LEVELS = {4: E2M1, 8: E4M3}
TOP_EXPONENT = {4: 2, 8: 8}


def block_byte(top, bits):
    """The scale's byte of a block whose largest magnitude is `top`."""
    if not np.isfinite(top):
        return 255
    if top == 0:
        return 0
    return max(int(np.frexp(top)[1]) - 1 - TOP_EXPONENT[bits], -127) + 127


def blocks(x, bits):
    """(codes with the sign on top [rows, blocks, 32], bytes [rows, blocks])"""
    rows, K = x.shape
    v = np.zeros((rows, -(-K // 32) * 32))
    v[:, :K] = x
    v = v.reshape(rows, -1, 32)
    levels = LEVELS[bits]
    codes, scales = np.zeros(v.shape, np.uint8), np.zeros(v.shape[:2], np.uint8)
    for i in np.ndindex(scales.shape):
        a = np.abs(v[i])
        scales[i] = block_byte(a.max() if np.isfinite(a).all() else np.inf, bits)
        if scales[i] == 255:
            continue
        a = np.minimum(a / 2.0 ** (int(scales[i]) - 127), levels[-1])
        up = np.clip(np.searchsorted(levels, a), 1, len(levels) - 1)
        lo, hi = a - levels[up - 1], levels[up] - a
        pick = np.where((hi < lo) | ((hi == lo) & (up % 2 == 0)), up, up - 1)           # (at the same distance the even code)
        codes[i] = pick + (np.signbit(v[i]) << (bits - 1))
    return codes, scales


def block_values(codes, scales, bits):
    levels = np.concatenate([LEVELS[bits], [np.nan] * (2 ** (bits - 1) - len(LEVELS[bits]))])
    v = levels[codes & (2 ** (bits - 1) - 1)] * np.where(codes >> (bits - 1), -1.0, 1.0)
    return (v * np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))[..., None]).reshape(codes.shape[0], -1)


def packed(codes, scales, bits):
    """(q, scales) as the library lays them out."""
    rows, kb, _ = codes.shape
    q = codes if bits == 8 else codes[..., 0::2] | (codes[..., 1::2] << 4)
    s = np.zeros((rows, -(-kb // 16) * 16), np.uint8)
    s[:, :kb] = scales
    return q.reshape(rows, -1).astype(np.uint8), s


def loss(x, w, target, v0, vocab):
    """(lse, logit, loss, Z): targets of the whole vocabulary, w its columns from v0 on."""
    z = x @ w.T
    top = z.max(axis=1, keepdims=True)
    lse = (top + np.log(np.exp(z - top).sum(axis=1, keepdims=True)))[:, 0]
    here = (target >= v0) & (target < v0 + w.shape[0]) & (target < vocab)
    logit = np.where(here, z[np.arange(len(z)), np.where(here, target - v0, 0)], 0.0)
    return lse, logit, np.where((target >= 0) & (target < vocab), lse - logit, 0.0), z


def loss_backward(x, w, target, v0, vocab, lse, dloss):
    """(dX, dW, dZ)"""
    z = x @ w.T
    at = (target - v0)[:, None] == np.arange(w.shape[0])
    counts = (target >= 0) & (target < vocab)
    dz = np.where(counts, dloss, 0.0)[:, None] * (np.exp(z - lse[:, None]) - (at & counts[:, None]))
    return dz @ w, dz.T @ x, dz
