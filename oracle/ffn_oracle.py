"""Oracle of the gated feed-forward block and of 4-bit microscaled matrices: numpy, 64 bits, from the formulas.
Test infrastructure only; shares no code with the library."""
from __future__ import annotations

import numpy as np
from scipy.special import ndtr

GELU_C = np.sqrt(2.0 / np.pi)
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def act(name: str, g: np.ndarray) -> np.ndarray:
    if name == "silu":
        return g / (1.0 + np.exp(-g))
    if name == "gelu":
        return g * ndtr(g)
    return 0.5 * g * (1.0 + np.tanh(GELU_C * (g + 0.044715 * g ** 3)))


def slope(name: str, g: np.ndarray) -> np.ndarray:
    if name == "silu":
        p = 1.0 / (1.0 + np.exp(-g))
        return p * (1.0 + g * (1.0 - p))
    if name == "gelu":
        return ndtr(g) + g * np.exp(-0.5 * g * g) / np.sqrt(2.0 * np.pi)
    t = np.tanh(GELU_C * (g + 0.044715 * g ** 3))
    return 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * GELU_C * (1.0 + 3 * 0.044715 * g * g)


def glu(name, x, wg, wu):
    """(H, G, U) with weights as [K,N]."""
    g, u = x @ wg, x @ wu
    return act(name, g) * u, g, u


def glu_backward(name, x, wg, wu, g, u, dh):
    """(dX, dWg, dWu, dG, dU) with weights as [K,N]."""
    dg, du = dh * u * slope(name, g), dh * act(name, g)
    return dg @ wg.T + du @ wu.T, x.T @ dg, x.T @ du, dg, du


def mx4_quantize(x: np.ndarray):
    """(codes [rows, blocks, 32], scale bytes [rows, blocks]) of a finite or not finite matrix."""
    rows, K = x.shape
    kb = -(-K // 32)
    v = np.zeros((rows, kb * 32))
    v[:, :K] = x
    v = v.reshape(rows, kb, 32)
    codes, scales = np.zeros(v.shape, np.uint8), np.zeros((rows, kb), np.uint8)
    for r in range(rows):
        for b in range(kb):
            blk = v[r, b]
            if not np.isfinite(blk).all():
                scales[r, b] = 255
                continue
            top = np.abs(blk).max()
            if top == 0:
                codes[r, b] = np.where(np.signbit(blk), 8, 0)
                continue
            e = max(int(np.floor(np.log2(top))) - 2, -127)
            if 2.0 ** (int(np.floor(np.log2(top))) + 1) <= top:        # (log2 rounded below a power of two)
                e += 1
            scales[r, b] = e + 127
            dist = np.abs(np.abs(blk)[:, None] / 2.0 ** e - E2M1[None, :])
            near = dist == dist.min(axis=1, keepdims=True)
            even = near & (np.arange(8) % 2 == 0)                       # of two at the same distance, the even code
            pick = np.where(even.any(axis=1), even.argmax(axis=1), near.argmax(axis=1))
            codes[r, b] = pick + np.where(np.signbit(blk), 8, 0)
    return codes, scales


def mx4_values(codes, scales):
    """[rows, 32 * blocks]"""
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    v = E2M1[codes & 7] * np.where(codes & 8, -1.0, 1.0) * s[..., None]
    return v.reshape(codes.shape[0], -1)


def mx4_pack(codes, scales):
    """(q, scales) as the library lays them out."""
    rows, kb, _ = codes.shape
    q = (codes[..., 0::2] | (codes[..., 1::2] << 4)).reshape(rows, kb * 16).astype(np.uint8)
    s = np.zeros((rows, -(-kb // 16) * 16), np.uint8)
    s[:, :kb] = scales
    return q, s


def mx4_unpack(q, scales):
    """(codes, scales without the padding)"""
    rows, kb = q.shape[0], q.shape[1] // 16
    codes = np.stack([q & 15, q >> 4], axis=-1).reshape(rows, kb, 32)
    return codes, scales[:, :kb]
