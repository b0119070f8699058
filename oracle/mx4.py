"""Microscaled 4-bit floating point from its definition: the block's power of two, the nearest E2M1 value by comparison, the layout of the products."""
from __future__ import annotations

import numpy as np

BLOCK = 32
LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def _blocks(x: np.ndarray) -> np.ndarray:
    return np.pad(x, ((0, 0), (0, -x.shape[1] % BLOCK))).reshape(x.shape[0], -1, BLOCK)


def quantize(x: np.ndarray, ceil: bool = False):
    """codes [rows, K] (sign in bit 3), scale bytes [rows, (K + 31) / 32] of x [rows, K] binary32."""
    v = _blocks(np.asarray(x, np.float64))
    bad = ~np.isfinite(v).all(-1)
    v = np.where(bad[..., None], 0.0, v)
    amax = np.abs(v).max(-1)
    m, e = np.frexp(amax)                                    # amax = m 2^e with m from .5 to 1: 2^(e-1) <= amax < 2^e
    log_scale = e - 1 - 2 + ((m > 0.75) if ceil else 0)
    log_scale = np.where(amax > 0, np.clip(log_scale, -127, 125), -127)
    a = np.abs(v) / np.ldexp(1.0, log_scale)[..., None]
    mid = (LEVELS[1:] + LEVELS[:-1]) / 2
    code = sum(((a > t) if i % 2 == 0 else (a >= t)).astype(np.uint8) for i, t in enumerate(mid))
    code = (code | (np.signbit(np.where(bad[..., None], 0.0, _blocks(np.asarray(x, np.float64)))) * 8)).astype(np.uint8)
    return code.reshape(x.shape[0], -1)[:, :x.shape[1]], np.where(bad, 255, log_scale + 127).astype(np.uint8)


def values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """What the codes stand for, binary64."""
    v = np.where(codes & 8, -1.0, 1.0) * LEVELS[codes & 7]
    scale = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(int) - 127))
    return (_blocks(v) * scale[..., None]).reshape(codes.shape[0], -1)[:, :codes.shape[1]]


def nibbles(codes: np.ndarray) -> np.ndarray:
    """Two codes to a byte, the even column's in the low half."""
    return (codes[:, ::2] | codes[:, 1::2] << 4).astype(np.uint8)


def layout(codes: np.ndarray, scales: np.ndarray):
    """The bytes of the codes and of the scales in the layout of the products: blocks of 16 rows by 128 codes, rows filled up to 16 and K to 256."""
    rows, K = codes.shape
    full = np.zeros((-(-rows // 16) * 16, -(-K // 256) * 256), np.uint8)
    full[:rows, :K] = codes
    r, k = full.shape[0] // 16, full.shape[1] // 128
    code_bytes = nibbles(full).reshape(r, 16, k, 4, 16).transpose(0, 2, 3, 1, 4).reshape(-1)
    s = np.zeros((full.shape[0], full.shape[1] // BLOCK), np.uint8)
    s[:rows, :scales.shape[1]] = scales
    return code_bytes, s.reshape(r, 16, k // 2, 2, 4).transpose(0, 2, 4, 1, 3).reshape(-1)


def linear_bwd(dy: np.ndarray, x: np.ndarray, Wt, ceil: bool = False):
    """dx, dW in binary64 of dy [M, N], x [M, K] and the quantized transpose Wt = (codes [K, N], scales)."""
    dx = values(*quantize(dy, ceil)) @ values(*Wt).T
    dW = values(*quantize(dy.T, ceil)) @ values(*quantize(x.T, ceil)).T
    return dx, dW
