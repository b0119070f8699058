"""Rows in 8-bit integers with a scale each, and their products: the binary32 steps of the definition, the sums exact."""
from __future__ import annotations

import numpy as np

F = np.float32


def quantize(x: np.ndarray):
    """codes [rows, K] int8, scales [rows] binary32 of x [rows, K] binary32."""
    x = np.asarray(x, F)
    bad = ~np.isfinite(x).all(-1)
    amax = np.abs(np.where(bad[:, None], F(0), x)).max(-1).astype(F) if x.shape[1] else np.zeros(x.shape[0], F)
    with np.errstate(all="ignore"):
        scale = (amax / F(127)).astype(F)
        factor = (F(127) * (F(1) / amax).astype(F)).astype(F)
    small = scale < F(2.0 ** -126)
    scale = np.where(small, np.where(amax > 0, F(2.0 ** -126), F(0)), scale).astype(F)
    factor = np.where(small, np.where(amax > 0, F(2.0 ** 126), F(0)), factor).astype(F)
    codes = np.rint(np.where(bad[:, None], F(0), x) * factor[:, None]).astype(np.int8)
    return codes, np.where(bad, F(np.nan), scale).astype(F)


def layout(codes: np.ndarray) -> np.ndarray:
    """The bytes of codes [rows, K] in blocks of 16 rows by 64 codes, 16 bytes of a row at a time, K filled up to 128."""
    rows, K = codes.shape
    full = np.zeros((-(-rows // 16) * 16, -(-K // 128) * 128), np.int8)
    full[:rows, :K] = codes
    r, k = full.shape[0] // 16, full.shape[1] // 64
    return full.reshape(r, 16, k, 4, 16).transpose(0, 2, 3, 1, 4).reshape(-1).view(np.uint8)


def matmul(a, sa, b, sb):
    """fl32(fl32(fl32(sum) sa) sb), [M, N] binary32."""
    exact = a.astype(np.float64) @ b.astype(np.float64).T               # whole numbers below 2^31: exact
    return ((exact.astype(F) * sa[:, None].astype(F)).astype(F) * sb[None, :].astype(F)).astype(F)
