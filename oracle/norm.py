"""Root-mean-square norm and its gradient, in binary64."""
from __future__ import annotations

import numpy as np


def forward(s: np.ndarray, g: np.ndarray, eps: float):
    """y, rstd of rows s."""
    s = s.astype(np.float64)
    rstd = 1.0 / np.sqrt((s * s).mean(-1) + eps)
    return s * rstd[:, None] * g, rstd


def backward(dy: np.ndarray, s: np.ndarray, rstd: np.ndarray, g: np.ndarray):
    """ds, dw."""
    n = s.astype(np.float64) * rstd.astype(np.float64)[:, None]
    a = dy.astype(np.float64) * g
    ds = rstd.astype(np.float64)[:, None] * (a - n * (a * n).mean(-1, keepdims=True))
    return ds, (dy.astype(np.float64) * n).sum(0)


def quantized_rows(s: np.ndarray, rstd: np.ndarray, g: np.ndarray) -> np.ndarray:
    """y in the binary32 steps of the library, from its rstd: what the codes are formed from."""
    F = np.float32
    return ((s.astype(F) * rstd.astype(F)[:, None]).astype(F) * g.astype(F)).astype(F)
