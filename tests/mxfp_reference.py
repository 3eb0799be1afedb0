"""A plain model of pools in four bits, in 64-bit floats on the CPU."""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(x):
    """x [..., 128] float64 holding float32 or bf16 values -> bytes [..., 64], scales [..., 4], as numpy uint8."""
    x = np.asarray(x, np.float64).reshape(*x.shape[:-1], 4, 32)
    top = np.abs(x).max(-1)
    fine = np.isfinite(top)
    m, k = np.frexp(np.where(fine, top, 0.0))                 # top = m 2^k with m in [0.5, 1): the least e with top <= 0.75 * 2^(e + 3)
    e = np.where((top > 0) & fine, np.maximum(np.where(m <= 0.75, k - 3, k - 2), -127), -127)
    y = np.minimum(np.abs(np.where(fine[..., None], x, 0.0)), 3 * 2.0 ** 126) / 2.0 ** e[..., None].astype(np.float64)
    off = np.abs(y[..., None] - GRID)
    # the nearest, of two as near the one of even code
    code = np.argmin(off + np.where(np.arange(8) % 2, 1e-12, 0.0), -1)
    code = np.where(fine[..., None], code + 8 * np.signbit(x), 0).astype(np.uint8).reshape(*x.shape[:-2], 64, 2)
    return code[..., 0] | code[..., 1] << 4, np.where(fine, e + 127, 255).astype(np.uint8)


def values(rows, scales):
    """bytes [..., 64], scales [..., 4] -> [..., 128] float64; NaN where a scale is 255."""
    code = np.stack([rows & 15, rows >> 4], -1).reshape(*rows.shape[:-1], 4, 32)
    x = GRID[code & 7] * np.where(code & 8, -1.0, 1.0) * 2.0 ** (scales[..., None].astype(np.float64) - 127)
    return np.where(scales[..., None] == 255, np.nan, x).reshape(*rows.shape[:-1], 128)
