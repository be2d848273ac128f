"""CPU oracle for products in 8-bit integers: quantisation of rows and columns, and the product.

TEST INFRASTRUCTURE ONLY: imported by tests, never by the product path; shares no code with the HIP kernels.

Quantisation is a rule in fp32 (a = max |v|, scale = a / 127, code = rint(v * (127 / a)), each operation rounded), so codes and scales
are exact and have to be met to the bit; everything behind them is in 64 bits.
"""
from __future__ import annotations

import numpy as np

F32 = np.float32


def quantise(v: np.ndarray):
    """Rows of v (fp32) -> (codes int64, scales fp32).  A row with an infinity or a NaN: scale NaN, codes 0."""
    v = np.asarray(v, dtype=F32)
    codes = np.zeros(v.shape, dtype=np.int64)
    scales = np.zeros(v.shape[0], dtype=F32)
    for r, row in enumerate(v):
        if not np.isfinite(row).all():
            scales[r] = np.nan
            continue
        a = np.abs(row).max()
        if a == 0:
            continue
        scales[r] = a / F32(127)
        up = F32(2.0 ** 100) if a < F32(2.0 ** -100) else F32(1)   # 127 / a would overflow
        codes[r] = np.rint(row * up * (F32(127) / (a * up))).astype(np.int64)
    return codes, scales


def product(x_codes, x_scales, w_codes, w_scales) -> np.ndarray:
    """[M, N] in fp64: rows of x_codes [M, K] times rows of w_codes [N, K], with their scales.  (Sums are whole numbers below 2^53: exact.)"""
    total = np.asarray(x_codes, dtype=np.float64) @ np.asarray(w_codes, dtype=np.float64).T
    return total * np.asarray(x_scales, dtype=np.float64)[:, None] * np.asarray(w_scales, dtype=np.float64)[None, :]
