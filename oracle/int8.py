"""Rows in 8-bit integers with a scale each, and their product: every step is exact or one fp32 rounding, so results are equal bit for bit."""
import numpy as np


def quantize_rows(x):
    """x [rows, k] (values of fp32): int8 codes and fp32 scales."""
    x = np.asarray(x, np.float32)
    amax = np.abs(x).max(1)
    fine = np.isfinite(amax)
    scale = np.where(fine, np.where(fine, amax, 0) / np.float32(127), np.nan).astype(np.float32)
    ok = fine & (scale > 0)
    ratio = np.zeros(x.shape)
    ratio[ok] = x[ok].astype(np.float64) / scale[ok].astype(np.float64)[:, None]   # (64 bits hold enough of the quotient to see ties)
    return np.clip(np.rint(ratio), -127, 127).astype(np.int8), scale


def product(xq, sx, wq, sw):
    """fp32 [m, n]: (float(sum) * sx) * sw"""
    s = xq.astype(np.float64) @ wq.astype(np.float64).T   # (integers below 2^53: exact)
    with np.errstate(invalid="ignore", over="ignore"):
        return (s.astype(np.float32) * sx[:, None]).astype(np.float32) * sw[None, :]


def operand_image(q):
    n, k = q.shape
    return np.ascontiguousarray(q.reshape(n // 32, 32, k // 128, 2, 4, 16).transpose(2, 0, 4, 3, 1, 5)).reshape(-1)
