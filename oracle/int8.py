"""The linear layer in 8-bit integers, in float64.

Written from the formulas: a row's scale is its largest magnitude over 127, held
in fp32; its integers are the quotients rounded half to even; y = sx sw (q w) + b.
A row of no normal scale counts as zeros, a row with a NaN or an infinity gives
NaN.  Numpy only.
"""
import numpy as np

SMALLEST_NORMAL = np.float64(2.0) ** -126


def quantize_rows(x):
    """(q float64 of whole numbers, scale float64 of an fp32 value) of fp32 rows."""
    x = np.asarray(x, np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        top = np.abs(x).max(axis=1) if x.shape[1] else np.zeros(len(x))
        finite = np.isfinite(x).all(axis=1)
        s = (np.where(finite, top, 0.0) / 127.0).astype(np.float32).astype(np.float64)
        s[s < SMALLEST_NORMAL] = 0.0
        q = np.where((s > 0)[:, None] & finite[:, None],
                     np.rint(np.where(finite[:, None], x, 0.0) / np.where(s > 0, s, 1.0)[:, None]),
                     0.0)
    s[~finite] = np.nan
    return q, s


def linear(x, wq, wscale, bias=None, relu=False):
    """relu(x in 8 bits times the quantised weights wq [outs][in], plus bias)."""
    q, s = quantize_rows(x)
    y = (q @ np.asarray(wq, np.float64).T) * s[:, None] * np.asarray(wscale, np.float64)
    if bias is not None:
        y = y + np.asarray(bias, np.float64)
    return np.where(y < 0, 0.0, y) if relu else y
