"""The linear layer in microscaled 4-bit floating point and its gradients, in float64.

Written from the formulas: 32 entries of a row share the least power of two s (from
2^-127 on, 2^125 at most) with max |x| < 7 s; an entry is the value nearest to x / s of 0, 1/2, 1,
3/2, 2, 3, 4, 6 and their negatives, of two equally near ones that with the even
code.  A block without a normal number counts as zeros, one with a NaN or an
infinity is NaN.  Numpy only.
"""
import numpy as np

from .dropout import factor, kept

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantize_rows(x):
    """(codes 0..15 [rows][cols], scale bytes [rows][blocks]) of fp32 rows."""
    x = np.asarray(x, np.float64)
    n, c = x.shape
    blocks = (c + 31) // 32
    y = np.zeros((n, blocks * 32))
    y[:, :c] = x
    y = y.reshape(n, blocks, 32)
    finite = np.isfinite(y).all(axis=2)
    top = np.abs(np.where(np.isfinite(y), y, 0.0)).max(axis=2)
    e = np.frexp(top)[1] - 4  # 7 2^e is below the largest
    for _ in range(3):
        e = np.where(top >= 7.0 * np.ldexp(1.0, e), e + 1, e)
    e = np.clip(e, -127, 125)
    zero = (top < 2.0 ** -126) | ~finite
    z = np.where(zero[..., None], 0.0, np.where(np.isfinite(y), y, 0.0)) \
        / np.ldexp(1.0, e)[..., None]
    away = np.abs(np.abs(z)[..., None] - VALUES)
    away[..., 1::2] += 1e-9  # of equally near ones the even code (distances: whole 2^-24)
    code = away.argmin(axis=3)
    nearest = np.abs(np.abs(z)[..., None] - VALUES).min(axis=3)
    assert (np.abs(np.abs(z) - VALUES[code]) == nearest).all()
    code = code + 8 * (np.signbit(z) & ~zero[..., None])
    scale = np.where(finite, np.where(zero, 0, e + 127), 255)
    return code.reshape(n, -1)[:, :c], scale


def values(code, scale):
    """What codes and scale bytes stand for."""
    n, c = code.shape
    s = np.where(scale == 255, np.nan, np.ldexp(1.0, scale.astype(np.int64) - 127))
    v = VALUES[code & 7] * np.where(code & 8, -1.0, 1.0)
    return v * np.repeat(s, 32, axis=1)[:, :c]


def rounded(x):
    return values(*quantize_rows(x))


def packed(code, scale):
    """The bytes of codes, zeros to a whole 128, and of scales, to a whole 16."""
    n, c = code.shape
    q = np.zeros((n, (c + 255) // 256 * 256), np.uint8)
    q[:, :c] = code
    s = np.zeros((n, (c + 511) // 512 * 16), np.uint8)
    s[:, :scale.shape[1]] = scale
    return q[:, ::2] | q[:, 1::2] << 4, s


def layer(xv, wv, bias=None, relu=False, dropout=None):
    """The layer of values: drop(relu(x w' + bias))."""
    y = xv @ wv.T
    if bias is not None:
        y = y + np.asarray(bias, np.float64)
    if relu:
        y = np.where(y < 0, 0.0, y)
    if dropout is not None:
        with np.errstate(invalid="ignore"):
            y = np.where(kept(*y.shape, *dropout), y * factor(dropout[0]), 0.0)
    return y


def passed(dy, y=None, dropout=None):
    """dz: the gradient behind the epilogue, held in fp32."""
    dz = np.asarray(dy, np.float64)
    if dropout is not None:
        dz = (dz * factor(dropout[0])).astype(np.float32).astype(np.float64)
        if y is None:
            dz = np.where(kept(*dz.shape, *dropout), dz, 0.0)
    return dz if y is None else np.where(y <= 0, 0.0, dz)


def gradients(dy, x, w, y=None, dropout=None):
    """(dx, dw, db), and the same sums of magnitudes for bounds of their errors."""
    dz = passed(dy, y, dropout)
    zr, zc, xc, wc = (rounded(v) for v in (dz, dz.T, np.asarray(x).T, np.asarray(w).T))
    sums = (zr @ wc.T, zc @ xc.T, dz.sum(axis=0))
    sizes = (np.abs(zr) @ np.abs(wc.T), np.abs(zc) @ np.abs(xc.T), np.abs(dz).sum(axis=0))
    return sums, sizes
