"""Dropout from a counter-based generator, in float64.

Written from Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1,
2, 3" (2011): Philox4x32 with 10 rounds.  Numpy and whole numbers only.
"""
import numpy as np

M = (0xD2511F53, 0xCD9E8D57)
W = (0x9E3779B9, 0xBB67AE85)
LOW = 0xFFFFFFFF


def philox(counter, key):
    """Four words of four counter words (whole numbers or arrays) and two key words."""
    c = [np.asarray(v, np.uint64) for v in counter]
    for r in range(10):
        k = [np.uint64((key[i] + r * W[i]) & LOW) for i in range(2)]
        p, q = np.uint64(M[0]) * c[0], np.uint64(M[1]) * c[2]
        low, s = np.uint64(LOW), np.uint64(32)
        c = [(q >> s) ^ c[1] ^ k[0], q & low, (p >> s) ^ c[3] ^ k[1], p & low]
    return c


def threshold(p):
    return int(np.rint(65536.0 * p))


def kept(rows, cols, p, seed, offset=0):
    """Which entries dropout keeps."""
    g, r = np.meshgrid(np.arange((cols + 7) // 8), np.arange(rows))
    offset &= (1 << 64) - 1
    w = philox((g, r, np.full_like(g, offset & LOW), np.full_like(g, offset >> 32)),
               (seed & LOW, seed >> 32))
    bits = np.empty(g.shape + (8,), np.uint64)
    for i in range(4):
        bits[..., 2 * i] = w[i] & np.uint64(0xFFFF)
        bits[..., 2 * i + 1] = w[i] >> np.uint64(16)
    return bits.reshape(rows, -1)[:, :cols] >= np.uint64(threshold(p))


def factor(p):
    """Of what is kept, held in fp32."""
    t = threshold(p)
    return np.float64(np.float32(65536.0 / (65536 - t))) if t < 65536 else 0.0


def dropout(x, p, seed, offset=0):
    x = np.asarray(x, np.float64)
    with np.errstate(invalid="ignore"):
        return np.where(kept(*x.shape, p, seed, offset), x * factor(p), 0.0)
