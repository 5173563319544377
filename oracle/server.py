"""The server's step with orthogonalised updates, in float64.

Written from the formulas: Newton-Schulz steps X <- a X + (b A + c A A) X with
A = X X' from X = G / |G|_F, and the step avg, d = g - avg, m = beta m + d,
u = d + beta m or m, W <- (1 - lr wd) W - lr sqrt(max(1, o / i)) orth(u).
The functions use operators only, so numpy arrays and torch tensors (of
float64) both go through them.
"""
import math

COEFFS = ((3.4445, -4.7750, 2.0315),) * 5


def newton_schulz(g, coeffs=COEFFS, disturb=None):
    """orth(g).  ``disturb(kind, step, value, noise)``, where given, returns what
    is kept of each stored value: kind "x", "gram" or "poly", ``noise`` a
    matrix the size of the sums' own roundings (a model of the arithmetic of
    fewer bits, for the tests' tolerances)."""
    keep = disturb or (lambda kind, step, v, noise: v)
    if g.shape[0] > g.shape[1]:
        return newton_schulz(g.T, coeffs, disturb).T
    norm = (g * g).sum() ** 0.5
    if float(norm) == 0.0:
        return g * 0.0
    x = g / norm

    def lengths(v, axis):
        return (v * v).sum(axis) ** 0.5

    x = keep("x", 0, x, None)
    for t, (a, b, c) in enumerate(coeffs):
        n = lengths(x, 1)
        s = keep("gram", t, x @ x.T, n[:, None] * n[None, :])
        n = lengths(s, 1)
        p = b * s + c * (s @ s)
        for i in range(p.shape[0]):
            p[i, i] += a
        p = keep("poly", t, p, abs(c) * n[:, None] * n[None, :])
        x = keep("x", t + 1, p @ x, lengths(p, 1)[:, None] * lengths(x, 0)[None, :])
    return x


def server_step(layers, replicas, weights, momentum, lr, beta, nesterov, weight_decay, plain_lr,
                plain_layers=(), coeffs=COEFFS):
    """New (layers, momentum): lists of (W, b) per layer, W as a matrix
    [out][rest]; ``replicas``: such a list per worker."""
    new, new_m = [], []
    for l, ((w, b), (mw, mb)) in enumerate(zip(layers, momentum), start=1):
        row, row_m = [], []
        for kind, x, m, own in (("w", w, mw, 0), ("b", b, mb, 1)):
            avg = sum(float(k) * r[l - 1][own] for k, r in zip(weights, replicas))
            d = x - avg
            m = beta * m + d
            u = d + beta * m if nesterov else m
            if kind == "w" and l not in plain_layers:
                s = math.sqrt(max(1.0, w.shape[0] / w.shape[1]))
                x = (1.0 - lr * weight_decay) * x - lr * s * newton_schulz(u, coeffs)
            else:
                x = x - plain_lr * u
            row.append(x)
            row_m.append(m)
        new.append(tuple(row))
        new_m.append(tuple(row_m))
    return new, new_m
