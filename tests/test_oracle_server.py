"""The oracle's Newton-Schulz steps and server's step, against their algebra."""
import numpy as np
import pytest

from oracle import server


def _scalar(s, coeffs=server.COEFFS):
    for a, b, c in coeffs:
        s = a * s + b * s ** 3 + c * s ** 5
    return s


@pytest.mark.parametrize("r,c", [(1, 1), (3, 3), (5, 12), (12, 5), (1, 7)])
def test_newton_schulz_is_the_polynomial_of_the_singular_values(r, c):
    g = np.random.default_rng(r * 31 + c).standard_normal((r, c))
    u, s, vt = np.linalg.svd(g, full_matrices=False)
    want = (u * _scalar(s / np.sqrt((s * s).sum()))) @ vt
    got = server.newton_schulz(g)
    # ten products of at most 12 terms, each step's errors grown at most 4 times
    assert np.abs(got - want).max() < 2.0 ** -52 * 4 ** 5 * 12 * 10


def test_newton_schulz_of_zeros_is_zero():
    assert not server.newton_schulz(np.zeros((3, 4))).any()


def test_server_step_of_plain_layers_is_the_average():
    rng = np.random.default_rng(0)
    layers = [(rng.standard_normal((3, 4)), rng.standard_normal(3))]
    reps = [[(w + 1.0 + k, b - k) for w, b in layers] for k in range(4)]
    zero = [(0 * w, 0 * b) for w, b in layers]
    new, m = server.server_step(layers, reps, [0.25] * 4, zero, 0.1, 0.0, False, 0.0, 1.0,
                                plain_layers=(1,))
    assert np.allclose(new[0][0], layers[0][0] + 2.5) and np.allclose(new[0][1], layers[0][1] - 1.5)
    assert np.allclose(m[0][0], -2.5)


def test_server_step_scales_tall_matrices_and_decays():
    rng = np.random.default_rng(1)
    layers = [(rng.standard_normal((8, 2)), rng.standard_normal(8))]
    reps = [[(w + rng.standard_normal(w.shape), b) for w, b in layers]]
    zero = [(0 * w, 0 * b) for w, b in layers]
    new, m = server.server_step(layers, reps, [1.0], zero, 0.1, 0.9, True, 0.5, 1.0)
    d = layers[0][0] - reps[0][0][0]
    want = 0.95 * layers[0][0] - 0.2 * server.newton_schulz(1.9 * d)
    assert np.allclose(new[0][0], want) and np.allclose(m[0][0], d)
