"""The oracle's 8-bit rows and layer."""
import numpy as np

from oracle import int8


def test_rows_by_hand():
    x = np.array([[127.0, 0.5, 1.5, -2.5, -63.5], [0, 0, 0, 0, 0], [1, np.nan, 0, 0, 0],
                  [np.inf, 1, 0, 0, 0], [1e-40, 0, 0, 0, 0], [-254.0, 1, 3, 5, 2]])
    q, s = int8.quantize_rows(x)
    assert s[0] == 1 and s[1] == 0 and np.isnan(s[2]) and np.isnan(s[3]) and s[4] == 0 and s[5] == 2
    assert np.array_equal(q[0], [127, 0, 2, -2, -64])
    assert not q[1:5].any()
    assert np.array_equal(q[5], [-127, 0, 2, 2, 1])


def test_entries_are_within_half_a_step():
    x = np.random.default_rng(0).standard_normal((50, 77)).astype(np.float32)
    q, s = int8.quantize_rows(x)
    assert np.abs(q).max() == 127
    assert (np.abs(q * s[:, None] - x) <= s[:, None] / 2 * (1 + 1e-12)).all()


def test_linear_is_the_product_of_what_the_integers_stand_for():
    rng = np.random.default_rng(1)
    x, w = rng.standard_normal((5, 40)).astype(np.float32), rng.standard_normal((7, 40))
    wq, ws = int8.quantize_rows(w.astype(np.float32))
    b = rng.standard_normal(7)
    q, s = int8.quantize_rows(x)
    want = (q * s[:, None]) @ (wq * ws[:, None]).T + b
    assert np.allclose(int8.linear(x, wq, ws, b), want)
    assert np.allclose(int8.linear(x, wq, ws, b, relu=True), np.maximum(want, 0))
