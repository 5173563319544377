"""The oracle of the 4-bit layer and of dropout: published vectors, borders by hand,
gradients against differences."""
import numpy as np
import pytest

from oracle import dropout, mx4


@pytest.mark.parametrize("counter,key,want", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))])
def test_philox_known_answers(counter, key, want):
    assert tuple(int(v) for v in dropout.philox(counter, key)) == want


def test_dropout_rate_and_mean():
    for p in (0.0, 0.1, 0.5, 0.9, 1.0):
        k = dropout.kept(400, 333, p, 7, 1 << 40)
        n = k.size
        assert abs(k.mean() - (1 - p)) <= 5 * np.sqrt(p * (1 - p) / n) + 2.0 ** -17
        x = np.ones((400, 333))
        assert abs(dropout.dropout(x, p, 7, 1 << 40).mean() - (p < 1)) <= (
            5 * np.sqrt(p / max(1 - p, 1e-9) / n) + 1e-6 if p < 1 else 0)
    assert not np.array_equal(dropout.kept(9, 9, 0.5, 1), dropout.kept(9, 9, 0.5, 1, 1))
    assert not np.array_equal(dropout.kept(9, 9, 0.5, 1), dropout.kept(9, 9, 0.5, 1 << 32))


def test_quantize_by_hand():
    x = np.zeros((1, 64), np.float32)
    x[0, :12] = [4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 6.9, -5, -0.1]
    x[0, 32:36] = [7, 1, -7, 3.5]  # from 7 on twice the scale
    code, s = mx4.quantize_rows(x)
    assert s.tolist() == [[127, 128]]
    assert code[0, :12].tolist() == [6, 0, 2, 2, 4, 4, 6, 6, 7, 7, 14, 8]
    assert code[0, 32:36].tolist() == [6, 1, 14, 4]
    assert mx4.values(code, s)[0, 32:36].tolist() == [8, 1, -8, 4]
    q, b = mx4.packed(code, s)
    assert q.shape == (1, 128) and b.shape == (1, 16)
    assert q[0, 0] == 6 and q[0, 1] == 0x22 and not q[0, 32:].any()


@pytest.mark.parametrize("x,scale", [(0.0, 0), (2.0 ** -127, 0), (2.0 ** -126, 0), (2.0 ** -125, 0),
                                     (7 * 2.0 ** -127, 1), (3.4e38, 252), (2.9e38, 252), (2.0 ** 126, 251), (np.inf, 255),
                                     (np.nan, 255)])
def test_scales_at_the_ends(x, scale):
    code, s = mx4.quantize_rows(np.array([[x, -x]], np.float32))
    assert s.tolist() == [[scale]]
    v = mx4.values(code, s)
    if scale == 255:
        assert np.isnan(v).all()
    elif abs(x) < 2.0 ** -126:
        assert not v.any() and not (code & 7).any()
    else:
        assert abs(v[0, 0] / float(np.float32(x)) - 1) <= (0.25 if x > 2.6e38 else 1 / 7)


def test_gradients_against_differences():
    """Entries that 4 bits hold, along rows and along columns: then the layer is its
    unrounded self, whose loss sum(c y) is piecewise linear, so that central
    differences of float64 are its gradients."""
    rng = np.random.default_rng(3)
    x, w, c = (rng.integers(-2, 3, s).astype(np.float64) for s in ((5, 6), (4, 6), (5, 4)))
    b, drop = np.full(4, 0.25), (0.25, 11, 2)
    y = mx4.layer(x, w, b, True, drop)

    def loss(x, w, b):
        return (c * mx4.layer(x, w, b, True, drop)).sum()

    (dx, dw, db), _ = mx4.gradients(c, x, w, y, drop)
    # dz is c times fp32's 4 / 3, which 4 bits round once more: to fp32's 4 / 3 at scale 1
    z = mx4.passed(c, y, drop)
    for got, what in ((db, 2), (dx, 0), (dw, 1)):
        args = [x, w, b]
        want = np.zeros(args[what].shape)
        for i in np.ndindex(*want.shape):
            up, down = args[what].copy(), args[what].copy()
            up[i] += 2.0 ** -6
            down[i] -= 2.0 ** -6
            args2, args3 = list(args), list(args)
            args2[what], args3[what] = up, down
            want[i] = (loss(*args2) - loss(*args3)) * 2.0 ** 5
        if what == 2:
            assert np.allclose(got, want, rtol=1e-6, atol=1e-9)
        elif what == 0:
            assert np.abs(got - want).max() <= (np.abs(mx4.rounded(z) - z) @ np.abs(w)).max() + 1e-6
        else:
            assert np.abs(got - want).max() <= (np.abs(mx4.rounded(z.T) - z.T)
                                                @ np.abs(x)).max() + 1e-6
    # without dropout all is exact
    y = mx4.layer(x, w, b, True)
    (dx, dw, db), _ = mx4.gradients(c, x, w, y)
    m = c * (y > 0)
    assert np.array_equal(dx, m @ w) and np.array_equal(dw, m.T @ x)
