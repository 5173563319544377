"""Argument checks of the operators on the global model, through the C ABI and
without a GPU: every call here is refused before anything is enqueued."""
import ctypes

import numpy as np
import pytest

import paper_2102_08550_amd as P

lib = P._lib()
BASE = 0x10000000  # addresses that nothing reads: the calls are refused
COEFFS = P._coeffs(P.NEWTON_SCHULZ)


def _mats(*specs):
    mats = (P._Matrix * len(specs))()
    for m, s in zip(mats, specs):
        m.rows, m.cols, m.x, m.x_ld, m.out, m.out_ld = s
    return mats


GOOD = (8, 12, BASE, 12, BASE + 0x10000, 12)
WS = BASE + 0x1000000


def _orth(mats, dtype=P.FP32, coeffs=COEFFS, ws=WS, nbytes=None, count=None):
    n = len(mats) if count is None else count
    need = lib.oscars_orthogonalize_workspace(mats, n)
    return lib.oscars_orthogonalize(mats, n, dtype, coeffs[0], coeffs[1], ws,
                                    need if nbytes is None else nbytes, None)


@pytest.mark.parametrize("bad", [
    (0, 12, BASE, 12, BASE + 0x10000, 12), (8, -1, BASE, 12, BASE + 0x10000, 12),
    (65537, 12, BASE, 12, BASE + 0x10000, 12), (8, 12, None, 12, BASE, 12),
    (8, 12, BASE, 12, None, 12), (8, 12, BASE, 11, BASE + 0x10000, 12),
    (8, 12, BASE, 12, BASE + 0x10000, 11), (8, 12, BASE + 2, 12, BASE + 0x10000, 12),
    (8, 12, BASE, 12, BASE + 0x10002, 12), (8, 12, WS, 12, BASE, 12), (8, 12, BASE, 12, WS, 12)])
def test_orthogonalize_refuses_a_matrix(bad):
    assert _orth(_mats(bad)) == P.E_INVALID
    assert _orth(_mats(GOOD, bad)) == P.E_INVALID


def test_orthogonalize_refuses_arguments():
    good = _mats(GOOD)
    need = lib.oscars_orthogonalize_workspace(good, 1)
    assert need > 0
    assert _orth(good, dtype=2) == P.E_INVALID
    assert _orth(good, ws=None) == P.E_INVALID
    assert _orth(good, ws=WS + 8) == P.E_INVALID
    assert _orth(good, nbytes=need - 1) == P.E_INVALID
    assert _orth(good, count=0) == P.E_INVALID
    assert _orth(_mats(*[GOOD] * 33)) == P.E_INVALID
    assert _orth(good, coeffs=(None, 5)) == P.E_INVALID
    assert _orth(good, coeffs=(COEFFS[0], 0)) == P.E_INVALID
    assert _orth(good, coeffs=P._coeffs(((1.0, 0.0, 0.0),) * 17)) == P.E_INVALID
    for c in ((100.0, 0.0, 0.0), (1.0, 300.0, 300.0), (float("nan"), 0.0, 0.0),
              (1.0, float("inf"), 0.0)):
        assert _orth(good, coeffs=P._coeffs((c,) * 2)) == P.E_INVALID, c
    assert lib.oscars_orthogonalize_workspace(None, 1) == 0
    assert lib.oscars_orthogonalize_workspace(_mats((0, 1, 1, 1, 1, 1)), 1) == 0


def test_orthogonalize_refuses_outputs_that_share_elements():
    out = BASE + 0x10000

    def pair(second, ld=12):
        return _orth(_mats((8, 12, BASE, 12, out, 24), (8, 12, BASE, 12, second, ld)))

    assert pair(out, 24) == P.E_INVALID
    assert pair(out + 4 * 11, 24) == P.E_INVALID   # one column in common
    assert pair(out + 4 * 13, 24) == P.E_INVALID   # wraps into the next row
    assert pair(out + 4 * 12, 23) == P.E_INVALID   # other strides
    assert pair(out + 4 * 24 * 7, 24) == P.E_INVALID


@pytest.mark.parametrize("step", [(100.0, 0.0, 0.0), (0.0, 500.0, 0.0)])
def test_one_step_past_the_range_is_refused(step):
    assert _orth(_mats(GOOD), coeffs=P._coeffs((step,))) == P.E_INVALID


def test_server_step_refuses_null():
    w = (ctypes.c_float * 1)(1.0)
    o = P._ServerOptions(0.1, 0.9, 0.0, 1.0, 1, 0, COEFFS[0], COEFFS[1])
    assert lib.oscars_server_step(None, BASE, BASE, w, BASE, BASE, BASE, ctypes.byref(o), WS,
                                  1 << 30) == P.E_INVALID
    assert lib.oscars_server_workspace(None) == 0


def test_python_checks_come_first():
    import torch
    x = torch.zeros(4, 5)
    with pytest.raises(TypeError):
        P.orthogonalize(x)  # not on a GPU
    with pytest.raises(TypeError):
        P.orthogonalize(x.double())
    with pytest.raises(ValueError):
        P.orthogonalize([x] * 33)
    with pytest.raises(ValueError):
        P.orthogonalize(torch.zeros(4, 5, 6))
    with pytest.raises(ValueError):
        P.orthogonalize(x[:, ::2])
    with pytest.raises(ValueError):
        P.orthogonalize(torch.zeros(1, 5).expand(4, 5))
    assert P._matrix_view(x, "x") == (4, 5, 5, False)
    assert P._matrix_view(x.mT, "x") == (4, 5, 5, True)
    assert P._matrix_view(x[:, 1:2], "x") == (4, 1, 5, False)
    assert P._matrix_view(x[2:3], "x") == (5, 1, 1, False)
    assert P._matrix_view(x.mT[1:2], "x") == (4, 1, 5, False)
    assert P._matrix_view(x[1:2, 2:3], "x") == (1, 1, 1, False)


def test_numbers_of_the_default_steps():
    assert np.allclose(P.NEWTON_SCHULZ, ((3.4445, -4.7750, 2.0315),) * 5)
