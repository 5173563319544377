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


@pytest.mark.parametrize("steps", [
    ((0.1, 0.0, 0.0),) * 8, ((0.1, 0.0, 0.0),) * 3, ((0.01, 1.0, 0.0), (1.5, -0.5, 0.0)),
    ((1.0, -1.0, 0.0), (1.5, -0.5, 0.0)), ((1.0, -1e-3, 0.0), (0.0, 0.0, 0.0), (1.0, 0.0, 0.0))])
def test_steps_that_shrink_are_refused(steps):
    """Iterates far below 1 fall out of fp16's range: by every step, for the small
    singular values only, for the largest one only, and all."""
    assert _orth(_mats(GOOD), coeffs=P._coeffs(steps)) == P.E_INVALID


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


def test_a_refused_round_leaves_no_momentum(monkeypatch):
    """The local steps' refusal comes before the momentum is made: under a stream's
    capture its zeros would never have been written."""
    import types

    import torch

    from paper_2102_08550_amd import rounds as R
    monkeypatch.setattr(R, "broadcast", lambda *a, **kw: None)
    run = R.OscarsRun.__new__(R.OscarsRun)
    run.ctx, run.cfg = types.SimpleNamespace(_stream=None), types.SimpleNamespace(K=2)
    run.g, run.replicas, run.n, run.momentum = torch.zeros(64), torch.zeros(128), 64, None

    def refuse(tau):
        raise P.OscarsError(P.E_STATE, "oscars_local_steps")

    run.local_steps = refuse
    with pytest.raises(P.OscarsError):
        run.round_server([1, 1], lr=0.1)
    assert run.momentum is None


# ------------------------------------------------------------------ 8 bits

Q, X, W, S, OUT = (BASE + k * 0x1000000 for k in range(2, 7))


def _quantize(**kw):
    a = dict(q=Q, q_ld=128, scale=S, x=X, x_ld=100, dtype=P.FP32, rows=4, cols=100)
    a.update(kw)
    return lib.oscars_quantize_rows(a["q"], a["q_ld"], a["scale"], a["x"], a["x_ld"], a["dtype"],
                                    a["rows"], a["cols"], None)


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(x=None), dict(scale=None), dict(q=Q + 8), dict(q_ld=120), dict(q_ld=96),
    dict(x_ld=99), dict(x=X + 2), dict(scale=S + 2), dict(dtype=2), dict(rows=-1), dict(cols=0),
    dict(cols=65537, x_ld=65537, q_ld=1 << 17), dict(rows=1 << 31), dict(x=Q), dict(scale=X),
    dict(scale=Q), dict(x=X + 1, dtype=P.BF16)])
def test_quantize_rows_refuses(bad):
    assert _quantize(**bad) == P.E_INVALID


def _linear(matmul=False, **kw):
    a = dict(out=OUT, out_ld=50, out_dtype=P.FP32, x=X, x_ld=128, dtype=P.FP32, xscale=S + 0x1000,
             wq=W, w_ld=112, wscale=S, bias=S + 0x8000, relu=1, rows=40, inf=100, outs=50, ws=Q,
             nbytes=None)
    a.update(kw)
    if matmul:
        return lib.oscars_matmul_quantized(a["out"], a["out_ld"], a["out_dtype"], a["x"], a["x_ld"],
                                    a["xscale"], a["wq"], a["w_ld"], a["wscale"], a["bias"],
                                    a["relu"], a["rows"], a["inf"], a["outs"], None)
    need = lib.oscars_linear_quantized_workspace(a["rows"], a["inf"])
    return lib.oscars_linear_quantized(a["out"], a["out_ld"], a["out_dtype"], a["x"], a["x_ld"],
                                a["dtype"], a["wq"], a["w_ld"], a["wscale"], a["bias"], a["relu"],
                                a["rows"], a["inf"], a["outs"], a["ws"],
                                need if a["nbytes"] is None else a["nbytes"], None)


@pytest.mark.parametrize("matmul", [False, True])
@pytest.mark.parametrize("bad", [
    dict(out=None), dict(x=None), dict(wq=None), dict(wscale=None), dict(out=OUT + 2),
    dict(out_ld=49), dict(out_dtype=7), dict(x_ld=99), dict(wq=W + 4), dict(w_ld=104),
    dict(w_ld=96), dict(wscale=S + 1), dict(bias=S + 3), dict(rows=-1), dict(rows=1 << 31),
    dict(inf=0), dict(inf=65537), dict(outs=0), dict(outs=65537), dict(out=X), dict(out=W),
    dict(out=S), dict(out=S + 0x8000), dict(out=OUT + 1, out_dtype=P.BF16)])
def test_linear_i8_refuses(bad, matmul):
    assert _linear(matmul, **bad) == P.E_INVALID


def test_linear_i8_refuses_workspace():
    need = lib.oscars_linear_quantized_workspace(40, 100)
    assert need >= 40 * 128 + 40 * 4 and lib.oscars_linear_quantized_workspace(16, 100) == 0
    assert lib.oscars_linear_quantized_workspace(-1, 100) == 0
    for bad in (dict(ws=None), dict(ws=Q + 8), dict(nbytes=need - 1), dict(ws=OUT), dict(ws=X),
                dict(ws=W), dict(ws=S), dict(dtype=3)):
        assert _linear(**bad) == P.E_INVALID, bad


def test_matmul_i8_refuses():
    for bad in (dict(xscale=None), dict(x=X + 8), dict(x_ld=112), dict(x_ld=136), dict(out=S + 0x1000)):
        assert _linear(True, **bad) == P.E_INVALID, bad


def test_int8_rows_too_far_apart():
    """A tile's 256 rows are addressed by 32 bits: 255 times the stride has to fit."""
    far, ld = OUT + (1 << 44), (1 << 23) + 16
    assert _linear(out=far, w_ld=ld) == P.E_INVALID
    assert _linear(True, out=far, w_ld=ld) == P.E_INVALID
    assert _linear(True, out=far, x_ld=ld) == P.E_INVALID
    assert _quantize(q=far & ~0xF, q_ld=ld) == P.E_INVALID


def test_no_rows_is_no_work():
    assert _quantize(rows=0) == P.OK
    assert _linear(rows=0, ws=None) == P.OK
    assert _linear(True, rows=0) == P.OK


def test_int8_model_refuses_null():
    loss, hits = ctypes.c_double(0.0), ctypes.c_int64(0)
    assert lib.oscars_quantized_model_bytes(None) == 0
    assert lib.oscars_quantize_model(None, BASE, BASE) == P.E_INVALID
    assert lib.oscars_evaluate_quantized(None, BASE, BASE, BASE, 1, ctypes.byref(loss),
                                  ctypes.byref(hits)) == P.E_INVALID


def _pretend(t):
    """A CPU tensor that says it is on a GPU: refusals come before its use."""
    import torch

    class OnGpu(torch.Tensor):
        is_cuda = property(lambda self: True)

    return t.as_subclass(OnGpu)


def test_quantize_rows_window_holds_its_padding(monkeypatch):
    """The zeros go to the next multiple of 128 columns, or to the row's end: a window
    of wider rows that ends before them is refused, and nothing is called."""
    import contextlib

    import torch
    calls = []

    class Lib:
        def oscars_quantize_rows(self, *a):
            calls.append(a)
            return P.OK

    monkeypatch.setattr(P, "_lib", Lib)
    monkeypatch.setattr(P, "_on_device", lambda device: contextlib.nullcontext())
    monkeypatch.setattr(P, "_stream_handle", lambda stream: None)
    buf = _pretend(torch.zeros(6, 384, dtype=torch.int8))
    scale = _pretend(torch.zeros(4))

    def quantize(cols, q, rows=4):
        return P.quantize_rows(_pretend(torch.zeros(rows, cols)), out=(q, scale[:rows]))

    for cols, q in ((40, buf[:4, 208:256]), (10, buf[:4, 240:256]), (40, buf[:4, 256:383]),
                    (129, buf[:4, :255]), (300, buf[:4, :320]), (40, buf[:4, 368:])):
        with pytest.raises(ValueError):
            quantize(cols, q)
    with pytest.raises(ValueError):  # one row of a wider tensor
        quantize(40, buf[5:, 208:256], rows=1)
    assert not calls
    whole = _pretend(torch.zeros(4, 48, dtype=torch.int8))
    for cols, q in ((40, buf[:4, 256:]), (40, buf[:4, 16:144]), (129, buf[:4, :256]),
                    (300, buf[:4]), (40, whole), (10, whole)):
        quantize(cols, q)
        assert calls[-1][1] == q.stride(0)
    assert len(calls) == 6
