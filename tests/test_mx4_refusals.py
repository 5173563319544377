"""Argument checks of the 4-bit layer and of dropout, through the C ABI and in Python,
without a GPU: every call here is refused before anything is enqueued."""
import ctypes

import pytest

import paper_2102_08550_amd as P

lib = P._lib()
BASE = 0x10000000  # addresses that nothing reads: the calls are refused
MB = 0x100000


def _drop(p=0.5, device=None):
    return P._Dropout(p, 1, 0, device)


def _call(fn, good, **change):
    args = dict(good, **change)
    return fn(*args.values())


QUANT = dict(q=BASE, q_ld=128, scale=BASE + MB, s_ld=16, x=BASE + 2 * MB, x_ld=100, dtype=P.FP32,
             rows=9, cols=100, transposed=0, stream=None)


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(q=BASE + 8), dict(q_ld=112), dict(q_ld=136), dict(q_ld=(1 << 23) + 16),
    dict(scale=None), dict(scale=BASE + MB + 4), dict(s_ld=8), dict(s_ld=24), dict(x=None),
    dict(x=BASE + 2 * MB + 2), dict(x_ld=99), dict(dtype=2), dict(rows=-1), dict(rows=1 << 31),
    dict(cols=0), dict(cols=(1 << 24) + 1, x_ld=1 << 25, q_ld=1 << 23, s_ld=1 << 20),
    dict(cols=257, x_ld=257), dict(x=BASE), dict(x=BASE + MB), dict(scale=BASE + 64),
    dict(transposed=1, rows=300), dict(transposed=1, rows=(1 << 24) + 1, q_ld=1 << 23, s_ld=1 << 20),
    dict(transposed=1, rows=1 << 23, cols=1 << 15, x_ld=1 << 15, q_ld=1 << 22, s_ld=1 << 18)])
def test_quantize_refuses(bad):
    assert _call(lib.oscars_quantize_micro, QUANT, **bad) == P.E_INVALID


VALUES = dict(out=BASE + 2 * MB, out_ld=100, dtype=P.FP32, q=BASE, q_ld=128, scale=BASE + MB,
              s_ld=16, rows=9, cols=100, stream=None)


@pytest.mark.parametrize("bad", [
    dict(out=None), dict(out_ld=99), dict(dtype=3), dict(q=None), dict(q=BASE + 1), dict(q_ld=64),
    dict(scale=None), dict(s_ld=0), dict(rows=-1), dict(cols=0), dict(cols=257, out_ld=300),
    dict(out=BASE), dict(out=BASE + MB)])
def test_dequantize_refuses(bad):
    assert _call(lib.oscars_dequantize_micro, VALUES, **bad) == P.E_INVALID


MATMUL = dict(out=BASE, out_ld=50, dtype=P.FP32, xq=BASE + MB, x_ld=128, xs=BASE + 2 * MB,
              xs_ld=16, wq=BASE + 3 * MB, w_ld=128, ws=BASE + 4 * MB, ws_ld=16,
              bias=BASE + 5 * MB, relu=1, dropout=None, rows=9, inputs=100, outs=50, stream=None)


@pytest.mark.parametrize("bad", [
    dict(out=None), dict(out_ld=49), dict(out=BASE + 2), dict(dtype=-1), dict(xq=None),
    dict(xq=BASE + MB + 8), dict(x_ld=120), dict(x_ld=64), dict(xs=None), dict(xs_ld=8),
    dict(wq=None), dict(w_ld=112), dict(ws=None), dict(ws=BASE + 4 * MB + 1), dict(ws_ld=17),
    dict(bias=BASE + 5 * MB + 2), dict(rows=-1), dict(rows=1 << 31), dict(inputs=0),
    dict(inputs=257), dict(outs=0), dict(outs=(1 << 24) + 1, out_ld=1 << 25),
    dict(inputs=(1 << 24) + 1), dict(out=BASE + MB), dict(out=BASE + 2 * MB),
    dict(out=BASE + 3 * MB), dict(out=BASE + 4 * MB), dict(out=BASE + 5 * MB),
    dict(dropout=_drop(-0.1)), dict(dropout=_drop(1.1)), dict(dropout=_drop(float("nan"))),
    dict(dropout=_drop(0.5, BASE + 6 * MB + 4)), dict(dropout=_drop(0.5, BASE + 8))])
def test_matmul_refuses(bad):
    assert _call(lib.oscars_matmul_micro, MATMUL, **bad) == P.E_INVALID


NEED = lib.oscars_linear_micro_workspace(40, 600)
LINEAR = dict(out=BASE, out_ld=50, out_dtype=P.FP32, x=BASE + MB, x_ld=600, dtype=P.BF16,
              wq=BASE + 3 * MB, w_ld=384, ws=BASE + 4 * MB, ws_ld=32, bias=None, relu=1,
              dropout=None, rows=40, inputs=600, outs=50, workspace=BASE + 6 * MB, nbytes=NEED,
              stream=None)


@pytest.mark.parametrize("bad", [
    dict(out=None), dict(x=None), dict(x=BASE + MB + 1), dict(x_ld=599), dict(dtype=2),
    dict(out_dtype=2), dict(wq=None), dict(w_ld=256), dict(ws_ld=16), dict(rows=-1),
    dict(inputs=0), dict(inputs=65537, x_ld=70000, w_ld=1 << 20, ws_ld=1 << 16),
    dict(workspace=None), dict(workspace=BASE + 6 * MB + 8), dict(nbytes=NEED - 1),
    dict(workspace=BASE), dict(workspace=BASE + MB), dict(workspace=BASE + 3 * MB),
    dict(out=BASE + MB), dict(dropout=_drop(2.0)), dict(bias=BASE)])
def test_linear_refuses(bad):
    assert _call(lib.oscars_linear_micro, LINEAR, **bad) == P.E_INVALID


def test_workspaces():
    assert lib.oscars_linear_micro_workspace(1, 65536) == 0
    assert lib.oscars_linear_micro_workspace(16, 1024) == 0
    assert lib.oscars_linear_micro_workspace(16, 1025) == 16 * (5 * 128 + 3 * 16)
    assert lib.oscars_linear_micro_workspace(32, 512) == 0
    assert lib.oscars_linear_micro_workspace(33, 10) > 0
    assert lib.oscars_linear_micro_workspace(-1, 10) == 0
    assert lib.oscars_linear_micro_backward_workspace(-1, 10, 10, 1) == 0
    assert lib.oscars_linear_micro_backward_workspace(10, 65537, 10, 1) == 0
    assert lib.oscars_linear_micro_backward_workspace(10, 10, 10, 1) > \
        lib.oscars_linear_micro_backward_workspace(10, 10, 10, 0) > 0


GRAD_NEED = lib.oscars_linear_micro_backward_workspace(40, 60, 50, 1)


def _gradients(**change):
    f = dict(rows=40, inputs=60, outs=50, dy=BASE, y=BASE + MB, x=BASE + 2 * MB, dy_ld=50, y_ld=50,
             x_ld=60, y_dtype=P.BF16, x_dtype=P.FP32, wtq=BASE + 3 * MB, wtscale=BASE + 4 * MB,
             wt_ld=128, wts_ld=16, dx=BASE + 5 * MB, dw=BASE + 6 * MB, db=BASE + 7 * MB, dx_ld=60,
             dw_ld=60)
    ws, n = change.pop("ws", BASE + 8 * MB), change.pop("n", GRAD_NEED)
    drop = change.pop("dropout", None)
    g = P._Gradients(**dict(f, **change))
    if drop is not None:
        g.dropout = ctypes.addressof(drop)
    return lib.oscars_linear_micro_backward(ctypes.byref(g), ws, n, None)


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(rows=(1 << 24) + 1), dict(inputs=0), dict(inputs=65537, x_ld=1 << 17),
    dict(outs=0), dict(dy=None), dict(dy=BASE + 1), dict(dy_ld=49), dict(y_ld=49),
    dict(y=BASE + MB + 1), dict(x=None), dict(x_ld=59), dict(y_dtype=2), dict(x_dtype=-1),
    dict(wtq=None), dict(wtscale=None), dict(wt_ld=64), dict(wts_ld=4), dict(dx_ld=59),
    dict(dx=BASE + 5 * MB + 2), dict(dw=None), dict(dw_ld=59), dict(db=BASE + 7 * MB + 1),
    dict(ws=None), dict(ws=BASE + 8 * MB + 4), dict(n=GRAD_NEED - 1), dict(ws=BASE),
    dict(ws=BASE + 6 * MB), dict(dx=BASE), dict(dx=BASE + 2 * MB), dict(dw=BASE + MB),
    dict(db=BASE + 6 * MB), dict(dw=BASE + 3 * MB), dict(dropout=_drop(-1.0)),
    dict(dropout=_drop(0.5, BASE + 6 * MB))])
def test_gradients_refuse(bad):
    assert _gradients(**bad) == P.E_INVALID


def test_gradients_refuse_null():
    assert lib.oscars_linear_micro_backward(None, BASE, 1 << 20, None) == P.E_INVALID


DROPOUT = dict(out=BASE, out_ld=50, x=BASE + MB, x_ld=50, dtype=P.FP32, options=_drop(), rows=9,
               cols=50, stream=None)


@pytest.mark.parametrize("bad", [
    dict(out=None), dict(out_ld=49), dict(x=None), dict(x_ld=49), dict(x=BASE + MB + 2),
    dict(dtype=2), dict(options=None), dict(options=_drop(1.5)), dict(rows=-1), dict(rows=1 << 31),
    dict(cols=0), dict(cols=1 << 31, x_ld=1 << 32, out_ld=1 << 32), dict(x=BASE + 4),
    dict(x=BASE, x_ld=51), dict(options=_drop(0.5, BASE)), dict(options=_drop(0.5, BASE + MB + 12))])
def test_dropout_refuses(bad):
    assert _call(lib.oscars_dropout, DROPOUT, **bad) == P.E_INVALID


def test_python_checks_come_first():
    import torch
    x = torch.zeros(4, 5)
    u = torch.zeros(4, 128, dtype=torch.uint8)
    for call in (lambda: P.quantize_mx4(x), lambda: P.dequantize_mx4(u, u, 5),
                 lambda: P.matmul_mx4(u, u, u, u, 5), lambda: P.linear_mx4(x, u, u),
                 lambda: P.linear_mx4_backward(x, x), lambda: P.dropout(x, 0.5, 1)):
        with pytest.raises(TypeError):  # not on a GPU
            call()
    for call in (lambda: P.linear_mx4(x, None, None), lambda: P.dequantize_mx4(None, None, 5),
                 lambda: P.matmul_mx4(u, u, u[0], u, 5), lambda: P.quantize_mx4(x.double())):
        with pytest.raises(TypeError):
            call()
    for bad in ((1.5, 1), (-0.1, 1), (float("nan"), 1), (0.5, -1), (0.5, 1 << 64), (0.5, 1, -1),
                (0.5, 1, 1 << 64)):
        with pytest.raises(ValueError):
            P._dropout_options(bad, x.device)
    with pytest.raises(TypeError):
        P._dropout_options((0.5, 1, torch.zeros(1, dtype=torch.int64)), x.device)
