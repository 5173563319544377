"""The layer in microscaled 4-bit floating point, its gradients and dropout, against
the oracle.

Codes and scales are equal.  Where all products and sums fit fp32 (entries from a
short range of scales) a product is equal too, whatever its order.  Else: a product
of two entries is exact, sums of 64 or 128 of them are added to the running sum by
one matrix instruction.  Counting a step (2^-23, whether it rounds or cuts) for each
of the at most 128 additions inside one and one for each instruction, a sum of K
products is off by at most (128 + K / 64 + 8) 2^-23 of the sum of their magnitudes
(8: the waves' sums, bias and dropout's factor), and the result by half a step of
its type on top.
"""
import numpy as np
import pytest

from _parity import say
from oracle import dropout as oracle_dropout
from oracle import mx4

pytestmark = pytest.mark.gpu

HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def P():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2102_08550_amd
    return paper_2102_08550_amd


def _bf16(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).bfloat16().float().numpy()


def _rows(rng, n, c, dtype, relu=False):
    x = rng.standard_normal((n, c)) * np.exp(rng.standard_normal(c))
    if relu:
        x = np.maximum(x, 0)
    x = x.astype(np.float32)
    return _bf16(x) if dtype == "bf16" else x


def _type(dtype):
    import torch
    return torch.float32 if dtype == "fp32" else torch.bfloat16


def _dev(x, dtype="fp32"):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda().to(_type(dtype))


def _host(t):
    return t.float().cpu().numpy().astype(np.float64)


def _codes(rng, n, c, spread=2):
    """Random codes and scales of a short range, on the host and packed on the device."""
    import torch
    code = rng.integers(0, 16, (n, c))
    scale = rng.integers(127 - spread, 128, (n, (c + 31) // 32))
    q, s = mx4.packed(code, scale)
    return mx4.values(code, scale), torch.from_numpy(q).cuda(), torch.from_numpy(s).cuda()


def _bound(xv, wv, b, want, dtype, gain=1.0):
    k = xv.shape[1]
    size = np.abs(xv) @ np.abs(wv).T + (0 if b is None else np.abs(b))
    return (128 + k / 64 + 8) * 2.0 ** -23 * size * gain + HALF[dtype] * np.abs(want) + 2.0 ** -126


# ------------------------------------------------------------------ quantisation

SHAPES = [(1, 1), (3, 7), (5, 31), (4, 32), (9, 33), (6, 255), (7, 256), (3, 257), (130, 784),
          (33, 513), (2, 2049), (257, 100), (511, 130), (1025, 8), (1, 65536)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("n,c", SHAPES)
def test_quantize(P, n, c, transposed, dtype):
    import torch
    x = _rows(np.random.default_rng(n * 100 + c), n, c, dtype)
    q, s = P.quantize_mx4(_dev(x, dtype), transposed=transposed)
    xt = x.T if transposed else x
    wq, ws = mx4.packed(*mx4.quantize_rows(xt))
    assert q.shape == wq.shape and s.shape == ws.shape
    assert np.array_equal(q.cpu().numpy(), wq) and np.array_equal(s.cpu().numpy(), ws)
    # an unaligned view, into windows of wider rows, whose surroundings stay
    base = torch.zeros(n, c + 5, dtype=_type(dtype), device="cuda")
    base[:, 3:3 + c] = _dev(x, dtype)
    big = torch.full((wq.shape[0] + 2, wq.shape[1] + 48), 99, dtype=torch.uint8, device="cuda")
    bis = torch.full((ws.shape[0] + 2, ws.shape[1] + 32), 98, dtype=torch.uint8, device="cuda")
    out = big[1:-1, 16:16 + wq.shape[1]], bis[1:-1, 16:16 + ws.shape[1]]
    P.quantize_mx4(base[:, 3:3 + c], transposed=transposed, out=out)
    assert torch.equal(out[0], q) and torch.equal(out[1], s)
    big[1:-1, 16:16 + wq.shape[1]] = 99
    bis[1:-1, 16:16 + ws.shape[1]] = 98
    assert (big == 99).all() and (bis == 98).all()
    # and back
    v = P.dequantize_mx4(q, s, xt.shape[1])
    assert np.array_equal(_host(v), mx4.rounded(xt))
    vb = P.dequantize_mx4(q, s, xt.shape[1], dtype=torch.bfloat16)  # 2 bits: as they are
    assert torch.equal(vb.float(), v)


@pytest.mark.parametrize("transposed", [False, True])
def test_quantize_borders(P, transposed):
    """Entries on and beside every border, for scales from end to end of the range."""
    rng = np.random.default_rng(5)
    mid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], np.float32)
    near = np.concatenate([mid, np.nextafter(mid, np.float32(9)), np.nextafter(mid, np.float32(0))])
    rows = []
    for e in list(range(-126, -110)) + list(range(-6, 7)) + [100, 124, 125]:
        for top in (4.0, 6.5, np.nextafter(np.float32(7), np.float32(0)), 7.0, 7.5):
            if np.float64(top) * 2.0 ** e > 3.4e38:
                continue
            row = np.zeros(32)
            row[:21] = near * rng.choice([-1, 1], 21)
            row[21] = top
            row[22:] = rng.uniform(-4, 4, 10)
            rows.append(np.ldexp(row.astype(np.float64), e).astype(np.float32))
    x = np.stack(rows)
    q, s = P.quantize_mx4(_dev(x.T if transposed else x), transposed=transposed)
    wq, ws = mx4.packed(*mx4.quantize_rows(x))
    assert np.array_equal(s.cpu().numpy(), ws)
    assert np.array_equal(q.cpu().numpy(), wq)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("transposed", [False, True])
def test_quantize_special_blocks(P, transposed, dtype):
    x = _rows(np.random.default_rng(1), 12, 96, dtype)
    x[0] = 0
    x[1, 3] = np.inf
    x[2, 40] = -np.inf
    x[3, 95] = np.nan
    x[4] = 2.0 ** -127            # no normal number
    x[5, :32] = 2.0 ** -126       # the least one
    x[5, 1] = -2.0 ** -127
    x[6, :32] = 2.0 ** -125
    x[7, 0] = 3.38e38
    x[8] = -0.0
    x = _bf16(x) if dtype == "bf16" else x
    q, s = P.quantize_mx4(_dev(x.T if transposed else x, dtype), transposed=transposed)
    wq, ws = mx4.packed(*mx4.quantize_rows(x))
    assert np.array_equal(s.cpu().numpy(), ws)
    assert np.array_equal(q.cpu().numpy(), wq)
    assert ws[1, 0] == 255 and ws[3, 2] == 255 and ws[0, 0] == 0 and ws[7, 0] == 252
    assert np.array_equal(_host(P.dequantize_mx4(q, s, 96)), mx4.rounded(x), equal_nan=True)


def test_quantize_rows_beyond_32_bits(P):
    """Entries more than 2^32 bytes from the first."""
    import torch
    n, c = 70000, 32768
    x = torch.zeros(n, c, dtype=torch.bfloat16, device="cuda")
    x[-1, -40:] = torch.arange(-20, 20, device="cuda", dtype=torch.bfloat16)
    q, s = P.quantize_mx4(x)
    v = P.dequantize_mx4(q[-2:], s[-2:], c)
    want = mx4.rounded(_host(x[-2:]))
    assert np.array_equal(_host(v), want)
    assert not q[:-1].any() and not s[:-1].any()
    d = P.dropout(x[-3:], 0.0, 1)
    assert torch.equal(d, x[-3:])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_columns_of_rows_far_apart(P, dtype):
    """Rows 2^24 entries apart and more: by columns, and in gradients by rows too."""
    import torch
    rng = np.random.default_rng(3)
    n, c = 70, 66
    x = _rows(rng, n, c, dtype)
    base = torch.full((n, (1 << 24) + 8), float("nan"), dtype=_type(dtype), device="cuda")
    base[:, :c] = _dev(x, dtype)
    far = base[:, :c]
    near = far.contiguous()
    q, s = P.quantize_mx4(far, transposed=True)
    wq, ws = mx4.packed(*mx4.quantize_rows(x.T))
    assert np.array_equal(q.cpu().numpy(), wq) and np.array_equal(s.cpu().numpy(), ws)
    wt = P.quantize_mx4(_dev(rng.standard_normal((c, c))), transposed=True)
    for y in (None, near):
        got = P.linear_mx4_backward(far, far, *wt, y=None if y is None else far)
        want = P.linear_mx4_backward(near, near, *wt, y=y)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    del base, far
    torch.cuda.empty_cache()


# ------------------------------------------------------------------ products

# outputs x inputs x rows over tiles of every size, their edges, one entry
PRODUCTS = [(1, 1, 1), (5, 33, 3), (33, 256, 31), (31, 257, 33), (40, 511, 64), (64, 513, 200),
            (1000, 700, 1100), (129, 100, 2500), (2300, 600, 2200), (4097, 40, 700),
            (3000, 1300, 3001)]


@pytest.mark.parametrize("outs,inputs,rows", PRODUCTS)
def test_product_exact(P, outs, inputs, rows):
    """Products whose every sum is a whole number of fp32: equal, in any order."""
    import torch
    rng = np.random.default_rng(outs + inputs + rows)
    xv, xq, xs = _codes(rng, rows, inputs)
    wv, wq, ws = _codes(rng, outs, inputs)
    want = xv @ wv.T
    assert (np.abs(xv) @ np.abs(wv).T).max() * 2 ** 6 < 2 ** 24
    y = P.matmul_mx4(xq, xs, wq, ws, inputs)
    assert np.array_equal(_host(y), want)
    # bias and ReLU, in fp32: one rounding
    b = rng.standard_normal(outs).astype(np.float32)
    y = P.matmul_mx4(xq, xs, wq, ws, inputs, bias=_dev(b), relu=True)
    both = (want.astype(np.float32) + b).astype(np.float32)
    assert np.array_equal(y.cpu().numpy(), np.where(both < 0, 0, both))
    # bf16, into a window of longer rows that is not aligned
    big = torch.full((rows + 2, outs + 7), 77.0, dtype=torch.bfloat16, device="cuda")
    out = big[1:-1, 3:3 + outs]
    P.matmul_mx4(xq, xs, wq, ws, inputs, bias=_dev(b), out=out)
    assert np.array_equal(out.float().cpu().numpy(), _bf16(both))
    big[1:-1, 3:3 + outs] = 77
    assert (big == 77).all()
    yb = P.matmul_mx4(xq, xs, wq, ws, inputs, bias=_dev(b), out_dtype=torch.bfloat16)
    assert np.array_equal(yb.float().cpu().numpy(), _bf16(both))


def test_product_of_strided_rows(P):
    """Operands inside wider, longer buffers that hold NaN around them."""
    import torch
    rng = np.random.default_rng(8)
    for rows, inputs, outs in ((37, 300, 50), (700, 520, 900)):
        xv, xq, xs = _codes(rng, rows, inputs)
        wv, wq, ws = _codes(rng, outs, inputs)

        def wide(t, extra):
            b = torch.full((t.shape[0] + 2, t.shape[1] + extra), 255, dtype=torch.uint8,
                           device="cuda")
            b[1:-1, 16:16 + t.shape[1]] = t
            return b[1:-1, 16:16 + t.shape[1]]

        y = P.matmul_mx4(wide(xq, 48), wide(xs, 32), wide(wq, 144), wide(ws, 16 * 5), inputs)
        assert np.array_equal(_host(y), xv @ wv.T)


@pytest.mark.parametrize("dtype,out_dtype", [("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32")])
@pytest.mark.parametrize("rows,inputs,outs", [
    (1, 8, 2), (1, 1, 1), (1, 4096, 515), (1, 65536, 40), (2, 784, 512), (16, 1024, 37),
    (16, 1025, 37), (7, 700, 100), (17, 784, 512), (32, 512, 33), (32, 8, 5), (33, 8, 5), (20, 519, 70), (200, 333, 130), (1300, 520, 700)])
def test_linear(P, rows, inputs, outs, dtype, out_dtype):
    import torch
    rng = np.random.default_rng(rows + inputs + outs)
    x = _rows(rng, rows, inputs, dtype, relu=True)
    w = (rng.standard_normal((outs, inputs)) / np.sqrt(inputs)).astype(np.float32)
    b = rng.standard_normal(outs).astype(np.float32)
    wq, ws = P.quantize_mx4(_dev(w))
    xv, wv = mx4.rounded(x), mx4.rounded(w)
    y = P.linear_mx4(_dev(x, dtype), wq, ws, bias=_dev(b), relu=True, out_dtype=_type(out_dtype))
    want = mx4.layer(xv, wv, b, True)
    assert (np.abs(_host(y) - want) <= _bound(xv, wv, b, want, out_dtype)).all()
    # the same as quantisation and product; unaligned rows
    base = torch.zeros(rows, inputs + 3, dtype=_type(dtype), device="cuda")
    base[:, 1:1 + inputs] = _dev(x, dtype)
    z = P.linear_mx4(base[:, 1:1 + inputs], wq, ws, bias=_dev(b), relu=True,
                     out_dtype=_type(out_dtype))
    assert torch.equal(z, y)
    xq, xs = P.quantize_mx4(_dev(x, dtype))
    m = P.matmul_mx4(xq, xs, wq, ws, inputs, bias=_dev(b), relu=True, out_dtype=_type(out_dtype))
    assert (np.abs(_host(m) - want) <= _bound(xv, wv, b, want, out_dtype)).all()
    # dropout in the epilogue: of the fp32 result, with its mask
    drop = (0.3, 12345678901234567, 5)
    d = P.linear_mx4(_dev(x, dtype), wq, ws, bias=_dev(b), relu=True, dropout=drop,
                     out_dtype=_type(out_dtype))
    y32 = P.linear_mx4(_dev(x, dtype), wq, ws, bias=_dev(b), relu=True, out_dtype=torch.float32)
    assert torch.equal(d, P.dropout(y32, *drop).to(_type(out_dtype)))
    d = P.matmul_mx4(xq, xs, wq, ws, inputs, bias=_dev(b), relu=True, dropout=drop,
                     out_dtype=_type(out_dtype))
    y32 = P.matmul_mx4(xq, xs, wq, ws, inputs, bias=_dev(b), relu=True)
    assert torch.equal(d, P.dropout(y32, *drop).to(_type(out_dtype)))


@pytest.mark.parametrize("rows", [1, 9, 40, 600])
def test_nan_and_infinity_stay_in_their_rows(P, rows):
    import torch
    rng = np.random.default_rng(rows)
    x = _rows(rng, rows, 600, "fp32")
    w = rng.standard_normal((530, 600)).astype(np.float32)
    w[7, 100], w[529, 599] = np.nan, np.inf
    bad = rows // 2
    x[bad, 599] = -np.inf
    wq, ws = P.quantize_mx4(_dev(w))
    y = _host(P.linear_mx4(_dev(x), wq, ws, relu=True))
    want = np.zeros((rows, 530), bool)
    want[bad], want[:, 7], want[:, 529] = True, True, True
    assert np.array_equal(np.isnan(y), want)
    d = _host(P.linear_mx4(_dev(x), wq, ws, relu=True, dropout=(0.5, 3)))
    kept = oracle_dropout.kept(rows, 530, 0.5, 3)
    assert np.array_equal(np.isnan(d), want & kept) and (d[~kept] == 0).all()


def test_rows_do_not_depend_on_others(P):
    """A row's result: the same alone in a tile and among others of the same call's tiles."""
    import torch
    rng = np.random.default_rng(2)
    x = _dev(_rows(rng, 300, 900, "bf16"), "bf16")
    wq, ws = P.quantize_mx4(_dev(rng.standard_normal((200, 900))))
    y = P.linear_mx4(x, wq, ws)
    again = P.linear_mx4(x.flip(0).contiguous(), wq, ws)
    assert torch.equal(again.flip(0), y)
    assert P.linear_mx4(x[:0], wq, ws).shape == (0, 200)
    assert P.quantize_mx4(x[:0])[0].shape == (0, 512)
    assert P.quantize_mx4(x[:0], transposed=True)[0].shape == (900, 0)


def test_dropout_of_a_product_in_two_launches(P):
    """Rows past 2^29, which go to a second launch: dropout counts them on."""
    import torch
    rows = 2 ** 29 + 70
    q = torch.zeros(rows, 128, dtype=torch.uint8, device="cuda")
    s = torch.zeros(rows, 16, dtype=torch.uint8, device="cuda")
    wq, ws = P.quantize_mx4(torch.ones(2, 1, device="cuda"))
    ones = torch.ones(2, device="cuda")
    y = P.matmul_mx4(q, s, wq, ws, 1, bias=ones, dropout=(0.5, 21, 4), out_dtype=torch.bfloat16)
    del q, s
    want = P.dropout(torch.ones(rows, 2, dtype=torch.bfloat16, device="cuda"), 0.5, 21, 4)
    same = torch.equal(y, want)
    del y, want
    torch.cuda.empty_cache()
    assert same


# rows, inputs, outputs that one launch does not hold (test_mx4_plan.py asks the plan)
TWO_LAUNCHES = (2 ** 30 + 70, 1, 2)


def test_product_of_more_rows_than_a_launch_holds(P):
    """The second launch's rows: dropout counts them on from the first's, operands and
    outputs are theirs.  160 GB."""
    import torch
    rows, inputs, outs = TWO_LAUNCHES
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 190 * 10 ** 9:
        pytest.skip("needs 190 GB of free device memory")
    x = torch.arange(300, device="cuda") % 7  # codes of the last rows' entries
    value = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4], device="cuda")[x].bfloat16()
    q = torch.zeros(rows, 128, dtype=torch.uint8, device="cuda")
    s = torch.zeros(rows, 16, dtype=torch.uint8, device="cuda")
    q[-300:, 0] = x.to(torch.uint8)
    s[-300:, 0] = 127
    wq, ws = P.quantize_mx4(torch.ones(outs, inputs, device="cuda"))
    ones = torch.ones(outs, device="cuda")
    y = P.matmul_mx4(q, s, wq, ws, inputs, bias=ones, dropout=(0.5, 21, 4),
                     out_dtype=torch.bfloat16)
    del q, s
    want = torch.ones(rows, outs, dtype=torch.bfloat16, device="cuda")
    want[-300:] += value[:, None]
    P.dropout(want, 0.5, 21, 4, out=want)  # times 2: exact
    same = torch.equal(y, want)
    del y, want
    torch.cuda.empty_cache()
    assert same


# ------------------------------------------------------------------ dropout

@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,c", [(1, 1), (3, 7), (64, 512), (5, 8), (37, 1001), (1000, 24),
                                 (2, 100000)])
@pytest.mark.parametrize("p", [0.0, 1e-6, 0.1, 0.5, 0.9999, 1.0])
def test_dropout(P, n, c, p, dtype):
    import torch
    x = _rows(np.random.default_rng(c), n, c, dtype)
    x[0, 0] = np.nan
    seed, offset = 0xFEDCBA9876543210, (3 << 32) + 5
    want = oracle_dropout.dropout(x, p, seed, offset).astype(np.float32)  # one rounding in fp32
    want = _bf16(want) if dtype == "bf16" else want
    t = _dev(x, dtype)
    y = P.dropout(t, p, seed, offset)
    assert np.array_equal(y.float().cpu().numpy(), want, equal_nan=True)
    # the offset from the device, a window of other rows, in place
    more = torch.tensor([offset], device="cuda")
    base = torch.full((n, c + 9), 5.0, dtype=_type(dtype), device="cuda")
    base[:, 1:1 + c] = t
    view = base[:, 1:1 + c]
    assert P.dropout(view, p, seed, more, out=view) is view
    assert np.array_equal(view.float().cpu().numpy(), want, equal_nan=True)
    assert (base[:, 0] == 5).all() and (base[:, 1 + c:] == 5).all()


def test_dropout_gradient_is_dropout(P):
    """Against differences: the mask of the forward call, applied to dy."""
    import torch
    rng = np.random.default_rng(0)
    x, dy = rng.standard_normal((2, 6, 21)).astype(np.float32)
    got = P.dropout(_dev(dy), 0.4, 9, 1).cpu().numpy()
    want = np.zeros_like(x, np.float64)
    for i in np.ndindex(*x.shape):
        up, down = x.astype(np.float64), x.astype(np.float64)
        up[i] += 0.5
        down[i] -= 0.5
        want[i] = (dy * (oracle_dropout.dropout(up, 0.4, 9, 1)
                         - oracle_dropout.dropout(down, 0.4, 9, 1))).sum()
    # 126 terms of fp64 cancel to the one that moved
    assert np.abs(got - want).max() <= 2.0 ** -24 * np.abs(want).max() + 1e-12


# ------------------------------------------------------------------ gradients

def _assert_gradients(P, got, dy, x, w, y, drop, x_dtype):
    sums, sizes = mx4.gradients(dy, x, w, y, drop)
    outs, rows = dy.shape[1], dy.shape[0]
    for what, g, want, size, k, dt in zip(("dx", "dw", "db"), got, sums, sizes,
                                          (outs, rows, None), (x_dtype, "fp32", "fp32")):
        if g is None:
            continue
        # db: sums in 64 bits, rounded once (rows 2^-53 of the magnitudes)
        steps = 128 + k / 64 + 8 if k else rows * 2.0 ** -29
        bound = steps * 2.0 ** -23 * size + HALF[dt] * np.abs(want) + 2.0 ** -126
        assert (np.abs(_host(g) - want) <= bound).all(), what


@pytest.mark.parametrize("relu", [True, False])
@pytest.mark.parametrize("p", [0.0, 0.25])
@pytest.mark.parametrize("x_dtype,y_dtype", [("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32")])
@pytest.mark.parametrize("rows,inputs,outs", [(1, 1, 1), (1, 40, 33), (31, 10, 65), (64, 512, 256),
                                              (257, 33, 129), (600, 260, 300), (1025, 700, 2)])
def test_gradients(P, rows, inputs, outs, x_dtype, y_dtype, p, relu):
    import torch
    rng = np.random.default_rng(rows + inputs + outs)
    x = _rows(rng, rows, inputs, x_dtype, relu=True)
    w = (rng.standard_normal((outs, inputs)) / np.sqrt(inputs)).astype(np.float32)
    dy = _rows(rng, rows, outs, y_dtype) * np.float32(2.0 ** -10)
    drop = (p, 77, 3) if p else None
    y = _rows(rng, rows, outs, y_dtype, relu=True) if relu else None
    if relu and p:
        y = np.where(oracle_dropout.kept(rows, outs, *drop), y, 0)
    wt, wts = P.quantize_mx4(_dev(w), transposed=True)
    dyd, xd = _dev(dy, y_dtype), _dev(x, x_dtype)
    yd = None if y is None else _dev(y, y_dtype)
    got = P.linear_mx4_backward(dyd, xd, wt, wts, y=yd, dropout=drop)
    assert got[0].dtype == xd.dtype and got[1].dtype == got[2].dtype == torch.float32
    _assert_gradients(P, got, dy, x, w, y, drop, x_dtype)
    # without dx; from and into windows; the same values
    def window(t, left):
        b = torch.full((t.shape[0], t.shape[1] + 11), 9.0, dtype=t.dtype, device="cuda")
        b[:, left:left + t.shape[1]] = t
        return b[:, left:left + t.shape[1]]
    dw = window(torch.zeros(outs, inputs, device="cuda"), 3)
    db = torch.empty(outs, device="cuda")
    some = P.linear_mx4_backward(window(dyd, 3), window(xd, 1), y=None if yd is None
                                 else window(yd, 5), dropout=drop, want_dx=False,
                                 out=(None, dw, db))
    assert some[0] is None
    assert torch.equal(dw, got[1]) and torch.equal(db, got[2])


@pytest.mark.parametrize("relu", [True, False])
@pytest.mark.parametrize("p", [0.0, 0.25])
@pytest.mark.parametrize("x_dtype,y_dtype", [("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32"),
                                             ("fp32", "bf16")])
@pytest.mark.parametrize("rows,inputs,outs", [(1, 2, 2), (64, 512, 256), (256, 30, 66),
                                              (257, 32, 130), (600, 260, 300)])
def test_gradients_without_dx(P, rows, inputs, outs, x_dtype, y_dtype, p, relu):
    """Of aligned tensors, up to 256 rows and more: dw and db are what they should be and
    what they are beside dx, whatever ran on the card before."""
    import torch
    rng = np.random.default_rng(rows + inputs + outs)
    x = _rows(rng, rows, inputs, x_dtype, relu=True)
    w = (rng.standard_normal((outs, inputs)) / np.sqrt(inputs)).astype(np.float32)
    dy = _rows(rng, rows, outs, y_dtype) * np.float32(2.0 ** -10)
    drop = (p, 77, 3) if p else None
    y = _rows(rng, rows, outs, y_dtype, relu=True) if relu else None
    if relu and p:
        y = np.where(oracle_dropout.kept(rows, outs, *drop), y, 0)
    dyd, xd = _dev(dy, y_dtype), _dev(x, x_dtype)
    yd = None if y is None else _dev(y, y_dtype)
    # gradients of other numbers first, on every CU
    P.linear_mx4_backward(torch.full((512, 32768), 3.0e5, device="cuda"),
                          torch.ones(512, 32, device="cuda"), want_dx=False)
    got = P.linear_mx4_backward(dyd, xd, y=yd, dropout=drop, want_dx=False)
    assert got[0] is None
    _assert_gradients(P, got, dy, x, w, y, drop, x_dtype)
    both = P.linear_mx4_backward(dyd, xd, *P.quantize_mx4(_dev(w), transposed=True), y=yd,
                                 dropout=drop)
    _assert_gradients(P, both, dy, x, w, y, drop, x_dtype)
    assert torch.equal(got[2], both[2])  # sums in one order; dw's tiles may be others
    # without db too
    lone = torch.empty_like(got[1])
    P.linear_mx4_backward(dyd, xd, y=yd, dropout=drop, want_dx=False, out=(None, lone, None))
    assert torch.equal(lone, got[1])


# rows, inputs, outputs whose dw takes tiles of 64, 128 and 256 (test_mx4_plan.py asks the plan)
LARGE_GRADIENTS = [(300, 1100, 1024), (600, 2048, 2048), (600, 4096, 4096)]


@pytest.mark.parametrize("want_dx", [True, False])
@pytest.mark.parametrize("relu", [True, False])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,inputs,outs", LARGE_GRADIENTS)
def test_gradients_in_large_tiles(P, rows, inputs, outs, dtype, relu, want_dx):
    """dw's tiles with the workgroups behind them that add up db's parts: against products
    in 64 bits of what quantize_mx4 makes of dz, x and w."""
    import torch
    rng = np.random.default_rng(rows + inputs + outs)
    x = _dev(_rows(rng, rows, inputs, dtype, relu=True), dtype)
    w = _dev(rng.standard_normal((outs, inputs)) / np.sqrt(inputs))
    dy = _dev(_rows(rng, rows, outs, dtype) * np.float32(2.0 ** -10), dtype)
    y = _dev(_rows(rng, rows, outs, dtype, relu=True), dtype) if relu else None
    wt = P.quantize_mx4(w, transposed=True)
    got = P.linear_mx4_backward(dy, x, *wt, y=y, want_dx=want_dx)
    dz = dy.float() if y is None else torch.where(y > 0, dy.float(), 0.0)

    def values(t, transposed, along):
        return P.dequantize_mx4(*P.quantize_mx4(t, transposed=transposed), along).double()

    zr, zc, xc = values(dz, False, outs), values(dz, True, rows), values(x, True, rows)
    wc = P.dequantize_mx4(*wt, outs).double()
    for what, g, a, b, k in (("dx", got[0], zr, wc, outs), ("dw", got[1], zc, xc, rows)):
        if g is None:
            assert what == "dx" and not want_dx
            continue
        b = b.t().contiguous()
        want, size = a @ b, a.abs() @ b.abs()
        half = HALF[dtype if what == "dx" else "fp32"]
        bound = (128 + k / 64 + 8) * 2.0 ** -23 * size + half * want.abs() + 2.0 ** -126
        assert ((g.double() - want).abs() <= bound).all(), what
    want, size = dz.double().sum(0), dz.double().abs().sum(0)
    # both sums in 64 bits, in orders of their own; one rounding
    assert ((got[2].double() - want).abs()
            <= 2 * rows * 2.0 ** -52 * size + HALF["fp32"] * want.abs()).all()


def test_gradients_of_no_rows(P):
    import torch
    wt, wts = P.quantize_mx4(torch.ones(5, 9, device="cuda"), transposed=True)
    dw, db = torch.full((5, 9), 3.0, device="cuda"), torch.full((5,), 3.0, device="cuda")
    dx = torch.empty(0, 9, device="cuda")
    e = torch.empty(0, 5, device="cuda")
    P.linear_mx4_backward(e, torch.empty(0, 9, device="cuda"), wt, wts, y=e, out=(dx, dw, db))
    assert not dw.any() and not db.any()


def test_gradients_of_masked_rows(P):
    """Rows that pass nothing on, a NaN of dy under the mask, and one that is seen."""
    import torch
    rng = np.random.default_rng(4)
    dy = rng.standard_normal((300, 50)).astype(np.float32)
    x = rng.standard_normal((300, 70)).astype(np.float32)
    w = rng.standard_normal((50, 70)).astype(np.float32)
    y = np.maximum(rng.standard_normal((300, 50)), 0).astype(np.float32)
    y[10:50] = 0
    y[60, 7], dy[60, 7] = 0, np.nan
    wt, wts = P.quantize_mx4(_dev(w), transposed=True)
    got = P.linear_mx4_backward(_dev(dy), _dev(x), wt, wts, y=_dev(y))
    clean = dy.copy()
    clean[60, 7] = 0
    _assert_gradients(P, got, clean, x, w, y, None, "fp32")
    assert not got[0][10:50].any()
    y[60, 7] = 1
    dx, dw, db = P.linear_mx4_backward(_dev(dy), _dev(x), wt, wts, y=_dev(y))
    bad = np.isnan(_host(dx))
    assert bad[60].all() and bad.sum() == 70
    bad = np.isnan(_host(dw))
    assert bad[7].all() and bad.sum() == 70
    assert np.isnan(_host(db)).sum() == 1 and np.isnan(float(db[7]))


def test_gradients_against_differences(P):
    """Entries that 4 bits hold along rows and columns: the layer is its unrounded self,
    linear between ReLU's borders, which the differences do not cross; central
    differences of the oracle's float64 are its gradients, exactly."""
    rng = np.random.default_rng(6)
    x, w, c = (rng.integers(-2, 3, s).astype(np.float64) for s in ((9, 14), (7, 14), (9, 7)))
    b = np.full(7, 0.25)
    wq, ws = P.quantize_mx4(_dev(w))
    y = P.linear_mx4(_dev(x), wq, ws, bias=_dev(b), relu=True)
    assert np.array_equal(_host(y), mx4.layer(x, w, b, True))
    wt, wts = P.quantize_mx4(_dev(w), transposed=True)
    got = P.linear_mx4_backward(_dev(c), _dev(x), wt, wts, y=y)
    args = [x, w, b]
    for k in range(3):
        want = np.zeros(args[k].shape)
        for i in np.ndindex(*want.shape):
            losses = []
            for sign in (1, -1):
                moved = [v.copy() for v in args]
                moved[k][i] += sign * 2.0 ** -6
                losses.append((c * mx4.layer(*moved, True)).sum())
            want[i] = (losses[0] - losses[1]) * 2.0 ** 5
        assert np.array_equal(_host(got[k]), want), k


# ------------------------------------------------------------------ together

def _same(a, b):
    import torch
    return torch.equal(a.view(torch.int32), b.view(torch.int32))


def _step(P, x, target, ws, bs, seed, offset, lr):
    """A training step of two layers; master weights in fp32."""
    import torch
    q = [P.quantize_mx4(w) for w in ws]
    qt = [P.quantize_mx4(w, transposed=True) for w in ws]
    drop = (0.25, seed, offset)
    h = P.linear_mx4(x, *q[0], bias=bs[0], relu=True, dropout=drop)
    z = P.linear_mx4(h, *q[1], bias=bs[1], out_dtype=torch.float32)
    dz = (z - target) * (1.0 / x.shape[0])
    dh, dw1, db1 = P.linear_mx4_backward(dz, h, *qt[1])
    _, dw0, db0 = P.linear_mx4_backward(dh, x, y=h, dropout=drop, want_dx=False)
    for w, d in ((ws[0], dw0), (ws[1], dw1), (bs[0], db0), (bs[1], db1)):
        w.sub_(lr * d)
    return h, z, dh


def test_training_step_together_and_captured(P):
    """A step eagerly against the oracle's pieces, then captured and replayed with the
    program counting dropout's offset up: every replay is what the eager step gives."""
    import torch
    rng = np.random.default_rng(9)
    x = _dev(_rows(rng, 96, 200, "fp32"))
    target = _dev(rng.standard_normal((96, 40)))
    w0 = [_dev(rng.standard_normal((144, 200)) / 14), _dev(rng.standard_normal((40, 144)) / 12)]
    b0 = [_dev(rng.standard_normal(144)), _dev(rng.standard_normal(40))]
    ws, bs = [w.clone() for w in w0], [b.clone() for b in b0]
    h, z, dh = _step(P, x, target, ws, bs, 5, 0, 0.1)
    hv, wv = mx4.rounded(_host(x)), mx4.rounded(_host(w0[0]))
    b = _host(b0[0])
    want = mx4.layer(hv, wv, b, True, (0.25, 5, 0))
    assert (np.abs(_host(h) - want) <= _bound(hv, wv, b, want, "fp32", gain=4 / 3)).all()
    hv, wv = mx4.rounded(_host(h)), mx4.rounded(_host(w0[1]))
    want = mx4.layer(hv, wv, _host(b0[1]))
    assert (np.abs(_host(z) - want) <= _bound(hv, wv, _host(b0[1]), want, "fp32")).all()
    dz = _host((z - target) * (1.0 / 96))
    got = P.linear_mx4_backward((z - target) * (1.0 / 96), h,
                                *P.quantize_mx4(w0[1], transposed=True))
    assert torch.equal(got[0], dh)
    _assert_gradients(P, got, dz, _host(h), _host(w0[1]), None, None, "fp32")

    eager_w, eager_b = [w.clone() for w in w0], [b.clone() for b in b0]
    ws, bs = [w.clone() for w in w0], [b.clone() for b in b0]
    offset = torch.zeros(1, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = _step(P, x, target, ws, bs, 5, offset, 0.1)
        offset.add_(1)
    offset.zero_()
    for step in range(4):
        graph.replay()
        want = _step(P, x, target, eager_w, eager_b, 5, step, 0.1)
        torch.cuda.synchronize()
        # bit by bit: the step is large for these inputs, and the last replays reach NaN
        assert all(_same(a, c) for a, c in zip(out, want)), step
        assert all(_same(a, c) for a, c in zip(ws + bs, eager_w + eager_b)), step
    assert int(offset) == 4


def test_captured_training_stays_finite(P):
    """Captured and replayed with a step that lets the weights settle: every replay is what
    the eager step gives, of finite numbers, and moves the weights."""
    import torch
    rng = np.random.default_rng(9)
    x = _dev(_rows(rng, 96, 200, "fp32"))
    target = _dev(rng.standard_normal((96, 40)))
    w0 = [_dev(rng.standard_normal((144, 200)) / 14), _dev(rng.standard_normal((40, 144)) / 12)]
    b0 = [_dev(rng.standard_normal(144)), _dev(rng.standard_normal(40))]
    eager_w, eager_b = [w.clone() for w in w0], [b.clone() for b in b0]
    ws, bs = [w.clone() for w in w0], [b.clone() for b in b0]
    offset = torch.zeros(1, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = _step(P, x, target, ws, bs, 5, offset, 2.0 ** -7)
        offset.add_(1)
    offset.zero_()
    before = w0
    for step in range(4):
        graph.replay()
        want = _step(P, x, target, eager_w, eager_b, 5, step, 2.0 ** -7)
        torch.cuda.synchronize()
        assert all(torch.isfinite(t).all() for t in (*out, *ws, *bs)), step
        assert all(_same(a, c) for a, c in zip(out, want)), step
        assert all(_same(a, c) for a, c in zip(ws + bs, eager_w + eager_b)), step
        assert not any(torch.equal(a, b) for a, b in zip(ws, before)), step
        before = [w.clone() for w in ws]
    assert int(offset) == 4


def test_two_graphs_and_another_stream(P):
    """Two captured calls with workspaces of their own, replayed in turns, and calls on a
    stream that is named, whose inputs the caller drops at once."""
    import torch
    rng = np.random.default_rng(12)
    wq, ws = P.quantize_mx4(_dev(rng.standard_normal((300, 500))))
    xs = [_dev(_rows(rng, 90 + i, 500, "fp32")) for i in range(2)]
    want = [P.linear_mx4(x, wq, ws) for x in xs]
    graphs, outs = [], []
    torch.cuda.synchronize()
    for x in xs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(P.linear_mx4(x, wq, ws))
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
        for o in outs:
            o.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    results = []
    for _ in range(5):
        x = xs[0].clone()
        side.wait_stream(torch.cuda.current_stream())
        results.append(P.linear_mx4(x, wq, ws, stream=side))
        q = P.quantize_mx4(x, stream=side)
        results.append(P.matmul_mx4(*q, wq, ws, 500, stream=side))
        d = P.dropout(x, 0.5, 1, stream=side)
        results.append(P.linear_mx4(d, wq, ws, stream=side))
        del x, q, d
        torch.empty(90, 500, device="cuda").fill_(float("nan"))
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    dropped = P.linear_mx4(P.dropout(xs[0], 0.5, 1), wq, ws)
    for r in results[::3] + results[1::3]:
        assert torch.equal(r, want[0])
    for r in results[2::3]:
        assert torch.equal(r, dropped)


# ------------------------------------------------------------------ models

def _losses(z, y):
    """(summed loss, rows whose label has the largest logit) in float64."""
    z = z.astype(np.float64)
    top = z.max(axis=1)
    mine = z[np.arange(len(z)), y]
    return float((np.log(np.exp(z - top[:, None]).sum(axis=1)) + top - mine).sum()), \
        int((mine == top).sum())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dims,n", [((24, 10), 7), ((784, 512, 256, 10), 300),
                                    ((1000, 520, 136, 40, 3), 257), ((64, 48, 10), 20000)])
def test_evaluate_mx4(P, dims, n, dtype):
    """Loss and hits from the logits that the layers give one by one (which the other
    tests hold to the oracle), and of a single layer from the oracle's."""
    import torch
    rng = np.random.default_rng(n)
    ctx = P.Context(dims, P.FP32 if dtype == "fp32" else P.BF16, 1, 8)
    try:
        init = [((2 * rng.random((o, i)) - 1).astype(np.float32) / np.sqrt(i),
                 (2 * rng.random(o) - 1).astype(np.float32) / np.sqrt(i))
                for i, o in zip(dims[:-1], dims[1:])]
        init = [(w.astype(np.float32), b.astype(np.float32)) for w, b in init]
        params = torch.from_numpy(ctx.pack(init)).cuda()
        x, y = _rows(rng, n, dims[0], dtype), rng.integers(0, dims[-1], n)
        model = ctx.quantize_model_mx4(params)
        passes = -(-n // 8192)
        rows = -(-n // passes)
        logits = []
        for at in range(0, n, rows):
            a = _dev(x[at:at + rows], dtype)
            for l, (w, b) in enumerate(init):
                last = l == len(init) - 1
                wq = P.quantize_mx4(_dev(w))
                a = P.matmul_mx4(*P.quantize_mx4(a), *wq, dims[l], bias=_dev(b), relu=not last,
                                 out_dtype=torch.float32 if last else _type(dtype))
            logits.append(a.cpu().numpy())
        z = np.concatenate(logits)
        want_loss, want_hits = _losses(z, y)
        dx = _dev(x, dtype)
        dy = torch.from_numpy(y.astype(np.int32)).cuda()
        loss, hits = ctx.evaluate_mx4(model, dx, dy)
        say(f"{dims} {dtype}: 4 bits {loss / n:.5f} {hits}, model {ctx.evaluate(params, dx, dy)}")
        assert hits == want_hits
        # a row's loss in fp32: the exponentials' sum and logarithm, and the difference of
        # logits, some 8 roundings of numbers up to |z| + log C
        size = np.abs(z).max() + np.log(dims[-1]) + 1
        assert abs(loss - want_loss) <= n * 8 * 2.0 ** -23 * size
        if len(dims) == 2:
            xv, wv = mx4.rounded(x), mx4.rounded(init[0][0])
            want = mx4.layer(xv, wv, init[0][1])
            assert (np.abs(z - want) <= _bound(xv, wv, init[0][1], want, "fp32")).all()
        again = ctx.evaluate_mx4(model, dx, dy, n_rows=max(1, n // 2))
        assert 0 <= again[1] <= hits
    finally:
        ctx.close()


def test_evaluate_mx4_refusals(P):
    import torch
    cnn = P.Context((8 * 8 * 3, 10), P.FP32, 1, 4, cnn=((8, 8, 3), ((16, 1),)))
    mlp = P.Context((24, 10), P.FP32, 1, 4)
    try:
        with pytest.raises(P.OscarsError):
            cnn.quantize_model_mx4(torch.zeros(cnn.n_pad, device="cuda"))
        params = torch.zeros(mlp.n_pad, device="cuda")
        model = mlp.quantize_model_mx4(params)
        x, y = torch.zeros(5, 24, device="cuda"), torch.zeros(5, dtype=torch.int32, device="cuda")
        with pytest.raises(ValueError):
            mlp.evaluate_mx4(model, x, y, n_rows=6)
        with pytest.raises(ValueError):
            mlp.evaluate_mx4(model[:-256], x, y)
        with pytest.raises(ValueError):
            mlp.quantize_model_mx4(params[:-64])
        with pytest.raises(TypeError):
            mlp.evaluate_mx4(model, x.bfloat16(), y)
        with pytest.raises(P.OscarsError):
            cnn.evaluate_mx4(torch.zeros(64, dtype=torch.uint8, device="cuda"),
                             torch.zeros(5, 192, device="cuda"), y)
    finally:
        cnn.close()
        mlp.close()


def test_rounds_and_paradigms_evaluate_in_4_bits(P):
    """run_paradigm with the 4-bit evaluation beside the ordinary and the 8-bit one:
    what the rounds by hand give; without it, records as before."""
    import torch
    import workload
    from paper_2102_08550_amd import controller as C
    from paper_2102_08550_amd import rounds as R
    cfg = workload.Config("mlp-mx4", (40, 32, 10), workload.FP32, K=2, n_rows=400, batch=16,
                          tau_rule="given", tau_given=(2, 2))
    ds, init = workload.gen_dataset(cfg), workload.gen_init(cfg)
    ev = workload.gen_eval_set(cfg, 100)
    sched = C.SpeedSchedule([1, 1])
    res = C.run_paradigm(cfg, ds, init, ev, "local", sched, 1.0, 1e9, local_steps=2, max_rounds=3,
                         int8_eval=True, mx4_eval=True)
    run = R.OscarsRun(cfg, ds, init)
    try:
        for _ in range(3):
            run.round([2] * 2)
        x, y = torch.from_numpy(ev.x).cuda(), torch.from_numpy(ev.y.astype(np.int32)).cuda()
        loss, hits = run.evaluate(x, y, mx4=True)
        with pytest.raises(ValueError):
            run.evaluate(x, y, int8=True, mx4=True)
    finally:
        run.close()
    last = res["records"][-1]
    assert last["eval_loss_mx4"] == loss / 100 and last["eval_acc_mx4"] == hits / 100
    assert {"eval_loss", "eval_loss_i8"} <= set(last)
    plain = C.run_paradigm(cfg, ds, init, ev, "local", sched, 1.0, 1e9, local_steps=2, max_rounds=1)
    assert not any("mx4" in k or "i8" in k for r in plain["records"] for k in r)
