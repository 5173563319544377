"""The linear layer in 8-bit integers against the oracle.

Integers and scales are equal.  The products' sums are exact, so an output is off
by the roundings behind them alone: fl(sum), fl(sx sw), their product and the
bias, each half a step of fp32 (4 2^-24 of what it rounds), and half a step of
the output's type (bf16: 2^-8 relative).  The same arithmetic in numpy's float32
gives the same bits, which is checked too.
"""
import numpy as np
import pytest

from _parity import say
from oracle import int8

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2102_08550_amd
    return paper_2102_08550_amd


def _bf16(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).bfloat16().float().numpy()


def _rows(rng, n, c, dtype):
    """Activations: some channels strong, half of them behind a ReLU."""
    x = rng.standard_normal((n, c)) * np.exp(rng.standard_normal(c))
    x[:, ::2] = np.maximum(x[:, ::2], 0)
    x = x.astype(np.float32)
    return _bf16(x) if dtype == "bf16" else x


def _dev(x, dtype):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t.bfloat16() if dtype == "bf16" else t


def _emulated(x, wq, ws, b, relu, bf16_out):
    """The kernels' own arithmetic: float32, rounding by rounding."""
    q, s = int8.quantize_rows(x)
    acc = (q @ wq.astype(np.float64).T).astype(np.float32)
    y = acc * (s.astype(np.float32)[:, None] * ws.astype(np.float32)[None, :])
    if b is not None:
        y = y + b
    if relu:
        y = np.where(y < 0, np.float32(0), y)
    return _bf16(y) if bf16_out else y


def _assert_layer(got, x, wq, ws, b, relu, where=""):
    bf16_out = "bfloat16" in str(got.dtype)
    y = got.float().cpu().numpy()
    want = int8.linear(x, wq, ws, b, relu)
    p = int8.linear(x, wq, ws)
    bound = 4 * 2.0 ** -24 * (np.abs(p) + (np.abs(b) if b is not None else 0)) + 2.0 ** -126
    if bf16_out:
        bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)
    assert (np.abs(y - want) <= bound).all(), where
    assert np.array_equal(y, _emulated(x, wq, ws, b, relu, bf16_out)), where


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,c", [(1, 1), (3, 7), (5, 8), (4, 127), (9, 128), (6, 513), (130, 784),
                                 (7, 1025), (33, 2049), (5, 4100), (3, 8200), (2, 65536)])
def test_quantize_rows(P, n, c, dtype):
    import torch
    x = _rows(np.random.default_rng(n * 100 + c), n, c, dtype)
    q, s = P.quantize_rows(_dev(x, dtype))
    wq, ws = int8.quantize_rows(x)
    assert q.shape == (n, -(-c // 128) * 128)
    assert np.array_equal(s.cpu().numpy(), ws.astype(np.float32))
    got = q.cpu().numpy()
    assert np.array_equal(got[:, :c], wq) and not got[:, c:].any()
    # an unaligned view, into rows longer than a block needs
    base = torch.zeros(n, c + 5, dtype=torch.float32 if dtype == "fp32" else torch.bfloat16,
                       device="cuda")
    base[:, 3:3 + c] = _dev(x, dtype)
    out = (torch.full((n, -(-c // 128) * 128 + 32), 99, dtype=torch.int8, device="cuda"),
           torch.empty(n, device="cuda"))
    P.quantize_rows(base[:, 3:3 + c], out=out)
    got2 = out[0].cpu().numpy()
    assert np.array_equal(got2[:, :-32], got) and (got2[:, -32:] == 99).all()
    assert torch.equal(out[1], s)


@pytest.mark.parametrize("cols", [10, 40, 130])
def test_quantize_rows_into_a_window(P, cols):
    """A window of wider rows: its padding is inside it and what lies around it
    stays; one that ends before its padding is refused."""
    import torch
    x = _rows(np.random.default_rng(cols), 5, cols, "fp32")
    wide = -(-cols // 128) * 128
    buf = torch.full((7, 16 + wide + 48), 99, dtype=torch.int8, device="cuda")
    scale = torch.full((7,), -1.0, device="cuda")
    q = buf[1:6, 16:16 + wide]
    P.quantize_rows(_dev(x, "fp32"), out=(q, scale[1:6]))
    want, s = int8.quantize_rows(x)
    assert np.array_equal(q[:, :cols].cpu().numpy(), want) and not q[:, cols:].any()
    assert np.array_equal(scale[1:6].cpu().numpy(), s.astype(np.float32))
    edge = buf.clone()
    edge[1:6, 16:16 + wide] = 99
    assert (edge == 99).all() and (scale[[0, 6]] == -1).all()
    keep = buf.clone()
    for narrow in (buf[1:6, 16:16 + wide - 1], buf[1:6, 32:16 + wide], buf[6:, 32:16 + wide]):
        with pytest.raises(ValueError):
            P.quantize_rows(_dev(x[:len(narrow)], "fp32"), out=(narrow, scale[1:1 + len(narrow)]))
    assert torch.equal(buf, keep)


def test_quantize_rows_next_to_a_half(P):
    """Quotients on and beside every half: the nearest fp32 values to (k + 1/2) s
    and their neighbours, for scales of every kind."""
    import torch
    rng = np.random.default_rng(5)
    rows = []
    for _ in range(300):
        top = np.float32(rng.uniform(1, 2) * 2.0 ** rng.integers(-110, 100))
        s = np.float32(np.float64(top) / 127)
        k = (np.arange(-127, 127) + 0.5) * np.float64(s)
        near = k.astype(np.float32)
        rows.append(np.concatenate([[top], near, np.nextafter(near, np.float32(np.inf)),
                                    np.nextafter(near, np.float32(-np.inf)), [0, -0.0, -top]]))
    x = np.stack(rows).astype(np.float32)
    x = np.where(np.abs(x) > x[:, :1], x[:, :1], x)
    exact = np.arange(-127, 127) + 0.5  # scale 1: halves themselves, ties to even
    x[0] = np.resize(np.concatenate([[127.0], exact]), x.shape[1])
    q, s = P.quantize_rows(torch.from_numpy(x).cuda())
    wq, ws = int8.quantize_rows(x)
    assert np.array_equal(s.cpu().numpy(), ws.astype(np.float32))
    assert np.array_equal(q.cpu().numpy()[:, :x.shape[1]], wq)


@pytest.mark.parametrize("c", [12, 700, 3000, 9000])
def test_quantize_rows_of_zeros_tiny_and_not_finite(P, c):
    import torch
    rng = np.random.default_rng(c)
    x = rng.standard_normal((7, c)).astype(np.float32)
    x[1] = 0
    x[2, c - 1] = np.nan
    x[3, 5] = -np.inf
    x[4] *= 1e-42  # no normal scale
    x[5] *= np.float32(3e38) / np.abs(x[5]).max()
    q, s = P.quantize_rows(torch.from_numpy(x).cuda())
    wq, ws = int8.quantize_rows(x)
    assert np.array_equal(s.cpu().numpy(), ws.astype(np.float32), equal_nan=True)
    assert np.array_equal(q.cpu().numpy()[:, :c], wq)


SIZES = [(1, 1, 1), (1, 8, 2), (2, 17, 10), (5, 64, 16), (16, 127, 17), (17, 128, 64),
         (1, 4096, 100), (3, 784, 512), (16, 4097, 33), (64, 200, 100), (100, 784, 130),
         (300, 1030, 257), (1, 65536, 3), (16, 9000, 40), (700, 33, 5)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,i,o", SIZES)
def test_linear_i8(P, n, i, o, dtype):
    import torch
    rng = np.random.default_rng(n + 10 * i + 100 * o)
    x = _rows(rng, n, i, dtype)
    w = (rng.uniform(-1, 1, (o, i)) / np.sqrt(i)).astype(np.float32)
    b = rng.uniform(-0.1, 0.1, o).astype(np.float32)
    wq, ws = int8.quantize_rows(w)
    dq, ds = P.quantize_rows(torch.from_numpy(w).cuda())
    dx, db = _dev(x, dtype), torch.from_numpy(b).cuda()
    _assert_layer(P.linear_i8(dx, dq, ds, bias=db, relu=True), x, wq, ws, b, True, "relu")
    _assert_layer(P.linear_i8(dx, dq, ds, out_dtype=torch.float32), x, wq, ws, None, False, "plain")
    _assert_layer(P.linear_i8(dx, dq, ds, bias=db, out_dtype=torch.bfloat16), x, wq, ws, b, False,
                  "bf16 out")
    # the two steps give the same bits
    xq, xs = P.quantize_rows(dx)
    two = P.matmul_i8(xq, xs, dq, ds, i, bias=db, relu=True)
    one = P.linear_i8(dx, dq, ds, bias=db, relu=True, out_dtype=torch.float32)
    assert torch.equal(one, two)


@pytest.mark.parametrize("n", [3, 90])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_linear_i8_strides_and_padding(P, n, dtype):
    """Rows apart and unaligned, weights whose rows hold other bytes behind their
    columns, a window of a larger output: nothing else is read into or written."""
    import torch
    rng = np.random.default_rng(n)
    i, o = 203, 77
    x = _rows(rng, n, i, dtype)
    base = _dev(np.full((n + 2, i + 60), 1e6, np.float32), dtype)
    base[1:n + 1, 7:7 + i] = _dev(x, dtype)
    wq, ws = int8.quantize_rows(rng.standard_normal((o, i)).astype(np.float32))
    w = torch.full((o + 1, 288), 77, dtype=torch.int8, device="cuda")
    w[:o, 16:16 + i] = torch.from_numpy(wq.astype(np.int8)).cuda()
    ds = torch.from_numpy(ws.astype(np.float32)).cuda()
    out = torch.full((n + 2, o + 9), -5.0, dtype=base.dtype, device="cuda")
    got = P.linear_i8(base[1:n + 1, 7:7 + i], w[:o, 16:16 + 240], ds, out=out[1:n + 1, 4:4 + o])
    _assert_layer(got, x, wq, ws, None, False)
    edge = out.clone()
    edge[1:n + 1, 4:4 + o] = -5.0
    assert (edge == -5.0).all()


@pytest.mark.parametrize("n,i,o", [(6200, 300, 2050), (4000, 130, 900), (4161, 3010, 2043),
                                   (4301, 4100, 4095)])
def test_linear_i8_large_tiles(P, n, i, o):
    import torch
    gen = torch.Generator("cuda")
    gen.manual_seed(3)
    x = torch.randn(n, i, generator=gen, device="cuda")
    dq, ds = P.quantize_rows(torch.randn(o, i, generator=gen, device="cuda"))
    xq, xs = P.quantize_rows(x)
    acc = (xq[:, :i].double() @ dq[:, :i].double().T).float()
    want = acc * (xs[:, None] * ds[None, :])
    assert torch.equal(P.linear_i8(x, dq, ds), want)
    got = P.linear_i8(x, dq, ds, relu=True, out_dtype=torch.bfloat16)
    assert torch.equal(got, want.clamp_min(0).bfloat16())


@pytest.mark.parametrize("n", [2, 40])
def test_linear_i8_longest_sums(P, n):
    """65536 products of 127 by 127, the largest sum: exact."""
    import torch
    x = torch.ones(n, 65536, device="cuda")
    x[1] = -1.0
    w = torch.full((20, 65536), 127, dtype=torch.int8, device="cuda")
    y = P.linear_i8(x, w, torch.ones(20, device="cuda"))
    s = np.float32(1.0 / 127)
    want = np.float32(65536 * 127 * 127) * s
    assert (y[0] == float(want)).all() and (y[1] == -float(want)).all()


def test_more_rows_than_threads_of_a_launch(P):
    """2^26 + 5 rows: four a workgroup of 256 threads would be 2^32 threads and more.
    Powers of two times 127: scales and integers are exact, whatever the division."""
    import torch
    n = (1 << 26) + 5
    at = torch.arange(n, device="cuda")
    k = torch.exp2((at % 11).float())
    sign = torch.where(at % 3 == 0, -1.0, 1.0)
    x = (127 * k * sign)[:, None]
    q, scale = P.quantize_rows(x, out=(torch.full((n, 16), 5, dtype=torch.int8, device="cuda"),
                                       torch.zeros(n, device="cuda")))
    assert torch.equal(scale, k)
    assert torch.equal(q[:, 0], (127 * sign).to(torch.int8))
    assert not q[:, 1:].any()


def test_outputs_past_32_bits(P):
    """4.5e9 outputs (9 GB): the last rows are those of a call of their own."""
    import torch
    n, i, o = 1_100_003, 100, 4096
    gen = torch.Generator("cuda")
    gen.manual_seed(5)
    x = torch.randn(n, i, generator=gen, device="cuda").bfloat16()
    w, ws = P.quantize_rows(torch.randn(o, i, generator=gen, device="cuda"))
    y = P.linear_i8(x, w, ws)
    for rows in (slice(0, 300), slice(524200, 524400), slice(n - 700, n)):
        assert torch.equal(y[rows], P.linear_i8(x[rows], w, ws))


def test_two_streams_at_once(P):
    import torch
    w, ws = P.quantize_rows(torch.randn(1000, 500, device="cuda"))
    xs = [torch.randn(n, 500, device="cuda") for n in (700, 3)]
    want = [P.linear_i8(x, w, ws) for x in xs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[] for _ in streams]
    for _ in range(10):
        for s, x, g in zip(streams, xs, got):
            with torch.cuda.stream(s):
                g.append(P.linear_i8(x, w, ws))
    torch.cuda.synchronize()
    assert all(torch.equal(y, v) for g, v in zip(got, want) for y in g)


@pytest.mark.parametrize("n", [4, 50])
def test_linear_i8_rows_not_finite_or_zero(P, n):
    import torch
    rng = np.random.default_rng(8)
    x = rng.standard_normal((n, 300)).astype(np.float32)
    x[1] = 0
    x[2, 299] = np.nan
    x[3, 0] = np.inf
    w = rng.standard_normal((40, 300)).astype(np.float32)
    dq, ds = P.quantize_rows(torch.from_numpy(w).cuda())
    b = torch.randn(40, device="cuda")
    y = P.linear_i8(torch.from_numpy(x).cuda(), dq, ds, bias=b, relu=True)
    assert torch.isnan(y[2:4]).all() and torch.isfinite(y[:2]).all() and torch.isfinite(y[4:]).all()
    assert torch.equal(y[1], b.clamp_min(0))


def test_int8_on_a_stream_and_in_a_graph(P):
    import torch
    w, ws = P.quantize_rows(torch.randn(200, 333, device="cuda"))
    for n in (5, 130):
        x = torch.randn(n, 333, device="cuda")
        want = P.linear_i8(x, w, ws)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        got = P.linear_i8(x, w, ws, stream=side)
        side.synchronize()
        assert torch.equal(got, want)
        out = torch.empty(n, 200, device="cuda")
        graphs = []
        for _ in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                P.linear_i8(x, w, ws, out=out)
            graphs.append(graph)
        for k in range(6):
            x.copy_(torch.randn(n, 333, device="cuda") * (k + 1))
            want = P.linear_i8(x, w, ws)
            out.fill_(7.0)
            graphs[k % 2].replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want), f"rows {n}, replay {k}"


def test_int8_rejects_and_empty(P):
    import torch
    x = torch.randn(4, 40, device="cuda")
    w, ws = P.quantize_rows(torch.randn(8, 40, device="cuda"))
    xq, xs = P.quantize_rows(x)
    with pytest.raises(TypeError):
        P.quantize_rows(x.double())
    with pytest.raises(TypeError):
        P.quantize_rows(x.cpu())
    with pytest.raises(ValueError):
        P.quantize_rows(x.mT[:, ::2])
    with pytest.raises(ValueError):  # one row for all
        P.linear_i8(x[:1].expand(4, 40), w, ws)
    with pytest.raises(P.OscarsError):  # rows of integers not 16 bytes apart
        P.quantize_rows(x, out=(torch.empty(4, 40, dtype=torch.int8, device="cuda"), xs))
    with pytest.raises(ValueError):
        P.quantize_rows(x, out=(torch.empty(4, 32, dtype=torch.int8, device="cuda"), xs))
    with pytest.raises(TypeError):
        P.linear_i8(x, w.float(), ws)
    with pytest.raises(ValueError):
        P.linear_i8(torch.randn(4, 200, device="cuda"), w, ws)
    with pytest.raises(ValueError):
        P.linear_i8(x, w, ws[:-1])
    with pytest.raises(ValueError):
        P.linear_i8(x, w, ws, out=torch.empty(8, 4, device="cuda"))
    with pytest.raises(TypeError):
        P.linear_i8(x, w, ws, out_dtype=torch.bfloat16, out=torch.empty(4, 8, device="cuda"))
    with pytest.raises(ValueError):  # the zero padding has to be there
        P.matmul_i8(xq[:, :64], xs, w, ws, 40)
    with pytest.raises(P.OscarsError):  # the output over the input
        P.linear_i8(x, w, ws, out=x[:, :8])
    empty = P.linear_i8(x[:0], w, ws)
    assert empty.shape == (0, 8)
    assert P.quantize_rows(x[:0])[0].shape == (0, 128)
    assert P.matmul_i8(xq[:0], xs[:0], w, ws, 40).shape == (0, 8)


# ------------------------------------------------------------------ a whole model

MODELS = [((264, 136, 72, 37), "bf16", 700), ((784, 512, 256, 10), "fp32", 1500),
          ((24, 10), "fp32", 3), ((40, 24, 200), "fp32", 9000)]


@pytest.mark.parametrize("dims,dtype,n", MODELS)
def test_evaluate_i8(P, dims, dtype, n):
    """The quantised model's loss and hits: every layer in the kernels' own
    arithmetic (equal bits), then the softmax in float64."""
    import torch
    import workload
    cfg = workload.Config("int8", dims, workload.BF16 if dtype == "bf16" else workload.FP32, K=1,
                          n_rows=10, batch=64, tau_rule="given", tau_given=(1,), seed=5)
    ctx = P.Context(dims, P.BF16 if dtype == "bf16" else P.FP32, 1, 64)
    try:
        init = workload.gen_init(cfg)
        params = torch.from_numpy(ctx.pack(init)).cuda()
        ev = workload.gen_eval_set(cfg, n)
        model = ctx.quantize_model(params)
        x = ev.x_f32()
        for l, (w, b) in enumerate(init):
            wq, ws = int8.quantize_rows(w)
            last = l == len(init) - 1
            x = _emulated(x, wq, ws, b, not last, dtype == "bf16" and not last)
        z = x.astype(np.float64)
        top = z.max(axis=1, keepdims=True)
        lse = np.log(np.exp(z - top).sum(axis=1)) + top[:, 0]
        mine = z[np.arange(n), ev.y]
        want_loss, want_hits = float((lse - mine).sum()), int((mine == top[:, 0]).sum())
        dx = torch.from_numpy(np.ascontiguousarray(ev.x).view(np.int16) if dtype == "bf16"
                              else ev.x).cuda()
        dy = torch.from_numpy(ev.y.astype(np.int32)).cuda()
        loss, hits = ctx.evaluate_i8(model, dx, dy)
        full, full_hits = ctx.evaluate(params, dx, dy)
        say(f"{dims} {dtype}: int8 {loss / n:.5f} {hits}, model {full / n:.5f} {full_hits}")
        assert hits == want_hits
        # a row's loss in fp32: the exponentials' sum and logarithm, and the
        # difference of logits, some 8 roundings of numbers up to |z| + log C
        size = np.abs(z).max() + np.log(dims[-1]) + 1
        assert abs(loss - want_loss) <= n * 8 * 2.0 ** -23 * size
        again = ctx.evaluate_i8(model, dx, dy, n_rows=max(1, n // 2))
        assert again[1] == int((mine == top[:, 0])[:max(1, n // 2)].sum())
    finally:
        ctx.close()


def test_evaluate_i8_refusals(P):
    import torch
    ctx = P.Context((8 * 8 * 3, 10), P.FP32, 1, 4, cnn=((8, 8, 3), ((16, 1),)))
    mlp = P.Context((24, 10), P.FP32, 1, 4)
    side = torch.cuda.Stream()
    try:
        with pytest.raises(P.OscarsError):
            ctx.quantize_model(torch.zeros(ctx.n_pad, device="cuda"))
        params = torch.zeros(mlp.n_pad, device="cuda")
        model = mlp.quantize_model(params)
        x, y = torch.zeros(5, 24, device="cuda"), torch.zeros(5, dtype=torch.int32, device="cuda")
        with pytest.raises(ValueError):
            mlp.evaluate_i8(model, x, y, n_rows=6)
        with pytest.raises(ValueError):
            mlp.evaluate_i8(model[:-256], x, y)
        with pytest.raises(TypeError):
            mlp.evaluate_i8(model, x.bfloat16(), y)
        with pytest.raises(P.OscarsError):
            ctx.evaluate_i8(torch.zeros(64, dtype=torch.uint8, device="cuda"),
                            torch.zeros(5, 192, device="cuda"), y)
        torch.cuda.synchronize()
        mlp.set_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            with pytest.raises(P.OscarsError) as ei:
                mlp.evaluate_i8(model, x, y)
        assert ei.value.status == P.E_STATE
    finally:
        ctx.close()
        mlp.close()
