"""Orthogonalisation by Newton-Schulz products and the server's step, against
the oracle in float64.

Tolerances.  What the kernels round is known: X, A and P are kept in 22 bits,
without lo lo; sums are fp32.  (Of bf16 matrices the model has the steps whose
errors grow no more than 16 times in 11 bits, more than the kernels need;
test_bf16_is_rounded_once has the closer bound.)  A step multiplies an error in
X by at most about 4 (the largest divided difference of its polynomial), so the
end error depends on the matrix.  It is modelled in float64: every stored value
moved by a uniform relative error of that many bits, every sum by a normal one
of 2^-24 of its operands' lengths, the result rounded to its type.  The kernel
may be off by 4 times the model's error in the Frobenius norm, and by 8 times
the model's largest in any entry, of the worst of eight draws of the model.
(One draw is no bound for a small matrix.  The error of a single entry is a
sum of some fifteen independent roundings, near normal: one draw of it falls
below a quarter of its standard deviation once in five, and then 4 times the
draw is less than one deviation.  All of eight do so once in 0.2^-8 = 390,000;
an error of a matrix of many entries hardly varies between draws.)
The coefficients are fp32 numbers, as the call takes them.
"""
import numpy as np
import pytest

from _parity import say
from oracle import server

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2102_08550_amd
    return paper_2102_08550_amd


COEFFS = tuple(tuple(float(np.float32(v)) for v in step) for step in server.COEFFS)


def _plain_steps(coeffs):
    """bf16: the steps kept in 11 bits."""
    out, amp = [], 1.0
    for a, _, _ in reversed(coeffs):
        amp *= max(1.0, abs(a))
        out.append(amp <= 16.0)
    return out[::-1]


def _model(g, dtype, coeffs, seed=0):
    """The oracle disturbed by roundings of the kernels' size."""
    import torch
    gen = torch.Generator(g.device)
    gen.manual_seed(seed)
    plain = _plain_steps(coeffs) + [False] if dtype == torch.bfloat16 else [False] * 17

    def disturb(kind, t, v, noise):
        last = kind == "x" and t == len(coeffs)
        bits = 2.0 ** -24 if last else 2.0 ** -11 if plain[t] and not (kind == "x" and t == 0) \
            else 2.0 ** -21
        v = v * (1 + bits * (2 * torch.rand(v.shape, generator=gen, device=v.device,
                                            dtype=v.dtype) - 1))
        if noise is not None:
            v = v + 2.0 ** -24 * noise * torch.randn(v.shape, generator=gen, device=v.device,
                                                     dtype=v.dtype)
        return v

    return server.newton_schulz(g.double(), coeffs, disturb).to(dtype).double()


def _f32(coeffs):
    return tuple(tuple(float(np.float32(v)) for v in step) for step in coeffs)


def _may(g, dtype, coeffs=COEFFS):
    """(norm, largest entry) of the model's error."""
    want = server.newton_schulz(g.double(), coeffs)
    errs = [(_model(g, dtype, coeffs, seed) - want).abs() for seed in range(8)]
    return max(float(e.norm()) for e in errs), max(float(e.max()) for e in errs)


def _check(got, g, coeffs=server.COEFFS, where=""):
    import torch
    coeffs = _f32(coeffs)
    want = server.newton_schulz(g.double(), coeffs)
    err = (got.double() - want).abs()
    norm, entry = _may(g, g.dtype, coeffs)
    rel = float(err.norm()) / (4 * norm)
    top = float(err.max()) / (8 * entry)
    say(f"  {where} {tuple(g.shape)} {g.dtype}: error {float(err.norm() / want.norm()):.2e}, "
        f"{rel:.2f} / {top:.2f} of what it may be")
    assert torch.isfinite(got).all()
    assert rel <= 1.0 and top <= 1.0


def _gradient(r, c, seed, strong=8, noise=0.3):
    import torch
    gen = torch.Generator("cuda")
    gen.manual_seed(seed)
    k = min(strong, r, c)
    u = torch.randn(r, k, generator=gen, device="cuda")
    v = torch.randn(k, c, generator=gen, device="cuda")
    s = 0.5 ** torch.arange(k, device="cuda", dtype=torch.float32)
    return 1e-3 * ((u * s) @ v + noise * torch.randn(r, c, generator=gen, device="cuda"))


SHAPES = [(1, 1), (1, 5), (7, 1), (2, 2), (10, 256), (31, 33), (64, 64), (65, 127), (32, 27),
          (128, 1152), (200, 129), (129, 257), (777, 66), (512, 784), (1030, 1100)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("r,c", SHAPES)
def test_orthogonalize(P, r, c, dtype):
    import torch
    g = _gradient(r, c, r * 7 + c).to(torch.float32 if dtype == "fp32" else torch.bfloat16)
    keep = g.clone()
    out = P.orthogonalize(g)
    _check(out, g, where="one")
    assert torch.equal(g, keep) and out.dtype == g.dtype


@pytest.mark.parametrize("shapes", [[(1, 5)], [(64, 64)], [(300, 40), (37, 2050)],
                                    [(512, 784), (256, 512), (10, 256)], [(1030, 1100)],
                                    [(2048, 2060)], [(3600, 3700)]])
@pytest.mark.parametrize("steps", [5, 1])
def test_bf16_is_rounded_once(P, shapes, steps):
    """A bf16 result is the 22-bit products' own, rounded at the end: off by half a
    step of bf16 beside what the fp32 matrix of the same values may be off by."""
    import torch
    gs = [_gradient(r, c, i + 40).bfloat16() for i, (r, c) in enumerate(shapes)]
    coeffs = COEFFS[:steps]
    for g, y in zip(gs, P.orthogonalize(gs, coeffs=coeffs)):
        want = server.newton_schulz(g.double(), coeffs)
        entry = 8 * _may(g.float(), torch.float32, coeffs)[1]
        # a value that close may lie in the next binade, with its larger steps
        exponent = torch.frexp(want.abs() + entry)[1]
        half = torch.ldexp(torch.ones_like(want), exponent - 9)
        over = float(((y.double() - want).abs() - half).max())
        say(f"  {tuple(g.shape)}: {over / entry:.2f} of what it may be beside half a step")
        assert over <= entry


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shapes", [[(512, 784), (256, 512), (10, 256)],
                                    [(300, 40), (40, 300), (1, 9), (64, 64), (1500, 700)],
                                    [(3600, 3700), (33, 900)],
                                    [(2900, 2950)], [(2048, 2060), (2100, 2040)]])
def test_orthogonalize_group(P, shapes, dtype):
    import torch
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    gs = [_gradient(r, c, i).to(dt) for i, (r, c) in enumerate(shapes)]
    outs = P.orthogonalize(gs)
    for g, o in zip(gs, outs):
        _check(o, g, where="group")
    again = P.orthogonalize(gs)
    assert all(torch.equal(a, b) for a, b in zip(outs, again))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_orthogonalize_strides_and_in_place(P, dtype):
    import torch
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    base = _gradient(150, 411, 5).to(dt)
    view = base[3:140, 5:300]  # rows apart, no 16-byte alignment
    _check(P.orthogonalize(view), view, where="view")
    out = torch.full((150, 500), 7.0, dtype=dt, device="cuda")
    P.orthogonalize(view, out=out[1:138, 33:328])
    _check(out[1:138, 33:328], view, where="into a window")
    edge = out.clone()
    edge[1:138, 33:328] = 7.0
    assert (edge == 7.0).all()
    turned = base[3:140, 5:300].mT
    res = P.orthogonalize(turned)
    assert res.stride(0) == 1
    _check(res, turned, where="by columns")
    column, row = base[:, 17:18], base[4:5, :]
    _check(P.orthogonalize(column), column, where="a column")
    _check(P.orthogonalize(row), row, where="a row")
    mine = view.clone()
    assert P.orthogonalize(mine, out=mine) is mine
    assert torch.equal(mine, P.orthogonalize(view.clone()))


@pytest.mark.parametrize("coeffs", [((1.5, -0.5, 0.0),), ((1.875, -1.25, 0.375),) * 8,
                                    ((3.4445, -4.7750, 2.0315), (2.0, -1.5, 0.5))])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_orthogonalize_other_coefficients(P, coeffs, dtype):
    import torch
    g = _gradient(90, 140, 3).to(torch.float32 if dtype == "fp32" else torch.bfloat16)
    _check(P.orthogonalize(g, coeffs=coeffs), g, coeffs, where=f"{len(coeffs)} steps")


@pytest.mark.parametrize("coeffs", [((0.1, 0.0, 0.0), (1.5, -0.5, 0.0)),
                                    ((0.07, 0.0, 0.0), (2.0, 0.0, 0.0)), ((1e-3, 0.0, 0.0),),
                                    ((0.26, 0.0, 0.0),) * 3, ((8.0, -8.0, 2.0), (0.01, 0.0, 0.0))])
def test_orthogonalize_steps_that_shrink(P, coeffs):
    """Down to a sixteenth of the norm in an iterate, as far as one likes in the
    result: full spectra, rank one, all singular values equal.  Less is refused."""
    import torch
    gen = torch.Generator("cuda")
    gen.manual_seed(6)
    a, b = (torch.randn(n, generator=gen, device="cuda") for n in (700, 900))
    flat = torch.linalg.qr(torch.randn(500, 400, generator=gen, device="cuda"))[0].contiguous()
    for g in (_gradient(90, 140, 3), torch.outer(a, b).contiguous(), flat):
        _check(P.orthogonalize(g, coeffs=coeffs), g, coeffs, where=f"{coeffs[0]}")
    for less in (((0.06, 0.0, 0.0),) + coeffs, ((0.1, 0.0, 0.0),) * 8):
        with pytest.raises(P.OscarsError):
            P.orthogonalize(flat, coeffs=less)


@pytest.mark.parametrize("scale", [1e-30, 1e-8, 1e8, 1e30])
def test_orthogonalize_is_free_of_scale(P, scale):
    g = _gradient(96, 200, 9) * scale
    _check(P.orthogonalize(g), g, where=f"times {scale}")


def test_orthogonalize_hard_spectra(P):
    """Singular values over four decades, rank one, and one entry alone."""
    import torch
    gen = torch.Generator("cuda")
    gen.manual_seed(1)
    q1 = torch.linalg.qr(torch.randn(160, 160, generator=gen, device="cuda"))[0]
    q2 = torch.linalg.qr(torch.randn(224, 160, generator=gen, device="cuda"))[0]
    decay = ((q1 * torch.logspace(0, -4, 160, device="cuda")) @ q2.T).contiguous()
    one = torch.zeros(70, 90, device="cuda")
    one[13, 57] = -3e-5
    rank1 = torch.outer(q1[:, 0], q2[:, 0]).contiguous()
    for g in (decay, one, rank1):
        _check(P.orthogonalize(g), g, where="spectrum")
        _check(P.orthogonalize(g.bfloat16()), g.bfloat16(), where="spectrum")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_orthogonalize_zeros_and_not_finite(P, dtype):
    """Zeros give zeros, a NaN or an infinity NaN, and neither reaches the others."""
    import torch
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    good = _gradient(70, 90, 2).to(dt)
    nan, inf = good.clone(), good.clone()
    nan[69, 89] = float("nan")
    inf[0, 3] = float("-inf")
    a, z, b, c, d = P.orthogonalize([good, torch.zeros_like(good), nan, inf, good.clone()])
    assert (z == 0).all() and torch.isnan(b).all() and torch.isnan(c).all()
    assert torch.equal(a, d)
    _check(a, good, where="beside them")


def test_orthogonalize_on_a_stream_and_in_a_graph(P):
    import torch
    gs = [_gradient(200, 333, 1), _gradient(64, 20, 2)]
    want = P.orthogonalize(gs)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = P.orthogonalize(gs, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs))
    x = [torch.zeros_like(g) for g in gs]
    outs = [torch.empty_like(g) for g in gs]
    graphs = []
    for _ in range(2):  # two graphs: workspaces of their own
        with torch.cuda.stream(side):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                P.orthogonalize(x, out=outs)
        graphs.append(graph)
    for k in range(6):
        for a, g in zip(x, gs):
            a.copy_(g * (k + 1) + 1e-4 * k)
        want = P.orthogonalize(x)
        for o in outs:
            o.fill_(-1.0)
        graphs[k % 2].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs)), f"replay {k}"


def test_orthogonalize_planes_past_32_bits(P):
    """8192 x 65536: planes of more than 2^31 bytes, at offsets past 2^32.  All but
    300 columns near the end are zero, and those are what they are beside fewer
    zeros: a rounding of 2^-21 is amplified by at most the product of the |a|, and
    each of the two results has its own."""
    import torch
    gen = torch.Generator("cuda")
    gen.manual_seed(4)
    cols = torch.randint(-9, 10, (8192, 300), generator=gen, device="cuda").float()
    wide = torch.zeros(8192, 65536, device="cuda")
    wide[:, 65216:65516] = cols
    narrow = torch.zeros(8192, 8200, device="cuda")
    narrow[:, :300] = cols
    got, want = P.orthogonalize(wide), P.orthogonalize(narrow)
    assert not got[:, :65216].any() and not got[:, 65516:].any() and not want[:, 300:].any()
    got, want = got[:, 65216:65516].double(), want[:, :300].double()
    amplified = np.prod([abs(a) for a, _, _ in COEFFS])
    assert float((got - want).norm() / want.norm()) <= 2 * 2.0 ** -21 * amplified


def test_two_streams_at_once(P):
    """Calls on two streams have workspaces of their own."""
    import torch
    gs = [_gradient(300, 410, 1), _gradient(64, 64, 2)]
    want = [P.orthogonalize(g) for g in gs]
    streams = [torch.cuda.Stream() for _ in gs]
    torch.cuda.synchronize()
    got = [[] for _ in gs]
    for k in range(8):
        for s, g, res in zip(streams, gs, got):
            if k % 2:
                res.append(P.orthogonalize(g, stream=s))
            else:
                with torch.cuda.stream(s):
                    res.append(P.orthogonalize(g))
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for res, w in zip(got, want) for o in res)


@pytest.mark.parametrize("scale", [2.0 ** -140, 2.0 ** -132, 2.0 ** 125])
def test_orthogonalize_at_the_ends_of_fp32(P, scale):
    """Entries below the normal numbers, and near the largest: the power of two
    changes nothing that the entries still hold (in bf16, whose smallest number is
    2^-133, 7 x 2^-140 is zero)."""
    import torch
    g = torch.randint(-7, 8, (40, 70), device="cuda").float()
    for v in (g, g.bfloat16()):
        held = ((v * scale).double() / scale).to(v.dtype)
        assert torch.equal(P.orthogonalize(v * scale), P.orthogonalize(held))


def test_orthogonalize_rejects(P):
    import torch
    g = torch.randn(8, 12, device="cuda")
    for bad in (torch.zeros(0, 4, device="cuda"), torch.zeros(4, device="cuda"),
                torch.zeros(2, 3, 4, device="cuda"), g[:, ::2]):
        with pytest.raises(ValueError):
            P.orthogonalize(bad)
    with pytest.raises(TypeError):
        P.orthogonalize(g.half())
    with pytest.raises(TypeError):
        P.orthogonalize([g, g.bfloat16()])
    with pytest.raises(TypeError):
        P.orthogonalize(g.cpu())
    with pytest.raises(ValueError):
        P.orthogonalize(g, out=torch.empty(12, 8, device="cuda"))
    with pytest.raises(ValueError):  # another order than x
        P.orthogonalize(g, out=torch.empty(12, 8, device="cuda").mT)
    with pytest.raises(ValueError):
        P.orthogonalize([])
    with pytest.raises(ValueError):
        P.orthogonalize([g] * 33)
    with pytest.raises(ValueError):
        P.orthogonalize(g, coeffs=((1.0, 2.0),))
    with pytest.raises(P.OscarsError):
        P.orthogonalize(g, coeffs=((100.0, 0.0, 0.0),) * 2)
    with pytest.raises(P.OscarsError):  # one output twice
        P.orthogonalize([g, g + 1], out=[torch.empty_like(g)] * 2)
    whole = torch.empty(8, 24, device="cuda")
    P.orthogonalize([g, g], out=[whole[:, :12], whole[:, 12:]])
    assert torch.equal(whole[:, :12], whole[:, 12:])


# ------------------------------------------------------------------ server's step

MLP = ((264, 136, 72, 37), None)
REG = ((24, 10), None)
DEEP = ((40,) + (24, 32) * 7 + (16, 5), None)  # 16 layers, the most
CNN = ((8 * 8 * 3, 10), ((8, 8, 3), ((16, 1), (16, 1), (16, 1, 1), (24, 2))))


def _server_inputs(ctx, seed, spread=3.0):
    import torch
    gen = np.random.default_rng(seed)
    g = [((gen.uniform(-1, 1, s) / np.sqrt(np.prod(s[1:]))).astype(np.float32),
          gen.uniform(-0.1, 0.1, s[0]).astype(np.float32)) for s in ctx.shapes]

    def moved(scale):
        return [((scale * _gradient(s[0], int(np.prod(s[1:])), int(gen.integers(1 << 30)))
                  ).cpu().numpy().reshape(s),
                 (scale * 1e-3 * gen.standard_normal(s[0])).astype(np.float32))
                for s in ctx.shapes]

    reps = [[(w - dw, b - db) for (w, b), (dw, db) in zip(g, moved(spread))]
            for _ in range(ctx.K)]
    mom = moved(5.0)
    dev = [torch.from_numpy(ctx.pack(v)).cuda() for v in (g, mom)]
    rep = torch.from_numpy(np.concatenate([ctx.pack(r) for r in reps])).cuda()
    return dev[0], rep, dev[1]


def _matrices(ctx, flat):
    import torch
    return [(torch.from_numpy(w.reshape(w.shape[0], -1).copy()).double(),
             torch.from_numpy(b.copy()).double())
            for w, b in ctx.unpack(flat.cpu().numpy())]


@pytest.mark.parametrize("model,K", [(MLP, 8), (MLP, 3), (REG, 1), (CNN, 5), (REG, 33), (REG, 64),
                                     (DEEP, 2)])
@pytest.mark.parametrize("nesterov,decay", [(True, 0.0), (False, 0.1)])
def test_server_step(P, model, K, nesterov, decay):
    import torch
    dims, cnn = model
    ctx = P.Context(dims, P.FP32, K, 4, cnn=cnn)
    try:
        g, reps, mom = _server_inputs(ctx, 11 + K)
        w = P.paper_weights(K)
        keep = [t.clone() for t in (g, reps, mom)]
        lr, beta, plain = 0.05, 0.9, 0.7
        plain_layers = (2,) if len(ctx.shapes) > 2 else ()
        out = (torch.full_like(g, float("nan")), torch.full_like(g, float("nan")))
        got = ctx.server_step(g, reps, w, mom, lr=lr, beta=beta, nesterov=nesterov,
                              weight_decay=decay, plain_lr=plain, plain_layers=plain_layers,
                              out=out)
        assert got is not None and got[0] is out[0] and got[1] is out[1]
        for a, b in zip((g, reps, mom), keep):
            assert torch.equal(a, b)
        # the average and the momentum are fp32 elementwise: the same bits
        avg = torch.empty_like(g)
        P.aggregate(avg, reps.clone(), w, K, ctx.n_pad, ctx.n_pad)
        d = g - avg
        m = float(np.float32(beta)) * mom + d
        assert torch.equal(out[1], m)
        u = d + float(np.float32(beta)) * m if nesterov else m
        flat = (g - float(np.float32(plain)) * u)
        want_plain = ctx.unpack(flat.cpu().numpy())
        got_layers = ctx.unpack(out[0].cpu().numpy())
        for l, ((gw, gb), (pw, pb)) in enumerate(zip(got_layers, want_plain), start=1):
            assert np.array_equal(gb, pb), f"bias {l}"
            wo, _ = ctx.layer_offsets(l)
            shape = (gw.shape[0], gw.size // gw.shape[0])
            if l in plain_layers:
                assert np.array_equal(gw, pw)
                continue
            um = u[wo:wo + gw.size].view(shape)
            x = g[wo:wo + gw.size].view(shape).double()
            rate = lr * max(1.0, shape[0] / shape[1]) ** 0.5
            want = (1 - lr * decay) * x - rate * server.newton_schulz(um.double(), COEFFS)
            _, entry = _may(um, torch.float32)
            err = (torch.from_numpy(gw.reshape(shape).copy()).cuda().double() - want).abs()
            # two products and a difference in fp32 behind the orthogonalisation
            assert float(err.max()) <= 8 * rate * entry + 3 * 2.0 ** -24 * float(
                x.abs().max() + rate), f"layer {l}"
        # padding stays zero
        mask = torch.ones_like(g, dtype=torch.bool)
        for l, s in enumerate(ctx.shapes, start=1):
            wo, bo = ctx.layer_offsets(l)
            mask[wo:wo + int(np.prod(s))] = False
            mask[bo:bo + s[0]] = False
        assert (out[0][mask] == 0).all() and (out[1][mask] == 0).all()
        # in place: the same bits
        ctx.server_step(g, reps, w, mom, lr=lr, beta=beta, nesterov=nesterov, weight_decay=decay,
                        plain_lr=plain, plain_layers=plain_layers)
        assert torch.equal(g, out[0]) and torch.equal(mom, out[1]) and torch.equal(reps, keep[1])
    finally:
        ctx.close()


def test_server_step_against_the_oracle(P):
    """The whole step in float64, every layer: the differences that the average's
    own fp32 sums make are part of what may differ."""
    import torch
    ctx = P.Context(MLP[0], P.FP32, 4, 4)
    try:
        g, reps, mom = _server_inputs(ctx, 3)
        keep = mom.clone()
        w = P.paper_weights(4)
        layers = _matrices(ctx, g)
        rl = [_matrices(ctx, r) for r in reps.view(4, -1)]
        new, m = server.server_step(layers, rl, w, _matrices(ctx, mom), 0.05, 0.9, True, 0.01, 0.7,
                                    coeffs=COEFFS)
        ctx.server_step(g, reps, w, mom, lr=0.05, weight_decay=0.01, plain_lr=0.7)
        mom0 = [mm for mm, _ in _matrices(ctx, keep)]
        for (a, b), (c, d), (mm, _), m0 in zip(_matrices(ctx, g), new, m, mom0):
            # u is off by the roundings of the average, the difference and the
            # momentum, 6 halves of 2^-23 of the largest weight at most; each of
            # the five steps makes an error at most 4 times as large; and the
            # kernels' own errors
            u = (mm - 0.9 * m0) + 0.9 * mm
            off = 6 * 2.0 ** -24 * float(a.abs().max()) * a.numel() ** 0.5 / float(u.norm())
            own, _ = _may(u.float(), torch.float32)
            assert float((a - c).norm()) <= 0.05 * (4.0 ** 5 * off + 4 * own) + float(
                a.norm()) * 3 * 2.0 ** -24
            assert float((b - d).abs().max()) <= 8 * 2.0 ** -24 * (1 + float(d.abs().max()))
        for (a, b), (c, d) in zip(_matrices(ctx, mom), m):
            assert float((a - c).abs().max()) <= 8 * 2.0 ** -24 * (1 + float(c.abs().max()))
    finally:
        ctx.close()


def test_server_step_plain_is_the_average(P):
    """beta = 0, plain_lr = 1, every layer plain: x - (x - avg), the average to the
    last bit where the difference is exact."""
    import torch
    ctx = P.Context(MLP[0], P.FP32, 8, 4)
    try:
        g, reps, mom = _server_inputs(ctx, 4, spread=0.1)
        w = P.paper_weights(8)
        avg = torch.empty_like(g)
        P.aggregate(avg, reps.clone(), w, 8, ctx.n_pad, ctx.n_pad)
        ctx.server_step(g, reps, w, mom, lr=0.1, beta=0.0, nesterov=False, plain_lr=1.0,
                        plain_layers=(1, 2, 3))
        assert float((g - avg).abs().max()) <= 2.0 ** -24 * 2 * float(avg.abs().max())
    finally:
        ctx.close()


def test_server_step_in_a_graph(P):
    import torch
    ctx = P.Context(MLP[0], P.FP32, 4, 4)
    side = torch.cuda.Stream()
    try:
        g, reps, mom = _server_inputs(ctx, 6)
        w = P.paper_weights(4)
        g2, mom2 = g.clone(), mom.clone()
        torch.cuda.synchronize()
        ctx.set_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            with torch.cuda.graph(graph, stream=side):
                ctx.server_step(g, reps, w, mom, lr=0.05)
        eager = P.Context(MLP[0], P.FP32, 4, 4)
        for k in range(5):
            graph.replay()
            torch.cuda.synchronize()
            eager.server_step(g2, reps, w, mom2, lr=0.05)
            torch.cuda.synchronize()
            assert torch.equal(g, g2) and torch.equal(mom, mom2), f"replay {k}"
        eager.close()
    finally:
        torch.cuda.synchronize()
        ctx.close()


def test_server_step_rejects(P):
    import torch
    ctx = P.Context(REG[0], P.FP32, 2, 4)
    try:
        g, reps, mom = _server_inputs(ctx, 1)
        w = P.paper_weights(2)
        ok = dict(lr=0.1)
        keep = [t.clone() for t in (g, reps, mom)]
        with pytest.raises(ValueError):
            ctx.server_step(g, reps, P.paper_weights(3), mom, **ok)
        with pytest.raises(ValueError):
            ctx.server_step(g, reps[:-1], w, mom, **ok)
        with pytest.raises(ValueError):
            ctx.server_step(g, reps, w, mom, plain_layers=(2,), **ok)
        with pytest.raises(TypeError):
            ctx.server_step(g.double(), reps, w, mom, **ok)
        for bad in (dict(lr=float("nan")), dict(lr=0.1, beta=float("inf")),
                    dict(lr=0.1, coeffs=((50.0, 0.0, 0.0),) * 2)):
            with pytest.raises(P.OscarsError):
                ctx.server_step(g, reps, w, mom, **bad)
        with pytest.raises(P.OscarsError):  # the new model over the momentum
            ctx.server_step(g, reps, w, mom, out=(mom, torch.empty_like(g)), **ok)
        with pytest.raises(P.OscarsError):  # over the replicas
            ctx.server_step(g, reps, w, mom, out=(reps, torch.empty_like(g)), **ok)
        with pytest.raises(P.OscarsError):
            ctx.server_step(g, reps, np.array([0.5, np.nan], np.float32), mom, **ok)
        for a, b in zip((g, reps, mom), keep):
            assert torch.equal(a, b)
    finally:
        ctx.close()
