"""The operators on the global model as a program uses them: rounds of local steps
that end with the server's step (OscarsRun.round_server), the model quantised
and evaluated after each, and the paradigm comparison on top of them.

Every step is checked on the models that the GPU had before it: the server's
step against the oracle in float64, within what fp32 roundings of u grow to in
five Newton-Schulz steps (each makes an error at most 4 times as large); the
quantised evaluation against the kernels' own arithmetic in numpy."""
import numpy as np
import pytest

import workload
from _parity import say
from oracle import int8, server

pytestmark = pytest.mark.gpu

COEFFS = tuple(tuple(float(np.float32(v)) for v in step) for step in server.COEFFS)
MLP32 = workload.Config("server-mlp-fp32", (64, 72, 10), workload.FP32, K=4, n_rows=600, batch=16,
                        tau_rule="given", tau_given=(1, 2, 2, 3), lr=0.05, seed=41, mean_scale=0.5)
MLP16 = workload.Config("server-mlp-bf16", (264, 136, 72, 37), workload.BF16, K=3, n_rows=500,
                        batch=32, tau_rule="given", tau_given=(3, 1, 2), lr=0.05, seed=42,
                        mean_scale=0.5)
CNN = workload.Config("server-cnn", (8 * 8 * 3, 10), workload.FP32, K=2, n_rows=200, batch=8,
                      tau_rule="given", tau_given=(2, 1), lr=0.05, seed=43, image=(8, 8, 3),
                      conv=((16, 1), (16, 1), (16, 1, 1), (24, 2)))
OPTS = dict(lr=0.02, beta=0.8, nesterov=True, weight_decay=0.01, plain_lr=0.9)


@pytest.fixture(scope="module")
def R():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2102_08550_amd import rounds
    return rounds


def _matrices(ctx, flat):
    import torch
    return [(torch.from_numpy(w.reshape(w.shape[0], -1).copy()).double(),
             torch.from_numpy(b.copy()).double())
            for w, b in ctx.unpack(flat.cpu().numpy())]


def _assert_step(run, g0, m0):
    layers, mom = _matrices(run.ctx, g0), _matrices(run.ctx, m0)
    reps = [_matrices(run.ctx, r) for r in run.replicas.view(run.cfg.K, -1)]
    new, new_m = server.server_step(layers, reps, run.weights, mom, OPTS["lr"], OPTS["beta"],
                                    OPTS["nesterov"], OPTS["weight_decay"], OPTS["plain_lr"],
                                    coeffs=COEFFS)
    for (gw, gb), (w, b), (mw, _), (m0w, _) in zip(_matrices(run.ctx, run.g), new, new_m, mom):
        d = mw - OPTS["beta"] * m0w
        u = d + OPTS["beta"] * mw
        top = float(gw.abs().max())
        off = 6 * 2.0 ** -24 * top * gw.numel() ** 0.5 / float(u.norm())
        # the kernels' 22-bit products: three roundings a step of 2^-21 of what is
        # kept, grown by the steps behind
        own = 3 * 2.0 ** -21 * sum(4.0 ** k for k in range(6))
        size = min(gw.shape) ** 0.5
        rate = OPTS["lr"] * max(1.0, gw.shape[0] / gw.shape[1]) ** 0.5
        bound = rate * (4.0 ** 5 * off + own) * size + 3 * 2.0 ** -24 * float(gw.norm())
        assert float((gw - w).norm()) <= bound
        assert float((gb - b).abs().max()) <= 16 * 2.0 ** -24 * (1 + float(b.abs().max()))
    for (gw, gb), (w, b) in zip(_matrices(run.ctx, run.momentum), new_m):
        for a, c in ((gw, w), (gb, b)):
            assert float((a - c).abs().max()) <= 8 * 2.0 ** -24 * (1 + float(c.abs().max()))


@pytest.mark.parametrize("cfg", [MLP32, MLP16, CNN], ids=lambda c: c.name)
def test_rounds_with_the_servers_step(R, cfg):
    import torch
    ds, init = workload.gen_dataset(cfg), workload.gen_init(cfg)
    ev = workload.gen_eval_set(cfg, 200)
    x = torch.from_numpy(np.ascontiguousarray(ev.x).view(np.int16) if cfg.dtype == workload.BF16
                         else np.ascontiguousarray(ev.x)).cuda()
    y = torch.from_numpy(ev.y.astype(np.int32)).cuda()
    run, other = R.OscarsRun(cfg, ds, init), R.OscarsRun(cfg, ds, init)
    try:
        for r in range(3):
            say(f"{cfg.name} round {r}")
            g0 = run.g.clone()
            m0 = torch.zeros_like(g0) if run.momentum is None else run.momentum.clone()
            run.round_server(cfg.tau_given, **OPTS)
            _assert_step(run, g0, m0)
            # the same steps one by one, out of place
            R.broadcast(other.g, other.replicas, cfg.K, other.n, other.n)
            other.local_steps(cfg.tau_given)
            out = (torch.empty_like(g0), torch.empty_like(g0))
            other.g, _ = other.ctx.server_step(other.g, other.replicas, other.weights, m0,
                                               out=out, **OPTS)
            assert torch.equal(run.g, other.g) and torch.equal(run.momentum, out[1])
            full = run.evaluate(x, y)
            assert np.isfinite(full[0])
            if cfg.is_cnn:
                continue
            a = ev.x_f32()
            layers = run.global_layers()
            for l, (w, b) in enumerate(layers):
                last = l == len(layers) - 1
                wq, ws = int8.quantize_rows(w)
                q, s = int8.quantize_rows(a)
                z = (q @ wq.T).astype(np.float32) * (s.astype(np.float32)[:, None]
                                                     * ws.astype(np.float32)[None, :]) + b
                a = z if last else np.where(z < 0, np.float32(0), z)
                if cfg.dtype == workload.BF16 and not last:
                    a = torch.from_numpy(a).bfloat16().float().numpy()
            z = a.astype(np.float64)
            mine, top = z[np.arange(len(z)), ev.y], z.max(axis=1)
            loss, hits = run.evaluate(x, y, int8=True)
            want = float((np.log(np.exp(z - top[:, None]).sum(axis=1)) + top - mine).sum())
            assert hits == int((mine == top).sum())
            assert abs(loss - want) <= len(z) * 8 * 2.0 ** -23 * (
                np.abs(z).max() + np.log(cfg.n_classes) + 1)
    finally:
        run.close()
        other.close()


def test_paradigm_with_the_servers_step(R):
    """run_paradigm with a server's step and the quantised evaluation beside the
    ordinary one: the same model as the rounds by hand, both measured each
    round; without them, records as before."""
    import torch
    from paper_2102_08550_amd import controller as C
    cfg = MLP32
    ds, init = workload.gen_dataset(cfg), workload.gen_init(cfg)
    ev = workload.gen_eval_set(cfg, 100)
    sched = C.SpeedSchedule([1, 1, 1, 1])
    res = C.run_paradigm(cfg, ds, init, ev, "local", sched, 1.0, 1e9, local_steps=2, max_rounds=3,
                         return_model=True, server=OPTS, int8_eval=True)
    run = R.OscarsRun(cfg, ds, init)
    try:
        for _ in range(3):
            run.round_server([2] * 4, **OPTS)
        for (a, b), (c, d) in zip(run.global_layers(), res["model"]):
            assert np.array_equal(a, c) and np.array_equal(b, d)
        x, y = torch.from_numpy(ev.x).cuda(), torch.from_numpy(ev.y.astype(np.int32)).cuda()
        loss, hits = run.evaluate(x, y, int8=True)
    finally:
        run.close()
    recs = res["records"]
    assert len(recs) == 4 and all({"eval_loss", "eval_acc", "eval_loss_i8", "eval_acc_i8"} <= set(r)
                                  for r in recs)
    assert recs[-1]["eval_loss_i8"] == loss / 100 and recs[-1]["eval_acc_i8"] == hits / 100
    plain = C.run_paradigm(cfg, ds, init, ev, "local", sched, 1.0, 1e9, local_steps=2, max_rounds=2)
    assert all("eval_loss_i8" not in r for r in plain["records"])


def test_a_captured_round_end(R):
    """The server's step and the quantisation of its result as one graph, replayed
    between rounds of local steps."""
    import torch
    cfg = MLP32
    ds, init = workload.gen_dataset(cfg), workload.gen_init(cfg)
    run, eager = R.OscarsRun(cfg, ds, init), R.OscarsRun(cfg, ds, init)
    side = torch.cuda.Stream()
    try:
        run.momentum, eager.momentum = torch.zeros_like(run.g), torch.zeros_like(run.g)
        run.quantized = run.ctx.quantize_model(run.g)
        main = torch.cuda.current_stream()
        torch.cuda.synchronize()
        run.ctx.set_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            run.ctx.server_step(run.g, run.replicas, run.weights, run.momentum, **OPTS)
            run.ctx.quantize_model(run.g, out=run.quantized)
        run.ctx.set_stream(main)
        for r in range(4):
            R.broadcast(run.g, run.replicas, cfg.K, run.n, run.n)
            run.local_steps(cfg.tau_given)
            graph.replay()
            torch.cuda.synchronize()
            eager.round_server(cfg.tau_given, **OPTS)
            want = eager.ctx.quantize_model(eager.g)
            torch.cuda.synchronize()
            assert torch.equal(run.g, eager.g) and torch.equal(run.momentum, eager.momentum), r
            off = 0
            for o, i in zip(cfg.dims[1:], cfg.dims[:-1]):
                # integers and scales; the layout is 256-byte parts
                n = o * (-(-i // 128) * 128)
                assert torch.equal(run.quantized[off:off + n], want[off:off + n])
                off += -(-n // 256) * 256
                assert torch.equal(run.quantized[off:off + 4 * o], want[off:off + 4 * o])
                off += 2 * (-(-4 * o // 256) * 256)
    finally:
        torch.cuda.synchronize()
        run.close()
        eager.close()


def test_rounds_on_the_contexts_own_stream(R):
    """A context on a stream of its own, rounds called under the default one, with
    other work on it: the rounds' copies follow the context's stream."""
    import torch
    cfg = MLP32
    ds, init = workload.gen_dataset(cfg), workload.gen_init(cfg)
    run, want = R.OscarsRun(cfg, ds, init), R.OscarsRun(cfg, ds, init)
    side = torch.cuda.Stream()
    other = torch.randn(2048, 2048, device="cuda")
    torch.cuda.synchronize()
    run.ctx.set_stream(side)
    try:
        for _ in range(4):
            want.round_server(cfg.tau_given, **OPTS)
        torch.cuda.synchronize()
        for _ in range(4):
            for _ in range(5):
                other = (other @ other).clamp(-1, 1)  # the default stream is behind
            run.round_server(cfg.tau_given, **OPTS)
        torch.cuda.synchronize()
        assert torch.equal(run.g, want.g) and torch.equal(run.momentum, want.momentum)
    finally:
        torch.cuda.synchronize()
        run.close()
        want.close()


def test_a_round_refused_under_capture_leaves_the_run_as_it_was(R):
    """The first round into a graph: the local steps refuse it, and the rounds after
    it are those of a run that never tried."""
    import torch
    cfg = MLP32
    ds, init = workload.gen_dataset(cfg), workload.gen_init(cfg)
    run, want = R.OscarsRun(cfg, ds, init), R.OscarsRun(cfg, ds, init)
    side, main = torch.cuda.Stream(), torch.cuda.current_stream()
    try:
        torch.cuda.synchronize()
        run.ctx.set_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            with pytest.raises(Exception) as ei:
                run.round_server(cfg.tau_given, **OPTS)
        assert "oscars_local_steps" in str(ei.value) and run.momentum is None
        run.ctx.set_stream(main)
        for _ in range(2):
            run.round_server(cfg.tau_given, **OPTS)
            want.round_server(cfg.tau_given, **OPTS)
        torch.cuda.synchronize()
        assert torch.equal(run.g, want.g) and torch.equal(run.momentum, want.momentum)
    finally:
        torch.cuda.synchronize()
        run.close()
        want.close()


def _late(side):
    """Some milliseconds of work, so that what follows on ``side`` runs late."""
    import torch
    with torch.cuda.stream(side):
        a = torch.randn(4096, 4096, device="cuda")
        for _ in range(40):
            a = (a @ a).clamp(-1, 1)
    return a


def test_inputs_dropped_behind_a_call_on_another_stream(R):
    """Tensors that the caller drops while a call on another stream has yet to read
    them: their memory is not given to the caller's own stream meanwhile."""
    import torch
    import paper_2102_08550_amd as P
    torch.manual_seed(3)
    x, g = torch.randn(777, 1000, device="cuda"), torch.randn(500, 640, device="cuda")
    w, ws = P.quantize_rows(torch.randn(300, 1000, device="cuda"))
    xq, xs = P.quantize_rows(x)
    cfg = MLP32
    run = R.OscarsRun(cfg, workload.gen_dataset(cfg), workload.gen_init(cfg))
    side = torch.cuda.Stream()
    mom = torch.zeros_like(run.g)
    reps = run.replicas + 0.01 * torch.randn_like(run.replicas)

    def step(*tensors):
        return run.ctx.server_step(tensors[0], tensors[1], run.weights, tensors[2], lr=0.05,
                                   out=(torch.empty_like(run.g), torch.empty_like(run.g)))

    calls = [("linear_i8", lambda s, a: P.linear_i8(a, w, ws, stream=s), (x,)),
             ("quantize_rows", lambda s, a: P.quantize_rows(a, stream=s), (x,)),
             ("matmul_i8", lambda s, a, b: P.matmul_i8(a, b, w, ws, 1000, stream=s), (xq, xs)),
             ("orthogonalize", lambda s, a: P.orthogonalize(a, stream=s), (g,)),
             ("quantize_model", lambda s, a: run.ctx.quantize_model(a), (run.g,)),
             ("server_step", lambda s, *t: step(*t), (run.g, reps, mom))]
    try:
        for name, call, args in calls:
            run.ctx.set_stream(None)
            want = call(None, *args)
            torch.cuda.synchronize()
            run.ctx.set_stream(side)
            keep = _late(side)
            mine = [a.clone() for a in args]
            side.wait_stream(torch.cuda.current_stream())  # the copies are there
            got = call(side, *mine)
            shapes = [(a.shape, a.dtype) for a in mine]
            del mine
            junk = [torch.full(s, 100, dtype=d, device="cuda") for s, d in shapes]
            torch.cuda.synchronize()
            pairs = zip(want, got) if isinstance(want, tuple) else [(want, got)]
            for a, b in pairs:
                if name == "quantize_model":  # integers of the first layer; the rest has gaps
                    a, b = a[:72 * 128], b[:72 * 128]
                assert torch.equal(a, b), name
            del keep, junk
    finally:
        torch.cuda.synchronize()
        run.close()


def test_a_named_stream_under_capture(R):
    """The operators captured with the capture's stream as an argument, on tensors of
    the default stream and on ones made and dropped during the capture."""
    import torch
    import paper_2102_08550_amd as P
    torch.manual_seed(4)
    x, g = torch.randn(90, 300, device="cuda"), torch.randn(70, 130, device="cuda")
    w, ws = P.quantize_rows(torch.randn(40, 300, device="cuda"))
    out = [torch.empty(90, 40, device="cuda"), torch.empty(90, 40, device="cuda"),
           torch.empty_like(g)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        P.linear_i8(x, w, ws, out=out[0], stream=side)
        xq, xs = P.quantize_rows(x * 2, stream=side)
        P.matmul_i8(xq, xs, w, ws, 300, out=out[1], stream=side)
        del xq, xs
        P.orthogonalize(g + 1, out=out[2], stream=side)
    for k in range(4):
        x.normal_()
        g.normal_()
        want = [P.linear_i8(x, w, ws), P.linear_i8(x * 2, w, ws), P.orthogonalize(g + 1)]
        for o in out:
            o.fill_(-3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out)), f"replay {k}"
    del x, g
    torch.cuda.synchronize()
