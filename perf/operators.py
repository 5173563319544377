"""The operators on the global model after a round's barrier, and how they are measured.

Three operators: the orthogonalisation of updates by Newton-Schulz products, the
server's step that averages the workers, keeps a momentum and applies the
orthogonalised update, and the linear layer in 8-bit integers with a scale for
each row of its input and each output channel.  ``run`` computes them in plain
torch operations or, where ``own`` is set, calls the framework.

Newton-Schulz (``orthogonalize``): for each matrix G, X_0 = G / |G|_F, then
for each step's (a, b, c): A = X X', X <- a X + (b A + c A A) X.

Server step (``server``): avg = sum_k w_k r_k as the framework's pairwise tree,
d = g - avg, m <- beta m + d, u = d + beta m (Nesterov) or m; each weight matrix
W [o][i] <- (1 - lr wd) W - lr sqrt(max(1, o / i)) orth(u), everything else
x <- x - plain_lr u.

Linear layer (``linear_i8``): row r of x has the scale s_r = max |x_r| / 127
(fp32) and the integers round-half-even(x / s_r); y = relu(s_r w_c sum q w + b).

Fields of a case:
  op        "orthogonalize", "server" or "linear_i8"
  shapes    orthogonalize: "512x784,256x512", the matrices of one call
  model     server: "784-512-256-10", an MLP's widths, or
            "32x32x3:32,64s2,64,64r:10", a convolutional model's image, conv
            channels (s2: stride 2, r: ends a residual block) and classes
  workers   server: replicas
  nesterov  server: which update
  decay     server: weight decay
  rows, inputs, outputs, relu     linear_i8
  dtype     "fp32" or "bf16"
"""
import math

import numpy as np
import torch

own = False

COEFFS = ((3.4445, -4.7750, 2.0315),) * 5
LR, BETA, PLAIN_LR = 0.02, 0.9, 0.7
PAD = 64  # a parameter segment starts at a multiple of this many elements


# ------------------------------------------------------------------ the cases

def _orth(name, shapes, dtype):
    return {"name": name, "op": "orthogonalize", "shapes": shapes, "dtype": dtype}


def _server(name, model, workers, nesterov=True, decay=0.0):
    return {"name": name, "op": "server", "model": model, "workers": workers,
            "nesterov": nesterov, "decay": decay, "dtype": "fp32"}


def _linear(name, rows, inputs, outputs, dtype, relu):
    return {"name": name, "op": "linear_i8", "rows": rows, "inputs": inputs, "outputs": outputs,
            "dtype": dtype, "relu": relu}


_RES = "32x32x3:32,32,32r,64s2,64,64r,128s2,128,128r:10"


def listed():
    return [
        # The weight matrices of the small MLP that the paradigms are compared
        # on: the least work, latency counts.
        _orth("orth-mlp-784-fp32", "512x784,256x512,10x256", "fp32"),
        # Matrices of no round size, wide and tall, in bf16.
        _orth("orth-ragged-bf16", "1023x517,37x2050,300x1777", "bf16"),
        # One wide layer's momentum held in bf16.
        _orth("orth-4096-bf16", "4096x4096", "bf16"),
        # Every matrix of the 4096-wide MLP, the largest call.
        _orth("orth-mlp-4096-fp32", "4096x4096,4096x4096,4096x4096,1000x4096", "fp32"),
        # The server's step of the residual network: ten small matrices.
        _server("server-res-k8", _RES, 8),
        # ... of the workload that measures iteration times.
        _server("server-1024-2048-k4", "1024-2048-2048-10", 4, nesterov=False, decay=0.01),
        # ... of the 4096-wide MLP with eight workers.
        _server("server-4096-k8", "4096-4096-4096-4096-1000", 8, decay=0.01),
        # One sample answered by a 4096-wide layer: a stream of weights.
        _linear("linear-1-4096-bf16", 1, 4096, 4096, "bf16", True),
        # A few samples by the small MLP's first layer.
        _linear("linear-17-784-fp32", 17, 784, 512, "fp32", True),
        # A mini-batch's last layer, 1000 classes, fp32 logits.
        _linear("linear-256-4096-1000", 256, 4096, 1000, "fp32", False),
        # Held-out evaluation of a wide layer over an odd number of rows.
        _linear("linear-8191-4096-bf16", 8191, 4096, 4096, "bf16", True),
        # ... of a layer of 2048, fp32 activations.
        _linear("linear-10000-2048-fp32", 10000, 2048, 2048, "fp32", True),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    limit = {}
    for c in listed():
        limit[c["op"]] = max(limit.get(c["op"], 0), work(c)["flops"])
    while True:
        op = rng.choice(["orthogonalize", "server", "linear_i8"])
        if op == "orthogonalize":
            c = {"op": op, "dtype": rng.choice(["fp32", "bf16"]),
                 "shapes": ",".join("%dx%d" % (_log(rng, 8, 4096), _log(rng, 8, 4096))
                                    for _ in range(rng.randint(1, 6)))}
        elif op == "server":
            if rng.random() < 0.3:
                ch = [_log(rng, 4, 32) * 4 for _ in range(3)]
                model = "32x32x3:%d,%ds2,%d,%ds2:%d" % (ch[0], ch[1], ch[1], ch[2],
                                                       _log(rng, 2, 100))
            else:
                model = "-".join(str(8 * _log(rng, 8, 512)) for _ in range(rng.randint(1, 4)))
                model += "-%d" % _log(rng, 2, 1000)
            c = {"op": op, "model": model, "workers": _log(rng, 1, 16),
                 "nesterov": rng.random() < 0.5, "decay": rng.choice([0.0, 0.01]),
                 "dtype": "fp32"}
        else:
            c = {"op": op, "rows": _log(rng, 1, 16384), "inputs": _log(rng, 8, 8192),
                 "outputs": _log(rng, 2, 8192), "dtype": rng.choice(["fp32", "bf16"]),
                 "relu": rng.random() < 0.5}
        if work(c)["flops"] <= limit[op]:
            return c


# ------------------------------------------------------------------ sizes

def _shapes(text):
    return [tuple(int(v) for v in s.split("x")) for s in text.split(",")]


def _model(text):
    """(widths, image and conv layers or None, [(rows, cols) of each weight matrix])."""
    if ":" not in text:
        dims = [int(v) for v in text.split("-")]
        return dims, None, [(o, i) for i, o in zip(dims[:-1], dims[1:])]
    image, conv, classes = text.split(":")
    image = tuple(int(v) for v in image.split("x"))
    layers, mats, cin = [], [], image[2]
    for s in conv.split(","):
        skip, s = s.endswith("r"), s.rstrip("r")
        ch, _, stride = s.partition("s")
        layers.append((int(ch), int(stride or 1), int(skip)))
        mats.append((int(ch), 9 * cin))
        cin = int(ch)
    mats.append((int(classes), cin))
    return [image[0] * image[1] * image[2], int(classes)], (image, tuple(layers)), mats


def _layout(mats):
    """Offsets of (weights, biases) of each layer, and the padded length."""
    at, out = 0, []
    for o, i in mats:
        w = at
        at += -(-o * i // PAD) * PAD
        out.append((w, at))
        at += -(-o // PAD) * PAD
    return out, at


def _orth_flops(shapes):
    """Products of the cheaper of two forms, symmetric results counted by half:
    on X itself, or on the Gram matrix alone with X once at each end."""
    total = 0
    for r, c in shapes:
        m, n, t = min(r, c), max(r, c), len(COEFFS)
        total += min(t * (3 * m * m * n + m ** 3), 3 * m * m * n + (4 * t - 3) * m ** 3)
    return total


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "orthogonalize":
        s = _shapes(case["shapes"])
        return {"bytes": 2 * size * sum(r * c for r, c in s), "flops": _orth_flops(s)}
    if case["op"] == "server":
        mats = _model(case["model"])[2]
        n = _layout(mats)[1]
        return {"bytes": 4 * n * (case["workers"] + 4),
                "flops": _orth_flops(mats) + n * (2 * case["workers"] + 6)}
    b, i, o = case["rows"], case["inputs"], case["outputs"]
    return {"bytes": size * b * (i + o) + i * o + 8 * o, "flops": 2 * b * i * o}


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator("cuda")
    g.manual_seed(seed)
    return g


def _gradient(g, r, c):
    """An averaged gradient: a few strong directions, as classes give, and noise."""
    k = min(8, r, c)
    u = torch.randn(r, k, generator=g, device="cuda")
    v = torch.randn(k, c, generator=g, device="cuda")
    s = 0.5 ** torch.arange(k, device="cuda", dtype=torch.float32)
    return 1e-3 * ((u * s) @ v + 0.3 * torch.randn(r, c, generator=g, device="cuda"))


def _flat(g, mats, spread):
    """A model's parameters: its initialisation, or a gradient in its layout."""
    places, n = _layout(mats)
    out = torch.zeros(n, device="cuda")
    for (o, i), (w, b) in zip(mats, places):
        if spread is None:
            a = 1.0 / math.sqrt(i)
            out[w:w + o * i] = a * (2 * torch.rand(o * i, generator=g, device="cuda") - 1)
            out[b:b + o] = a * (2 * torch.rand(o, generator=g, device="cuda") - 1)
        else:
            out[w:w + o * i] = spread * _gradient(g, o, i).view(-1)
            out[b:b + o] = spread * 1e-3 * torch.randn(o, generator=g, device="cuda")
    return out


def _weights_i8(g, o, i):
    """A layer's weights in integers: rows padded with zeros to 16 bytes, a scale each."""
    a = 1.0 / math.sqrt(i)
    w = (a * (2 * torch.rand(o, i, generator=g, device="cuda") - 1)).double()
    s = (w.abs().amax(1) / 127).float()
    q = torch.zeros(o, -(-i // 16) * 16, dtype=torch.int8, device="cuda")
    q[:, :i] = torch.round(w / s.double()[:, None]).clamp(-127, 127).to(torch.int8)
    return q, s


def _inputs(case, seed):
    g = _gen(seed)
    dt = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    if case["op"] == "orthogonalize":
        return {"x": [_gradient(g, r, c).to(dt) for r, c in _shapes(case["shapes"])]}
    if case["op"] == "server":
        mats, k = _model(case["model"])[2], case["workers"]
        x = _flat(g, mats, None)
        replicas = torch.empty(k * x.numel(), device="cuda")
        for row in replicas.view(k, -1):
            # the worker's steps: its own gradients, and what all workers share
            torch.sub(x, _flat(g, mats, 3.0), out=row)
        return {"global": x, "replicas": replicas, "momentum": _flat(g, mats, 5.0),
                "weights": np.full(k, 1.0 / k, np.float32)}
    b, i, o = case["rows"], case["inputs"], case["outputs"]
    # activations behind a ReLU: half of them zero, some channels stronger
    x = torch.randn(b, i, generator=g, device="cuda").relu_()
    x *= torch.exp(0.5 * torch.randn(i, generator=g, device="cuda"))
    q, s = _weights_i8(g, o, i)
    bias = (2 * torch.rand(o, generator=g, device="cuda") - 1) / math.sqrt(i)
    return {"x": x.to(dt), "wq": q, "wscale": s, "bias": bias}


def prepare(case, seed):
    state = _inputs(case, seed)
    state["case"] = case
    if case["op"] == "server":
        dims, cnn, state["mats"] = _model(case["model"])
        if own:
            import paper_2102_08550_amd as P
            state["ctx"] = P.Context(dims, P.FP32, case["workers"], 8, cnn=cnn)
            state["out"] = (torch.empty_like(state["global"]), torch.empty_like(state["global"]))
    elif own:
        # the tensors that a program hands its results on in
        if case["op"] == "orthogonalize":
            state["out"] = [torch.empty_like(x) for x in state["x"]]
        else:
            state["out"] = torch.empty(case["rows"], case["outputs"], dtype=state["x"].dtype,
                                       device="cuda")
    return state


# ------------------------------------------------------------------ plain forms

def _newton_schulz(g):
    x = g.float()
    tall = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if tall else x
    x = x / torch.sqrt(torch.sum(x.double() * x.double())).float()
    for a, b, c in COEFFS:
        s = x @ x.t()
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.t() if tall else x


def _average(replicas, weights, k):
    """The framework's pairwise tree: leaves w_k r_k, padded to a power of two with zeros."""
    rows = replicas.view(k, -1)
    leaves = [float(weights[j]) * rows[j] for j in range(k)]
    size = 1
    while size < k:
        size *= 2
    leaves += [torch.zeros_like(leaves[0])] * (size - k)
    while len(leaves) > 1:
        leaves = [leaves[j] + leaves[j + 1] for j in range(0, len(leaves), 2)]
    return leaves[0]


def _plain_server(state):
    case, x, m = state["case"], state["global"], state["momentum"]
    d = x - _average(state["replicas"], state["weights"], case["workers"])
    m = BETA * m + d
    u = d + BETA * m if case["nesterov"] else m
    out = x - PLAIN_LR * u
    for (o, i), (w, _) in zip(state["mats"], _layout(state["mats"])[0]):
        t = _newton_schulz(u[w:w + o * i].view(o, i)).reshape(-1)
        out[w:w + o * i] = ((1 - LR * case["decay"]) * x[w:w + o * i]
                            - LR * math.sqrt(max(1.0, o / i)) * t)
    return out, m


def _plain_linear(state):
    x, i = state["x"].float(), state["case"]["inputs"]
    # the quotients in 64 bits: in 32, one next to a half rounds to the other integer
    s = (x.abs().amax(1, keepdim=True).double() / 127).float()
    q = torch.round(x.double() / torch.where(s > 0, s, torch.ones_like(s)).double()).float()
    acc = q @ state["wq"][:, :i].float().t()
    y = acc * (s * state["wscale"]) + state["bias"]
    if state["case"]["relu"]:
        y = torch.clamp_min(y, 0.0)
    return y.to(state["x"].dtype)


def run(state):
    op = state["case"]["op"]
    if own:
        import paper_2102_08550_amd as P
        if op == "orthogonalize":
            return P.orthogonalize(state["x"], out=state["out"], coeffs=COEFFS)
        if op == "server":
            return state["ctx"].server_step(
                state["global"], state["replicas"], state["weights"], state["momentum"], lr=LR,
                beta=BETA, nesterov=state["case"]["nesterov"], weight_decay=state["case"]["decay"],
                plain_lr=PLAIN_LR, coeffs=COEFFS, out=state["out"])
        return P.linear_i8(state["x"], state["wq"], state["wscale"], bias=state["bias"],
                           relu=state["case"]["relu"], out=state["out"])
    if op == "orthogonalize":
        return [_newton_schulz(x).to(x.dtype) for x in state["x"]]
    if op == "server":
        return _plain_server(state)
    return _plain_linear(state)


# ------------------------------------------------------------------ 64 bits

def _orth64(g):
    """From the definition: the polynomial in G's own products, long side last."""
    g = g.double()
    if g.shape[0] > g.shape[1]:
        return _orth64(g.mT.contiguous()).mT
    y = g.div(g.square().sum().sqrt())
    eye = torch.eye(g.shape[0], dtype=torch.float64, device=g.device)
    for a, b, c in COEFFS:
        gram = torch.mm(y, y.mT.contiguous())
        y = torch.mm(a * eye + b * gram + c * torch.mm(gram, gram), y)
    return y


def exact(case, seed):
    data = _inputs(case, seed)
    if case["op"] == "orthogonalize":
        return [_orth64(x) for x in data["x"]]
    if case["op"] == "server":
        mats = _model(case["model"])[2]
        x = data["global"].double()
        avg = torch.zeros_like(x)
        for w, r in zip(data["weights"], data["replicas"].view(case["workers"], -1)):
            avg += float(w) * r.double()
        d = x - avg
        m = d + BETA * data["momentum"].double()
        u = BETA * m + d if case["nesterov"] else m
        y = x - PLAIN_LR * u
        for (o, i), (at, _) in zip(mats, _layout(mats)[0]):
            part = slice(at, at + o * i)
            y[part] = x[part] - LR * (case["decay"] * x[part] + math.sqrt(max(1.0, o / i))
                                      * _orth64(u[part].view(o, i)).reshape(-1))
        return y, m
    x, w = data["x"].double(), data["wq"][:, :case["inputs"]].double()
    s = (x.abs().max(dim=1).values / 127).float().double()  # the scale is held in 32 bits
    q = torch.where(s[:, None] > 0, x / s[:, None], torch.zeros_like(x)).round()
    y = torch.mm(q, w.t().contiguous()) * s[:, None] * data["wscale"].double() + data["bias"].double()
    return y.clamp(min=0) if case["relu"] else y
