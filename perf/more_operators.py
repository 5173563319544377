"""The linear layer in microscaled 4-bit floating point, for answers and for
training, and dropout, and how they are measured.

Five operators: the quantisation to 4 bits and back, the product of quantised
rows, the whole layer, its gradients, and dropout from a counter-based
generator.  ``run`` computes them in plain torch operations or, where ``own`` is
set, calls the framework.

4 bits (``quantize``): 32 consecutive entries of a row share a scale, the
smallest power of two s with max |x| < 7 s; each entry is x / s rounded to the
nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives, ties to the even code.
A block whose largest magnitude is below 2^-126 counts as zeros.  ``columns``
quantises along the columns of x instead and gives the rows of x' in 4 bits.

Layer (``product`` takes quantised rows, ``linear`` quantises them itself):
y = drop(relu(sum_k Q(x)_k Q(w)_k + b)).

Gradients (``backward``, straight through the rounding): dz = dy where the layer
passed its output on, times dropout's factor, held in 32 bits;
dx = Q(dz) Q(w') along the outputs, dw = Q(dz') Q(x') along the rows, db = sum dz.

Dropout (``dropout``): t = round(65536 p); entry (r, c) is dropped where its 16
bits of Philox4x32-10 (Salmon et al., 2011) are below t, and multiplied by
65536 / (65536 - t) (fp32) elsewhere.  Key: the seed; counter: (c / 8, r,
offset's low and high word); entry c takes half c mod 2 (low first) of word
(c mod 8) / 2.

Fields of a case:
  op        "quantize", "product", "linear", "backward" or "dropout"
  rows, inputs, outputs    the layer's sizes (quantize, dropout: rows, inputs)
  dtype     "fp32" or "bf16", of activations and their gradients
  relu      the layer ends in a ReLU
  p         dropout's probability
  columns   quantize: along the columns
"""
import functools
import math

import torch

own = False

OFFSET = 3  # of dropout's counter


# ------------------------------------------------------------------ the cases

def _case(name, op, rows, inputs, outputs, dtype, relu=False, p=0.0, columns=False):
    return {"name": name, "op": op, "rows": rows, "inputs": inputs, "outputs": outputs,
            "dtype": dtype, "relu": relu, "p": p, "columns": columns}


def listed():
    return [
        # Held-out samples of the small MLP's width, to look at what 4 bits keep.
        _case("quantize-10000-784-bf16", "quantize", 10000, 784, 0, "bf16"),
        # A wide layer's weights by input, as the gradient of x takes them.
        _case("quantize-4096-columns-fp32", "quantize", 4096, 4096, 0, "fp32", columns=True),
        # A mini-batch that is quantised already, through the last layer: logits.
        _case("product-256-4096-1000-fp32", "product", 256, 4096, 1000, "fp32"),
        # Held-out evaluation of a wide layer, many rows: matrix work alone.
        _case("product-8192-4096-bf16", "product", 8192, 4096, 4096, "bf16", relu=True),
        # One sample answered by a 4096-wide layer: a stream of weights.
        _case("linear-1-4096-bf16", "linear", 1, 4096, 4096, "bf16", relu=True),
        # A few samples by the small MLP's first layer.
        _case("linear-17-784-512-fp32", "linear", 17, 784, 512, "fp32", relu=True),
        # A training batch of an odd number of rows through a wide layer.
        _case("linear-8191-4096-bf16", "linear", 8191, 4096, 4096, "bf16", relu=True, p=0.1),
        # The gradients of the small MLP's second layer, one mini-batch.
        _case("backward-64-512-256-fp32", "backward", 64, 512, 256, "fp32", relu=True, p=0.25),
        # ... of a wide layer, one worker's mini-batch.
        _case("backward-256-4096-bf16", "backward", 256, 4096, 4096, "bf16", relu=True),
        # ... of a wide layer over a large ragged batch.
        _case("backward-8191-4096-2048-bf16", "backward", 8191, 4096, 2048, "bf16", relu=True,
              p=0.1),
        # A small batch's activations: the least work, latency counts.
        _case("dropout-64-512-fp32", "dropout", 64, 512, 0, "fp32", p=0.25),
        # A large batch's activations of a wide layer.
        _case("dropout-16384-4096-bf16", "dropout", 16384, 4096, 0, "bf16", p=0.1),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    limit = {}
    for c in listed():
        w = work(c)
        limit[c["op"]] = max(limit.get(c["op"], 0), w["flops"] or w["bytes"])
    while True:
        op = rng.choice(["quantize", "product", "linear", "backward", "dropout"])
        flat = op in ("quantize", "dropout")
        c = {"op": op, "rows": _log(rng, 1, 16384), "inputs": _log(rng, 8, 8192),
             "outputs": 0 if flat else _log(rng, 2, 8192),
             "dtype": rng.choice(["fp32", "bf16"]),
             "relu": not flat and rng.random() < 0.7,
             "p": 0.0 if op == "quantize" else rng.choice([0.1, 0.25, 0.5]),
             "columns": op == "quantize" and rng.random() < 0.5}
        if op != "dropout" and rng.random() < 0.5:
            c["p"] = 0.0
        w = work(c)
        if (w["flops"] or w["bytes"]) <= limit[op]:
            return c


def _packed(rows, cols):
    """Bytes of rows in 4 bits: two entries a byte, a scale for each 32."""
    return rows * ((cols + 1) // 2 + (cols + 31) // 32)


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    b, i, o = case["rows"], case["inputs"], case["outputs"]
    if case["op"] == "quantize":  # x, its 4 bits, and the values that they stand for
        there = _packed(i, b) if case["columns"] else _packed(b, i)
        return {"bytes": size * b * i + there + 4 * b * i, "flops": 0}
    if case["op"] == "dropout":
        return {"bytes": 2 * size * b * i, "flops": 0}
    if case["op"] == "backward":
        y = 1 if case["relu"] else 0
        return {"bytes": size * b * (2 * i + (1 + y) * o) + _packed(i, o) + 4 * o * (i + 1),
                "flops": 4 * b * i * o}
    x = _packed(b, i) if case["op"] == "product" else size * b * i
    return {"bytes": x + _packed(o, i) + 4 * o + size * b * o, "flops": 2 * b * i * o}


# ------------------------------------------------------------------ inputs

def _inputs(case, seed):
    g = torch.Generator("cuda")
    g.manual_seed(seed)
    dt = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    b, i, o = case["rows"], case["inputs"], case["outputs"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    # activations: some channels stronger; behind a ReLU where they feed a layer
    x = normal(b, i)
    if case["op"] != "dropout" and not case["columns"]:
        x.relu_()
    x *= torch.exp(0.5 * normal(i))
    data = {"x": x.to(dt), "seed": 1000003 * (seed + 1)}
    if o == 0:
        return data
    data["w"] = (2 * torch.rand(o, i, generator=g, device="cuda") - 1) / math.sqrt(i)
    if case["op"] != "backward":
        data["bias"] = (2 * torch.rand(o, generator=g, device="cuda") - 1) / math.sqrt(i)
        return data
    data["dy"] = (1e-3 * normal(b, o) * torch.exp(0.5 * normal(b, 1))).to(dt)
    if case["relu"]:  # the layer's own output: about half of it is zero
        data["y"] = normal(b, o).relu_().to(dt)
    return data


def prepare(case, seed):
    state = _inputs(case, seed)
    state["case"] = case
    state["dropout"] = (case["p"], state["seed"], OFFSET) if case["p"] > 0 else None
    op = case["op"]
    # what a program keeps between calls: the weights in 4 bits, and the batch
    # where the call takes it quantised
    if own:
        import paper_2102_08550_amd as P
        if op == "backward":
            state["wq"] = P.quantize_mx4(state["w"], transposed=True)
        elif op in ("product", "linear"):
            state["wq"] = P.quantize_mx4(state["w"])
        if op == "product":
            state["xq"] = P.quantize_mx4(state["x"])
    else:
        if op == "backward":
            state["wq"] = _plain_mx4(state["w"].t())
        elif op in ("product", "linear"):
            state["wq"] = _plain_mx4(state["w"])
        if op == "product":
            state["xq"] = _plain_mx4(state["x"])
    return state


# ------------------------------------------------------------------ plain forms

@functools.lru_cache(maxsize=4)
def _powers(device):
    return torch.tensor([2.0 ** k for k in range(-160, 160)], dtype=torch.float64, device=device)


def _plain_mx4(x):
    """The values that the rows of x have in 4 bits, in fp32."""
    x = x.float()
    rows, cols = x.shape
    blocks = -(-cols // 32)
    v = torch.zeros(rows, blocks * 32, device=x.device)
    v[:, :cols] = x
    v = v.view(rows, blocks, 32)
    top = v.abs().amax(2, keepdim=True)
    m, e = torch.frexp(top)  # top = m 2^e, m from 1/2 on
    e = torch.clamp_min(e - 3 + (m >= 0.875).to(e.dtype), -127)
    scale = _powers(x.device)[e.long() + 160]  # exact, which exp2 on a GPU need not be
    v = v.double() / scale
    a = v.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    v = torch.round(v / step) * step * scale
    v = torch.where(top < 2.0 ** -126, torch.zeros_like(v), v)
    return v.view(rows, blocks * 32)[:, :cols].float().contiguous()


def _times(a, c):
    """a c mod 2^32 and a c / 2^32 of a's 32-bit words, in int64."""
    low, high = a & 0xFFFF, a >> 16
    p0, p1 = low * c, high * c
    mid = (p0 >> 16) + (p1 & 0xFFFF)
    return ((mid & 0xFFFF) << 16) | (p0 & 0xFFFF), (p1 >> 16) + (mid >> 16)


def _plain_keep(rows, cols, dropout, device):
    """Where dropout keeps an entry, and the factor there."""
    p, seed, offset = dropout
    t = int(round(65536 * p))
    groups = -(-cols // 8)
    c0 = torch.arange(groups, device=device).expand(rows, groups)
    c1 = torch.arange(rows, device=device)[:, None].expand(rows, groups)
    c2 = torch.full_like(c0, offset & 0xFFFFFFFF)
    c3 = torch.full_like(c0, offset >> 32)
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        l0, h0 = _times(c0, 0xD2511F53)
        l1, h1 = _times(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = torch.stack((c0, c1, c2, c3), 2)
    bits = torch.stack((words & 0xFFFF, words >> 16), 3).reshape(rows, groups * 8)[:, :cols]
    factor = torch.tensor(65536.0 / (65536 - t) if t < 65536 else 0.0, device=device)
    return bits >= t, factor


def _plain_drop(x, dropout):
    if dropout is None:
        return x
    keep, factor = _plain_keep(x.shape[0], x.shape[1], dropout, x.device)
    return torch.where(keep, x * factor, torch.zeros_like(x))


def _plain_layer(state, x):
    y = x @ state["wq"].t() + state["bias"]
    if state["case"]["relu"]:
        y = torch.clamp_min(y, 0.0)
    return _plain_drop(y, state["dropout"]).to(state["x"].dtype)


def _plain_backward(state):
    dy = state["dy"].float()
    if state["case"]["relu"]:  # y says what passed, dropout's choice among it
        t = int(round(65536 * state["case"]["p"]))
        dz = torch.where(state["y"] > 0, dy * torch.tensor(65536.0 / (65536 - t)),
                         torch.zeros_like(dy))
    else:
        dz = _plain_drop(dy, state["dropout"])
    dx = _plain_mx4(dz) @ state["wq"].t()
    dw = _plain_mx4(dz.t()) @ _plain_mx4(state["x"].t()).t()
    return dx.to(state["x"].dtype), dw, dz.double().sum(0).float()


def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        import paper_2102_08550_amd as P
        if op == "quantize":
            q, s = P.quantize_mx4(state["x"], transposed=case["columns"])
            return P.dequantize_mx4(q, s, state["x"].shape[0 if case["columns"] else 1])
        if op == "product":
            return P.matmul_mx4(*state["xq"], *state["wq"], case["inputs"], bias=state["bias"],
                                relu=case["relu"], dropout=state["dropout"],
                                out_dtype=state["x"].dtype)
        if op == "linear":
            return P.linear_mx4(state["x"], *state["wq"], bias=state["bias"], relu=case["relu"],
                                dropout=state["dropout"])
        if op == "backward":
            return P.linear_mx4_backward(state["dy"], state["x"], *state["wq"], y=state.get("y"),
                                         dropout=state["dropout"])
        return P.dropout(state["x"], *state["dropout"])
    if op == "quantize":
        return _plain_mx4(state["x"].t() if case["columns"] else state["x"])
    if op == "product":
        return _plain_layer(state, state["xq"])
    if op == "linear":
        return _plain_layer(state, _plain_mx4(state["x"]))
    if op == "backward":
        return _plain_backward(state)
    return _plain_drop(state["x"].float(), state["dropout"]).to(state["x"].dtype)


# ------------------------------------------------------------------ 64 bits

def _mx4_64(x):
    """Rows in 4 bits from the definition: the least s with max |x| < 7 s, and a
    step up at each border between two values."""
    x = x.double()
    n, c = x.shape
    y = torch.nn.functional.pad(x, (0, -c % 32)).reshape(-1, 32)
    top = y.abs().max(dim=1, keepdim=True).values
    field = torch.floor(torch.log2(top.clamp(min=2.0 ** -126))).long() - 4 + 1023
    s = (field << 52).view(torch.float64)  # a power of two by its exponent
    for _ in range(3):
        s = torch.where(top >= 7 * s, 2 * s, s)
    s = s.clamp(min=2.0 ** -127)
    y = torch.where(top < 2.0 ** -126, torch.zeros_like(y), y / s)
    a = y.abs()
    v = 0.5 * ((a > 0.25).double() + (a >= 0.75) + (a > 1.25) + (a >= 1.75))
    v = v + (a > 2.5).double() + (a >= 3.5).double() + 2.0 * (a > 5)
    return (y.sign() * v * s).reshape(n, -1)[:, :c].contiguous()


def _mulhilo(a, m):
    """High and low word of the product of 32-bit words, which 64 bits hold wrapped."""
    low = (a * m) & 0xFFFFFFFF
    high = ((a >> 8) * m + (((a & 0xFF) * m) >> 8)) >> 24
    return high, low


def _kept64(shape, p, seed, offset):
    """One counter after the other in the order of the entries."""
    n, c = shape
    t = round(p * 65536)
    per = (c + 7) // 8
    at = torch.arange(n * per, device="cuda")
    x = [at % per, at // per, torch.full_like(at, offset % 2 ** 32),
         torch.full_like(at, offset // 2 ** 32)]
    for r in range(10):
        ka = (seed % 2 ** 32 + r * 0x9E3779B9) % 2 ** 32
        kb = (seed // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32
        ha, la = _mulhilo(x[0], 0xD2511F53)
        hb, lb = _mulhilo(x[2], 0xCD9E8D57)
        x = [hb ^ x[1] ^ ka, lb, ha ^ x[3] ^ kb, la]
    halves = torch.empty(n * per, 8, dtype=torch.int64, device="cuda")
    for k in range(4):
        halves[:, 2 * k] = x[k] % 65536
        halves[:, 2 * k + 1] = x[k] // 65536
    kept = (halves.reshape(n, per * 8)[:, :c] >= t).double()
    return kept if t == 65536 else kept * _factor64(p)


def _factor64(p):
    t = round(p * 65536)
    return torch.tensor(65536 / (65536 - t)).double().item()  # held in 32 bits


def exact(case, seed):
    data = _inputs(case, seed)
    x, p = data["x"], case["p"]
    op = case["op"]
    if op == "quantize":
        return _mx4_64(x.mT if case["columns"] else x)
    if op == "dropout":
        return x.double() * _kept64(x.shape, p, data["seed"], OFFSET)
    if op == "backward":
        dz = data["dy"].double()
        if case["relu"]:
            dz = dz * (data["y"] > 0) * _factor64(p)
        elif p > 0:
            dz = dz * _kept64(dz.shape, p, data["seed"], OFFSET)
        held = dz.float()  # in 32 bits
        dx = torch.mm(_mx4_64(held), _mx4_64(data["w"].mT).mT.contiguous())
        dw = torch.mm(_mx4_64(held.mT), _mx4_64(x.mT).mT.contiguous())
        return dx, dw, held.double().sum(dim=0)
    y = torch.mm(_mx4_64(x), _mx4_64(data["w"]).mT.contiguous()) + data["bias"].double()
    if case["relu"]:
        y = y.clamp(min=0)
    return y * _kept64(y.shape, p, data["seed"], OFFSET) if p > 0 else y
