"""The 8-bit operators (rows in 8 bits with a scale each, and the products that read them): their cases, inputs and plain forms.

Three families share one format - a row of int8 values in [-127, 127] with one 32-bit scale:

  norm    h = x + residual, y = h * w / sqrt(mean(h^2) + eps), y's rows in 8 bits; and the gradient
  rows    rows in 8 bits: of a matrix (weights per output channel), or of silu(gate) * up; and the latter's gradient
  linear  y = (xq . wq^T) * token scale * channel scale + bias, the sum of products exact

Rows in 8 bits are returned as the values they stand for, in bf16 (the type in which a fine-tuning step reads them).
"""
import math

import torch

own = False

EPS = 1e-6
F32, BF16 = "f32", "bf16"
TYPES = {F32: torch.float32, BF16: torch.bfloat16}


# ---- cases -------------------------------------------------------------------------------------------------
def listed():
    return [
        # one token in a decoding step: the norm in front of a block, launch latency
        {"name": "norm token", "op": "norm", "rows": 1, "cols": 4096, "type": BF16},
        # a long prompt at an even width: the ordinary large call, bound by memory
        {"name": "norm prompt", "op": "norm", "rows": 16384, "cols": 8192, "type": BF16},
        # a training step of a pruned variant, its width whatever channels were left
        {"name": "norm backward", "op": "norm_back", "rows": 8192, "cols": 4099, "type": BF16},
        # a rebuilt weight matrix in 32 bits, an odd number of rows and columns, quantised per output channel
        {"name": "rows weights", "op": "rows", "rows": 2741, "cols": 5003, "type": F32},
        # one token between the two products of a gated block
        {"name": "rows gate token", "op": "gate", "rows": 1, "cols": 14336, "type": BF16},
        # a long prompt there: gate and up are the halves of one product's output
        {"name": "rows gate prompt", "op": "gate", "rows": 8192, "cols": 14336, "type": BF16},
        # its gradient in a training step
        {"name": "rows gate backward", "op": "gate_back", "rows": 4096, "cols": 11003, "type": BF16},
        # one token against a square layer: the weights are read once
        {"name": "linear token", "op": "linear", "rows": 1, "in": 4096, "out": 4096, "type": BF16, "bias": False},
        # some users' tokens decoded together, a wide layer
        {"name": "linear batch", "op": "linear", "rows": 24, "in": 4096, "out": 14336, "type": BF16, "bias": False},
        # a pruned layer with a bias: odd widths, 32-bit output, a short prompt
        {"name": "linear pruned", "op": "linear", "rows": 333, "in": 5003, "out": 2741, "type": F32, "bias": True},
        # an ordinary prompt
        {"name": "linear prompt", "op": "linear", "rows": 2048, "in": 4096, "out": 4096, "type": BF16, "bias": True},
        # a long prompt through a wide layer: bound by the tensor cores
        {"name": "linear long prompt", "op": "linear", "rows": 8192, "in": 8192, "out": 14336, "type": BF16, "bias": False},
    ]


def _spread(rng, lo, hi):
    """A whole number in [lo, hi], even over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm_back", "rows", "gate", "gate_back", "linear", "linear", "linear"])
    kind = rng.choice([BF16, BF16, F32])
    if op == "linear":
        n_in, n_out = _spread(rng, 64, 14336), _spread(rng, 64, 14336)
        if rng.random() < 0.4:  # widths of a model that was not pruned
            n_in, n_out = max(64, n_in // 64 * 64), max(64, n_out // 64 * 64)
        return {"op": op, "rows": _spread(rng, 1, 4096), "in": n_in, "out": n_out, "type": kind, "bias": rng.random() < 0.5}
    cols = _spread(rng, 64, 14336)
    if rng.random() < 0.4:
        cols = max(64, cols // 64 * 64)
    return {"op": op, "rows": _spread(rng, 1, max(1, min(16384, (1 << 26) // cols))), "cols": cols, "type": kind}


def work(case):
    e = 4 if case["type"] == F32 else 2
    if case["op"] == "linear":
        m, k, n = case["rows"], case["in"], case["out"]
        return {"bytes": m * k + n * k + m * n * e + 4 * (m + n) + (4 * n if case["bias"] else 0), "flops": 2 * m * n * k}
    t, d = case["rows"], case["cols"]
    each = {"norm": (3 * e + 3, 8), "norm_back": (4 * e, 12), "rows": (e + 3, 3), "gate": (2 * e + 3, 8), "gate_back": (5 * e, 14)}[case["op"]]
    vectors = {"norm": 4 * t + 4 * d, "norm_back": 8 * d}.get(case["op"], 4 * t if case["op"] != "gate_back" else 0)
    return {"bytes": t * d * each[0] + vectors, "flops": t * d * each[1]}


# ---- inputs ------------------------------------------------------------------------------------------------
def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _rows_in_8_bits(x):
    """(int8 rows, padded to start on 16 bytes; scales): how a user's quantised tensors look."""
    top = x.abs().amax(1)
    q = torch.round(x * (127.0 / top)[:, None]).to(torch.int8)
    rows, cols = x.shape
    padded = torch.zeros(rows, (cols + 15) // 16 * 16, dtype=torch.int8, device=x.device)
    padded[:, :cols] = q
    return padded, top / 127.0


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind = TYPES[case["type"]]
    s = {}
    if case["op"] == "linear":
        m, k, n = case["rows"], case["in"], case["out"]
        # activations with a few channels much larger than the rest, weights of a trained layer's size
        channel = torch.exp(0.5 * _normal(g, k))
        s["xq"], s["xs"] = _rows_in_8_bits(_normal(g, m, k) * channel)
        s["wq"], s["ws"] = _rows_in_8_bits(_normal(g, n, k) * (k ** -0.5))
        s["bias"] = 0.1 * _normal(g, n) if case["bias"] else None
        return s
    t, d = case["rows"], case["cols"]
    if case["op"] in ("norm", "norm_back"):
        s["weight"] = 1.0 + 0.2 * _normal(g, d)
        channel = torch.exp(0.5 * _normal(g, d))
        if case["op"] == "norm":
            s["x"], s["residual"] = _normal(g, t, d).to(kind), (2.0 * _normal(g, t, d) * channel).to(kind)
        else:
            s["h"], s["dy"], s["dh"] = (2.0 * _normal(g, t, d) * channel).to(kind), _normal(g, t, d).to(kind), _normal(g, t, d).to(kind)
    elif case["op"] == "rows":
        s["x"] = (_normal(g, t, d) * (d ** -0.5)).to(kind)
    else:
        both = torch.empty(t, 2 * d, dtype=kind, device="cuda")  # one product writes both
        both.copy_(_normal(g, t, 2 * d))
        s["gate"], s["up"] = both[:, :d], both[:, d:]
        if case["op"] == "gate_back":
            s["dy"] = _normal(g, t, d).to(kind)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:  # the buffers and handles that a user's program keeps
        from paper_2309_06973_b200 import runtime as R
        kind = TYPES[case["type"]]
        if case["op"] == "linear":
            m, k, n = case["rows"], case["in"], case["out"]
            s["tokens"] = R.RowsQ8.of(s["xq"], s["xs"], k)
            s["layer"] = R.LinearQ8(R.RowsQ8.of(s["wq"], s["ws"], k), s["bias"])
            s["y"] = torch.empty(m, n, dtype=kind, device="cuda")
            return s
        t, d = case["rows"], case["cols"]
        new = lambda: torch.empty(t, d, dtype=kind, device="cuda")  # noqa: E731
        if case["op"] in ("norm", "rows", "gate"):
            s["out"] = R.RowsQ8(t, d, values=True)
        if case["op"] == "norm":
            s["h"] = new()
        elif case["op"] == "norm_back":
            s["dx"], s["dw"] = new(), torch.empty(d, device="cuda")
            s["space"] = R.rmsnorm_q8_backward_workspace(t, d)
        elif case["op"] == "gate_back":
            both = torch.empty(t, 2 * d, dtype=kind, device="cuda")
            s["dgate"], s["dup"] = both[:, :d], both[:, d:]
        s["R"] = R
    return s


# ---- one pass ----------------------------------------------------------------------------------------------
def _plain_values(y):
    top = y.abs().amax(1, keepdim=True)
    scale = top / 127.0
    q = torch.where(top > 0, torch.round(y * (127.0 / top)), torch.zeros_like(y))
    return (q * scale).to(torch.bfloat16), scale[:, 0]


def _plain(s):
    case = s["case"]
    op, kind = case["op"], TYPES[case["type"]]
    if op == "linear":
        k = case["in"]
        y = (s["xq"][:, :k].float() @ s["wq"][:, :k].float().t()) * s["xs"][:, None] * s["ws"][None, :]
        return {"y": (y if s["bias"] is None else y + s["bias"]).to(kind)}
    if op == "norm":
        h = s["x"].float() + s["residual"].float()
        values, scale = _plain_values(h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["weight"])
        return {"h": h.to(kind), "values": values, "scale": scale}
    if op == "norm_back":
        h, dy = s["h"].float(), s["dy"].float()
        r = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
        g = dy * s["weight"]
        dx = r * g - h * (r * r * r * (g * h).mean(1, keepdim=True)) + s["dh"].float()
        return {"dx": dx.to(kind), "dw": (dy * h * r).sum(0)}
    if op == "rows":
        values, scale = _plain_values(s["x"].float())
        return {"values": values, "scale": scale}
    gate, up = s["gate"].float(), s["up"].float()
    sig = 1.0 / (1.0 + torch.exp(-gate))
    if op == "gate":
        values, scale = _plain_values(gate * sig * up)
        return {"values": values, "scale": scale}
    dy = s["dy"].float()
    return {"dgate": (dy * up * sig * (1.0 + gate * (1.0 - sig))).to(kind), "dup": (dy * gate * sig).to(kind)}


def run(s):
    if not own:
        return _plain(s)
    op = s["case"]["op"]
    if op == "linear":
        s["layer"](s["tokens"], s["y"])
        return {"y": s["y"]}
    R = s["R"]
    if op == "norm":
        R.rmsnorm_q8(s["x"], s["weight"], EPS, s["out"], residual=s["residual"], h=s["h"])
        return {"h": s["h"], "values": s["out"].values, "scale": s["out"].scale}
    if op == "norm_back":
        R.rmsnorm_q8_backward(s["dy"], s["h"], s["weight"], EPS, s["dx"], s["dw"], dh=s["dh"], workspace=s["space"])
        return {"dx": s["dx"], "dw": s["dw"]}
    if op == "gate_back":
        R.silu_gate_q8_backward(s["dy"], s["gate"], s["up"], s["dgate"], s["dup"])
        return {"dgate": s["dgate"], "dup": s["dup"]}
    if op == "rows":
        R.quantize_rows(s["x"], s["out"])
    else:
        R.silu_gate_q8(s["gate"], s["up"], s["out"])
    return {"values": s["out"].values, "scale": s["out"].scale}


# ---- the definition in 64 bits -----------------------------------------------------------------------------
def exact(case, seed):
    s = {k: v.double() if torch.is_tensor(v) else v for k, v in _inputs(case, seed).items()}
    op = case["op"]

    def rounded(y):  # a row's largest magnitude becomes 127 steps
        step = torch.linalg.vector_norm(y, ord=math.inf, dim=1) / 127
        return {"values": torch.round(y / step.unsqueeze(1)) * step.unsqueeze(1), "scale": step}

    if op == "linear":
        k = case["in"]
        y = torch.mm(s["xq"][:, :k], s["wq"][:, :k].T)
        y.mul_(s["xs"].unsqueeze(1)).mul_(s["ws"])
        return {"y": y if s["bias"] is None else y.add_(s["bias"])}
    if op == "norm":
        h = s["residual"] + s["x"]
        root = torch.sqrt(torch.linalg.vector_norm(h, dim=1, keepdim=True).square() / case["cols"] + EPS)
        return {"h": h, **rounded(h / root * s["weight"])}
    if op == "norm_back":
        n = case["cols"]
        root = torch.sqrt(torch.linalg.vector_norm(s["h"], dim=1, keepdim=True).square() / n + EPS)
        unit = s["h"] / root
        g = s["weight"] * s["dy"]
        along = torch.linalg.vecdot(g, unit, dim=1).unsqueeze(1) / n
        return {"dx": (g - unit * along) / root + s["dh"], "dw": torch.einsum("td,td->d", s["dy"], unit)}
    if op == "rows":
        return rounded(s["x"])
    half = torch.tanh(s["gate"] / 2)  # sigmoid(g) = (1 + tanh(g / 2)) / 2
    act = s["gate"] * (1 + half) / 2
    if op == "gate":
        return rounded(act * s["up"])
    slope = (1 + half) / 2 + s["gate"] * (1 - half * half) / 4
    return {"dgate": s["dy"] * s["up"] * slope, "dup": s["dy"] * act}
