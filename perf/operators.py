"""Layers in the clear, in 8-bit integers, as cases that can be timed and compared.

A network that this library evaluates on ciphertexts has a clear side: layers in front of the bits
that the client encrypts, the clear twin of an encrypted layer, layers behind decrypted scores.
Three operators make it up.

  linear   acc = x w^T in integers (x: [m][k] int8 tokens, w: [n][k] int8 channels), then either
           acc * x_scale[token] * w_scale[channel] + bias as f32, bf16 or f16, or, in whole numbers,
           acc + bias as int32, its sign as +-1 (int8) or as a bit (uint8); sign(0) = +1
  norm     h = x + residual;  y = h / sqrt(mean(h^2) + eps) * weight;  y in 8 bits, a scale a row
  gate     y = act(gate) * up (or act(gate) alone);  y in 8 bits, a scale a row

"In 8 bits, a scale a row": scale = max|y| / 127 and q = y / scale, rounded to the nearest whole
number, ties to even.  q is returned as the values that it stands for, q * scale, in bfloat16 (a
whole number of 8 bits needs no more).
"""
import math

import torch

own = False

EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16,
         "i32": torch.int32, "sign": torch.int8, "bits": torch.uint8}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "i32": 4, "sign": 1, "bits": 1}

# what a drawn case costs at most: the largest listed one of its operator
MOST_PRODUCTS = 8192 * 8192 * 10240
MOST_ELEMENTS = 8192 * 8192


def listed():
    return [
        # one token of a generated answer through a square layer: the weights are read once
        {"name": "linear_token", "op": "linear", "m": 1, "k": 4096, "n": 4096, "out": "bf16", "bias": False},
        # sixteen answers at once through the widening layer of a feed-forward block
        {"name": "linear_16", "op": "linear", "m": 16, "k": 4096, "n": 10240, "out": "f16", "bias": False},
        # the clear twin of the 784 -> 512 layer with +-1 weights, for 64 images: signs for the next layer
        {"name": "linear_sign_784x512", "op": "linear", "m": 64, "k": 784, "n": 512, "out": "sign", "bias": True},
        # exact sums of a tabular layer over a data set, odd sizes: what thresholds are chosen from
        {"name": "linear_sums_1704", "op": "linear", "m": 1999, "k": 1704, "n": 257, "out": "i32", "bias": True},
        # a short prompt, ragged in every direction
        {"name": "linear_333", "op": "linear", "m": 333, "k": 2050, "n": 1111, "out": "f32", "bias": True},
        # a prompt through a square layer
        {"name": "linear_prompt", "op": "linear", "m": 4096, "k": 4096, "n": 4096, "out": "bf16", "bias": False},
        # the largest: a long prompt through the narrowing layer of a feed-forward block
        {"name": "linear_long", "op": "linear", "m": 8192, "k": 10240, "n": 8192, "out": "bf16", "bias": False},
        # one token's norm: a launch and little else
        {"name": "norm_token", "op": "norm", "m": 1, "k": 4096, "type": "bf16", "residual": True},
        # a prompt's norm, rows that are no whole number of vectors
        {"name": "norm_777", "op": "norm", "m": 777, "k": 1001, "type": "f32", "residual": False},
        # a long prompt's norm with the residual stream
        {"name": "norm_long", "op": "norm", "m": 8192, "k": 8192, "type": "bf16", "residual": True},
        # sixteen answers at once between the two products of a feed-forward block
        {"name": "gate_16", "op": "gate", "m": 16, "k": 10240, "type": "bf16", "act": "silu", "up": True},
        # a prompt between the two products
        {"name": "gate_prompt", "op": "gate", "m": 4096, "k": 10240, "type": "f16", "act": "gelu", "up": True},
    ]


def _spread(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["linear", "linear", "norm", "gate"])
    if op == "linear":
        while True:
            case = {"op": op, "m": _spread(rng, 1, 8192), "k": _spread(rng, 64, 10240), "n": _spread(rng, 10, 10240),
                    "out": rng.choice(["f32", "bf16", "f16", "bf16", "i32", "sign", "bits"]), "bias": rng.random() < 0.5}
            if rng.random() < 0.6:          # widths are whole numbers of 64 more often than not
                case["k"], case["n"] = -(-case["k"] // 64) * 64, -(-case["n"] // 64) * 64
            if case["m"] * case["k"] * case["n"] <= MOST_PRODUCTS:
                return case
    while True:
        case = {"op": op, "m": _spread(rng, 1, 8192), "k": _spread(rng, 64, 16384), "type": rng.choice(["f32", "bf16", "f16"])}
        if rng.random() < 0.6:
            case["k"] = -(-case["k"] // 64) * 64
        if op == "norm":
            case["residual"] = rng.random() < 0.6
        else:
            case.update(act=rng.choice(["silu", "gelu", "relu", "identity"]), up=rng.random() < 0.75)
        if case["m"] * case["k"] <= MOST_ELEMENTS // (2 if case["type"] == "f32" else 1):
            return case


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    m, k = case["m"], case["k"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    if case["op"] == "linear":
        n, whole = case["n"], case["out"] in ("i32", "sign", "bits")
        if whole:                           # +-1 inputs and +-1/0 weights, as a binary layer has them
            x = (2 * torch.randint(0, 2, (m, k), generator=g, device="cuda") - 1).to(torch.int8)
            w = (torch.randint(-1, 2, (n, k), generator=g, device="cuda")).to(torch.int8)
            bias = torch.randint(-20, 21, (n,), generator=g, device="cuda", dtype=torch.int32) if case["bias"] else None
            return {"x": x, "w": w, "x_scale": None, "w_scale": None, "bias": bias}
        x = (normal(m, k) * 32).round_().clamp_(-127, 127).to(torch.int8)
        w = (normal(n, k) * 40).round_().clamp_(-127, 127).to(torch.int8)
        return {"x": x, "w": w, "x_scale": 0.02 * torch.exp(0.5 * normal(m)), "w_scale": 0.001 * torch.exp(0.3 * normal(n)),
                "bias": normal(n) if case["bias"] else None}
    t = TYPES[case["type"]]
    # a few channels are an order of magnitude larger than the rest, as a network's activations have them
    spread = torch.where(torch.rand(k, generator=g, device="cuda") < 0.005, 8.0, 1.0)
    if case["op"] == "norm":
        return {"x": normal(m, k).mul_(spread).to(t), "residual": (2 * normal(m, k)).to(t) if case["residual"] else None,
                "weight": (1 + 0.1 * normal(k)).to(t)}
    return {"gate": (2 * normal(m, k)).to(t), "up": normal(m, k).mul_(spread).to(t) if case["up"] else None}


def prepare(case, seed):
    state = dict(case, **_inputs(case, seed))
    m, k = case["m"], case["k"]
    # a serving program keeps the buffers that its layers write
    if case["op"] == "linear":
        state["to"] = torch.empty(m, case["n"], dtype=TYPES[case["out"]], device="cuda")
        return state
    state["q"] = torch.empty(m, k, dtype=torch.int8, device="cuda")
    state["scale"] = torch.empty(m, dtype=torch.float32, device="cuda")
    state["values"] = torch.empty(m, k, dtype=torch.bfloat16, device="cuda")
    if case.get("residual"):
        state["sum"] = torch.empty(m, k, dtype=TYPES[case["type"]], device="cuda")
    return state


def _plain_linear(s):
    if s["out"] in ("i32", "sign", "bits"):     # sums that have to be exact
        acc = s["x"].double() @ s["w"].double().t()
        if s["bias"] is not None:
            acc = acc + s["bias"]
        if s["out"] == "i32":
            return acc.to(torch.int32)
        one = acc >= 0
        return one.to(torch.uint8) if s["out"] == "bits" else (2 * one.to(torch.int8) - 1)
    y = (s["x"].float() @ s["w"].float().t()) * s["x_scale"][:, None] * s["w_scale"]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(TYPES[s["out"]])


def _plain_rows(y):
    scale = y.abs().amax(dim=1, keepdim=True) / 127
    q = torch.round(torch.where(scale > 0, y / scale, torch.zeros_like(y)))
    return {"values": (q * scale).to(torch.bfloat16), "scale": scale[:, 0]}


def _plain_norm(s):
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    y = h * torch.rsqrt((h * h).mean(dim=1, keepdim=True) + EPS) * s["weight"].float()
    got = _plain_rows(y)
    if s["residual"] is not None:
        got["sum"] = h.to(TYPES[s["type"]])
    return got


def _plain_gate(s):
    y = s["gate"].float()
    if s["act"] == "silu":
        y = y / (1 + torch.exp(-y))
    elif s["act"] == "gelu":
        y = 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    elif s["act"] == "relu":
        y = torch.where(y > 0, y, torch.zeros_like(y))
    return _plain_rows(y if s["up"] is None else y * s["up"].float())


def _own(s):
    import paper_1806_03461_amd as T
    if s["op"] == "linear":
        T.bnn_dense_clear(s["x"], s["w"], s["to"], x_scale=s["x_scale"], w_scale=s["w_scale"], bias=s["bias"])
        return s["to"]
    if s["op"] == "norm":
        T.bnn_rms_norm_clear(s["x"], s["weight"], EPS, s["q"], s["scale"], residual=s["residual"], total=s.get("sum"))
    else:
        T.bnn_gate_clear(s["gate"], s["up"], s["act"], s["q"], s["scale"])
    torch.mul(s["q"], s["scale"][:, None], out=s["values"])
    got = {"values": s["values"], "scale": s["scale"]}
    if "sum" in s:
        got["sum"] = s["sum"]
    return got


def run(state):
    if own:
        return _own(state)
    return {"linear": _plain_linear, "norm": _plain_norm, "gate": _plain_gate}[state["op"]](state)


def work(case):
    m, k = case["m"], case["k"]
    if case["op"] == "linear":
        n, whole = case["n"], case["out"] in ("i32", "sign", "bits")
        scales = 0 if whole else 4 * (m + n)
        return {"bytes": m * k + n * k + m * n * SIZE[case["out"]] + scales + (4 * n if case["bias"] else 0), "flops": 2 * m * n * k}
    size = SIZE[case["type"]]
    if case["op"] == "norm":
        # x and weight in, with the residual one row more in and one out; 8 bits a value and a scale a row out
        return {"bytes": m * k * (size * (3 if case["residual"] else 1) + 1) + k * size + 4 * m, "flops": 6 * m * k}
    return {"bytes": m * k * (size * (2 if case["up"] else 1) + 1) + 4 * m, "flops": 10 * m * k}


def _to_8_bits(y):
    """Values and scales of rows in 64 bits, a block of rows at a time in the caller."""
    top = torch.linalg.vector_norm(y, ord=math.inf, dim=1)
    steps = torch.where(top > 0, 127 / top, torch.zeros_like(top))
    return torch.round(y * steps[:, None]) * (top / 127)[:, None], top / 127


def exact(case, seed):
    s, m = _inputs(case, seed), case["m"]
    block = max(1, (1 << 25) // max(case["k"], case.get("n", 1)))
    parts = []
    if case["op"] == "linear":
        wt = s["w"].to(torch.float64).t().contiguous()
        b = None if s["bias"] is None else s["bias"].to(torch.float64)
        for i in range(0, m, block):
            y = torch.matmul(s["x"][i:i + block].to(torch.float64), wt)
            if s["x_scale"] is not None:
                y.mul_(torch.outer(s["x_scale"][i:i + block].double(), s["w_scale"].double()))
            if b is not None:
                y.add_(b)
            if case["out"] == "i32":
                y = y.to(torch.int32)
            elif case["out"] in ("sign", "bits"):
                y = torch.where(y < 0, -1 if case["out"] == "sign" else 0, 1).to(TYPES[case["out"]])
            parts.append(y)
        return torch.cat(parts)
    sums = []
    for i in range(0, m, block):
        at = slice(i, i + block)
        if case["op"] == "norm":
            h = s["x"][at].to(torch.float64)
            if s["residual"] is not None:
                h = h + s["residual"][at].to(torch.float64)
                sums.append(h)
            rms = torch.sqrt(torch.sum(h ** 2, dim=1) / case["k"] + EPS)
            y = s["weight"].to(torch.float64) * (h / rms[:, None])
        else:
            v = s["gate"][at].to(torch.float64)
            y = {"silu": lambda: v * torch.sigmoid(v), "gelu": lambda: v * torch.special.ndtr(v),
                 "relu": lambda: v.clamp(min=0), "identity": lambda: v}[case["act"]]()
            if s["up"] is not None:
                y = y * s["up"][at].to(torch.float64)
        parts.append(_to_8_bits(y))
    got = {"values": torch.cat([p[0] for p in parts]), "scale": torch.cat([p[1] for p in parts])}
    if sums:
        got["sum"] = torch.cat(sums)
    return got
