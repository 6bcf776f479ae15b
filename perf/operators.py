"""The operators of an 8-bit transformer layer as a benchmark sees them: cases, inputs, plain forms, 64-bit values.

Five operators, which a program uses together:

* ``checkpoint``  -- activations to 8-bit codes with one scale per token, and back (what is kept between the two passes);
* ``linear``      -- codes times weights, with scales per token and channel, bias, activation and residual;
* ``gated``       -- both projections of a gated feed-forward block, the activation and the product;
* ``gated_grad``  -- the gradient of that block's two projections, from the codes and the gradient of its output;
* ``product``     -- a bfloat16 gradient times 8-bit codes whose scales lie along the summed axis: the gradient of the
  input (against the weights) and the gradient of the weights (against the kept activations).
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "f16": 2, "bf16": 2}
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def listed():
    return [
        # the tokens of eight sequences in flight, before a projection: latency
        {"name": "checkpoint 8x4096", "op": "checkpoint", "m": 8, "n": 4096, "type": "bf16"},
        # a training batch's activations, kept in 8 bits for the backward pass
        {"name": "checkpoint 16384x4096", "op": "checkpoint", "m": 16384, "n": 4096, "type": "bf16"},
        # one token through an attention block's output projection, onto the residual stream
        {"name": "linear 1x4096x4096", "op": "linear", "m": 1, "n": 4096, "k": 4096, "type": "bf16", "act": "none",
         "bias": False, "residual": True},
        # every edge ragged and no pitch aligned: bias, activation and residual at once, 32-bit output
        {"name": "linear 1000x3001x777", "op": "linear", "m": 1000, "n": 3001, "k": 777, "type": "f32", "act": "gelu",
         "bias": True, "residual": True},
        # a long prompt batch through the second projection of a feed-forward block, onto the residual stream
        {"name": "linear 16384x4096x11008", "op": "linear", "m": 16384, "n": 4096, "k": 11008, "type": "bf16",
         "act": "none", "bias": False, "residual": True},
        # sixteen tokens of as many sequences through a gated block: the weights' bytes count
        {"name": "gated 16x11008x4096", "op": "gated", "m": 16, "f": 11008, "k": 4096, "type": "bf16", "act": "silu"},
        # an encoder-sized block on a short batch
        {"name": "gated 1024x4096x1024", "op": "gated", "m": 1024, "f": 4096, "k": 1024, "type": "f16", "act": "gelu"},
        # a long prompt batch through a large gated block
        {"name": "gated 16384x14336x4096", "op": "gated", "m": 16384, "f": 14336, "k": 4096, "type": "bf16",
         "act": "silu"},
        # the gradient of a small odd-sized block
        {"name": "gated_grad 257x1001x777", "op": "gated_grad", "m": 257, "f": 1001, "k": 777, "type": "f16",
         "act": "gelu_tanh"},
        # the gradient of a large block over a training batch
        {"name": "gated_grad 8192x11008x4096", "op": "gated_grad", "m": 8192, "f": 11008, "k": 4096, "type": "bf16",
         "act": "silu"},
        # gradient of the input of an encoder-sized block: the two projections stacked along the summed axis
        {"name": "product 1024x1024x8192", "op": "product", "m": 1024, "n": 1024, "k": 8192, "type": "bf16",
         "a_order": 0},
        # gradient of the stacked weights of a large block: the sum runs over the tokens of a training batch
        {"name": "product 22016x4096x8192", "op": "product", "m": 22016, "n": 4096, "k": 8192, "type": "bf16",
         "a_order": 1},
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    odd = rng.random() < 0.25          # models' widths are multiples of 16 as a rule

    def width(lo, hi):
        v = spread(lo, hi)
        return v if odd else max(16, v // 16 * 16)

    while True:
        case = {"op": rng.choice(["checkpoint", "linear", "gated", "gated_grad", "product"]), "m": spread(1, 16384),
                "type": rng.choice(["bf16", "bf16", "f16", "f32"])}
        if case["op"] == "checkpoint":
            case.update(n=width(64, 16384))
        elif case["op"] == "linear":
            case.update(n=width(64, 14336), k=width(64, 14336), act=rng.choice(ACTS), bias=rng.random() < 0.5,
                        residual=rng.random() < 0.5)
        elif case["op"] == "gated" or case["op"] == "gated_grad":
            case.update(f=width(64, 14336), k=width(64, 8192), act=rng.choice(ACTS))
        else:                          # both orders of the gradient; its results are held in bfloat16
            case.update(m=width(64, 22016), n=width(64, 8192), k=width(64, 22016), type="bf16",
                        a_order=rng.randrange(2))
        top = max(work(c)["flops"] for c in listed())
        most = max(work(c)["bytes"] for c in listed())
        w = work(case)
        if w["flops"] <= top and w["bytes"] <= most:
            return case


def work(case):
    size = SIZES[case["type"]]
    m = case["m"]
    if case["op"] == "checkpoint":     # in, codes out and in again, out
        n = case["n"]
        return {"bytes": m * n * (2 * size + 2) + 8 * m, "flops": 4 * m * n}
    if case["op"] == "linear":
        n, k = case["n"], case["k"]
        b = m * k + n * k + 4 * (m + n) + size * m * n
        return {"bytes": b + (4 * n if case["bias"] else 0) + (size * m * n if case["residual"] else 0),
                "flops": 2 * m * n * k}
    if case["op"] == "product":
        n, k = case["n"], case["k"]
        return {"bytes": 2 * m * k + n * k + 4 * k + size * m * n, "flops": 2 * m * n * k}
    f, k = case["f"], case["k"]
    tiles = 1 if case["op"] == "gated" else 3
    return {"bytes": m * k + 2 * f * k + 4 * (m + 2 * f) + tiles * size * m * f, "flops": 4 * m * f * k}


def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)

    def codes(rows, cols, spread):     # what rounding normally distributed values to 8 bits gives
        x = torch.randn(rows, cols, device=dev, generator=gen).mul_(spread)
        return x.round_().clamp_(-127, 127).to(torch.int8)

    def scales(n, mean):
        return (torch.rand(n, device=dev, generator=gen) + 0.5) * mean

    def values(rows, cols, kind):
        return torch.randn(rows, cols, device=dev, generator=gen).to(TYPES[kind])

    s = dict(case)
    m, kind = case["m"], case["type"]
    out = TYPES[kind]
    if case["op"] == "checkpoint":
        # tokens of different magnitudes, a few channels far above the rest
        n = case["n"]
        x = torch.randn(m, n, device=dev, generator=gen) * scales(m, 1.0)[:, None]
        x[:, ::97] *= 8
        s.update(x=x.to(out), q=torch.empty(m, n, dtype=torch.int8, device=dev), y=torch.empty(m, n, dtype=out, device=dev),
                 scale=torch.empty(m, dtype=torch.float32, device=dev))
    elif case["op"] == "linear":
        n, k = case["n"], case["k"]
        s.update(a=codes(m, k, 30), a_scale=scales(m, 1 / 30), b=codes(n, k, 40), b_scale=scales(n, 1 / (40 * math.sqrt(k))),
                 bias_v=torch.randn(n, device=dev, generator=gen) if case["bias"] else None,
                 residual_v=values(m, n, kind) if case["residual"] else None,
                 c=torch.empty(m, n, dtype=out, device=dev))
    elif case["op"] == "product":
        # a gradient as it leaves the block's backward pass, and codes with a scale for each row
        n, k = case["n"], case["k"]
        a = values(k, m, "bf16") if case["a_order"] else values(m, k, "bf16")
        s.update(a=a, b=codes(k, n, 30), b_scale=scales(k, 1 / (30 * math.sqrt(k))),
                 c=torch.empty(m, n, dtype=out, device=dev))
    else:
        f, k = case["f"], case["k"]
        # the two projections' weights lie one behind the other, as the input's gradient reads them
        w, w_scale = codes(2 * f, k, 40), scales(2 * f, 1 / (40 * math.sqrt(k)))
        s.update(x=codes(m, k, 30), x_scale=scales(m, 1 / 30), w=w, w_scale=w_scale, wg=w[:f], wu=w[f:],
                 g_scale=w_scale[:f], u_scale=w_scale[f:])
        if case["op"] == "gated":
            s.update(h=torch.empty(m, f, dtype=out, device=dev))
        else:
            d = torch.empty(m, 2 * f, dtype=out, device=dev)
            s.update(dh=values(m, f, kind), dg=d[:, :f], du=d[:, f:])
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _act(x, act):
    if act == "relu":
        return torch.where(x > 0, x, torch.zeros_like(x))
    if act == "gelu":
        return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x)))
    if act == "silu":
        return x / (1 + torch.exp(-x))
    return x


def _slope(x, act):
    if act == "relu":
        return (x > 0).to(x.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) * (1 / math.sqrt(2 * math.pi))
    if act == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x))
        return 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * x * x)
    if act == "silu":
        e = 1 / (1 + torch.exp(-x))
        return e * (1 + x * (1 - e))
    return torch.ones_like(x)


def _plain(s):
    out = TYPES[s["type"]]
    if s["op"] == "checkpoint":
        x = s["x"].float()
        top = x.abs().amax(dim=1)
        scale = top / 127
        q = torch.round(x * (127 / top)[:, None])
        return {"values": (q * scale[:, None]).to(out), "scale": scale}
    if s["op"] == "linear":
        y = (s["a"].float() @ s["b"].float().t()) * s["a_scale"][:, None] * s["b_scale"]
        if s["bias"]:
            y = y + s["bias_v"]
        y = _act(y, s["act"])
        if s["residual"]:
            y = y + s["residual_v"].float()
        return y.to(out)
    if s["op"] == "product":
        a = s["a"].float()
        return ((a.t() if s["a_order"] else a) @ (s["b"].float() * s["b_scale"][:, None])).to(out)
    f = s["f"]
    z = (s["x"].float() @ s["w"].float().t()) * s["x_scale"][:, None] * s["w_scale"]
    g, u = z[:, :f], z[:, f:]
    if s["op"] == "gated":
        return (_act(g, s["act"]) * u).to(out)
    dh = s["dh"].float()
    return {"dg": (dh * u * _slope(g, s["act"])).to(out), "du": (dh * _act(g, s["act"])).to(out)}


# ------------------------------------------------------------------------------------------------ the framework's calls
def _own(s):
    from paper_2506_11728_b200 import binding as mg
    kind = mg.TYPES[s["type"]]
    m = s["m"]
    if s["op"] == "checkpoint":
        n = s["n"]
        mg.mipgemm_quantize_rows(kind, m, n, s["x"], n, s["q"], n, s["scale"])
        mg.mipgemm_dequantize_rows(kind, m, n, s["q"], n, s["scale"], s["y"], n)
        return {"values": s["y"], "scale": s["scale"]}
    if s["op"] == "linear":
        n, k = s["n"], s["k"]
        mg.mipgemm_s8s8_linear(kind, mg.ACTIVATIONS[s["act"]], m, n, k, s["a"], k, s["a_scale"], s["b"], k, s["b_scale"],
                               s["bias_v"], s["residual_v"], n, s["c"], n)
        return s["c"]
    if s["op"] == "product":
        n, k = s["n"], s["k"]
        mg.mipgemm_bf16s8_product(kind, s["a_order"], m, n, k, s["a"], m if s["a_order"] else k, s["b"], n, s["b_scale"],
                                  s["c"], n)
        return s["c"]
    f, k, act = s["f"], s["k"], mg.ACTIVATIONS[s["act"]]
    block = (s["x"], k, s["x_scale"], s["wg"], k, s["g_scale"], s["wu"], k, s["u_scale"])
    if s["op"] == "gated":
        mg.mipgemm_s8s8_gated(kind, act, m, f, k, *block, s["h"], f)
        return s["h"]
    mg.mipgemm_s8s8_gated_grad(kind, act, m, f, k, *block, s["dh"], f, s["dg"], 2 * f, s["du"], 2 * f)
    return {"dg": s["dg"], "du": s["du"]}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op, act = case["op"], case.get("act")
    wide = torch.float64

    def phi(x):                        # the normal distribution's integral
        return torch.special.ndtr(x)

    def cubic(x):
        return 2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)

    def f(x):
        return {"none": lambda: x, "relu": lambda: x.clamp(min=0), "gelu": lambda: x * phi(x),
                "gelu_tanh": lambda: x * torch.sigmoid(cubic(x)), "silu": lambda: x * torch.sigmoid(x)}[act]()

    def df(x):
        if act == "none":
            return torch.ones_like(x)
        if act == "relu":
            return (x > 0).to(wide)
        if act == "gelu":
            return phi(x) + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
        inner = cubic(x) if act == "gelu_tanh" else x
        slope = 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * x * x) if act == "gelu_tanh" else 1.0
        e = torch.sigmoid(inner)
        return e + x * e * (1 - e) * slope

    if op == "checkpoint":
        x = s["x"].to(wide)
        step = x.abs().amax(dim=1, keepdim=True) / 127
        return {"values": torch.round(x / step) * step, "scale": step[:, 0]}
    if op == "product":
        b = s["b_scale"].to(wide)[:, None] * s["b"].to(wide)
        a = s["a"].to(wide)
        return torch.matmul(a.t() if case["a_order"] else a, b)
    if op == "linear":
        left = s["a_scale"].to(wide)[:, None] * s["a"].to(wide)
        z = torch.matmul(left, (s["b_scale"].to(wide)[:, None] * s["b"].to(wide)).t())
        if case["bias"]:
            z += s["bias_v"].to(wide)
        y = f(z)
        if case["residual"]:
            y = y + s["residual_v"].to(wide)
        return y
    x = s["x_scale"].to(wide)[:, None] * s["x"].to(wide)
    w = s["w_scale"].to(wide)[:, None] * s["w"].to(wide)
    g, u = x @ w[:case["f"]].t(), x @ w[case["f"]:].t()
    if op == "gated":
        return f(g) * u
    dh = s["dh"].to(wide)
    return {"dg": dh * u * df(g), "du": dh * f(g)}
