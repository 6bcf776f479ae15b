"""Operators of a transformer layer in 8-bit floating point as a benchmark sees them: cases, inputs, plain forms, 64-bit values.

Five operators, which a program uses together:

* ``codes``     -- a matrix to 8-bit floating point with a float32 scale for each block of 128 and back: blocks along the rows
  (operands of the forward pass), along the columns (operands of the weights' gradient), both from one reading, or squares
  (weights, which are read along either axis);
* ``product``   -- C (+)= A B of such codes: the forward product, the gradient of the input (against the weights as they lie)
  and the gradient of the weights (the sum runs over the tokens);
* ``step``      -- what stands between two blocks: y = s x + dropout(gate * norm(z)), h = norm(y), h also as codes;
* ``step_grad`` -- its backward pass, the gradients of gate, weights and biases included;
* ``dropout``   -- the same step without norms: a block's output onto the residual stream through a mask that is drawn from
  a counter and never stored, and the gradient through the same mask.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "f16": 2, "bf16": 2}
FORMATS = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}
LEAST = {"e4m3": 2.0 ** -119, "e5m2": 2.0 ** -112}       # blocks below this hold zeros
NORMS = ("none", "rms", "layer")
EPS = 1e-5


def listed():
    return [
        # the tokens of eight sequences in flight, before a projection: latency
        {"name": "codes 8x4096", "op": "codes", "m": 8, "n": 4096, "type": "bf16", "format": "e4m3", "form": "rows"},
        # a training batch's activations: codes along the rows for this product, along the columns for the weights' gradient
        {"name": "codes 16384x4096", "op": "codes", "m": 16384, "n": 4096, "type": "bf16", "format": "e4m3", "form": "both"},
        # one token through a projection: the weights' bytes count
        {"name": "product 1x4096x4096", "op": "product", "m": 1, "n": 4096, "k": 4096, "type": "bf16", "what": "forward",
         "a_format": "e4m3", "bias": False, "accumulate": False},
        # every edge ragged, no pitch aligned, a bias, 32-bit output
        {"name": "product 1000x3001x777", "op": "product", "m": 1000, "n": 3001, "k": 777, "type": "f32", "what": "forward",
         "a_format": "e4m3", "bias": True, "accumulate": False},
        # a long prompt batch through the second projection of a feed-forward block
        {"name": "product 16384x4096x11008", "op": "product", "m": 16384, "n": 4096, "k": 11008, "type": "bf16",
         "what": "forward", "a_format": "e4m3", "bias": False, "accumulate": False},
        # gradient of a projection's weights over a training batch, added to what earlier batches gave
        {"name": "product 11008x4096x8192", "op": "product", "m": 11008, "n": 4096, "k": 8192, "type": "f32",
         "what": "weight_grad", "a_format": "e5m2", "bias": False, "accumulate": True},
        # eight tokens between two blocks of a decoder, straight to the next projection's codes: latency
        {"name": "step 8x4096", "op": "step", "m": 8, "n": 4096, "type": "bf16", "post": "none", "pre": "rms", "gate": 0,
         "drop": 0.0, "scale": 1.0, "codes": "e4m3"},
        # a training batch between two blocks: norms on both sides, a gate for each channel, dropout
        {"name": "step 16384x4096", "op": "step", "m": 16384, "n": 4096, "type": "bf16", "post": "rms", "pre": "rms",
         "gate": 16384, "drop": 0.1, "scale": 1.0, "codes": "none"},
        # the gradient at an odd width: means subtracted, a gate for each sequence of 64 tokens
        {"name": "step_grad 257x1001", "op": "step_grad", "m": 257, "n": 1001, "type": "f32", "post": "layer", "pre": "layer",
         "gate": 64, "drop": 0.1, "scale": 0.5},
        # the gradient over a training batch
        {"name": "step_grad 16384x4096", "op": "step_grad", "m": 16384, "n": 4096, "type": "bf16", "post": "rms",
         "pre": "rms", "gate": 16384, "drop": 0.1, "scale": 1.0},
        # an encoder-sized block's output onto the residual stream, a short batch
        {"name": "dropout 512x768", "op": "dropout", "m": 512, "n": 768, "type": "f16", "drop": 0.1},
        # a large training batch
        {"name": "dropout 16384x8192", "op": "dropout", "m": 16384, "n": 8192, "type": "bf16", "drop": 0.1},
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    odd = rng.random() < 0.25          # models' widths are multiples of 16 as a rule

    def width(lo, hi):
        v = spread(lo, hi)
        return v if odd else max(16, v // 16 * 16)

    while True:
        case = {"op": rng.choice(["codes", "product", "product", "step", "step_grad", "dropout"]), "m": spread(1, 16384),
                "type": rng.choice(["bf16", "bf16", "f16", "f32"])}
        if case["op"] == "codes":
            case.update(n=width(64, 16384), format=rng.choice(["e4m3", "e4m3", "e5m2"]),
                        form=rng.choice(["rows", "columns", "both", "squares"]))
        elif case["op"] == "product":
            what = rng.choice(["forward", "forward", "input_grad", "weight_grad"])
            if what == "weight_grad":          # its rows are channels, the sum runs over the tokens
                case.update(m=width(64, 14336), k=spread(1, 16384))
            else:
                case.update(k=width(64, 14336))
            case.update(n=width(64, 14336), what=what, a_format="e4m3" if what == "forward" else rng.choice(["e4m3", "e5m2"]),
                        bias=what == "forward" and rng.random() < 0.5, accumulate=rng.random() < 0.3)
        elif case["op"] == "dropout":
            case.update(n=width(64, 16384), drop=rng.choice([0.05, 0.1, 0.25, 0.5]))
        else:
            m = case["m"]
            case.update(n=width(64, 16384), post=rng.choice(NORMS), pre=rng.choice(NORMS),
                        gate=rng.choice([0, 1, m, max(1, m // rng.randint(2, 9))]), drop=rng.choice([0.0, 0.1, 0.3]),
                        scale=rng.choice([1.0, 1.0, 0.5]))
            if case["op"] == "step":
                case.update(codes=rng.choice(["none", "s8", "e4m3"]) if case["pre"] != "none" and case["type"] != "f32"
                            else "none")
        top = max(work(c)["flops"] for c in listed())
        most = max(work(c)["bytes"] for c in listed())
        w = work(case)
        if w["flops"] <= top and w["bytes"] <= most:
            return case


def _blocks(n):
    return (n + 127) // 128


def work(case):
    m, n, size = case["m"], case["n"], SIZES[case["type"]]
    if case["op"] == "codes":          # in; codes out and in again, out
        sets = 2 if case["form"] == "both" else 1
        return {"bytes": m * n * (size + sets * (2 + size)) + 8 * sets * m * n // 128, "flops": 4 * sets * m * n}
    if case["op"] == "product":
        k = case["k"]
        scales = m * _blocks(k) + (n * _blocks(k) if case["what"] == "weight_grad" else _blocks(n) * _blocks(k))
        b = m * k + n * k + 4 * scales + size * m * n * (2 if case["accumulate"] else 1) + (4 * n if case["bias"] else 0)
        return {"bytes": b, "flops": 2 * m * n * k}
    if case["op"] == "dropout":        # there: x, z in and y out; back: dy in and dz out
        return {"bytes": 5 * size * m * n, "flops": 5 * m * n}
    gate = _blocks_of(m, case["gate"]) * n * size
    vectors = (4 * n if case["post"] != "none" else 0) + (4 * n if case["pre"] != "none" else 0)
    pre = case["pre"] != "none"
    if case["op"] == "step":
        out = size + ((1 if case["codes"] != "none" else size) if pre else 0)
        return {"bytes": m * n * (2 * size + out) + gate + vectors, "flops": 16 * m * n}
    return {"bytes": m * n * size * ((3 if pre else 1) + 3) + 2 * (gate + vectors), "flops": 32 * m * n}


def _blocks_of(m, rows):
    return (m + rows - 1) // rows if rows else 0


def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, device=dev, generator=gen)

    def scales(n, mean):
        return (torch.rand(n, device=dev, generator=gen) + 0.5) * mean

    def tokens(rows, cols):            # of different magnitudes, a few channels far above the rest
        x = normal(rows, cols) * scales(rows, 1.0)[:, None]
        x[:, ::97] *= 8
        return x

    s = dict(case)
    m, n, op, out = case["m"], case["n"], case["op"], TYPES[case["type"]]

    def values(rows=m, cols=n):
        return normal(rows, cols).to(out)

    def room(rows=m, cols=n, kind=out):
        return torch.empty(rows, cols, dtype=kind, device=dev)

    if op == "codes":
        fmt = FORMATS[case["format"]]
        s["x"] = tokens(m, n).to(out)
        for side in ("rows", "columns", "squares"):
            if case["form"] in (side, "both") and not (case["form"] == "both" and side == "squares"):
                shape = {"rows": (_blocks(n), m), "columns": (_blocks(m), n), "squares": (_blocks(m), _blocks(n))}[side]
                s.update({side + "_q": room(kind=fmt), side + "_scale": room(*shape, kind=torch.float32), side + "_y": room()})
    elif op == "product":
        k, what = case["k"], case["what"]
        a_cols, b_cols = what == "weight_grad", what != "forward"

        def operand(rows, cols, form, fmt, mean):
            x = tokens(rows, cols) * mean
            codes, scale = _encode(x, form, fmt)
            return codes, scale
        s["a"], s["a_scale"] = operand(*((k, m, "columns") if a_cols else (m, k, "rows")), case["a_format"], 1.0)
        s["b"], s["b_scale"] = operand(*((k, n) if b_cols else (n, k)), "columns" if a_cols else "squares", "e4m3",
                                       1 / math.sqrt(k))
        s["bias_v"] = normal(n) if case["bias"] else None
        s["before"] = values() if case["accumulate"] else None
        s["c"] = room()
    elif op == "dropout":
        s.update(x=values(), z=values(), dy=values(), y=room(), dz=room(), key=int(seed) * 2 + 1,
                 counter=torch.tensor([seed % 1000], dtype=torch.int64, device=dev))
    else:
        post, pre = case["post"], case["pre"]
        s.update(x=tokens(m, n).to(out), z=values(), key=int(seed) * 2 + 1,
                 counter=torch.tensor([seed % 1000], dtype=torch.int64, device=dev),
                 gate_v=values(_blocks_of(m, case["gate"]), n) if case["gate"] else None,
                 post_w=1 + 0.1 * normal(n) if post != "none" else None, post_b=0.1 * normal(n) if post == "layer" else None,
                 pre_w=1 + 0.1 * normal(n) if pre != "none" else None, pre_b=0.1 * normal(n) if pre == "layer" else None)
        s["y"] = room()
        if op == "step":
            s["stats"] = room(m, 4, torch.float32) if case["codes"] == "none" else None
            if pre != "none":
                s["h"] = room() if case["codes"] == "none" else None
                if case["codes"] != "none":
                    s["q"] = room(kind=torch.int8 if case["codes"] == "s8" else FORMATS[case["codes"]])
                    s["q_scale"] = room(1 if case["codes"] == "s8" else _blocks(n), m, torch.float32)
                    s["back"] = room()
        else:
            # what the forward pass left: y, and the rows' statistics
            st = _step(dict(s, codes="none"), torch.float32)
            s.update(y=st["y"].to(out), stats=st["stats"], dy=values(), dh=values() if pre != "none" else None,
                     dx=room(), dz=room(), dgate=torch.empty_like(s["gate_v"]) if case["gate"] else None)
            for name in ("post_w", "post_b", "pre_w", "pre_b"):
                s["d" + name] = torch.empty_like(s[name]) if s[name] is not None else None
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _split(x, form):
    """x, filled up with zeros, by blocks: the axes to reduce over come last."""
    m, n = x.shape
    rows, cols = {"rows": (1, 128), "columns": (128, 1), "squares": (128, 128)}[form]
    x = torch.nn.functional.pad(x, (0, -n % cols, 0, -m % rows))
    return x.reshape(x.shape[0] // rows, rows, x.shape[1] // cols, cols)


def _join(b, m, n):
    return b.reshape(b.shape[0] * b.shape[1], -1)[:m, :n]


def _encode(x, form, fmt):
    """Codes of x, and the scales as they are kept: [column block][row], [row block][column] or [row block][column block]."""
    m, n = x.shape
    b = _split(x.float(), form)
    top = b.abs().amax(dim=(1, 3), keepdim=True)
    live = top >= LEAST[fmt]
    most = torch.full_like(top, LARGEST[fmt])
    mult = torch.where(live, most / top, torch.zeros_like(top))
    scale = torch.where(live, top / most, torch.zeros_like(top))
    q = _join(b * mult, m, n).to(FORMATS[fmt])
    scale = scale[:, 0, :, 0]
    return q, (scale.t() if form == "rows" else scale).contiguous()


def _decode(q, scale, form):
    """The float32 values that codes stand for."""
    m, n = q.shape
    scale = scale.t() if form == "rows" else scale
    return _join(_split(q.float(), form) * scale[:, None, :, None], m, n)


def _philox(counter, key):
    """Philox 4x32-10 on four int64 tensors that hold 32-bit words."""
    low = 0xFFFFFFFF

    def product(a, c):                 # high and low word of the 64-bit product, by 16-bit halves of the constant
        p0, p1 = a * (c & 0xFFFF), a * (c >> 16)
        mid = (p0 >> 16) + p1
        return mid >> 16, ((mid & 0xFFFF) << 16) | (p0 & 0xFFFF)

    c0, c1, c2, c3 = counter
    k0, k1 = key & low, key >> 32 & low

    def after(c0, c1, c2, c3, k0, k1):
        h0, l0 = product(c0, 0xD2511F53)
        h1, l1 = product(c2, 0xCD9E8D57)
        return h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0

    for r in range(10):
        c0, c1, c2, c3 = after(c0, c1, c2, c3, (k0 + r * 0x9E3779B9) & low, (k1 + r * 0xBB67AE85) & low)
    return c0, c1, c2, c3


def _kept(m, n, drop, key, counter):
    """1 / (1 - rate) where an element is kept, 0 where it is dropped."""
    bar = round(drop * 65536)          # the rate is a multiple of 2^-16
    groups = (n + 7) // 8
    g = torch.arange(m * groups, device=counter.device, dtype=torch.int64)
    step = counter.expand(m * groups)
    words = torch.stack(_philox((g & 0xFFFFFFFF, g >> 32, step & 0xFFFFFFFF, step >> 32), key), dim=1)
    halves = torch.stack((words & 0xFFFF, words >> 16), dim=2).reshape(m, groups * 8)[:, :n]
    return (halves >= bar).float() * (65536.0 / (65536 - bar))


def _norm(x, kind, w, b):
    mean = x.mean(dim=1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
    d = x - mean
    rstd = 1 / torch.sqrt((d * d).mean(dim=1, keepdim=True) + EPS)
    y = d * rstd * w
    return (y + b if b is not None else y), mean, rstd


def _spread(v, m, rows):
    """Rows of a gate by row of the matrix it applies to."""
    return v if rows == 1 else v.repeat_interleave(rows, dim=0)[:m]


def _step(s, wide):
    m = s["m"]
    none = torch.zeros(m, 1, dtype=wide, device=s["z"].device)
    v, pm, pr = s["z"].to(wide), none, none
    if s["post"] != "none":
        v, pm, pr = _norm(v, s["post"], s["post_w"], s["post_b"])
    if s["gate"]:
        v = v * _spread(s["gate_v"].to(wide), m, s["gate"])
    if s["drop"]:
        v = v * _kept(m, s["n"], s["drop"], s["key"], s["counter"])
    y = s["scale"] * s["x"].to(wide) + v
    r, qm, qr = {"y": y}, none, none
    if s["pre"] != "none":
        r["h"], qm, qr = _norm(y, s["pre"], s["pre_w"], s["pre_b"])
    r["stats"] = torch.cat((pm, pr, qm, qr), dim=1)
    return r


def _back(g, hat, rstd, kind):
    """Through a norm: gradient of its input from g = w * gradient of its output."""
    d = g - hat * (g * hat).mean(dim=1, keepdim=True)
    if kind == "layer":
        d = d - g.mean(dim=1, keepdim=True)
    return d * rstd


def _sums(x, rows):
    """Sums over groups of rows."""
    m, n = x.shape
    return torch.nn.functional.pad(x, (0, 0, 0, -m % rows)).reshape(-1, rows, n).sum(dim=1)


def _plain(s):
    op, out, m, n = s["op"], TYPES[s["type"]], s["m"], s["n"]
    if op == "codes":
        forms = ("rows", "columns") if s["form"] == "both" else (s["form"],)
        r = {}
        for form in forms:
            q, scale = _encode(s["x"], form, s["format"])
            r[form] = {"values": _decode(q, scale, form).to(out), "scale": scale}
        return r
    if op == "product":
        over = s["what"] == "weight_grad"
        a = _decode(s["a"], s["a_scale"], "columns" if over else "rows")
        b = _decode(s["b"], s["b_scale"], "columns" if over else "squares")
        c = (a.t() if over else a) @ (b.t() if s["what"] == "forward" else b)
        if s["bias"]:
            c = c + s["bias_v"]
        if s["accumulate"]:
            c = c + s["before"].float()
        return c.to(out)
    if op == "dropout":
        keep = _kept(m, n, s["drop"], s["key"], s["counter"])
        return {"y": (s["x"].float() + keep * s["z"].float()).to(out), "dz": (keep * s["dy"].float()).to(out)}
    if op == "step":
        r = _step(s, torch.float32)
        if s["codes"] == "none":
            return {k: v if k == "stats" else v.to(out) for k, v in r.items()}
        h = r["h"]
        if s["codes"] == "s8":
            top = h.abs().amax(dim=1)
            back, scale = torch.round(h * (127 / top)[:, None]) * (top / 127)[:, None], (top / 127)[None]
        else:
            q, scale = _encode(h, "rows", s["codes"])
            back = _decode(q, scale, "rows")
        return {"y": r["y"].to(out), "values": back.to(out), "scale": scale}
    dy, r = s["dy"].float(), {}
    pm, pr, qm, qr = s["stats"].split(1, dim=1)
    if s["pre"] != "none":
        dh, hat = s["dh"].float(), (s["y"].float() - qm) * qr
        dy = dy + _back(dh * s["pre_w"], hat, qr, s["pre"])
        r["dpre_w"] = (dh * hat).sum(dim=0)
        if s["pre"] == "layer":
            r["dpre_b"] = dh.sum(dim=0)
    r["dx"] = (s["scale"] * dy).to(out)
    g = dy * _kept(m, n, s["drop"], s["key"], s["counter"]) if s["drop"] else dy
    u = hat = s["z"].float()
    if s["post"] != "none":
        hat = (u - pm) * pr
        u = hat * s["post_w"]
        if s["post"] == "layer":
            u = u + s["post_b"]
    if s["gate"]:
        r["dgate"] = _sums(g * u, s["gate"]).to(out)
        g = g * _spread(s["gate_v"].float(), m, s["gate"])
    if s["post"] != "none":
        r["dpost_w"] = (g * hat).sum(dim=0)
        if s["post"] == "layer":
            r["dpost_b"] = g.sum(dim=0)
        g = _back(g * s["post_w"], hat, pr, s["post"])
    r["dz"] = g.to(out)
    return r


# ------------------------------------------------------------------------------------------------ the framework's calls
def _own(s):
    from paper_2506_11728_b200 import binding as mg
    kind, op, m, n = mg.TYPES[s["type"]], s["op"], s["m"], s["n"]
    if op == "codes":
        fmt, form = mg.F8_FORMATS[s["format"]], s["form"]
        if form == "squares":
            mg.mipgemm_f8_quantize_squares(kind, fmt, m, n, s["x"], n, s["squares_q"], n, s["squares_scale"], _blocks(n))
        else:
            rows, cols = form in ("rows", "both"), form in ("columns", "both")
            mg.mipgemm_f8_quantize(kind, fmt, m, n, s["x"], n, s["rows_q"] if rows else None, n,
                                   s["rows_scale"] if rows else None, m, s["columns_q"] if cols else None, n,
                                   s["columns_scale"] if cols else None, n)
        r = {}
        for side in ("rows", "columns") if form == "both" else (form,):
            scale = s[side + "_scale"]
            mg.mipgemm_f8_dequantize(kind, fmt, mg.F8_BLOCKS[side], m, n, s[side + "_q"], n, scale, scale.shape[1],
                                     s[side + "_y"], n)
            r[side] = {"values": s[side + "_y"], "scale": scale}
        return r
    if op == "product":
        k, what = s["k"], s["what"]
        a_order = mg.MN_CONTIGUOUS if what == "weight_grad" else mg.K_CONTIGUOUS
        b_order = mg.K_CONTIGUOUS if what == "forward" else mg.MN_CONTIGUOUS
        mg.mipgemm_f8f8_product(kind, mg.F8_FORMATS[s["a_format"]], mg.F8_FORMATS["e4m3"], a_order, b_order,
                                mg.F8_BLOCKS["columns" if what == "weight_grad" else "squares"], m, n, k,
                                s["a"], s["a"].shape[1], s["a_scale"], m, s["b"], s["b"].shape[1], s["b_scale"],
                                s["b_scale"].shape[1], s["bias_v"], s["before"], n, s["c"], n)
        return s["c"]
    if op == "dropout":
        mg.mipgemm_norm_step(kind, mg.NORMS["none"], mg.NORMS["none"], m, n, X=s["x"], ldx=n, Z=s["z"], ldz=n, drop=s["drop"],
                             seed=s["key"], counter=s["counter"], Y=s["y"], ldy=n)
        mg.mipgemm_norm_step_grad(kind, mg.NORMS["none"], mg.NORMS["none"], m, n, dY=s["dy"], lddy=n, drop=s["drop"],
                                  seed=s["key"], counter=s["counter"], dZ=s["dz"], lddz=n)
        return {"y": s["y"], "dz": s["dz"]}
    same = dict(x_scale=s["scale"], Z=s["z"], ldz=n, post_weight=s["post_w"], post_bias=s["post_b"], gate=s["gate_v"],
                ldgate=n, gate_rows=s["gate"], drop=s["drop"], seed=s["key"], counter=s["counter"], pre_weight=s["pre_w"],
                Y=s["y"], ldy=n, stats=s["stats"])
    post, pre = mg.NORMS[s["post"]], mg.NORMS[s["pre"]]
    if op == "step":
        r = {"y": s["y"]}
        if s["codes"] == "none":
            mg.mipgemm_norm_step(kind, post, pre, m, n, EPS, X=s["x"], ldx=n, pre_bias=s["pre_b"], H=s.get("h"), ldh=n, **same)
            return dict(r, h=s["h"], stats=s["stats"]) if s["pre"] != "none" else dict(r, stats=s["stats"])
        mg.mipgemm_norm_step(kind, post, pre, m, n, EPS, X=s["x"], ldx=n, pre_bias=s["pre_b"], codes=mg.CODES[s["codes"]],
                             Q=s["q"], ldq=n, q_scale=s["q_scale"], ldqs=m, **same)
        if s["codes"] == "s8":
            mg.mipgemm_dequantize_rows(kind, m, n, s["q"], n, s["q_scale"], s["back"], n)
        else:
            mg.mipgemm_f8_dequantize(kind, mg.F8_FORMATS[s["codes"]], mg.F8_BLOCKS["rows"], m, n, s["q"], n, s["q_scale"], m,
                                     s["back"], n)
        return dict(r, values=s["back"], scale=s["q_scale"])
    mg.mipgemm_norm_step_grad(kind, post, pre, m, n, dY=s["dy"], lddy=n, dH=s["dh"], lddh=n, dX=s["dx"], lddx=n, dZ=s["dz"],
                              lddz=n, dgate=s["dgate"], lddgate=n, dpost_weight=s["dpost_w"], dpost_bias=s["dpost_b"],
                              dpre_weight=s["dpre_w"], dpre_bias=s["dpre_b"], **same)
    return {k: s[k] for k in ("dx", "dz", "dgate", "dpost_w", "dpost_b", "dpre_w", "dpre_b") if s[k] is not None}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op, m, n = case["op"], case["m"], case["n"]
    wide = torch.float64

    def scale_of(scale, form, rows, cols):
        """Scales by element."""
        scale = scale.to(wide)
        if form == "rows":
            return scale.repeat_interleave(128, dim=0)[:cols].t()
        if form == "columns":
            return scale.repeat_interleave(128, dim=0)[:rows]
        return scale.repeat_interleave(128, dim=0)[:rows].repeat_interleave(128, dim=1)[:, :cols]

    def tops(x, form):
        """Largest magnitude of each block, laid out as the scales are."""
        rows, cols = x.shape
        if form == "rows":
            return torch.stack([p.abs().amax(dim=1) for p in x.split(128, dim=1)])
        if form == "columns":
            return torch.stack([p.abs().amax(dim=0) for p in x.split(128, dim=0)])
        return torch.stack([torch.stack([t.abs().amax() for t in p.split(128, dim=1)]) for p in x.split(128, dim=0)])

    def rounded(v, fmt):
        """To the nearest value of the format."""
        bits, least = (3, -6) if fmt == "e4m3" else (2, -14)
        place = torch.exp2((torch.frexp(v)[1] - 1).clamp(min=least).to(wide) - bits)
        return torch.round(v / place) * place

    def codes(x, form, fmt):
        top = tops(x, form)
        per = scale_of(top, form, *x.shape) / LARGEST[fmt]
        return {"values": torch.where(per > 0, rounded(x / per, fmt) * per, torch.zeros_like(x)), "scale": top / LARGEST[fmt]}

    if op == "codes":
        if m * n > 2 ** 26 or (case["form"] == "squares" and m * n > 2 ** 24):
            return None
        return {f: codes(s["x"].to(wide), f, case["format"]) for f in (("rows", "columns") if case["form"] == "both" else
                                                                      (case["form"],))}
    if op == "product":
        k = case["k"]
        form = {"forward": ("rows", "squares", (m, k), (n, k)), "input_grad": ("rows", "squares", (m, k), (k, n)),
                "weight_grad": ("columns", "columns", (k, m), (k, n))}[case["what"]]
        a = s["a"].to(wide) * scale_of(s["a_scale"], form[0], *form[2])
        b = s["b"].to(wide) * scale_of(s["b_scale"], form[1], *form[3])
        c = torch.matmul(a.t() if form[0] == "columns" else a, b.t() if case["what"] == "forward" else b)
        if case["bias"]:
            c += s["bias_v"].to(wide)
        if case["accumulate"]:
            c += s["before"].to(wide)
        return c

    def keep():
        """The generator again, on 64-bit products split at 2^31 instead of 2^16."""
        bar = round(case["drop"] * 65536)
        if not bar:
            return torch.ones((), dtype=wide, device="cuda")
        mask = 2 ** 32 - 1

        def wide_product(a, c):        # a < 2^32, c < 2^32: (a * c) >> 32 and (a * c) mod 2^32
            top, rest = a >> 31, a & (2 ** 31 - 1)
            p = rest * c               # below 2^63
            hi, lo = p >> 32, p & mask
            q = (top * c) << 31        # top is 0 or 1
            lo2 = lo + (q & mask)
            return (hi + (q >> 32) + (lo2 >> 32)) & mask, lo2 & mask
        width = -(-n // 8)
        g = torch.arange(m, device="cuda")[:, None] * width + torch.arange(width, device="cuda")
        step = int(s["counter"])
        c = [g & mask, g >> 32, torch.full_like(g, step & mask), torch.full_like(g, step >> 32)]
        k0, k1 = s["key"] & mask, (s["key"] >> 32) & mask
        for _ in range(10):
            h0, l0 = wide_product(c[0], 0xD2511F53)
            h1, l1 = wide_product(c[2], 0xCD9E8D57)
            c = [h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0]
            k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
        bits = torch.stack([(c[i // 2] >> (16 * (i % 2))) & 0xFFFF for i in range(8)], dim=-1).flatten(1)[:, :n]
        return (bits >= bar).to(wide) / (1 - bar / 65536)

    if op == "dropout":
        k = keep()
        return {"y": s["x"].to(wide) + s["z"].to(wide) * k, "dz": s["dy"].to(wide) * k}

    def hat(x, kind):
        mean = x.mean(dim=1, keepdim=True) if kind == "layer" else 0 * x[:, :1]
        var = ((x - mean) ** 2).mean(dim=1, keepdim=True)
        return (x - mean) / (var + EPS).sqrt(), mean, (var + EPS).rsqrt()

    def gates():
        rows = torch.arange(m, device="cuda") // max(1, case["gate"])
        return s["gate_v"].to(wide)[rows] if case["gate"] else torch.ones((), dtype=wide, device="cuda")

    def affine(x, w, b):
        if w is not None:
            x = x * w.to(wide)
        return x if b is None else x + b.to(wide)

    if op == "step":
        zero = torch.zeros(m, 1, dtype=wide, device="cuda")
        z, pm, pr = s["z"].to(wide), zero, zero
        if case["post"] != "none":
            z, pm, pr = hat(z, case["post"])
        y = case["scale"] * s["x"].to(wide) + keep() * gates() * affine(z, s["post_w"], s["post_b"])
        r, qm, qr = {"y": y}, zero, zero
        if case["pre"] != "none":
            h, qm, qr = hat(y, case["pre"])
            r["h"] = affine(h, s["pre_w"], s["pre_b"])
        if case["codes"] == "none":
            return dict(r, stats=torch.cat((pm, pr, qm, qr), dim=1))
        if case["codes"] == "s8":
            per = r["h"].abs().amax(dim=1, keepdim=True) / 127
            return {"y": y, "values": torch.round(r["h"] / per) * per, "scale": per.t()}
        return dict(codes(r["h"], "rows", case["codes"]), y=y)

    # the backward pass: the statistics are inputs, as the forward pass left them
    pm, pr, qm, qr = (s["stats"][:, i:i + 1].to(wide) for i in range(4))

    def through(g, h, r, kind):
        return r * (g - (g.mean(dim=1, keepdim=True) if kind == "layer" else 0) - h * (g * h).mean(dim=1, keepdim=True))

    r, dy = {}, s["dy"].to(wide)
    if case["pre"] != "none":
        h, dh = (s["y"].to(wide) - qm) * qr, s["dh"].to(wide)
        r["dpre_w"] = (h * dh).sum(dim=0)
        if case["pre"] == "layer":
            r["dpre_b"] = dh.sum(dim=0)
        dy = dy + through(s["pre_w"].to(wide) * dh, h, qr, case["pre"])
    r["dx"] = case["scale"] * dy
    dv = dy * keep()
    z = s["z"].to(wide)
    h = (z - pm) * pr if case["post"] != "none" else z
    if case["gate"]:
        total = dv * affine(h, s["post_w"], s["post_b"])
        r["dgate"] = torch.stack([p.sum(dim=0) for p in total.split(case["gate"])]) if case["gate"] > 1 else total
    du = dv * gates()
    if case["post"] != "none":
        r["dpost_w"] = (du * h).sum(dim=0)
        if case["post"] == "layer":
            r["dpost_b"] = du.sum(dim=0)
        du = through(du * s["post_w"].to(wide), h, pr, case["post"])
    return dict(r, dz=du)
