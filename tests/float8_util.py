"""64-bit forms of the operators in 8-bit floating point and of the step between two blocks, and what their tests share.
Written out from the definitions in NumPy; nothing here calls the library."""
import numpy as np

FORMATS = ("e4m3", "e5m2")
LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}
LEAST = {"e4m3": 2.0 ** -119, "e5m2": 2.0 ** -112}
MANTISSA = {"e4m3": 3, "e5m2": 2}
LOWEST = {"e4m3": -6, "e5m2": -14}        # exponent of the smallest normal value


def f8_type(fmt):
    import torch
    return {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}[fmt]


def nearest(v, fmt):
    """v (float64) to the nearest value of the format, ties to even; magnitudes beyond the largest stay there."""
    v = np.asarray(v, dtype=np.float64)
    e = np.maximum(np.frexp(v)[1] - 1, LOWEST[fmt])
    step = np.ldexp(1.0, e - MANTISSA[fmt])
    return np.clip(np.round(v / step) * step, -LARGEST[fmt], LARGEST[fmt])      # (np.round: ties to even)


def spread(scale, blocks, rows, cols):
    """Scales as they are stored, by element."""
    s = np.asarray(scale, dtype=np.float64)
    if blocks == "rows":
        return np.repeat(s, 128, axis=0)[:cols, :rows].T
    if blocks == "columns":
        return np.repeat(s, 128, axis=0)[:rows, :cols]
    return np.repeat(np.repeat(s, 128, axis=0), 128, axis=1)[:rows, :cols]


def scale_shape(blocks, rows, cols):
    b = lambda n: (n + 127) // 128  # noqa: E731
    return {"rows": (b(cols), rows), "columns": (b(rows), cols), "squares": (b(rows), b(cols))}[blocks]


def tops(x, blocks):
    rows, cols = x.shape
    out = np.zeros(scale_shape(blocks, rows, cols))
    for i in range(out.shape[0]):
        if blocks == "rows":
            out[i] = np.abs(x[:, 128 * i:128 * i + 128]).max(axis=1)
        elif blocks == "columns":
            out[i] = np.abs(x[128 * i:128 * i + 128]).max(axis=0)
        else:
            for j in range(out.shape[1]):
                out[i, j] = np.abs(x[128 * i:128 * i + 128, 128 * j:128 * j + 128]).max()
    return out


def encode(x, blocks, fmt):
    """(code values, scales) by the rule: both quotients and the product rounded in binary32."""
    with np.errstate(all="ignore"):
        top = tops(x, blocks).astype(np.float32)
        largest = np.float32(LARGEST[fmt])
        live = (top >= LEAST[fmt]) & np.isfinite(top)
        scale = np.where(live, top / largest, np.float32(0)).astype(np.float32)
        mult = np.where(live, largest / np.where(live, top, 1), np.float32(0)).astype(np.float32)
        product = x.astype(np.float32) * spread(mult, blocks, *x.shape).astype(np.float32)
        q = np.where(spread(mult, blocks, *x.shape) == 0, 0.0, nearest(product.astype(np.float64), fmt))
        scale[~np.isfinite(top)] = np.nan
    return q, scale


def philox(counter, key):
    """Philox4x32-10 on Python integers: four words."""
    low = 2 ** 32 - 1
    c, k = list(counter), list(key)
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & low, (p0 >> 32) ^ c[3] ^ k[1], p0 & low]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    return c


def kept(rows, cols, drop, seed, counter=0):
    """What a kept element is multiplied with, 0 where it is dropped."""
    bar, low = round(drop * 65536), 2 ** 32 - 1
    out = np.ones((rows, cols))
    if not bar:
        return out
    groups = (cols + 7) // 8
    for i in range(rows):
        for g in range(groups):
            n = i * groups + g
            w = philox([n & low, n >> 32, counter & low, counter >> 32], [seed & low, seed >> 32])
            for j in range(8 * g, min(8 * g + 8, cols)):
                half = (w[(j % 8) // 2] >> (16 * (j % 2))) & 0xFFFF
                out[i, j] = 1 / (1 - bar / 65536) if half >= bar else 0.0
    return out


def hat(x, kind, eps):
    mean = x.mean(axis=1, keepdims=True) if kind == "layer" else np.zeros((x.shape[0], 1))
    rstd = 1 / np.sqrt(((x - mean) ** 2).mean(axis=1, keepdims=True) + eps)
    return (x - mean) * rstd, mean, rstd


def through(g, h, rstd, kind):
    """Through a norm, backward: g the gradient of the normalised value."""
    mean = g.mean(axis=1, keepdims=True) if kind == "layer" else 0.0
    return rstd * (g - mean - h * (g * h).mean(axis=1, keepdims=True))


def ones(v, n):
    return np.ones(n) if v is None else np.asarray(v, dtype=np.float64)


def zeros(v, n):
    return np.zeros(n) if v is None else np.asarray(v, dtype=np.float64)


def step(c):
    """c: x, z (or None), post, pre, weights, gate, gate_rows, mask (or 1), x_scale, eps.  Returns y, h, stats."""
    some = c["z"] if c["z"] is not None else c["x"]
    m, n = some.shape
    stats = np.zeros((m, 4))
    v = np.zeros((m, n)) if c["z"] is None else c["z"]
    if c["post"] != "none":
        v, mean, rstd = hat(v, c["post"], c["eps"])
        stats[:, :2] = np.concatenate((mean, rstd), axis=1)
        v = v * ones(c["post_w"], n) + zeros(c["post_b"], n)
    if c["gate"] is not None:
        v = v * c["gate"][np.arange(m) // c["gate_rows"]]
    v = v * c["mask"]
    y = v + (0 if c["x"] is None else c["x_scale"] * c["x"])
    h = None
    if c["pre"] != "none":
        h, mean, rstd = hat(y, c["pre"], c["eps"])
        stats[:, 2:] = np.concatenate((mean, rstd), axis=1)
        h = h * ones(c["pre_w"], n) + zeros(c["pre_b"], n)
    return y, h, stats


def step_grad(c, y, stats, dy, dh):
    """Gradients by the formulas, from the y and the statistics that are handed over."""
    m, n = y.shape
    pm, pr, qm, qr = (stats[:, i:i + 1] for i in range(4))
    r, g = {}, np.zeros((m, n)) if dy is None else dy
    if c["pre"] != "none":
        h = (y - qm) * qr
        r["dpre_w"], r["dpre_b"] = (dh * h).sum(axis=0), dh.sum(axis=0)
        g = g + through(dh * ones(c["pre_w"], n), h, qr, c["pre"])
    r["dx"] = c["x_scale"] * g
    k = g * c["mask"]
    if c["z"] is None:
        return r
    h = c["z"] if c["post"] == "none" else (c["z"] - pm) * pr
    if c["gate"] is not None:
        u = h if c["post"] == "none" else h * ones(c["post_w"], n) + zeros(c["post_b"], n)
        r["dgate"] = np.zeros(c["gate"].shape)
        np.add.at(r["dgate"], np.arange(m) // c["gate_rows"], k * u)
        k = k * c["gate"][np.arange(m) // c["gate_rows"]]
    if c["post"] != "none":
        r["dpost_w"], r["dpost_b"] = (k * h).sum(axis=0), k.sum(axis=0)
        k = through(k * ones(c["post_w"], n), h, pr, c["post"])
    r["dz"] = k
    return r
