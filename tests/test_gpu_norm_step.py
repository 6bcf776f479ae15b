"""The step between two blocks, forward and backward, against 64 bits."""
import numpy as np
import pytest

import float8_util as f
import layer_util as u

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mg():
    from paper_2506_11728_b200 import binding
    return binding


LAYOUTS = {"dense": (0, 0), "padded": (16, 16), "odd": (3, 1)}
EPS = 1e-5


def case(rng, M, N, kind, post, pre, gate_rows, drop, x_scale=1.0, has_x=True, has_z=True, weights=True):
    c = dict(post=post, pre=pre, eps=EPS, x_scale=float(np.float32(x_scale)), gate_rows=gate_rows or 1, seed=int(rng.integers(1 << 62)),
             counter=int(rng.integers(1 << 40)), drop=drop)
    c["x"] = u.rounded(rng.standard_normal((M, N)) * 2 + 0.3, kind) if has_x else None
    c["z"] = u.rounded(rng.standard_normal((M, N)) + 0.5, kind) if has_z else None
    c["gate"] = u.rounded(rng.standard_normal(((M + gate_rows - 1) // gate_rows, N)), kind) if gate_rows else None
    for side in ("post", "pre"):
        c[side + "_w"] = (1 + 0.2 * rng.standard_normal(N)).astype(np.float32) if c[side] != "none" and weights else None
        c[side + "_b"] = (0.2 * rng.standard_normal(N)).astype(np.float32) if c[side] == "layer" and weights else None
    c["mask"] = f.kept(M, N, drop, c["seed"], c["counter"])
    return c


def device(c, kind, layout, M, N):
    """Keyword arguments of both calls, and what keeps their memory alive."""
    import torch
    pad, shift = LAYOUTS[layout]
    keep, kw = [], dict(x_scale=c["x_scale"], gate_rows=c["gate_rows"], drop=c["drop"], seed=c["seed"])
    for name, arg, ld in (("z", "Z", "ldz"), ("gate", "gate", "ldgate")):
        if c[name] is not None:
            m = u.Matrix(c[name].shape[0], N, kind, N + pad, shift, c[name])
            keep.append(m)
            kw[arg], kw[ld] = m.ptr, m.ld
    for name, arg in (("post_w", "post_weight"), ("post_b", "post_bias"), ("pre_w", "pre_weight"), ("pre_b", "pre_bias")):
        if c[name] is not None:
            v = torch.zeros(N + 4, device="cuda")
            at = v[1:1 + N] if layout == "odd" else v[:N]
            at.copy_(torch.from_numpy(c[name]))
            keep.append(v)
            kw[arg] = at
    kw["counter"] = torch.tensor([c["counter"]], dtype=torch.int64, device="cuda")
    return kw, keep


def forward(mg, c, kind, layout, M, N, codes="none", want_y=True, want_h=True):
    import torch
    pad, shift = LAYOUTS[layout]
    kw, keep = device(c, kind, layout, M, N)
    X = u.Matrix(M, N, kind, N + pad, shift, c["x"]) if c["x"] is not None else None
    Y, H = u.Matrix(M, N, kind, N + pad, shift), u.Matrix(M, N, kind, N + pad, shift)
    stats = torch.full((M, 4), -5.0, device="cuda")
    more = {}
    if X:
        more.update(X=X.ptr, ldx=X.ld)
    if want_y:
        more.update(Y=Y.ptr, ldy=Y.ld)
    if want_h and c["pre"] != "none":
        more.update(H=H.ptr, ldh=H.ld)
    Q = S = None
    if codes != "none":
        Q = u.Matrix(M, N, "u8", N + pad, shift)
        S = torch.full((1 if codes == "s8" else (N + 127) // 128, M + pad), -5.0, device="cuda")
        more.update(codes=mg.CODES[codes], Q=Q.ptr, ldq=Q.ld, q_scale=S, ldqs=M + pad)
    mg.mipgemm_norm_step(mg.TYPES[kind], mg.NORMS[c["post"]], mg.NORMS[c["pre"]], M, N, EPS, stats=stats, **kw, **more)
    assert mg.mipgemm_device_status() == mg.OK
    assert Y.unchanged() and H.unchanged() and (Q is None or Q.unchanged())
    return Y, H, stats.double().cpu().numpy(), Q, S


def arithmetic(N):
    """Relative error of binary32 along one norm, in units of the magnitudes that enter: sums of N terms by trees (a thread's
    own at most 32, then at most 10 levels), a quotient, a root, three products: below 64 * 2^-24, and the sums' share falls
    under the root.  Doubled, for the second norm reads what the first one wrote."""
    return 128 * 2.0 ** -24


def check(got, want, size, kind, what):
    tol = u.ROUND[kind] * np.abs(want) * 1.01 + u.TINY[kind] + arithmetic(0) * size
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, int(bad.sum()), bad.size, got[bad][:3], want[bad][:3], np.broadcast_to(tol, want.shape)[bad][:3])


def sizes(c, y, h):
    """What the magnitudes of the terms add up to, behind each norm (a bound for the error's unit)."""
    n = y.shape[1]
    v = np.zeros_like(y) if c["z"] is None else np.abs(c["z"])
    if c["post"] != "none":
        _, mean, rstd = f.hat(c["z"], c["post"], EPS)
        v = (v + np.abs(mean) + 1 / rstd) * rstd * np.abs(f.ones(c["post_w"], n)) + np.abs(f.zeros(c["post_b"], n))
    if c["gate"] is not None:
        v = v * np.abs(c["gate"])[np.arange(y.shape[0]) // c["gate_rows"]]
    v = v * c["mask"] + (0 if c["x"] is None else np.abs(c["x_scale"] * c["x"]))
    if h is None:
        return v, None
    _, mean, rstd = f.hat(y, c["pre"], EPS)
    spread = np.sqrt((v * v).mean(axis=1, keepdims=True))
    return v, (v + np.abs(mean) + np.abs(y - mean) * (1 + spread * rstd)) * rstd * np.abs(f.ones(c["pre_w"], n)) + np.abs(f.zeros(c["pre_b"], n))


SHAPES = [(1, 1), (5, 7), (3, 8), (9, 64), (130, 72), (7, 256), (33, 257), (6, 768), (4, 1001), (3, 4096), (2, 4104), (3, 5000), (2, 8200), (2, 16384), (1, 20001), (2, 32768)]
MIXES = [("rms", "rms", 0, 0.0), ("layer", "layer", 3, 0.1), ("none", "rms", 1, 0.25), ("none", "layer", 0, 0.0), ("rms", "none", 2, 0.5), ("layer", "none", 0, 0.0),
         ("none", "none", 0, 0.1), ("none", "none", 1, 0.0), ("rms", "layer", 1000000, 0.3)]


@pytest.mark.parametrize("kind", u.TYPES)
@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("M,N", SHAPES)
def test_forward(mg, M, N, layout, kind):
    rng = np.random.default_rng([M, N, 2])
    for i, (post, pre, gate, drop) in enumerate(MIXES):
        if N > 1001 and (i + M + len(kind) + len(layout)) % 4:
            continue
        c = case(rng, M, N, kind, post, pre, gate, drop, x_scale=(1.0, 0.7)[i % 2], has_x=i != 3 or True)
        Y, H, stats, _, _ = forward(mg, c, kind, layout, M, N)
        y, h, st = f.step(c)
        sy, sh = sizes(c, y, h)
        check(Y.get(), y, sy, kind, (post, pre, "y"))
        if h is not None:
            check(H.get(), h, sh, kind, (post, pre, "h"))
        big = np.abs(st).copy()
        if post != "none":
            big[:, 0] += np.abs(c["z"]).mean(axis=1)
            big[:, 1] *= 1 + (np.abs(st[:, 0]) * st[:, 1]) ** 2
        if pre != "none":
            spread = np.sqrt((sy * sy).mean(axis=1))
            big[:, 2] += sy.mean(axis=1)
            big[:, 3] *= 1 + (spread * st[:, 3]) ** 2
        assert (np.abs(stats - st) <= arithmetic(N) * big).all(), (post, pre)


@pytest.mark.parametrize("M,N", [(1, 5), (20, 128), (130, 300), (4, 4096), (3, 5008), (2, 20001)])
@pytest.mark.parametrize("layout", list(LAYOUTS))
def test_x_or_z_alone_and_no_weights(mg, M, N, layout):
    rng = np.random.default_rng([M, N, 3])
    for has_x, has_z, post in ((True, False, "none"), (False, True, "rms"), (False, True, "none")):
        c = case(rng, M, N, "bf16", post, "layer", 0, 0.0, has_x=has_x, has_z=has_z, weights=False)
        Y, H, stats, _, _ = forward(mg, c, "bf16", layout, M, N)
        y, h, st = f.step(c)
        sy, sh = sizes(c, y, h)
        check(Y.get(), y, sy, "bf16", "y")
        check(H.get(), h, sh, "bf16", "h")


@pytest.mark.parametrize("codes", ["s8", "e4m3", "e5m2"])
@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("M,N", SHAPES[:-2] + [(2, 20000)])
def test_codes_of_h(mg, M, N, layout, codes):
    """float32 in and out: codes come from the unrounded h, which H then holds, so they follow from H by the rules."""
    rng = np.random.default_rng([M, N, 4])
    for post, pre in (("none", "rms"), ("rms", "layer")):
        c = case(rng, M, N, "f32", post, pre, 0, 0.0)
        Y, H, _, Q, S = forward(mg, c, "f32", layout, M, N, codes)
        h = H.get()
        got_s = S[:, :M].cpu().numpy()
        assert bool((S[:, M:] == -5).all())
        if codes == "s8":
            top = np.abs(h).max(axis=1).astype(np.float32)
            assert np.array_equal(got_s[0], top / np.float32(127))
            want = np.round((h.astype(np.float32) * (np.float32(127) / top)[:, None]).astype(np.float64))
            got = Q.view.contiguous().view(__import__("torch").int8).double().cpu().numpy()
        else:
            want, scale = f.encode(h, "rows", codes)
            assert np.array_equal(got_s, scale)
            got = Q.view.contiguous().view(f.f8_type(codes)).double().cpu().numpy()
        assert np.array_equal(got, want)
        # the same codes without y and h being written, and from 16-bit operands within a step
        Q2 = forward(mg, c, "f32", layout, M, N, codes, want_y=False, want_h=False)[3]
        assert np.array_equal(Q2.get(), Q.get())


@pytest.mark.parametrize("codes", ["s8", "e4m3", "e5m2"])
def test_rows_without_a_scale(mg, codes):
    """A row of zeros gives codes 0 and scale 0; a NaN spoils its row's norm, and with it all its blocks."""
    rng = np.random.default_rng(5)
    M, N = 6, 384
    c = case(rng, M, N, "f32", "none", "rms", 0, 0.0)
    c["z"][1], c["x"][1] = 0, 0
    c["x"][3, 200] = np.nan
    c["x"][4, 1] = np.inf
    Y, H, _, Q, S = forward(mg, c, "f32", "dense", M, N, codes)
    s, q = S.cpu().numpy(), Q.get()
    assert (s[:, 1] == 0).all() and (q[[1, 3, 4]] == 0).all() and np.isnan(s[:, [3, 4]]).any(axis=0).all()
    assert np.isfinite(s[:, [0, 2, 5]]).all() and (q[[0, 2, 5]] != 0).any()


def test_dropped_places_hold_zero_whatever_was_there(mg):
    rng = np.random.default_rng(6)
    M, N = 9, 40
    c = case(rng, M, N, "bf16", "none", "none", 0, 0.4)
    bad = c["mask"] == 0
    z = c["z"].copy()
    c["z"] = np.where(bad, np.nan, z)
    c["z"][0] = np.where(bad[0], np.inf, z[0])
    Y, *_ = forward(mg, c, "bf16", "dense", M, N)
    c["z"] = np.where(bad, 0, z)
    check(Y.get(), f.step(c)[0], np.abs(c["z"]) * c["mask"] + np.abs(c["x"]), "bf16", "y")


def test_mask_is_a_function_of_seed_counter_and_place(mg):
    """The same mask whatever the pitch, type and the rest of the step; another one for another seed or counter; the counter is
    read when a captured call is replayed; rates are kept."""
    import torch
    M, N, drop = 512, 1024, 0.25
    one = torch.ones(M, N, device="cuda")
    ctr = torch.zeros(1, dtype=torch.int64, device="cuda")

    def draw(seed, kind=torch.float32, ld=N):
        z = torch.ones(M, ld, device="cuda", dtype=kind)
        y = torch.empty(M, ld, device="cuda", dtype=kind)
        mg.mipgemm_norm_step({torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}[kind], 0, 0, M, N, Z=z, ldz=ld, drop=drop, seed=seed, counter=ctr, Y=y, ldy=ld)
        return y[:, :N] != 0
    a = draw(7)
    assert torch.equal(a, draw(7, torch.bfloat16)) and torch.equal(a, draw(7, torch.float16, N + 5)) and not torch.equal(a, draw(8))
    # 2^19 draws: five deviations
    assert abs(float(a.float().mean()) - 0.75) < 5 * (0.75 * 0.25 / (M * N)) ** 0.5
    y = torch.empty(M, N, device="cuda")
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g, stream=s):
        mg.mipgemm_norm_step(0, 0, 0, M, N, Z=one, ldz=N, drop=drop, seed=7, counter=ctr, Y=y, ldy=N)
    seen = []
    for i in (0, 1, 0, (1 << 32) + 1):
        ctr.fill_(i)
        g.replay()
        torch.cuda.synchronize()
        seen.append(y != 0)
    assert torch.equal(seen[0], a) and torch.equal(seen[2], a) and not torch.equal(seen[1], a) and not torch.equal(seen[3], seen[1])


def test_y_may_be_x_or_z(mg):
    import torch
    M, N = 33, 1000
    x, z = torch.randn(M, N, device="cuda").bfloat16(), torch.randn(M, N, device="cuda").bfloat16()
    y, h, h2 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    args = (2, 1, 2, M, N, EPS)
    mg.mipgemm_norm_step(*args, X=x, ldx=N, Z=z, ldz=N, Y=y, ldy=N, H=h, ldh=N)
    for which in (0, 1):
        both = [x.clone(), z.clone()]
        mg.mipgemm_norm_step(*args, X=both[0], ldx=N, Z=both[1], ldz=N, Y=both[which], ldy=N, H=h2, ldh=N)
        assert torch.equal(both[which], y) and torch.equal(h2, h) and torch.equal(both[1 - which], (x, z)[1 - which])


# ------------------------------------------------------------------------------------------------ backward
def backward(mg, c, kind, layout, M, N, y, stats, dy, dh, without=()):
    import torch
    pad, shift = LAYOUTS[layout]
    kw, keep = device(c, kind, layout, M, N)
    kw.pop("pre_bias", None)
    more, outs = {}, {}
    for name, arg, ld, v in (("y", "Y", "ldy", y if c["pre"] != "none" else None), ("dy", "dY", "lddy", dy), ("dh", "dH", "lddh", dh)):
        if v is not None:
            m = u.Matrix(M, N, kind, N + pad, shift, v)
            keep.append(m)
            more[arg], more[ld] = m.ptr, m.ld
    for name, ld, rows in (("dX", "lddx", M), ("dZ", "lddz", M), ("dgate", "lddgate", c["gate"].shape[0] if c["gate"] is not None else 0)):
        if name in without or not rows or (name == "dZ" and c["z"] is None):
            continue
        outs[name] = u.Matrix(rows, N, kind, N + pad, shift)
        more[name], more[ld] = outs[name].ptr, outs[name].ld
    for side in ("post", "pre"):
        for what, when in (("weight", c[side] != "none"), ("bias", c[side] == "layer")):
            name = "d%s_%s" % (side, what)
            if when and name not in without:
                outs[name] = torch.full((N,), -3.0, device="cuda")
                more[name] = outs[name]
    s = torch.from_numpy(np.ascontiguousarray(stats)).float().cuda()
    mg.mipgemm_norm_step_grad(mg.TYPES[kind], mg.NORMS[c["post"]], mg.NORMS[c["pre"]], M, N, stats=s, **kw, **more)
    assert mg.mipgemm_device_status() == mg.OK
    for m in outs.values():
        assert not isinstance(m, u.Matrix) or m.unchanged()
    return {k: v.get() if isinstance(v, u.Matrix) else v.double().cpu().numpy() for k, v in outs.items()}


def grad_sizes(c, y, stats, dy, dh):
    """Magnitudes of the terms of each gradient."""
    m, n = y.shape
    pm, pr, qm, qr = (stats[:, i:i + 1] for i in range(4))
    r, g = {}, np.zeros((m, n)) if dy is None else np.abs(dy)

    def norm(g, h, rstd):
        return rstd * (g + g.mean(axis=1, keepdims=True) + np.abs(h) * (g * np.abs(h)).mean(axis=1, keepdims=True))
    if c["pre"] != "none":
        h = (np.abs(y) + np.abs(qm)) * qr
        r["dpre_weight"], r["dpre_bias"] = (np.abs(dh) * h).sum(axis=0), np.abs(dh).sum(axis=0)
        g = g + norm(np.abs(dh) * np.abs(f.ones(c["pre_w"], n)), h, qr)
    r["dX"] = abs(c["x_scale"]) * g
    k = g * c["mask"]
    if c["z"] is None:
        return r
    h = np.abs(c["z"]) if c["post"] == "none" else (np.abs(c["z"]) + np.abs(pm)) * pr
    if c["gate"] is not None:
        w = h if c["post"] == "none" else h * np.abs(f.ones(c["post_w"], n)) + np.abs(f.zeros(c["post_b"], n))
        r["dgate"] = np.zeros(c["gate"].shape)
        np.add.at(r["dgate"], np.arange(m) // c["gate_rows"], k * w)
        k = k * np.abs(c["gate"])[np.arange(m) // c["gate_rows"]]
    if c["post"] != "none":
        r["dpost_weight"], r["dpost_bias"] = (k * h).sum(axis=0), k.sum(axis=0)
        k = norm(k * np.abs(f.ones(c["post_w"], n)), h, pr)
    r["dZ"] = k
    return r


def check_grad(mg, c, kind, layout, M, N, rng, without=(), has_dy=True):
    y, h, st = f.step(c)
    y, st = u.rounded(y, kind), st.astype(np.float32).astype(np.float64)
    dy = u.rounded(rng.standard_normal((M, N)), kind) if has_dy else None
    dh = u.rounded(rng.standard_normal((M, N)), kind) if c["pre"] != "none" else None
    got = backward(mg, c, kind, layout, M, N, y, st, dy, dh, without)
    want, size = f.step_grad(c, y, st, dy, dh), grad_sizes(c, y, st, dy, dh)
    names = {"dX": "dx", "dZ": "dz", "dgate": "dgate", "dpost_weight": "dpost_w", "dpost_bias": "dpost_b", "dpre_weight": "dpre_w", "dpre_bias": "dpre_b"}
    for k, v in got.items():
        # column sums: rows are added one after the other, at most M of them in a thread's sum
        extra = M * 2.0 ** -24 * size[k] if k not in ("dX", "dZ") else 0
        w = want[names[k]]
        tol = arithmetic(N) * size[k] + extra + (u.ROUND[kind] * np.abs(w) * 1.01 + u.TINY[kind] if k in ("dX", "dZ", "dgate") else 0)
        bad = ~(np.abs(v - w) <= tol)
        assert not bad.any(), (k, c["post"], c["pre"], c["gate_rows"], int(bad.sum()), v[bad][:3], w[bad][:3])
    return got


GRAD_SHAPES = SHAPES + [(600, 64), (1000, 24), (400, 520), (700, 136)]


@pytest.mark.parametrize("kind", u.TYPES)
@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("M,N", GRAD_SHAPES)
def test_backward(mg, M, N, layout, kind):
    rng = np.random.default_rng([M, N, 7])
    for i, (post, pre, gate, drop) in enumerate(MIXES):
        if M * N > 20000 and (i + M + len(kind) + len(layout)) % 4:
            continue
        c = case(rng, M, N, kind, post, pre, gate, drop, x_scale=(1.0, 0.7)[i % 2])
        check_grad(mg, c, kind, layout, M, N, rng)


@pytest.mark.parametrize("gate_rows", [1, 2, 3, 7, 64, 100, 299, 300, 301])
@pytest.mark.parametrize("N", [24, 200, 520, 4200])
def test_gradient_of_a_shared_gate(mg, N, gate_rows):
    """Gate rows shared by few rows, by many, by all; the last one by what is left."""
    rng = np.random.default_rng([N, gate_rows])
    M = 300 if N < 4000 else 30
    c = case(rng, M, N, "f32", "rms", "rms", gate_rows, 0.0)
    check_grad(mg, c, "f32", "dense", M, N, rng)


def test_more_gate_rows_than_workers(mg):
    rng = np.random.default_rng(9)
    for M, N, rows in ((2000, 24, 2), (900, 600, 3), (901, 40, 5)):
        c = case(rng, M, N, "bf16", "layer", "none", rows, 0.0)
        check_grad(mg, c, "bf16", "dense", M, N, rng)


def test_outputs_may_be_left_out(mg):
    rng = np.random.default_rng(10)
    M, N = 50, 264
    c = case(rng, M, N, "f32", "layer", "layer", 10, 0.1)
    every = {"dX", "dZ", "dgate", "dpost_weight", "dpost_bias", "dpre_weight", "dpre_bias"}
    for keep in [{k} for k in sorted(every)] + [{"dX", "dZ"}, {"dpost_bias", "dpre_weight"}, every - {"dgate"}]:
        got = check_grad(mg, c, "f32", "dense", M, N, np.random.default_rng(11), without=every - keep)
        assert set(got) == keep
    check_grad(mg, c, "f32", "dense", M, N, rng, has_dy=False)


def test_no_rows_give_zero_sums(mg):
    import torch
    N = 40
    w = [torch.ones(N, device="cuda") for _ in range(4)]
    mg.mipgemm_norm_step_grad(0, 2, 2, 0, N, dpost_weight=w[0], dpost_bias=w[1], dpre_weight=w[2], dpre_bias=w[3])
    assert all(bool((v == 0).all()) for v in w)


def test_gradients_are_the_same_every_time_and_in_place(mg):
    import torch
    M, N = 400, 1000
    t = {k: torch.randn(M, N, device="cuda").bfloat16() for k in ("dy", "dh", "y", "z")}
    stats = torch.rand(M, 4, device="cuda") + 0.5

    def run(dx, dz, **src):
        a = dict(t, **src)
        w = [torch.empty(N, device="cuda") for _ in range(2)]
        mg.mipgemm_norm_step_grad(2, 1, 1, M, N, dY=a["dy"], lddy=N, dH=a["dh"], lddh=N, Y=a["y"], ldy=N, Z=a["z"], ldz=N, stats=stats, drop=0.1, seed=5,
                                  dX=dx, lddx=N, dZ=dz, lddz=N, dpost_weight=w[0], dpre_weight=w[1])
        return [dx, dz] + w
    first = run(torch.empty_like(t["z"]), torch.empty_like(t["z"]))
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(first, run(torch.empty_like(t["z"]), torch.empty_like(t["z"]))))
    for i, j in (("dy", "dh"), ("z", "dy"), ("y", "z")):
        a, b = t[i].clone(), t[j].clone()
        assert all(torch.equal(p, q) for p, q in zip(first, run(a, b, **{i: a, j: b}))), (i, j)


def test_gradients_against_differences(mg):
    """float32: the loss's difference along a direction is the gradients' product with it."""
    import torch
    M, N, e = 20, 200, 2.0 ** -7
    rng = np.random.default_rng(12)
    for post, pre in (("layer", "rms"), ("rms", "layer")):
        c = case(rng, M, N, "f32", post, pre, 7, 0.2, x_scale=0.5)
        dy, dh = rng.standard_normal((M, N)), rng.standard_normal((M, N))
        Y, H, st, _, _ = forward(mg, c, "f32", "dense", M, N)
        got = backward(mg, c, "f32", "dense", M, N, Y.get(), st, u.rounded(dy, "f32"), u.rounded(dh, "f32"))

        def loss(c):
            y, h, _, _, _ = forward(mg, c, "f32", "dense", M, N)
            return (dy * y.get()).sum() + (dh * h.get()).sum()
        for name, grad in (("x", "dX"), ("z", "dZ"), ("gate", "dgate"), ("post_w", "dpost_weight"), ("pre_w", "dpre_weight")):
            d = rng.standard_normal(c[name].shape)
            up, down = (dict(c, **{name: (c[name] + s * d).astype(c[name].dtype)}) for s in (e, -e))
            slope, exact = (loss(up) - loss(down)) / (2 * e), (got[grad] * d).sum()
            # the forward pass in 64 bits gives what the difference's own curvature is worth
            l64 = [(lambda r: (dy * r[0]).sum() + (dh * r[1]).sum())(f.step(v)) for v in (up, down)]
            curve = abs((l64[0] - l64[1]) / (2 * e) - exact)
            noise = 2 * 128 * 2.0 ** -24 * (np.abs(dy).sum() * 4 + np.abs(dh).sum() * 4) / (2 * e) / 16
            assert abs(slope - exact) <= curve + noise + 1e-3 * abs(exact), (post, pre, name)


# ------------------------------------------------------------------------------------------------ rows that lie on no boundary
def placed(t, pitch, shift):
    """A copy of `t` whose rows are `pitch` elements apart, the first one `shift` elements into its memory."""
    import torch
    room = torch.full((t.shape[0] * pitch + 64,), 7.0, dtype=t.dtype, device="cuda")
    at = room[shift:shift + t.shape[0] * pitch].view(t.shape[0], pitch)
    at[:, :t.shape[1]].copy_(t)
    return at


@pytest.mark.parametrize("kind", u.TYPES)
@pytest.mark.parametrize("post,pre,gate_rows,drop", [("rms", "rms", 0, 0.1), ("layer", "rms", 1, 0.0), ("none", "layer", 50, 0.2), ("rms", "none", 1400, 0.0), ("none", "none", 1, 0.3)])
@pytest.mark.parametrize("M,N", [(1300, 1000), (700, 520), (610, 8192), (5, 1000), (3, 20000)])
def test_where_rows_lie_changes_no_bit(mg, M, N, post, pre, gate_rows, drop, kind):
    """Many rows and few, at 16-byte boundaries and at none, in place and not: one arithmetic, so the same bits."""
    import torch
    torch.manual_seed(M + N)
    dtype = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}[kind]
    new = lambda rows: torch.randn(rows, N, device="cuda").to(dtype)
    x, z, dy, dh = (new(M) for _ in range(4))
    gate = new((M + gate_rows - 1) // gate_rows) if gate_rows else None
    post_w, pre_w = torch.randn(N + 1, device="cuda"), torch.randn(N + 1, device="cuda")
    seen = []
    for pitch, shift, in_place in ((N, 0, False), (N + 1, 1, False), (N + 3, 2, True), (N + 8, 0, True)):
        put = lambda t: placed(t, pitch, shift)
        X, Z, DY, DH = (put(t) for t in (x, z, dy, dh))
        Y = X if in_place else put(torch.zeros_like(x))
        H = put(torch.zeros_like(x))
        stats = torch.zeros(M, 4, device="cuda")
        w = {}
        for name, v, there in (("post_weight", post_w, post != "none"), ("pre_weight", pre_w, pre != "none")):
            if there:
                w[name] = v[:N] if pitch % 8 == 0 else torch.cat([v[:1], v[:N]])[1:]
        g = put(gate) if gate_rows else None
        shared = dict(w, Z=Z, ldz=pitch, gate=g, ldgate=pitch if gate_rows else 0, gate_rows=gate_rows or 1, drop=drop, seed=3)
        norms = (mg.TYPES[kind], mg.NORMS[post], mg.NORMS[pre], M, N)
        mg.mipgemm_norm_step(*norms, EPS, X=X, ldx=pitch, Y=Y, ldy=pitch, **({"H": H, "ldh": pitch} if pre != "none" else {}), stats=stats, **shared)
        out = [Y[:, :N].clone(), H[:, :N].clone(), stats.clone()]
        back, sums = {}, {}
        if pre != "none":
            back.update(dH=DH, lddh=pitch, Y=Y, ldy=pitch)
            sums["dpre_weight"] = torch.zeros(N, device="cuda")
        if post != "none":
            sums["dpost_weight"] = torch.zeros(N, device="cuda")
        dg = put(torch.zeros_like(gate)) if gate_rows else None
        if gate_rows:
            back.update(dgate=dg, lddgate=pitch)
        dx, dz = (DY, Z) if in_place else (put(torch.zeros_like(x)), put(torch.zeros_like(x)))
        mg.mipgemm_norm_step_grad(*norms, dY=DY, lddy=pitch, stats=stats, dX=dx, lddx=pitch, dZ=dz, lddz=pitch, **back, **sums, **shared)
        out += [dx[:, :N].clone(), dz[:, :N].clone(), *sums.values()] + ([dg[:, :N].clone()] if gate_rows else [])
        for t in (Y, H, dx, dz):
            behind = t[:, N:]
            assert bool((behind == 7.0).all())
        seen.append(out)
    for other in seen[1:]:
        assert all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(seen[0], other))
