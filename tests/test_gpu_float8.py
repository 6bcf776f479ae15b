"""8-bit floating-point codes and their product, against 64 bits."""
import numpy as np
import pytest

import float8_util as f
import layer_util as u

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mg():
    from paper_2506_11728_b200 import binding
    binding.mipgemm_set_tuning()
    return binding


def bytes_of(rows, cols, ld=None, shift=0, fmt=None, values=None):
    """A matrix of codes (as bytes) in a larger poisoned buffer; values: what the codes stand for."""
    import torch
    m = u.Matrix(rows, cols, "u8", ld, shift)
    if values is not None:
        m.view.copy_(torch.from_numpy(np.ascontiguousarray(values)).to(f.f8_type(fmt)).view(torch.uint8))
    return m


def code_values(m, fmt):
    import torch
    return m.view.contiguous().view(f.f8_type(fmt)).double().cpu().numpy()


def room(shape, pad=0):
    import torch
    return torch.full((shape[0], shape[1] + pad), -7.0, device="cuda")


LAYOUTS = {"dense": (0, 0), "padded": (16, 16), "odd": (3, 1)}
SHAPES = [(1, 1), (1, 128), (3, 129), (128, 128), (127, 255), (130, 200), (257, 1000), (8, 4096), (300, 72), (1000, 40)]


def tokens(rng, M, N, kind):
    x = rng.standard_normal((M, N)) * 2.0 ** rng.integers(-6, 7, (M, 1))
    x[:, ::37] *= 30
    x[rng.random((M, N)) < 0.02] = 0
    return u.rounded(x, kind)


@pytest.mark.parametrize("fmt", f.FORMATS)
@pytest.mark.parametrize("kind", u.TYPES)
@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("M,N", SHAPES)
def test_codes_are_the_rules_bit_for_bit(mg, M, N, layout, kind, fmt):
    """Codes and scales follow from a rule with three roundings: nothing is left open."""
    pad, shift = LAYOUTS[layout]
    rng = np.random.default_rng([M, N, 1])
    x = tokens(rng, M, N, kind)
    if kind == "f16":
        x = u.rounded(np.clip(x, -60000, 60000), kind)
    X = u.Matrix(M, N, kind, N + pad, shift, x)
    t, ff = mg.TYPES[kind], mg.F8_FORMATS[fmt]
    for sides in (("rows",), ("columns",), ("rows", "columns"), ("squares",)):
        Q = {s: bytes_of(M, N, N + pad, shift) for s in sides}
        S = {s: room(f.scale_shape(s, M, N), pad) for s in sides}
        if sides == ("squares",):
            mg.mipgemm_f8_quantize_squares(t, ff, M, N, X.ptr, X.ld, Q["squares"].ptr, Q["squares"].ld, S["squares"], S["squares"].shape[1])
        else:
            r, c = "rows" in sides, "columns" in sides
            mg.mipgemm_f8_quantize(t, ff, M, N, X.ptr, X.ld, Q["rows"].ptr if r else None, N + pad, S["rows"] if r else None,
                                   S["rows"].shape[1] if r else 0, Q["columns"].ptr if c else None, N + pad, S["columns"] if c else None,
                                   S["columns"].shape[1] if c else 0)
        assert mg.mipgemm_device_status() == mg.OK
        for s in sides:
            q, scale = f.encode(x, s, fmt)
            assert np.array_equal(S[s][:, :scale.shape[1]].cpu().numpy(), scale), (sides, s)
            assert bool((S[s][:, scale.shape[1]:] == -7).all())
            assert np.array_equal(code_values(Q[s], fmt), q) and Q[s].unchanged()
            Y = u.Matrix(M, N, kind, N + pad, shift)
            mg.mipgemm_f8_dequantize(t, ff, mg.F8_BLOCKS[s], M, N, Q[s].ptr, Q[s].ld, S[s], S[s].shape[1], Y.ptr, Y.ld)
            want = (q.astype(np.float32) * f.spread(scale, s, M, N).astype(np.float32)).astype(np.float64)
            assert np.array_equal(Y.get(), u.rounded(want, kind)) and Y.unchanged()


@pytest.mark.parametrize("fmt", f.FORMATS)
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("N", [256, 250])
def test_blocks_without_a_scale(mg, N, kind, fmt):
    """Zeros, magnitudes below the limit, infinities and NaNs, each in a block of its own."""
    import torch
    M = 256
    x = np.ones((M, N))
    x[0, :128] = 0
    x[1, :128] = f.LEAST[fmt] * 0.5
    x[2, :128] = f.LEAST[fmt]
    x[3, 5] = np.inf
    x[4, 130] = -np.inf
    x[5, 131] = np.nan
    X = u.Matrix(M, N, kind, values=x)
    Qr, Qc, Qs = (bytes_of(M, N) for _ in range(3))
    Sr, Sc, Ss = (room(f.scale_shape(s, M, N)) for s in ("rows", "columns", "squares"))
    t, ff = mg.TYPES[kind], mg.F8_FORMATS[fmt]
    mg.mipgemm_f8_quantize(t, ff, M, N, X.ptr, N, Qr.ptr, N, Sr, M, Qc.ptr, N, Sc, N)
    mg.mipgemm_f8_quantize_squares(t, ff, M, N, X.ptr, N, Qs.ptr, N, Ss, Ss.shape[1])
    for s, Q, S in (("rows", Qr, Sr), ("columns", Qc, Sc), ("squares", Qs, Ss)):
        q, scale = f.encode(x, s, fmt)
        assert np.array_equal(S.cpu().numpy(), scale, equal_nan=True) and np.array_equal(code_values(Q, fmt), q)
        Y = u.Matrix(M, N, kind)
        mg.mipgemm_f8_dequantize(t, ff, mg.F8_BLOCKS[s], M, N, Q.ptr, N, S, S.shape[1], Y.ptr, N)
        assert np.array_equal(np.isnan(Y.get()), np.isnan(f.spread(scale, s, M, N)))
    assert torch.isnan(Ss[0, 0]) and float(Sr[0, 0]) == 0 and float(Sr[0, 1]) == 0 and float(Sr[0, 2]) > 0


def test_more_rows_than_one_launch_takes(mg):
    """65535 tiles is what the grid's second dimension holds."""
    import torch
    M, N = 65535 * 128 + 130, 8
    x = torch.arange(M, device="cuda", dtype=torch.float32).remainder_(251).add_(1)[:, None].expand(M, N).to(torch.bfloat16).contiguous()
    q, qc, y = (torch.empty(M, N, dtype=torch.uint8, device="cuda") for _ in range(3))
    s, sc = torch.empty(1, M, device="cuda"), torch.empty((M + 127) // 128, N, device="cuda")
    mg.mipgemm_f8_quantize(2, 0, M, N, x, N, q, N, s, M, qc, N, sc, N)
    y = torch.empty_like(x)
    mg.mipgemm_f8_dequantize(2, 0, 0, M, N, q, N, s, M, y, N)
    largest = torch.full((M,), 448.0, device="cuda")            # (a quotient; a tensor over a number is a product with its reciprocal)
    assert torch.equal(s[0], x[:, 0].float() / largest) and torch.equal(y, x)
    mg.mipgemm_f8_dequantize(2, 0, 1, M, N, qc, N, sc, N, y, N)
    assert float(((y - x).abs() / x).max()) <= 2.0 ** -4 + 2.0 ** -8
    top = x[:65535 * 128, 0].float().view(-1, 128).amax(dim=1)
    assert torch.equal(sc[:65535, 0], top / largest[:65535]) and float(sc[-1, 0]) > 0


# ------------------------------------------------------------------------------------------------ the product
KINDS = {  # a_order, b_order, b_blocks
    "forward": (0, 0, "squares"), "forward_rows": (0, 0, "rows"), "input_grad": (0, 1, "squares"), "weight_grad": (1, 1, "columns"),
    "a_columns": (1, 0, "squares"), "a_columns_rows": (1, 0, "rows"), "a_rows_columns": (0, 1, "columns"), "a_columns_squares": (1, 1, "squares"),
}
SIZES = [(1, 1, 1), (1, 128, 128), (3, 33, 17), (16, 256, 144), (17, 300, 2700), (32, 130, 1200), (64, 200, 5000), (5, 1000, 9000), (100, 40, 129), (128, 128, 256), (129, 257, 200), (200, 520, 328),
         (300, 300, 1000), (64, 1000, 40), (520, 640, 136), (8, 2048, 512), (2000, 24, 96), (40, 48, 0), (256, 264, 4096)]


def operands(M, N, K, what, layout, seed=0, small=False, a_fmt="e4m3", b_fmt="e4m3"):
    import torch
    rng = np.random.default_rng([M, N, K, seed])
    ao, bo, bb = KINDS[what]
    pad, shift = LAYOUTS[layout]
    ashape, bshape = (K, M) if ao else (M, K), (K, N) if bo else (N, K)
    ablocks = "columns" if ao else "rows"
    r = {}
    for name, shape, blocks, fmt in (("a", ashape, ablocks, a_fmt), ("b", bshape, bb, b_fmt)):
        sshape = f.scale_shape(blocks, *shape)
        if small:                          # integers whose products and sums are exact
            v, s = rng.integers(-4, 5, shape).astype(np.float64), 2.0 ** rng.integers(-2, 3, sshape)
        else:
            v = f.nearest(rng.standard_normal(shape) * f.LARGEST[fmt] / 5, fmt)
            s = ((rng.random(sshape) + 0.5) / f.LARGEST[fmt]).astype(np.float32).astype(np.float64)
        S = room((max(sshape[0], 1), max(sshape[1], 1)), pad)
        S[:sshape[0], :sshape[1]] = torch.from_numpy(s).float()
        r[name] = v * f.spread(s, blocks, *shape)
        r[name.upper()] = bytes_of(shape[0], shape[1], max(shape[1] + pad, 1), shift, fmt, v)
        r["s" + name] = S
    a = r["a"].T if ao else r["a"]
    b = r["b"] if bo else r["b"].T
    return rng, a, b, r


def call(mg, kind, what, M, N, K, r, bias, R, C, a_fmt="e4m3", b_fmt="e4m3", ldr=None):
    ao, bo, bb = KINDS[what]
    mg.mipgemm_f8f8_product(mg.TYPES[kind], mg.F8_FORMATS[a_fmt], mg.F8_FORMATS[b_fmt], ao, bo, mg.F8_BLOCKS[bb], M, N, K,
                            r["A"].ptr, r["A"].ld, r["sa"], r["sa"].shape[1], r["B"].ptr, r["B"].ld, r["sb"], r["sb"].shape[1],
                            u.vector(bias), R.ptr if R else None, R.ld if R else 0, C.ptr, C.ld)
    assert mg.mipgemm_device_status() == mg.OK


FORMS = {"auto": {}, "pair": dict(force_path=2), "single": dict(force_path=1), "split": dict(force_path=1, split_k=3), "pair_split": dict(force_path=2, split_k=2),
         "shares_1": dict(split_k=1), "shares_2": dict(split_k=2), "shares_8": dict(split_k=8)}


@pytest.fixture(params=list(FORMS))
def form(request, mg):
    mg.mipgemm_set_tuning(**FORMS[request.param])
    yield request.param
    mg.mipgemm_set_tuning()


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("what", list(KINDS))
@pytest.mark.parametrize("M,N,K", SIZES)
def test_small_integers_are_exact(mg, form, M, N, K, what, layout):
    """Integers and power-of-two scales: products and sums are exact in binary32, so a wrong index, a lost term, a term
    counted twice or a wrong scale shows."""
    if layout == "padded" and form != "auto":
        pytest.skip("the forms differ in what they do with whole and with odd rows")
    if form.startswith("shares") and M > 32:
        pytest.skip("the few-token kernel's shares of K")
    rng, a, b, r = operands(M, N, K, what, layout, small=True)
    pad, shift = LAYOUTS[layout]
    C = u.Matrix(M, N, "f32", N + pad, shift)
    call(mg, "f32", what, M, N, K, r, None, None, C)
    assert np.array_equal(C.get(), a @ b) and C.unchanged()


@pytest.mark.parametrize("kind", u.TYPES)
@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("what", ["forward", "input_grad", "weight_grad"])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_product(mg, M, N, K, what, layout, kind):
    formats = [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2")][(M + N + K) % 3]
    rng, a, b, r = operands(M, N, K, what, layout, 1, False, *formats)
    pad, shift = LAYOUTS[layout]
    for has_bias, residual in ((False, None), (True, "own"), (True, "other"), (False, "odd")):
        c0 = u.rounded(rng.standard_normal((M, N)), kind)
        bias = rng.standard_normal(N).astype(np.float32) if has_bias else None
        C = u.Matrix(M, N, kind, N + pad, shift, c0)
        R = {None: None, "own": C, "other": u.Matrix(M, N, kind, N + 8, 8, c0), "odd": u.Matrix(M, N, kind, N + 5, 3, c0)}[residual]
        call(mg, kind, what, M, N, K, r, bias, R, C, *formats)
        more = (0 if bias is None else bias.astype(np.float64)) + (c0 if residual else 0)
        want = a @ b + more
        total = np.abs(a) @ np.abs(b) + np.abs(more)
        # the documented bound: K products and their scales in binary32; two more additions; one rounding to the type
        tol = total * (K + 8) * 2.0 ** -23 + u.ROUND[kind] * np.abs(want) * 1.01 + u.TINY[kind]
        assert (np.abs(C.get() - want) <= tol).all() and C.unchanged()


def test_scales_may_be_left_out(mg):
    M, N, K = 130, 140, 300
    rng, a, b, r = operands(M, N, K, "forward", "dense", 2, small=True)
    raw_a, raw_b = code_values(r["A"], "e4m3"), code_values(r["B"], "e4m3")
    C = u.Matrix(M, N, "f32")
    mg.mipgemm_f8f8_product(0, 0, 0, 0, 0, 2, M, N, K, r["A"].ptr, r["A"].ld, None, 0, r["B"].ptr, r["B"].ld, None, 0, None, None, 0, C.ptr, N)
    assert np.array_equal(C.get(), raw_a @ raw_b.T)


@pytest.mark.parametrize("what", ["forward", "weight_grad"])
def test_nan_scales_reach_their_rows_and_columns_alone(mg, what):
    M, N, K = 300, 400, 512
    rng, a, b, r = operands(M, N, K, what, "dense", 3, small=True)
    r["sa"][1, 7] = float("nan")
    r["sb"].view(-1)[1] = float("inf")
    C = u.Matrix(M, N, "bf16")
    call(mg, "bf16", what, M, N, K, r, None, None, C)
    got = C.get()
    assert np.isnan(got[7]).all()
    bad = np.zeros((M, N), bool)
    bad[7] = True
    bad[:, 1 if what == "weight_grad" else slice(0, 128)] = True        # sb[0, 1]: column 1, or columns below 128 in block 1
    assert np.array_equal(np.isfinite(got), ~bad) or what == "weight_grad" and np.isfinite(got[~bad]).all()


@pytest.mark.parametrize("what", ["forward", "weight_grad"])
def test_a_code_that_is_no_number_stays_in_its_row(mg, what):
    """Rows behind the last one and columns behind the last block are never mixed in."""
    M, N, K = 100, 130, 140
    rng, a, b, r = operands(M, N, K, what, "padded", 4, small=True)
    r["A"].view[3, 5] = 0x7F                       # NaN of e4m3
    C = u.Matrix(M, N, "f32")
    call(mg, "f32", what, M, N, K, r, None, None, C)
    got, row = C.get(), 5 if what == "weight_grad" else 3
    assert np.isnan(got[row]).all() and np.array_equal(np.delete(got, row, 0), np.delete(a @ b, row, 0))


def test_product_is_the_same_every_time(mg, form):
    M, N, K = 520, 520, 1100
    rng, a, b, r = operands(M, N, K, "weight_grad", "dense", 5)
    C = [u.Matrix(M, N, "f32") for _ in range(3)]
    for c in C:
        call(mg, "f32", "weight_grad", M, N, K, r, None, None, c)
    assert np.array_equal(C[0].get(), C[1].get()) and np.array_equal(C[0].get(), C[2].get())


def test_codes_and_products_make_a_layer_and_its_gradients(mg):
    """Y = X W^T from codes of X and W, and from the same codes of W and column codes of dY and X the two gradients: each
    is the exact product of what the codes stand for, and the bilinear form ties them together."""
    import torch
    M, N, K = 300, 260, 392
    rng = np.random.default_rng(8)
    x, w, dy = (u.rounded(rng.standard_normal(s), "bf16") for s in ((M, K), (N, K), (M, N)))
    X, W, D = u.Matrix(M, K, "bf16", values=x), u.Matrix(N, K, "bf16", values=w), u.Matrix(M, N, "bf16", values=dy)
    bl = lambda n: (n + 127) // 128  # noqa: E731
    new = lambda *s: torch.empty(*s, dtype=torch.uint8, device="cuda")  # noqa: E731
    fl = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
    xr, xrs, xc, xcs = new(M, K), fl(bl(K), M), new(M, K), fl(bl(M), K)
    dr, drs, dc, dcs = new(M, N), fl(bl(N), M), new(M, N), fl(bl(M), N)
    wq, ws = new(N, K), fl(bl(N), bl(K))
    mg.mipgemm_f8_quantize(2, 0, M, K, X.ptr, K, xr, K, xrs, M, xc, K, xcs, K)
    mg.mipgemm_f8_quantize(2, 1, M, N, D.ptr, N, dr, N, drs, M, dc, N, dcs, N)
    mg.mipgemm_f8_quantize_squares(2, 0, N, K, W.ptr, K, wq, K, ws, bl(K))
    Y, dX, dW = fl(M, N), fl(M, K), torch.zeros(N, K, device="cuda")
    mg.mipgemm_f8f8_product(0, 0, 0, 0, 0, 2, M, N, K, xr, K, xrs, M, wq, K, ws, bl(K), None, None, 0, Y, N)
    mg.mipgemm_f8f8_product(0, 1, 0, 0, 1, 2, M, K, N, dr, N, drs, M, wq, K, ws, bl(K), None, None, 0, dX, K)
    mg.mipgemm_f8f8_product(0, 1, 0, 1, 1, 1, N, K, M, dc, N, dcs, N, xc, K, xcs, K, None, dW, K, dW, K)
    assert mg.mipgemm_device_status() == mg.OK

    def back(q, s, blocks, fmt):
        v = q.view(f.f8_type(fmt)).double().cpu().numpy()
        return v * f.spread(s.cpu().numpy(), blocks, *v.shape)
    vx, vxc, vw = back(xr, xrs, "rows", "e4m3"), back(xc, xcs, "columns", "e4m3"), back(wq, ws, "squares", "e4m3")
    vd, vdc = back(dr, drs, "rows", "e5m2"), back(dc, dcs, "columns", "e5m2")
    for got, p, q in ((Y, vx, vw.T), (dX, vd, vw), (dW, vdc.T, vxc)):
        assert (np.abs(got.double().cpu().numpy() - p @ q) <= (p.shape[1] + 8) * 2.0 ** -23 * (np.abs(p) @ np.abs(q))).all()
    # codes are within half a step of what they were made from: 2^-4 (e4m3), 2^-3 (e5m2) relative, or of the smallest step
    assert (np.abs(vx - x) <= 2.0 ** -4 * np.abs(x) + np.repeat(np.abs(x).max(axis=1, keepdims=True), K, 1) * 2.0 ** -10 / 448 * 1.01).all()
    assert (np.abs(vd - dy) <= 2.0 ** -3 * np.abs(dy) + np.abs(dy).max(axis=1, keepdims=True) * 2.0 ** -17 / 57344 * 1.01).all()


@pytest.mark.parametrize("what", ["forward", "input_grad"])
def test_constant_weights_fetched_early(mg, what):
    """Under the promise the few-token kernel fetches weights before the kernel in front of it is over; tokens and scales are
    still read behind it."""
    import torch
    M, N, K = 7, 640, 1500
    rng, a, b, r = operands(M, N, K, what, "padded", 13, small=True)
    C = [u.Matrix(M, N, "f32") for _ in range(6)]
    buf = r["B"].buf
    mg.mipgemm_register_constant_weights(buf)
    try:
        ao, bo, bb = KINDS[what]
        for c in C:
            r["A"].view.copy_(r["A"].view.clone())                     # (a kernel in front that writes the tokens)
            mg.mipgemm_f8f8_product(0, 0, 0, ao, bo, mg.F8_BLOCKS[bb], M, N, K, r["A"].ptr, r["A"].ld, r["sa"], r["sa"].shape[1], r["B"].ptr,
                                    r["B"].ld, r["sb"], r["sb"].shape[1], None, None, 0, c.ptr, N)
        assert mg.mipgemm_device_status() == mg.OK and mg.mipgemm_last_path() & mg.PATH_MASK == mg.PATH_SKINNY
    finally:
        mg.mipgemm_unregister_constant_weights(buf)
    assert all(np.array_equal(c.get(), a @ b) for c in C)
    torch.cuda.synchronize()


def test_captured_calls_use_their_own_scratch(mg):
    """Two graphs of calls that need scratch (odd pitches, K in shares), replayed on two streams at once."""
    import torch
    M, N, K = 130, 200, 2100
    work = []
    for seed in (10, 11):
        rng, a, b, r = operands(M, N, K, "forward", "odd", seed, small=True)
        C = u.Matrix(M, N, "f32")
        call(mg, "f32", "forward", M, N, K, r, None, None, C)                # (kernels are loaded before the capture)
        g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(g, stream=s):
            ao, bo, bb = KINDS["forward"]
            mg.mipgemm_f8f8_product(0, 0, 0, ao, bo, mg.F8_BLOCKS[bb], M, N, K, r["A"].ptr, r["A"].ld, r["sa"], r["sa"].shape[1], r["B"].ptr,
                                    r["B"].ld, r["sb"], r["sb"].shape[1], None, None, 0, C.ptr, N)
        work.append((g, s, C, a @ b, r))
    for g, s, C, _, _ in work:
        C.view.fill_(-1)
    torch.cuda.synchronize()
    for _ in range(20):
        for g, s, *_ in work:
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for _, _, C, want, _ in work:
        assert np.array_equal(C.get(), want)


def test_waits_that_run_out_are_reported(mg):
    """The signal that a block's products are ready is withheld: the kernel unwinds and says so; the next call is whole."""
    import torch
    for M, N, path in ((300, 300, 2), (300, 300, 1), (9, 300, 0)):
        K = 1200
        rng, a, b, r = operands(M, N, K, "forward", "dense", 12, small=True)
        C = u.Matrix(M, N, "f32")
        mg.mipgemm_set_tuning(force_path=path)
        mg.mipgemm_debug_set(1, 20_000_000)
        ao, bo, bb = KINDS["forward"]
        try:
            mg.mipgemm_f8f8_product(0, 0, 0, ao, bo, mg.F8_BLOCKS[bb], M, N, K, r["A"].ptr, r["A"].ld, r["sa"], r["sa"].shape[1], r["B"].ptr,
                                    r["B"].ld, r["sb"], r["sb"].shape[1], None, None, 0, C.ptr, N)
            assert mg.mipgemm_device_status() == mg.ERR_TIMEOUT
        finally:
            mg.mipgemm_debug_set()
            torch.cuda.synchronize()
        mg.mipgemm_set_tuning(force_path=path, stages=3, split_k=1)    # (another plan: the kept one holds the test's limit)
        call(mg, "f32", "forward", M, N, K, r, None, None, C)
        assert np.array_equal(C.get(), a @ b)
        mg.mipgemm_set_tuning()
