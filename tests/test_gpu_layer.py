"""Operators of the 8-bit layer against their definitions in 64 bits: linear, gated, gated_grad.

Every output element is held to the error that binary32 arithmetic behind an exact integer sum can have
(layer_util.ARITH) plus one rounding to the output's type; with power-of-two scales and 32-bit outputs the
arithmetic is exact and the comparison is for equality."""
import numpy as np
import pytest

import layer_util as u

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mg():
    from paper_2506_11728_b200 import binding
    return binding


# (M, N, K): single elements, tile edges from both sides, one to sixteen tokens, ragged everything, empty sums
SIZES = [(1, 1, 1), (1, 16, 128), (2, 33, 64), (3, 250, 65), (8, 160, 1152), (16, 2400, 256), (7, 2401, 1040),
         (17, 64, 96), (33, 100, 384), (127, 129, 130), (128, 256, 128), (129, 257, 144), (300, 520, 400),
         (64, 2500, 512), (513, 1000, 272), (40, 48, 0), (1, 4096, 2048), (9, 3000, 1000), (5, 4112, 16)]
# how the matrices lie: (extra pitch of 8-bit operands, their base offset, extra pitch of floating matrices, offset)
LAYOUTS = {"dense": (0, 0, 0, 0), "padded": (16, 16, 8, 8), "odd": (3, 1, 1, 1)}


def layer_case(M, N, K, kind, act, layout, unsigned=False, seed=0, spread=1.0):
    rng = np.random.default_rng([M, N, K, seed])
    p8, o8, pf, of = LAYOUTS[layout]
    A = u.codes(rng, M, K, unsigned)
    a_scale = u.scales(rng, M, spread / 74)
    def weights():
        w = u.codes(rng, N, K)
        return w, u.scales(rng, N, 1 / (74 * max(K, 1) ** 0.5))
    def floats():
        return u.rounded(rng.standard_normal((M, N)), kind)
    def m8(x, kind8="s8"):
        return u.Matrix(x.shape[0], x.shape[1], kind8, x.shape[1] + p8 if p8 else max(x.shape[1], 1), o8, x)
    def mf(values=None):
        return u.Matrix(M, N, kind, N + pf, of, values)
    return rng, A, a_scale, weights, floats, m8, mf


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("M,N,K", SIZES)
def test_linear(mg, M, N, K, layout):
    for i, (kind, act) in enumerate([("bf16", "none"), ("f32", "gelu"), ("f16", "silu"), ("f32", "relu"), ("bf16", "gelu_tanh")]):
        unsigned = i == 3
        rng, A, a_s, weights, floats, m8, mf = layer_case(M, N, K, kind, act, layout, unsigned, i)
        W, w_s = weights()
        bias = rng.standard_normal(N).astype(np.float32) if i in (1, 2) else None
        res = floats() if i in (0, 1, 4) else None
        a, w, c = m8(A, "u8" if unsigned else "s8"), m8(W), mf()
        r = mf(res) if res is not None else None
        fn = mg.mipgemm_u8s8_linear if unsigned else mg.mipgemm_s8s8_linear
        fn(mg.TYPES[kind], mg.ACTIVATIONS[act], M, N, K, a.ptr, a.ld, u.vector(a_s), w.ptr, w.ld, u.vector(w_s), u.vector(bias),
           r.ptr if r else None, r.ld if r else 0, c.ptr, c.ld)
        assert mg.mipgemm_device_status() == mg.OK
        z = u.sums(A, W) * a_s[:, None].astype(np.float64) * w_s.astype(np.float64)
        b = np.zeros(N) if bias is None else bias.astype(np.float64)
        want = u.act(z + b, act) + (0 if res is None else res)
        u.check(c.get(), want, 1 + np.abs(z) + np.abs(b) + (0 if res is None else np.abs(res)), kind, "%s %s" % (kind, act))
        assert c.unchanged()


@pytest.mark.parametrize("M,N,K", SIZES)
def test_linear_power_of_two_scales_are_exact(mg, M, N, K):
    """Sums below 2^24, scales that are powers of two, 32-bit output: nothing is rounded."""
    rng = np.random.default_rng(7)
    A, W = rng.integers(-60, 61, (M, K)).astype(np.int8), rng.integers(-60, 61, (N, K)).astype(np.int8)
    a_s, w_s = 2.0 ** rng.integers(-3, 4, M), 2.0 ** rng.integers(-3, 4, N)
    a, w, c = u.Matrix(M, K, "s8", max(K, 1), 0, A), u.Matrix(N, K, "s8", max(K, 1), 0, W), u.Matrix(M, N, "f32")
    mg.mipgemm_s8s8_linear(0, 0, M, N, K, a.ptr, a.ld, u.vector(a_s), w.ptr, w.ld, u.vector(w_s), None, None, 0, c.ptr, c.ld)
    assert mg.mipgemm_device_status() == mg.OK
    assert np.array_equal(c.get(), u.sums(A, W) * a_s[:, None] * w_s)
    # no scales at all: the plain product
    mg.mipgemm_s8s8_linear(0, 0, M, N, K, a.ptr, a.ld, None, w.ptr, w.ld, None, None, None, 0, c.ptr, c.ld)
    assert np.array_equal(c.get(), u.sums(A, W))


@pytest.mark.parametrize("M,N,K", [(1, 4096, 256), (12, 2500, 384), (200, 300, 160), (700, 264, 1024)])
@pytest.mark.parametrize("kind", u.TYPES)
def test_linear_residual_in_place(mg, M, N, K, kind):
    rng, A, a_s, weights, floats, m8, mf = layer_case(M, N, K, kind, "none", "dense")
    W, w_s = weights()
    res = floats()
    a, w, c = m8(A), m8(W), mf(res)
    mg.mipgemm_s8s8_linear(mg.TYPES[kind], 0, M, N, K, a.ptr, a.ld, u.vector(a_s), w.ptr, w.ld, u.vector(w_s), None, c.ptr, c.ld, c.ptr, c.ld)
    assert mg.mipgemm_device_status() == mg.OK
    z = u.sums(A, W) * a_s[:, None].astype(np.float64) * w_s.astype(np.float64)
    u.check(c.get(), z + res, np.abs(z) + np.abs(res), kind)


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("M,F,K", SIZES)
def test_gated(mg, M, F, K, layout):
    for i, (kind, act) in enumerate([("bf16", "silu"), ("f32", "gelu"), ("f16", "gelu_tanh"), ("f32", "relu"), ("f32", "none")]):
        rng, X, x_s, weights, floats, m8, mf = layer_case(M, F, K, kind, act, layout, seed=i)
        (Wg, g_s), (Wu, u_s) = weights(), weights()
        x, wg, wu, h = m8(X), m8(Wg), m8(Wu), mf()
        mg.mipgemm_s8s8_gated(mg.TYPES[kind], mg.ACTIVATIONS[act], M, F, K, x.ptr, x.ld, u.vector(x_s), wg.ptr, wg.ld, u.vector(g_s),
                              wu.ptr, wu.ld, u.vector(u_s), h.ptr, h.ld)
        assert mg.mipgemm_device_status() == mg.OK
        G = u.sums(X, Wg) * x_s[:, None].astype(np.float64) * g_s.astype(np.float64)
        U = u.sums(X, Wu) * x_s[:, None].astype(np.float64) * u_s.astype(np.float64)
        u.check(h.get(), u.act(G, act) * U, (1 + np.abs(G)) * np.abs(U), kind, "%s %s" % (kind, act))
        assert h.unchanged()


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("M,F,K", SIZES)
def test_gated_grad(mg, M, F, K, layout):
    for i, (kind, act) in enumerate([("bf16", "silu"), ("f32", "gelu"), ("f16", "gelu_tanh"), ("f32", "relu"), ("f32", "none")]):
        rng, X, x_s, weights, floats, m8, mf = layer_case(M, F, K, kind, act, layout, seed=i)
        (Wg, g_s), (Wu, u_s) = weights(), weights()
        d = floats()
        x, wg, wu, dh = m8(X), m8(Wg), m8(Wu), mf(d)
        p, o = LAYOUTS[layout][2:]
        both = u.Matrix(M, 2 * F, kind, 2 * F + p, o)          # the two results as halves of one matrix
        mg.mipgemm_s8s8_gated_grad(mg.TYPES[kind], mg.ACTIVATIONS[act], M, F, K, x.ptr, x.ld, u.vector(x_s), wg.ptr, wg.ld, u.vector(g_s),
                                   wu.ptr, wu.ld, u.vector(u_s), dh.ptr, dh.ld, both.ptr, both.ld, both.ptr + F * u.size(kind), both.ld)
        assert mg.mipgemm_device_status() == mg.OK
        G = u.sums(X, Wg) * x_s[:, None].astype(np.float64) * g_s.astype(np.float64)
        U = u.sums(X, Wu) * x_s[:, None].astype(np.float64) * u_s.astype(np.float64)
        got = both.get()
        # at G = 0 the derivative of relu jumps; a sum of 0 is exact, so no case hangs between the two sides
        u.check(got[:, :F], d * U * u.slope(G, act), np.abs(d) * np.abs(U) * (1 + np.abs(G)), kind, "dG %s %s" % (kind, act))
        u.check(got[:, F:], d * u.act(G, act), np.abs(d) * (1 + np.abs(G)), kind, "dU %s %s" % (kind, act))
        assert both.unchanged()


@pytest.mark.parametrize("act", u.ACTS)
def test_gated_grad_against_differences_of_the_forward_pass(mg, act):
    """L = sum(dH * H).  Scaling column j of the gate by 1 +- e changes L by 2 e sum_i dG_ij G_ij (+ e^3), and the
    same for the other projection, which is linear."""
    M, F, K, e = 24, 40, 96, 2.0 ** -7
    rng, X, x_s, weights, floats, m8, mf = layer_case(M, F, K, "f32", act, "dense", seed=3)
    (Wg, g_s), (Wu, u_s) = weights(), weights()
    d = floats()
    x, wg, wu, dh = m8(X), m8(Wg), m8(Wu), mf(d)
    dg, du = mf(), mf()
    mg.mipgemm_s8s8_gated_grad(0, mg.ACTIVATIONS[act], M, F, K, x.ptr, x.ld, u.vector(x_s), wg.ptr, wg.ld, u.vector(g_s), wu.ptr, wu.ld,
                               u.vector(u_s), dh.ptr, dh.ld, dg.ptr, dg.ld, du.ptr, du.ld)
    def loss(gs, us):
        h = mf()
        mg.mipgemm_s8s8_gated(0, mg.ACTIVATIONS[act], M, F, K, x.ptr, x.ld, u.vector(x_s), wg.ptr, wg.ld, u.vector(gs), wu.ptr, wu.ld,
                              u.vector(us), h.ptr, h.ld)
        return (d * h.get()).sum(axis=0)
    one = np.float32(1)
    by_g = (loss(g_s * (one + np.float32(e)), u_s) - loss(g_s * (one - np.float32(e)), u_s)) / (2 * e)
    by_u = (loss(g_s, u_s * (one + np.float32(e))) - loss(g_s, u_s * (one - np.float32(e)))) / (2 * e)
    G = u.sums(X, Wg) * x_s[:, None].astype(np.float64) * g_s.astype(np.float64)
    U = u.sums(X, Wu) * x_s[:, None].astype(np.float64) * u_s.astype(np.float64)
    # third derivatives of the activations are below 2 in magnitude: e^2 |G|^3 / 3 per element; the rounding of the
    # two losses, ARITH each, is divided by e
    tol_g = (np.abs(d * U) * (e * e * np.abs(G) ** 3 + 2 * u.ARITH / e * (1 + np.abs(G)))).sum(axis=0)
    tol_u = (np.abs(d * U) * 2 * u.ARITH / e * (1 + np.abs(G))).sum(axis=0)
    assert (np.abs((dg.get() * G).sum(axis=0) - by_g) <= tol_g).all()
    assert (np.abs((du.get() * U).sum(axis=0) - by_u) <= tol_u).all()


def test_infinite_and_nan_scales_reach_exactly_their_rows_and_columns(mg):
    """A row quantized from infinities has scale NaN: its outputs are NaN, no others are."""
    for M, N, K in [(4, 2400, 256), (150, 300, 160)]:
        rng, A, a_s, weights, floats, m8, mf = layer_case(M, N, K, "f32", "silu", "dense")
        W, w_s = weights()
        a_s[M // 2] = np.nan
        w_s[5] = np.inf
        a, w, c, h = m8(A), m8(W), mf(), mf()
        mg.mipgemm_s8s8_linear(0, 0, M, N, K, a.ptr, a.ld, u.vector(a_s), w.ptr, w.ld, u.vector(w_s), None, None, 0, c.ptr, c.ld)
        got = c.get()
        want = np.isfinite(u.sums(A, W) * a_s[:, None].astype(np.float64) * w_s.astype(np.float64))
        assert np.array_equal(np.isfinite(got), want)
        mg.mipgemm_s8s8_gated(0, 4, M, N, K, a.ptr, a.ld, u.vector(a_s), w.ptr, w.ld, None, w.ptr, w.ld, None, h.ptr, h.ld)
        assert np.array_equal(np.isnan(h.get()).any(axis=1), np.isnan(a_s))


def test_extreme_activations_saturate(mg):
    """Sums far outside the exponential's range: the limits of the activations, never NaN."""
    M, N, K = 3, 64, 512
    A = np.full((M, K), 127, np.int8)
    W = np.where(np.arange(N)[:, None] % 2 == 0, 127, -128) * np.ones((N, K), np.int64)
    W = W.astype(np.int8)
    a, w = u.Matrix(M, K, "s8", K, 0, A), u.Matrix(N, K, "s8", K, 0, W)
    for act in u.ACTS:
        c = u.Matrix(M, N, "f32")
        mg.mipgemm_s8s8_linear(0, mg.ACTIVATIONS[act], M, N, K, a.ptr, K, None, w.ptr, K, None, None, None, 0, c.ptr, N)
        z = u.sums(A, W)
        want = z if act == "none" else np.maximum(z, 0)
        assert np.array_equal(c.get(), want), act
        dg, du = u.Matrix(M, N, "f32"), u.Matrix(M, N, "f32")
        dh = u.Matrix(M, N, "f32", values=np.ones((M, N)))
        mg.mipgemm_s8s8_gated_grad(0, mg.ACTIVATIONS[act], M, N, K, a.ptr, K, None, w.ptr, K, None, w.ptr, K, None, dh.ptr, N, dg.ptr, N, du.ptr, N)
        step = np.ones_like(z) if act == "none" else (z > 0)
        assert np.array_equal(dg.get(), z * step) and np.array_equal(du.get(), want), act


def test_gated_grad_in_place(mg):
    """dG may be dH itself: every element is read before it is written."""
    for M, F, K in [(5, 300, 128), (200, 513, 160)]:
        rng, X, x_s, weights, floats, m8, mf = layer_case(M, F, K, "bf16", "silu", "dense")
        (Wg, g_s), (Wu, u_s) = weights(), weights()
        d = floats()
        x, wg, wu = m8(X), m8(Wg), m8(Wu)
        outs = []
        for where in (None, "g", "u"):
            dh, dg, du = mf(d), mf(), mf()
            g, v = (dh if where == "g" else dg), (dh if where == "u" else du)
            mg.mipgemm_s8s8_gated_grad(2, 4, M, F, K, x.ptr, x.ld, u.vector(x_s), wg.ptr, wg.ld, u.vector(g_s), wu.ptr, wu.ld, u.vector(u_s),
                                       dh.ptr, dh.ld, g.ptr, g.ld, v.ptr, v.ld)
            outs.append((g.get(), v.get()))
        for other in outs[1:]:
            assert np.array_equal(outs[0][0], other[0]) and np.array_equal(outs[0][1], other[1])


def test_results_do_not_depend_on_the_run(mg):
    """Two calls on the same operands give the same bits (integer sums, no floating atomics)."""
    import torch
    for M, N, K in [(4, 4096, 1024), (700, 900, 528)]:
        rng, A, a_s, weights, floats, m8, mf = layer_case(M, N, K, "f32", "silu", "dense")
        W, w_s = weights()
        a, w = m8(A), m8(W)
        outs = []
        for _ in range(2):
            c = mf()
            mg.mipgemm_s8s8_gated(0, 4, M, N, K, a.ptr, a.ld, u.vector(a_s), w.ptr, w.ld, u.vector(w_s), w.ptr, w.ld, u.vector(w_s), c.ptr, c.ld)
            outs.append(c.view.clone())
        assert torch.equal(outs[0], outs[1])


def test_other_streams_and_chains(mg):
    """A chain on a side stream -- quantize, linear, quantize, gated, quantize, linear -- equals the same chain with a
    synchronisation after every call: each launch waits for what it reads."""
    import torch
    M, K, N = 37, 512, 640
    rng = np.random.default_rng(5)
    x0 = torch.from_numpy(rng.standard_normal((M, K)).astype(np.float32)).cuda().bfloat16()
    w1, w2, w3 = (u.Matrix(n, k, "s8", k, 0, u.codes(rng, n, k)) for n, k in ((N, K), (2 * N, N), (K, N)))
    s1, s2, s3 = (u.vector(u.scales(rng, n, 1 / (74 * k ** 0.5))) for n, k in ((N, K), (2 * N, N), (K, N)))
    def chain(sync):
        q1, q2, q3 = (torch.empty(M, k, dtype=torch.int8, device="cuda") for k in (K, N, N))
        t = [torch.empty(M, device="cuda") for _ in range(3)]
        y, h = (torch.empty(M, N, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        out = x0.clone()
        steps = [
            lambda: mg.mipgemm_quantize_rows(2, M, K, x0, K, q1, K, t[0]),
            lambda: mg.mipgemm_s8s8_linear(2, 2, M, N, K, q1, K, t[0], w1.ptr, K, s1, None, None, 0, y, N),
            lambda: mg.mipgemm_quantize_rows(2, M, N, y, N, q2, N, t[1]),
            lambda: mg.mipgemm_s8s8_gated(2, 4, M, N, N, q2, N, t[1], w2.ptr, N, s2, w2.ptr + N * N, N, s2[N:], h, N),
            lambda: mg.mipgemm_quantize_rows(2, M, N, h, N, q3, N, t[2]),
            lambda: mg.mipgemm_s8s8_linear(2, 0, M, K, N, q3, N, t[2], w3.ptr, N, s3, None, out, K, out, K)]
        for f in steps:
            f()
            if sync:
                torch.cuda.synchronize()
        return out
    want = chain(True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        with torch.cuda.stream(side):
            got = chain(False)
        side.synchronize()
        assert torch.equal(got, want)


def test_offsets_beyond_32_bits(mg):
    """Pitches that put the rows of every matrix more than 2^32 bytes apart from the first."""
    import torch
    M, N, K = 3, 48, 64
    ld8, ldf = (1 << 31) + 64, (1 << 30) + 32
    rng = np.random.default_rng(11)
    A, W = u.codes(rng, M, K), u.codes(rng, N, K)
    a_s, w_s = u.scales(rng, M, 1 / 74), u.scales(rng, N, 1 / (74 * K ** 0.5))
    buf = torch.empty(2 * ld8 + K, dtype=torch.int8, device="cuda")
    for i in range(M):
        buf[i * ld8:i * ld8 + K] = torch.from_numpy(A[i]).cuda()
    w = u.Matrix(N, K, "s8", K, 0, W)
    c = torch.empty(2 * ldf + N, dtype=torch.float32, device="cuda")
    mg.mipgemm_s8s8_linear(0, 0, M, N, K, buf, ld8, u.vector(a_s), w.ptr, K, u.vector(w_s), None, None, 0, c, ldf)
    z = u.sums(A, W) * a_s[:, None].astype(np.float64) * w_s.astype(np.float64)
    got = np.stack([c[i * ldf:i * ldf + N].double().cpu().numpy() for i in range(M)])
    u.check(got, z, np.abs(z), "f32")
    del c
    x = torch.empty(2 * ldf + N, dtype=torch.bfloat16, device="cuda")
    q = torch.empty(2 * ld8 + N, dtype=torch.int8, device="cuda")
    sc = torch.empty(M, device="cuda")
    vals = u.rounded(rng.standard_normal((M, N)), "bf16")
    for i in range(M):
        x[i * ldf:i * ldf + N] = torch.from_numpy(vals[i]).cuda().bfloat16()
    mg.mipgemm_quantize_rows(2, M, N, x, ldf, q, ld8, sc)
    x.zero_()
    mg.mipgemm_dequantize_rows(2, M, N, q, ld8, sc, x, ldf)
    got = np.stack([x[i * ldf:i * ldf + N].double().cpu().numpy() for i in range(M)])
    step = np.abs(vals).max(axis=1, keepdims=True) / 127
    assert (np.abs(got - vals) <= step * 0.501 + np.abs(vals) * 2.0 ** -8).all()
