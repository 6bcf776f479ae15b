"""Layer operators: kernel forms, host-side state and long queues.

The forms are reached by sizes (and, where a size would be large, by mipgemm_set_tuning); each is compared with the
definition in 64 bits.  Nothing here faults or hangs the GPU: the expiry tests withhold a signal inside the kernel, so
that a bounded wait runs out after a fraction of a millisecond and the kernel returns with an error status."""
import numpy as np
import pytest

import layer_util as u

pytestmark = pytest.mark.gpu


@pytest.fixture
def mg():
    from paper_2506_11728_b200 import binding
    binding.mipgemm_set_tuning()
    yield binding
    binding.mipgemm_set_tuning()
    binding.mipgemm_set_weights_constant(0)
    binding.mipgemm_set_workspace(None)


def problem(M, N, K, seed=0, kind="bf16"):
    rng = np.random.default_rng([M, N, K, seed])
    A, W, V = u.codes(rng, M, K), u.codes(rng, N, K), u.codes(rng, N, K)
    a_s, w_s, v_s = u.scales(rng, M, 1 / 74), u.scales(rng, N, 1 / (74 * K ** 0.5)), u.scales(rng, N, 1 / (74 * K ** 0.5))
    d = u.rounded(rng.standard_normal((M, N)), kind)
    G = u.sums(A, W) * a_s[:, None].astype(np.float64) * w_s
    U = u.sums(A, V) * a_s[:, None].astype(np.float64) * v_s
    dev = dict(A=u.Matrix(M, K, "s8", values=A), W=u.Matrix(N, K, "s8", values=W), V=u.Matrix(N, K, "s8", values=V),
               a_s=u.vector(a_s), w_s=u.vector(w_s), v_s=u.vector(v_s), d=u.Matrix(M, N, kind, values=d))
    return dev, d, G, U


def run_all(mg, M, N, K, kind="bf16", seed=0):
    """linear with residual, gated and gated_grad on one problem; returns the path of each."""
    p, d, G, U = problem(M, N, K, seed, kind)
    t, paths = mg.TYPES[kind], []
    c = u.Matrix(M, N, kind)
    mg.mipgemm_s8s8_linear(t, 0, M, N, K, p["A"].ptr, K, p["a_s"], p["W"].ptr, K, p["w_s"], None, p["d"].ptr, N, c.ptr, N)
    paths.append(mg.mipgemm_last_path())
    u.check(c.get(), G + d, 1 + np.abs(G) + np.abs(d), kind, "linear")
    h = u.Matrix(M, N, kind)
    mg.mipgemm_s8s8_gated(t, 4, M, N, K, p["A"].ptr, K, p["a_s"], p["W"].ptr, K, p["w_s"], p["V"].ptr, K, p["v_s"], h.ptr, N)
    paths.append(mg.mipgemm_last_path())
    u.check(h.get(), u.act(G, "silu") * U, (1 + np.abs(G)) * np.abs(U), kind, "gated")
    dg, du = u.Matrix(M, N, kind), u.Matrix(M, N, kind)
    mg.mipgemm_s8s8_gated_grad(t, 4, M, N, K, p["A"].ptr, K, p["a_s"], p["W"].ptr, K, p["w_s"], p["V"].ptr, K, p["v_s"], p["d"].ptr, N,
                               dg.ptr, N, du.ptr, N)
    paths.append(mg.mipgemm_last_path())
    u.check(dg.get(), d * U * u.slope(G, "silu"), np.abs(d) * np.abs(U) * (1 + np.abs(G)), kind, "dG")
    u.check(du.get(), d * u.act(G, "silu"), np.abs(d) * (1 + np.abs(G)), kind, "dU")
    assert mg.mipgemm_device_status() == mg.OK
    return paths


@pytest.mark.parametrize("kind", u.TYPES)
@pytest.mark.parametrize("block_n", [64, 128, 192, 256])
@pytest.mark.parametrize("form", ["one", "pair"])
def test_every_dense_tile(mg, kind, block_n, form):
    path = mg.PATH_DENSE if form == "one" else mg.PATH_DENSE_PAIR
    mg.mipgemm_set_tuning(block_n=block_n, split_k=1, force_path=path)
    for M, N, K in [(300, 416, 272), (140, 1000, 2304)]:       # 16 and 8 epilogue warps for 16-bit types
        assert [x & mg.PATH_MASK for x in run_all(mg, M, N, K, kind)] == [path] * 3


@pytest.mark.parametrize("kind", u.TYPES)
@pytest.mark.parametrize("form", ["one", "pair"])
@pytest.mark.parametrize("split", [2, 3, 5])
def test_split_k(mg, kind, form, split):
    path = mg.PATH_DENSE if form == "one" else mg.PATH_DENSE_PAIR
    mg.mipgemm_set_tuning(split_k=split, force_path=path)
    for M, N, K in [(150, 197, 4000), (257, 96, 2600)]:
        for x in run_all(mg, M, N, K, kind):
            assert x & mg.PATH_MASK == path and x & mg.PATH_SPLITK


@pytest.mark.parametrize("M", [1, 2, 5, 16, 17, 32, 33, 47, 64])
def test_few_tokens(mg, M):
    for N, K in [(160, 6400), (1000, 6272), (4096, 6144)]:
        for x in run_all(mg, M, N, K):
            assert x & mg.PATH_MASK == mg.PATH_SKINNY


@pytest.mark.parametrize("split", [1, 2, 4, 8])
def test_few_tokens_cluster_sizes(mg, split):
    """17 k-blocks over up to 8 CTAs: shares of unequal length, some of them empty."""
    mg.mipgemm_set_tuning(split_k=split)
    for K in (2176, 2170 + 6, 64, 1152):
        run_all(mg, 7, 300, K)
        run_all(mg, 23, 129, K, "f32")


def test_unsigned_few_tokens(mg):
    M, N, K = 9, 260, 1040
    rng = np.random.default_rng(3)
    A, W = u.codes(rng, M, K, True), u.codes(rng, N, K)
    a, w, c = u.Matrix(M, K, "u8", values=A), u.Matrix(N, K, "s8", values=W), u.Matrix(M, N, "f32")
    mg.mipgemm_u8s8_linear(0, 0, M, N, K, a.ptr, K, None, w.ptr, K, None, None, None, 0, c.ptr, N)
    z = u.sums(A, W)
    u.check(c.get(), z, np.abs(z), "f32")


@pytest.mark.parametrize("M", [3, 40, 300])
def test_largest_sums(mg, M):
    """Every product -128 * -128 at the largest K: 2147467264, the largest sum there is, and its conversion."""
    N, K = 32, 131071
    a = u.Matrix(M, K, "s8", K + 1, values=np.full((M, K), -128, np.int8))
    w = u.Matrix(N, K, "s8", K + 1, values=np.where(np.arange(N)[:, None] % 2, 127, -128) * np.ones((N, K), np.int64))
    c = u.Matrix(M, N, "f32")
    mg.mipgemm_s8s8_linear(0, 0, M, N, K, a.ptr, K + 1, None, w.ptr, K + 1, None, None, None, 0, c.ptr, N)
    want = np.where(np.arange(N) % 2, -128.0 * 127 * K, 128.0 * 128 * K).astype(np.float32).astype(np.float64)
    assert np.array_equal(c.get(), np.broadcast_to(want, (M, N)))


@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("form", ["one", "pair"])
@pytest.mark.parametrize("split", [1, 2, 3])
def test_product_forms(mg, order, form, split):
    """Small integers, so that every form gives the same exact numbers; with and without the sum to add to."""
    path = mg.PATH_DENSE if form == "one" else mg.PATH_DENSE_PAIR
    mg.mipgemm_set_tuning(split_k=split, force_path=path)
    for M, N, K in [(300, 197, 900), (129, 264, 1000), (520, 256, 830)]:
        rng = np.random.default_rng([M, N, K])
        a = rng.integers(-8, 9, (M, K)).astype(np.float64)
        b = rng.integers(-128, 128, (K, N)).astype(np.int8)
        s = 2.0 ** rng.integers(-2, 3, K)
        A, B = u.Matrix(*((K, M) if order else (M, K)), "bf16", values=a.T if order else a), u.Matrix(K, N, "s8", values=b)
        want = a @ (s[:, None] * b)
        for accumulate in (0, 1):
            c0 = rng.integers(-100, 101, (M, N)).astype(np.float64)
            C = u.Matrix(M, N, "f32", values=c0)
            mg.mipgemm_bf16s8_product(0, order, M, N, K, A.ptr, A.ld, B.ptr, N, u.vector(s), C.ptr, N, accumulate)
            x = mg.mipgemm_last_path()
            assert x & mg.PATH_MASK == path and bool(x & mg.PATH_SPLITK) == (split > 1)
            assert np.array_equal(C.get(), want + (c0 if accumulate else 0))
        assert mg.mipgemm_device_status() == mg.OK


def test_a_split_that_the_size_does_not_allow(mg):
    """Asked for by mipgemm_set_tuning, it is not taken: the call chooses among those that there are."""
    for split in (6, 9, 16):
        mg.mipgemm_set_tuning(split_k=split)
        run_all(mg, 150, 197, 300)
        run_all(mg, 5, 197, 300)
        A = u.Matrix(150, 100, "bf16", 104, values=np.ones((150, 100)))
        B = u.Matrix(100, 64, "s8", values=np.full((100, 64), 3))
        C = u.Matrix(150, 64, "f32")
        mg.mipgemm_bf16s8_product(0, 0, 150, 64, 100, A.ptr, 104, B.ptr, 64, None, C.ptr, 64)
        assert (C.get() == 300).all()


def test_long_queues_with_scratch(mg):
    """Re-pitched operands, a pair kernel over a split K and the kernel that adds its parts, many calls in flight, on two
    alternating sets of buffers: this combination once stopped making progress.  (Bounded: waits run out after 20 ms.)"""
    import torch
    mg.mipgemm_debug_set(0, 20_000_000)
    try:
        M, N, K = 3893, 197, 12113
        rng = np.random.default_rng(1)
        sets = []
        for _ in range(2):
            a = torch.randn(K, M, device="cuda").bfloat16()
            b = torch.from_numpy(u.codes(rng, K, N)).cuda()
            sets.append((a, b, u.vector(u.scales(rng, K, 1e-3)), torch.empty(M, N, dtype=torch.bfloat16, device="cuda")))
        first = []
        for a, b, s, c in sets:
            mg.mipgemm_bf16s8_product(2, 1, M, N, K, a, M, b, N, s, c, N)
            first.append(c.clone())
        for i in range(60):
            a, b, s, c = sets[i & 1]
            mg.mipgemm_bf16s8_product(2, 1, M, N, K, a, M, b, N, s, c, N)
        assert mg.mipgemm_device_status() == mg.OK
        for (a, b, s, c), want in zip(sets, first):
            assert torch.equal(c, want)                       # the parts are added in the same order every time
            exact = a.double().t() @ (s.double()[:, None] * b.double())
            assert (c.double() - exact).norm() <= 2.0 ** -8 * exact.norm()
    finally:
        mg.mipgemm_debug_set(0, 0)


@pytest.mark.parametrize("M,K", [(4, 512), (300, 512)])
def test_waits_run_out_and_kernels_return(mg, M, K):
    """The "accumulator ready" signal is withheld: the waits expire after 0.2 ms, the status says so once, and the next
    ordinary calls are right."""
    import torch
    N = 256
    p, d, G, U = problem(M, N, K)
    c = u.Matrix(M, N, "bf16")
    g = torch.randn(M, K, device="cuda").bfloat16()
    w = u.Matrix(K, N, "s8", values=u.codes(np.random.default_rng(2), K, N))
    mg.mipgemm_debug_set(1, 200_000)
    try:
        mg.mipgemm_s8s8_gated(2, 4, M, N, K, p["A"].ptr, K, p["a_s"], p["W"].ptr, K, p["w_s"], p["V"].ptr, K, p["v_s"], c.ptr, N)
        assert mg.mipgemm_device_status() == mg.ERR_TIMEOUT
        mg.mipgemm_s8s8_linear(2, 0, M, N, K, p["A"].ptr, K, p["a_s"], p["W"].ptr, K, p["w_s"], None, p["d"].ptr, N, c.ptr, N)
        assert mg.mipgemm_device_status() == mg.ERR_TIMEOUT
        mg.mipgemm_bf16s8_product(2, 0, M, N, K, g, K, w.ptr, N, None, c.ptr, N)
        assert mg.mipgemm_device_status() == mg.ERR_TIMEOUT
    finally:
        mg.mipgemm_debug_set(0, 0)
    assert mg.mipgemm_device_status() == mg.OK
    run_all(mg, M, N, K)


def test_lent_workspace(mg):
    """With a lent buffer the re-pitched operands lie there, K is not split, and too small a buffer is refused."""
    import torch
    M, N, K = 150, 96, 4001
    p, d, G, U = problem(M, N, K)
    need = mg.mipgemm_workspace_query_gemm(M, N, K, p["A"].ptr, K, p["W"].ptr, K, 0, N)
    assert need > 0
    buf = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    base = (buf.data_ptr() + 255) // 256 * 256
    c = u.Matrix(M, N, "f32")
    args = (0, 0, M, N, K, p["A"].ptr, K, p["a_s"], p["W"].ptr, K, p["w_s"], None, None, 0, c.ptr, N)
    mg.mipgemm_set_workspace(base, need - 1)
    assert mg.mipgemm_s8s8_linear(*args, check=False) == mg.ERR_WORKSPACE
    mg.mipgemm_set_workspace(base, need)
    mg.mipgemm_s8s8_linear(*args)
    assert mg.mipgemm_last_path() & mg.PATH_REPACK and not mg.mipgemm_last_path() & mg.PATH_SPLITK
    u.check(c.get(), G, np.abs(G), "f32")
    mg.mipgemm_set_workspace(None)


def test_scratch_blocks_belong_to_their_stream(mg):
    """Calls that need scratch, on two streams at once and after the blocks have been released."""
    import torch
    M, N, K = 200, 130, 1501
    p, d, G, U = problem(M, N, K, kind="f32")
    outs = [[u.Matrix(M, N, "f32") for _ in range(6)] for _ in range(2)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for i in range(6):
        for s, st in enumerate(streams):
            mg.mipgemm_s8s8_linear(0, 0, M, N, K, p["A"].ptr, K, p["a_s"], p["W"].ptr, K, p["w_s"], None, None, 0, outs[s][i].ptr, N, stream=st)
        if i == 3:
            mg.mipgemm_release_staging()
    torch.cuda.synchronize()
    for group in outs:
        for c in group:
            u.check(c.get(), G, np.abs(G), "f32")


def test_captured_in_a_graph(mg):
    """Operands that need scratch, a split K and the few-token form, captured once and replayed on changed inputs."""
    import torch
    for M, N, K in [(3, 130, 501), (150, 96, 4001), (300, 416, 256)]:
        p, d, G, U = problem(M, N, K, kind="f32")
        c = u.Matrix(M, N, "f32")
        call = lambda: mg.mipgemm_s8s8_linear(0, 0, M, N, K, p["A"].ptr, K, p["a_s"], p["W"].ptr, K, p["w_s"], None, None, 0, c.ptr, N)
        call()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        p["a_s"].mul_(2.0)
        c.view.zero_()
        g.replay()
        torch.cuda.synchronize()
        u.check(c.get(), 2 * G, 2 * np.abs(G), "f32")


@pytest.mark.parametrize("K", [1024, 1003])
@pytest.mark.parametrize("how", ["switch", "range"])
def test_constant_weights_promise(mg, how, K):
    """Early fetch of the weights changes no result, in a chain whose tokens come from the previous call.  With K = 1003 the
    weights are re-pitched in each call, into scratch that the previous call's weights lay in: those are not constant."""
    import torch
    M = 4
    rng = np.random.default_rng(8)
    W = [u.Matrix(K, K, "s8", values=u.codes(rng, K, K)) for _ in range(3)]
    s = u.vector(u.scales(rng, K, 1 / (74 * K ** 0.5)))
    x = torch.from_numpy(rng.standard_normal((M, K)).astype(np.float32)).cuda().bfloat16()
    def chain():
        y = x.clone()
        q, t = torch.empty(M, K, dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
        for i in range(9):
            w = W[i % 3]
            mg.mipgemm_quantize_rows(2, M, K, y, K, q, K, t)
            mg.mipgemm_s8s8_linear(2, 4, M, K, K, q, K, t, w.ptr, K, s, None, y, K, y, K)
        torch.cuda.synchronize()
        return y
    want = chain()
    if how == "switch":
        mg.mipgemm_set_weights_constant(1)
    else:
        for w in W:
            mg.mipgemm_register_constant_weights(w.buf)
    try:
        for _ in range(4):
            assert torch.equal(chain(), want)
    finally:
        mg.mipgemm_set_weights_constant(0)
        if how == "range":
            for w in W:
                mg.mipgemm_unregister_constant_weights(w.buf)
    assert mg.mipgemm_device_status() == mg.OK


def test_plan_cache_serves_layer_calls(mg):
    run_all(mg, 5, 256, 256)
    on, hits, misses = mg.mipgemm_plan_cache_stats()
    p, d, G, U = problem(5, 256, 256, 1)
    c = u.Matrix(5, 256, "f32")
    for _ in range(3):
        mg.mipgemm_s8s8_linear(0, 0, 5, 256, 256, p["A"].ptr, 256, p["a_s"], p["W"].ptr, 256, p["w_s"], None, None, 0, c.ptr, 256)
    if on:
        on, hits2, misses2 = mg.mipgemm_plan_cache_stats()
        assert hits2 - hits == 2 and misses2 - misses == 1
    # scales, bias and activation are not part of a plan
    mg.mipgemm_s8s8_linear(0, 1, 5, 256, 256, p["A"].ptr, 256, None, p["W"].ptr, 256, None, None, None, 0, c.ptr, 256)
    assert (c.get() >= 0).all() and c.get().max() > 100


def test_two_threads_two_streams(mg):
    import threading
    import torch
    res, err = {}, []
    def work(i):
        try:
            torch.cuda.set_device(0)
            st = torch.cuda.Stream()
            M, N, K = (5, 300, 777) if i else (260, 200, 777)
            p, d, G, U = problem(M, N, K, i, "f32")
            torch.cuda.synchronize()
            outs = [u.Matrix(M, N, "f32") for _ in range(10)]
            for c in outs:
                mg.mipgemm_s8s8_linear(0, 0, M, N, K, p["A"].ptr, K, p["a_s"], p["W"].ptr, K, p["w_s"], None, None, 0, c.ptr, N, stream=st)
            st.synchronize()
            for c in outs:
                u.check(c.get(), G, np.abs(G), "f32")
        except Exception as e:          # noqa: BLE001 (reported by the main thread)
            err.append(e)
    ts = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    [t.start() for t in ts]
    [t.join() for t in ts]
    assert not err, err
