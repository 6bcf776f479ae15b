"""Kernels of the 8-bit layer whose waits run out, in every form: they return, say so once, and what runs after them on the
same SMs is right.  The "accumulator ready" signal is withheld, so that waits expire after 0.2 ms; with more tiles than
CTAs the producers are stopped in the middle of their work."""
import numpy as np
import pytest

import layer_util as u
from test_gpu_layer_paths import mg, problem, run_all  # noqa: F401 (mg is a fixture)

pytestmark = pytest.mark.gpu

SIZES = [(300, 416, 1024), (2500, 1544, 1300)]       # one tile a CTA, several


def expire(mg, call):
    mg.mipgemm_debug_set(1, 200_000)
    try:
        call()
        assert mg.mipgemm_device_status() == mg.ERR_TIMEOUT
        assert mg.mipgemm_device_status() == mg.OK
    finally:
        mg.mipgemm_debug_set(0, 0)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("split", [1, 2])
@pytest.mark.parametrize("form", ["one", "pair"])
def test_layer_kernel(mg, form, split, kind):
    mg.mipgemm_set_tuning(block_n=64, split_k=split, force_path=mg.PATH_DENSE if form == "one" else mg.PATH_DENSE_PAIR)
    t = mg.TYPES[kind]
    for M, N, K in SIZES[:1] if split > 1 else SIZES:
        p, d, G, U = problem(M, N, K, kind=kind)
        c, c2 = u.Matrix(M, N, kind), u.Matrix(M, N, kind)
        block = (p["A"].ptr, K, p["a_s"], p["W"].ptr, K, p["w_s"], p["V"].ptr, K, p["v_s"])
        for call in (lambda: mg.mipgemm_s8s8_linear(t, 2, M, N, K, *block[:6], None, p["d"].ptr, N, c.ptr, N),
                     lambda: mg.mipgemm_s8s8_gated(t, 4, M, N, K, *block, c.ptr, N),
                     lambda: mg.mipgemm_s8s8_gated_grad(t, 4, M, N, K, *block, p["d"].ptr, N, c.ptr, N, c2.ptr, N)):
            expire(mg, call)
        run_all(mg, M, N, K, kind)


@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("split", [1, 2])
@pytest.mark.parametrize("form", ["one", "pair"])
def test_product_kernel(mg, form, split, order):
    mg.mipgemm_set_tuning(split_k=split, force_path=mg.PATH_DENSE if form == "one" else mg.PATH_DENSE_PAIR)
    for M, N, K in [(300, 416, 1000), (4100, 2608, 1000)][:1 if split > 1 else 2]:
        rng = np.random.default_rng([M, N, K])
        a = rng.integers(-8, 9, (M, K)).astype(np.float64)
        b = rng.integers(-128, 128, (K, N)).astype(np.int8)
        s = 2.0 ** rng.integers(-2, 3, K)
        A, B = u.Matrix(*((K, M) if order else (M, K)), "bf16", M + 4 if order else K, 0, a.T if order else a), u.Matrix(K, N, "s8", values=b)
        for kind in ("bf16", "f32"):
            C = u.Matrix(M, N, kind)
            call = lambda: mg.mipgemm_bf16s8_product(mg.TYPES[kind], order, M, N, K, A.ptr, A.ld, B.ptr, N, u.vector(s), C.ptr, N)
            expire(mg, call)
            call()
            assert mg.mipgemm_device_status() == mg.OK
            assert np.array_equal(C.get(), u.rounded(a @ (s[:, None] * b), kind))
