"""Kernels of the 8-bit layer whose waits run out, in every form: they return, say so once, and what runs after them on the
same SMs is right.  The "accumulator ready" signal is withheld, so that waits expire after 0.2 ms; with more tiles than
CTAs the producers are stopped in the middle of their work."""
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
