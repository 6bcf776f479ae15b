"""Scales at the ends of the range in which the 8-bit floating-point product's error bound is stated."""
import numpy as np
import pytest

import layer_util as u
import test_gpu_float8 as base

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mg():
    from paper_2506_11728_b200 import binding
    binding.mipgemm_set_tuning()
    yield binding
    binding.mipgemm_set_tuning()


@pytest.mark.parametrize("ea,eb", [(-63, -63), (-126, 0), (0, -126), (-120, 118), (118, -120), (57, 57), (0, 110), (110, 0)])
@pytest.mark.parametrize("what", ["forward", "forward_rows", "input_grad", "weight_grad"])
@pytest.mark.parametrize("M,N,K,path", [(9, 200, 300, 0), (40, 200, 300, 1), (300, 520, 300, 2)])
def test_products_at_the_ends_are_exact(mg, M, N, K, path, what, ea, eb):
    """Integers times powers of two: |sum| <= 300 * 16 < 2^13, with scales up to 2^114 below 2^127 and with those from 2^-126 normal, so
    nothing is rounded."""
    rng, a, b, r = base.operands(M, N, K, what, "padded", 9, small=True)
    r["sa"].fill_(2.0 ** ea)
    r["sb"].fill_(2.0 ** eb)
    ao, bo, _ = base.KINDS[what]
    va, vb = base.code_values(r["A"], "e4m3"), base.code_values(r["B"], "e4m3")
    want = (va.T if ao else va) @ (vb if bo else vb.T) * 2.0 ** (ea + eb)
    mg.mipgemm_set_tuning(force_path=path)
    C = u.Matrix(M, N, "f32")
    base.call(mg, "f32", what, M, N, K, r, None, None, C)
    assert np.array_equal(C.get(), want)
