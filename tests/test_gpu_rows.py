"""Rows to 8-bit codes and back, against the rule evaluated in binary32 and the definition in 64 bits."""
import numpy as np
import pytest

import layer_util as u

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mg():
    from paper_2506_11728_b200 import binding
    return binding


SHAPES = [(1, 1), (1, 7), (2, 16), (3, 33), (8, 4096), (5, 4097), (257, 64), (1000, 72), (3, 5000), (4, 11008),
          (2, 40000), (1, 200001), (33, 2048), (130, 1024)]


def rule(x):
    """The documented rule, every step rounded in binary32."""
    x = x.astype(np.float32)
    top = np.abs(x).max(axis=1) if x.shape[1] else np.zeros(x.shape[0], np.float32)
    scale, q = np.zeros(x.shape[0], np.float32), np.zeros(x.shape, np.int64)
    for i in range(x.shape[0]):
        if not np.isfinite(x[i]).all():
            scale[i] = np.nan
        elif top[i] >= np.float32(2.0 ** -119):
            scale[i] = top[i] / np.float32(127)
            q[i] = np.rint(x[i] * (np.float32(127) / top[i]))
    return q, scale


@pytest.mark.parametrize("kind", u.TYPES)
@pytest.mark.parametrize("M,N", SHAPES)
@pytest.mark.parametrize("pad,shift", [(0, 0), (16, 16), (3, 1)])
def test_codes_follow_the_rule_bit_for_bit(mg, M, N, kind, pad, shift):
    rng = np.random.default_rng([M, N])
    x = u.rounded(rng.standard_normal((M, N)) * 2.0 ** rng.integers(-10, 10, (M, 1)), kind)
    X = u.Matrix(M, N, kind, N + pad, shift, x)
    Q = u.Matrix(M, N, "s8", N + pad, shift)
    S = u.Matrix(1, M, "f32")
    mg.mipgemm_quantize_rows(mg.TYPES[kind], M, N, X.ptr, X.ld, Q.ptr, Q.ld, S.ptr)
    assert mg.mipgemm_device_status() == mg.OK
    q, scale = rule(x)
    assert np.array_equal(Q.get(), q) and np.array_equal(S.get()[0], scale)
    assert Q.unchanged() and S.unchanged()
    # half a step of the row's largest magnitude, and the rounding of the quotient (127 units of 2^-23)
    assert (np.abs(q * scale[:, None].astype(np.float64) - x) <= scale[:, None] * (0.5 + 2.0 ** -15)).all()
    # and back: the product, rounded once
    Y = u.Matrix(M, N, kind, N + pad, shift)
    mg.mipgemm_dequantize_rows(mg.TYPES[kind], M, N, Q.ptr, Q.ld, S.ptr, Y.ptr, Y.ld)
    back = u.rounded((q.astype(np.float32) * scale[:, None]).astype(np.float64), kind)
    assert np.array_equal(Y.get(), back) and Y.unchanged()


@pytest.mark.parametrize("kind", u.TYPES)
@pytest.mark.parametrize("N", [9, 512, 9000, 70000])
def test_rows_of_zeros_infinities_and_tiny_values(mg, kind, N):
    x = np.zeros((7, N))
    x[1, N // 2] = np.inf
    x[2, N - 1] = np.nan
    x[3, 0] = -np.inf
    x[4] = u.rounded(np.full(N, 1e-40), kind)              # below the smallest row that is kept (0 in f16)
    x[5] = u.rounded(np.linspace(-6e-5, 6e-5, N), kind)    # subnormal in f16
    x[6, ::3] = u.rounded(np.array([6e4]), kind)[0]
    X, Q, S = u.Matrix(7, N, kind, values=x), u.Matrix(7, N, "s8"), u.Matrix(1, 7, "f32")
    mg.mipgemm_quantize_rows(mg.TYPES[kind], 7, N, X.ptr, N, Q.ptr, N, S.ptr)
    q, scale = rule(x)
    assert np.array_equal(Q.get(), q)
    assert np.array_equal(S.get()[0], scale, equal_nan=True)
    Y = u.Matrix(7, N, kind)
    mg.mipgemm_dequantize_rows(mg.TYPES[kind], 7, N, Q.ptr, N, S.ptr, Y.ptr, N)
    y = Y.get()
    assert np.isnan(y[1:4]).all() and (y[0] == 0).all() and (y[4] == 0).all()


def test_no_columns(mg):
    S = u.Matrix(1, 5, "f32")
    mg.mipgemm_quantize_rows(0, 5, 0, None, 0, None, 0, S.ptr)
    assert (S.get() == 0).all() and S.unchanged()
