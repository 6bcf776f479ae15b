"""bfloat16 gradients times 8-bit codes with scales along the summed axis, against 64 bits."""
import numpy as np
import pytest

import layer_util as u

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mg():
    from paper_2506_11728_b200 import binding
    return binding


SIZES = [(1, 1, 1), (1, 64, 64), (3, 33, 17), (16, 128, 72), (100, 40, 129), (128, 256, 64), (129, 257, 65), (256, 128, 200),
         (300, 520, 328), (257, 1000, 136), (640, 136, 1000), (8, 2048, 512), (2000, 24, 96), (40, 48, 0), (200, 264, 4096)]
LAYOUTS = {"dense": (0, 0), "padded": (16, 16), "odd": (3, 1)}


def operands(M, N, K, order, layout, seed=0, small=False):
    rng = np.random.default_rng([M, N, K, order, seed])
    pad, shift = LAYOUTS[layout]
    shape = (K, M) if order else (M, K)
    a = rng.integers(-8, 9, shape).astype(np.float64) if small else u.rounded(rng.standard_normal(shape), "bf16")
    b = rng.integers(-128, 128, (K, N)).astype(np.int8)
    s = 2.0 ** rng.integers(-2, 3, K) if small else u.scales(rng, K, 1 / 74)
    A = u.Matrix(shape[0], shape[1], "bf16", shape[1] + pad if shape[1] + pad else 1, shift, a)
    B = u.Matrix(K, N, "s8", N + pad, shift, b)
    return rng, (a.T if order else a), b.astype(np.float64), s.astype(np.float32), A, B


@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("M,N,K", SIZES)
def test_small_integers_are_exact(mg, M, N, K, layout, order):
    """Integers and power-of-two scales: operands, products and sums are exact in every type involved, so a wrong index,
    a lost term or a term counted twice shows."""
    rng, a, b, s, A, B = operands(M, N, K, order, layout, small=True)
    pad, shift = LAYOUTS[layout]
    C = u.Matrix(M, N, "f32", N + pad, shift)
    mg.mipgemm_bf16s8_product(0, order, M, N, K, A.ptr, A.ld, B.ptr, B.ld, u.vector(s), C.ptr, C.ld)
    assert mg.mipgemm_device_status() == mg.OK
    assert np.array_equal(C.get(), a @ (s[:, None] * b)) and C.unchanged()


@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("M,N,K", SIZES)
def test_product(mg, M, N, K, layout, kind, order):
    rng, a, b, s, A, B = operands(M, N, K, order, layout, 1)
    pad, shift = LAYOUTS[layout]
    for scale, accumulate in ((s, 0), (None, 0), (s, 1)):
        c0 = u.rounded(rng.standard_normal((M, N)), kind)
        C = u.Matrix(M, N, kind, N + pad, shift, c0)
        mg.mipgemm_bf16s8_product(mg.TYPES[kind], order, M, N, K, A.ptr, A.ld, B.ptr, B.ld, u.vector(scale), C.ptr, C.ld, accumulate)
        assert mg.mipgemm_device_status() == mg.OK
        left = b if scale is None else scale[:, None].astype(np.float64) * b
        want = a @ left + (c0 if accumulate else 0)
        total = np.abs(a) @ np.abs(left) + (np.abs(c0) if accumulate else 0)
        # a scaled code is rounded to bfloat16 (2^-8 of itself at most), unscaled codes are exact; K additions in binary32
        tol = total * ((0 if scale is None else 2.0 ** -8) + (K + 2) * 2.0 ** -23) + u.ROUND[kind] * np.abs(want) * 1.01 + 1e-30
        assert (np.abs(C.get() - want) <= tol).all()
        assert C.unchanged()


def test_rounding_of_the_scaled_codes_averages_out(mg):
    """The rounding errors of the scaled codes are independent of each other: over a long sum their share of the
    result's norm stays that of one rounding (2^-8 at most, 2^-9.5 on average)."""
    M, N, K = 256, 256, 4096
    rng, a, b, s, A, B = operands(M, N, K, 0, "dense", 2)
    C = u.Matrix(M, N, "f32")
    mg.mipgemm_bf16s8_product(0, 0, M, N, K, A.ptr, A.ld, B.ptr, B.ld, u.vector(s), C.ptr, C.ld)
    want = a @ (s[:, None].astype(np.float64) * b)
    assert np.linalg.norm(C.get() - want) <= 2.0 ** -9 * np.linalg.norm(want)


def test_product_is_the_gradient_of_linear(mg):
    """Raising one code of X by one changes L = sum(dY * Y), Y = linear(X, W), by x_scale * dX: the forward pass is
    linear in the codes, so the difference is the derivative.  The same for the weights."""
    M, N, K = 20, 48, 64
    rng = np.random.default_rng(9)
    X, W = rng.integers(-100, 100, (M, K)).astype(np.int8), rng.integers(-100, 100, (N, K)).astype(np.int8)
    xs, ws = u.scales(rng, M, 1 / 74), u.scales(rng, N, 1 / 600)
    dY = u.rounded(rng.standard_normal((M, N)), "bf16")
    d = u.Matrix(M, N, "bf16", values=dY)
    x, w = u.Matrix(M, K, "s8", values=X), u.Matrix(N, K, "s8", values=W)
    dX, dW = u.Matrix(M, K, "f32"), u.Matrix(N, K, "f32")
    mg.mipgemm_bf16s8_product(0, 0, M, K, N, d.ptr, N, w.ptr, K, u.vector(ws), dX.ptr, K)
    mg.mipgemm_bf16s8_product(0, 1, N, K, M, d.ptr, N, x.ptr, K, u.vector(xs), dW.ptr, K)
    def loss(Xc, Wc):
        a, b, y = u.Matrix(M, K, "s8", values=Xc), u.Matrix(N, K, "s8", values=Wc), u.Matrix(M, N, "f32")
        mg.mipgemm_s8s8_linear(0, 0, M, N, K, a.ptr, K, u.vector(xs), b.ptr, K, u.vector(ws), None, None, 0, y.ptr, N)
        return (dY * y.get()).sum()
    base = loss(X, W)
    size = (np.abs(dY) @ (np.abs(W) * ws[:, None])).max()
    for i, k in [(0, 0), (7, 63), (19, 31)]:
        X2 = X.copy()
        X2[i, k] += 1
        assert abs((loss(X2, W) - base) - xs[i] * dX.get()[i, k]) <= xs[i] * size * 2.0 ** -7
    size = (np.abs(dY).T @ (np.abs(X) * xs[:, None])).max()
    for j, k in [(0, 0), (47, 63), (21, 5)]:
        W2 = W.copy()
        W2[j, k] += 1
        assert abs((loss(X, W2) - base) - ws[j] * dW.get()[j, k]) <= ws[j] * size * 2.0 ** -7


def test_nan_and_infinite_scales_stay_in_the_sum(mg):
    M, N, K = 130, 140, 96
    rng, a, b, s, A, B = operands(M, N, K, 1, "dense", 4)
    s[70] = np.nan
    C = u.Matrix(M, N, "bf16")
    mg.mipgemm_bf16s8_product(2, 1, M, N, K, A.ptr, A.ld, B.ptr, B.ld, u.vector(s), C.ptr, C.ld)
    assert np.isnan(C.get()).all()
