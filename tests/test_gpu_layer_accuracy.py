"""Activations and their gradients where they are small: relative accuracy of their negative tails, in every kernel form.

One product of two codes times a power of two is the activation's argument, so that nothing is rounded before it.  The
bounds come from the formulas, in units of the binary32 half unit h = 2^-24, relative to the terms that are added:
  * a sigmoid of y: the exponential's argument is rounded where it is formed (silu: the product with log2 e and that
    constant, 1.5 y h; gelu_tanh: up to six roundings and three constants, 7.5 y h), the instruction has 2 units (4 h), the
    sum and the reciprocal 3 h, the product with x 1 h (9 with the other factors, which are exact here);
  * the normal integral: 14 h of its polynomial (1.3 of the fit, the rest from t with 3 h and the evaluation, found by trying
    every t), 1.25 x^2 h and 4 h of the exponential, the products 3 h (22 with one more in the slope).
The slopes add up terms with these errors; 12 h more cover the factors between them.
"""
import numpy as np
import pytest

import layer_util as u
from test_gpu_layer_paths import mg  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu

H = 2.0 ** -24
#: kernel forms: M, N, K, tuning.  (K beyond 1 is zeros.)
FORMS = {"dense": (200, 256, 128, dict(split_k=1)), "few": (16, 256, 128, {}), "split": (200, 256, 1024, dict(split_k=2)),
         "odd": (201, 251, 1, dict(split_k=1))}


def phi(x):
    import torch
    return torch.special.log_ndtr(torch.from_numpy(x)).exp().numpy()


def reference(z, kind):
    """The activation, its slope, and the relative rounding of the terms of each, for z < 0."""
    if kind == "gelu":
        cdf, pdf = phi(z), np.exp(-z * z / 2) / np.sqrt(2 * np.pi)
        err = (1.25 * z * z + 22) * H
        return z * cdf, cdf + z * pdf, err, err * (cdf + np.abs(z) * pdf)
    if kind == "silu":
        inner, d, err = z, 1.0, (1.5 * np.abs(z) + 9) * H
    else:
        c = np.sqrt(2 / np.pi)
        inner, d = 2 * c * (z + 0.044715 * z ** 3), 2 * c * (1 + 3 * 0.044715 * z * z)
        err = (7.5 * np.abs(inner) + 9) * H
    e = np.exp(inner) / (1 + np.exp(inner))
    slope = e + z * e * (1 - e) * d
    return z * e, slope, err, (err + 12 * H) * (e + np.abs(z) * e * (1 - e) * d)


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_small_values_keep_their_relative_size(mg, form, act):
    M, N, K, tuning = FORMS[form]
    mg.mipgemm_set_tuning(**tuning)
    rng = np.random.default_rng(17)
    # arguments -a b / 1024, from -12.5 (gelu; -80 in a sigmoid's exponent) to -2^-10
    A, W = np.zeros((M, K), np.int8), np.zeros((N, K), np.int8)
    A[:, 0], W[:, 0] = rng.integers(1, 128, M), -rng.integers(1, 101, N)
    V = np.zeros((N, K), np.int8)
    V[:, 0] = 1
    step = {"gelu": 2.0 ** -10, "gelu_tanh": 2.0 ** -11, "silu": 2.0 ** -8}[act]
    z = A[:, :1].astype(np.float64) * W[:, 0] * step
    assert z.min() >= {"gelu": -12.5, "gelu_tanh": -9.0, "silu": -80.0}[act]
    value, slope, err, slope_err = reference(z, act)
    a, w, v = (u.Matrix(*x.shape, "s8", values=x) for x in (A, W, V))
    s = u.vector(np.full(N, step))
    c = u.Matrix(M, N, "f32")
    mg.mipgemm_s8s8_linear(0, mg.ACTIVATIONS[act], M, N, K, a.ptr, K, None, w.ptr, K, s, None, None, 0, c.ptr, N)
    path = mg.mipgemm_last_path()
    assert (path & mg.PATH_MASK == mg.PATH_SKINNY) == (form == "few") and bool(path & mg.PATH_SPLITK) == (form == "split")
    assert (np.abs(c.get() - value) <= err * np.abs(value)).all()
    # the gradients, with dH = 1 and U = a (an exact integer): dG = a slope, dU = value
    dh, dg, du = u.Matrix(M, N, "f32", values=np.ones((M, N))), u.Matrix(M, N, "f32"), u.Matrix(M, N, "f32")
    mg.mipgemm_s8s8_gated_grad(0, mg.ACTIVATIONS[act], M, N, K, a.ptr, K, None, w.ptr, K, s, v.ptr, K, None, dh.ptr, N, dg.ptr, N, du.ptr, N)
    assert mg.mipgemm_device_status() == mg.OK
    U = A[:, :1].astype(np.float64)
    assert (np.abs(du.get() - value) <= err * np.abs(value)).all()
    assert (np.abs(dg.get() - U * slope) <= U * slope_err).all()
    # 16-bit results: one rounding more
    c = u.Matrix(M, N, "bf16")
    mg.mipgemm_s8s8_linear(mg.TYPES["bf16"], mg.ACTIVATIONS[act], M, N, K, a.ptr, K, None, w.ptr, K, s, None, None, 0, c.ptr, N)
    assert (np.abs(c.get() - value) <= (err + u.ROUND["bf16"] * 1.01) * np.abs(value)).all()


def test_the_far_tail_is_zero_or_tiny(mg):
    """Below the exponential's range the activations are 0 within 1e-35, with no NaN on the way."""
    M = N = 128
    A, W = np.full((M, 1), 127, np.int8), -np.arange(N).astype(np.int8).reshape(N, 1)
    a, w, c = u.Matrix(M, 1, "s8", values=A), u.Matrix(N, 1, "s8", values=W), u.Matrix(M, N, "f32")
    z = u.sums(A, W)
    for act in ("gelu", "gelu_tanh", "silu"):
        mg.mipgemm_s8s8_linear(0, mg.ACTIVATIONS[act], M, N, 1, a.ptr, 1, None, w.ptr, 1, None, None, None, 0, c.ptr, N)
        assert (np.abs(c.get())[z < -110] <= 1e-35).all() and not np.isnan(c.get()).any()


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("act", u.ACTS)
def test_slopes_at_large_finite_arguments(mg, form, act):
    """|G| up to 1e30, whose square is beyond binary32: the slopes are 1 and 0 (1 and 1 without an activation), not NaN."""
    M, N, K, tuning = FORMS[form]
    mg.mipgemm_set_tuning(**tuning)
    A, W, V = np.zeros((M, K), np.int8), np.zeros((N, K), np.int8), np.zeros((N, K), np.int8)
    A[:, 0], W[:, 0], V[:, 0] = 1, np.where(np.arange(N) % 2, -1, 1), 3
    size = 10.0 ** np.linspace(3, 30, N)
    a, w, v = (u.Matrix(*x.shape, "s8", values=x) for x in (A, W, V))
    dh, dg, du = u.Matrix(M, N, "f32", values=np.full((M, N), 2.0)), u.Matrix(M, N, "f32"), u.Matrix(M, N, "f32")
    mg.mipgemm_s8s8_gated_grad(0, mg.ACTIVATIONS[act], M, N, K, a.ptr, K, None, w.ptr, K, u.vector(size), v.ptr, K, None, dh.ptr, N, dg.ptr, N,
                               du.ptr, N)
    positive = W[:, 0] > 0
    G = W[:, 0] * size.astype(np.float32).astype(np.float64)
    assert np.array_equal(dg.get(), np.broadcast_to(np.where(positive | (act == "none"), 6.0, 0.0), (M, N)))
    assert np.array_equal(du.get(), np.broadcast_to((2 * np.where(positive | (act == "none"), G, 0.0)).astype(np.float32), (M, N)))


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
def test_a_nan_of_the_gate_reaches_its_gradient(mg, form, act):
    """A gate row quantized from an infinity or a NaN has scale NaN: both gradients of its column are NaN, no others."""
    M, N, K, tuning = FORMS[form]
    mg.mipgemm_set_tuning(**tuning)
    A, W = np.zeros((M, K), np.int8), np.zeros((N, K), np.int8)
    A[:, 0], W[:, 0] = 1, np.where(np.arange(N) % 2, -1, 1)
    scale = np.ones(N)
    scale[[3, 10, N - 1]] = np.nan
    a, w = u.Matrix(M, K, "s8", values=A), u.Matrix(N, K, "s8", values=W)
    for kind in ("f32", "bf16"):
        dh, dg, du = u.Matrix(M, N, kind, values=np.ones((M, N))), u.Matrix(M, N, kind), u.Matrix(M, N, kind)
        mg.mipgemm_s8s8_gated_grad(mg.TYPES[kind], mg.ACTIVATIONS[act], M, N, K, a.ptr, K, None, w.ptr, K, u.vector(scale), w.ptr, K, None,
                                   dh.ptr, N, dg.ptr, N, du.ptr, N)
        for got in (dg.get(), du.get()):
            assert np.array_equal(np.isnan(got), np.broadcast_to(np.isnan(scale), (M, N)))
