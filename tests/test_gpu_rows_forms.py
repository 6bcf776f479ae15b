"""Rows to 8-bit codes and back in the kernel forms that large shapes reach: four vectors a thread from 2048 rows on, four rows
a thread from 2^20 sixteens on, several rows a block, each with remainders in rows and in vectors; bit for bit."""
import numpy as np
import pytest

import layer_util as u
from test_gpu_rows import mg  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu

# rows short enough for one warp (16, 272), beyond (2064, 4112), a row of 65536 elements (the wide form's longest) and one more,
# M either side of 2048 and of 2^20 / (N / 16), never a multiple of 4
SHAPES = [(2047, 16), (2049, 16), (2051, 272), (2050, 2064), (4099, 4112), (16387, 1040), (262, 65536), (261, 65552), (2055, 1008), (70001, 240)]


def rule(x):
    """The documented rule, every step rounded in binary32 (x finite, every row's largest magnitude above 2^-119)."""
    x = x.astype(np.float32)
    top = np.abs(x).max(axis=1, keepdims=True)
    return np.rint(x * (np.float32(127) / top)).astype(np.int8), (top / np.float32(127))[:, 0]


@pytest.mark.parametrize("kind", u.TYPES)
@pytest.mark.parametrize("M,N", SHAPES)
def test_codes_and_values(mg, M, N, kind):
    import torch
    rng = np.random.default_rng([M, N])
    x = torch.from_numpy((rng.standard_normal((M, N), np.float32) * np.float32(2) ** rng.integers(-8, 9, (M, 1)).astype(np.float32)))
    x = x.to(u.torch_type(kind))
    q, scale = rule(x.float().numpy())
    # a row's pitch of 32 bytes more, so that the rows' ends show
    pad = 32 // u.size(kind)
    X = torch.full((M, N + pad), 77, dtype=x.dtype, device="cuda")
    X[:, :N] = x.cuda()
    Q = torch.full((M, N + 32), 77, dtype=torch.int8, device="cuda")
    S = torch.full((M + 8,), 77.0, device="cuda")
    mg.mipgemm_quantize_rows(mg.TYPES[kind], M, N, X, N + pad, Q, N + 32, S)
    assert bool((Q[:, :N].cpu() == torch.from_numpy(q)).all()) and np.array_equal(S[:M].cpu().numpy(), scale)
    assert bool((Q[:, N:] == 77).all()) and bool((S[M:] == 77).all())
    Y = torch.full((M, N + pad), 77, dtype=x.dtype, device="cuda")
    mg.mipgemm_dequantize_rows(mg.TYPES[kind], M, N, Q, N + 32, S, Y, N + pad)
    back = torch.from_numpy(q.astype(np.float32) * scale[:, None]).to(x.dtype)
    assert bool((Y[:, :N].cpu() == back).all()) and bool((Y[:, N:] == 77).all())
    assert mg.mipgemm_device_status() == mg.OK


@pytest.mark.parametrize("kind", u.TYPES)
def test_special_rows_among_many(mg, kind):
    """Rows of zeros, infinities and NaN at the beginning, at the end and inside groups of four rows."""
    import torch
    M, N = 4098, 4112
    g = torch.Generator(device="cuda").manual_seed(1)
    X = torch.randn(M, N, device="cuda", generator=g).to(u.torch_type(kind))
    X[[0, 5, 2047, M - 1]] = 0
    X[1, 0], X[6, N - 1], X[M - 2, 17] = float("inf"), float("-inf"), float("nan")
    Q, S, Y = torch.empty(M, N, dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda"), torch.empty_like(X)
    mg.mipgemm_quantize_rows(mg.TYPES[kind], M, N, X, N, Q, N, S)
    mg.mipgemm_dequantize_rows(mg.TYPES[kind], M, N, Q, N, S, Y, N)
    bad = torch.zeros(M, dtype=torch.bool, device="cuda")
    bad[[1, 6, M - 2]] = True
    zero = torch.zeros_like(bad)
    zero[[0, 5, 2047, M - 1]] = True
    assert torch.equal(torch.isnan(S), bad) and torch.equal(S == 0, zero)
    assert bool((Q[bad | zero] == 0).all()) and bool(torch.isnan(Y[bad]).all()) and bool((Y[zero] == 0).all())
    rest = ~(bad | zero)
    assert bool((Q[rest].abs().amax(dim=1) == 127).all()) and not bool(torch.isnan(Y[rest]).any())
