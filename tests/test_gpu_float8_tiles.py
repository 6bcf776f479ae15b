"""8-bit floating-point products of many tiles a CTA and few blocks of K, where the warps of the dense kernel are whole tiles apart:
every element of C, against products that are exact."""
import pytest

import float8_util as f

pytestmark = pytest.mark.gpu


@pytest.fixture
def mg():
    from paper_2506_11728_b200 import binding
    binding.mipgemm_set_tuning()
    yield binding
    binding.mipgemm_set_tuning()


def operand(g, rows, cols, blocks):
    """Codes of small integers with powers of two as scales, at a pitch of whole 16 bytes: (codes, pitch, scales, values)."""
    import torch
    pitch = (cols + 15) // 16 * 16
    v = torch.randint(-4, 5, (rows, cols), generator=g, device="cuda").float()
    q = torch.zeros(rows, pitch, dtype=torch.uint8, device="cuda")
    q[:, :cols] = v.to(torch.float8_e4m3fn).view(torch.uint8)
    s = torch.exp2(torch.randint(-2, 3, f.scale_shape(blocks, rows, cols), generator=g, device="cuda").float())
    if blocks == "rows":
        wide = s.repeat_interleave(128, 0)[:cols].t()
    elif blocks == "columns":
        wide = s.repeat_interleave(128, 0)[:rows]
    else:
        wide = s.repeat_interleave(128, 0)[:rows].repeat_interleave(128, 1)[:, :cols]
    return q, pitch, s, v * wide


def product(mg, M, N, K, what, kind, residual, seed=0):
    """The call's C and what it has to be: |sum| <= 257 * 4 * 4 * 4 * 4 in units of 2^-4, below 2^24, so binary32 holds every partial sum."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(1000003 * K + M + seed)
    dtype = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[kind]
    back = what == "weight_grad"
    A, lda, sa, a = operand(g, *((K, M) if back else (M, K)), "columns" if back else "rows")
    bb = {"forward": "squares", "forward_rows": "rows", "weight_grad": "columns"}[what]
    B, ldb, sb, b = operand(g, *((K, N) if back else (N, K)), bb)
    before = torch.randint(-8, 9, (M, N), generator=g, device="cuda").to(dtype) if residual else None
    C = before.clone() if residual else torch.full((M, N), float("nan"), dtype=dtype, device="cuda")
    r = C if residual == "own" else before
    mg.mipgemm_f8f8_product(mg.TYPES[kind], 0, 0, int(back), int(back), mg.F8_BLOCKS[bb], M, N, K, A, lda, sa, sa.shape[1], B, ldb, sb, sb.shape[1], None,
                            r, N if residual else 0, C, N)
    path = mg.mipgemm_last_path() & mg.PATH_MASK
    assert mg.mipgemm_device_status() == mg.OK
    want = a.t() @ b if back else a @ b.t()
    if residual:
        want += before.float()
    return C, want.to(dtype), path


@pytest.mark.parametrize("K", [1, 64, 100, 128, 129, 200, 256, 257])
@pytest.mark.parametrize("what", ["forward", "weight_grad"])
@pytest.mark.parametrize("form,M,N", [("pair", 8190, 8448), ("pair", 8190, 8450), ("single", 8190, 4224)])
def test_every_tile_is_stored_at_its_place(mg, form, M, N, what, K):
    """14 tiles a CTA or pair; rows of C at 16-byte boundaries (stored by TMA) and at none."""
    import torch
    mg.mipgemm_set_tuning(force_path=2 if form == "pair" else 1)
    for kind, residual in (("f32", None), ("bf16", "own"), ("f32", "other"), ("f16", None)):
        C, want, path = product(mg, M, N, K, what, kind, residual)
        assert path == (mg.PATH_DENSE_PAIR if form == "pair" else mg.PATH_DENSE)
        assert torch.equal(C, want), (kind, residual)


@pytest.mark.parametrize("M,N,K,what", [(16384, 4096, 64, "forward"), (8192, 8192, 128, "forward_rows"), (100, 128256, 128, "forward"), (100, 128250, 256, "forward"),
                                        (11008, 4096, 100, "weight_grad"), (14336, 4096, 1, "weight_grad"), (40, 100000, 200, "forward_rows"),
                                        (130, 60000, 129, "weight_grad")])
def test_short_sums_as_they_are_planned(mg, M, N, K, what):
    import torch
    for kind, residual in (("f32", "own"), ("bf16", None)):
        C, want, _ = product(mg, M, N, K, what, kind, residual, 1)
        assert torch.equal(C, want), (kind, residual)


@pytest.mark.parametrize("formats", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2")])
@pytest.mark.parametrize("what", ["forward", "forward_rows", "input_grad", "weight_grad"])
@pytest.mark.parametrize("form,M,N,K", [("pair", 6000, 5128, 700), ("single", 4000, 3001, 1300), ("pair", 5129, 6001, 389)])
def test_every_element_of_many_tiles(mg, form, M, N, K, what, formats):
    """Codes over the formats' whole range, any scales, several tiles a CTA and several blocks of K: the documented bound, against 64 bits."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(M + K)
    orders = {"forward": (0, 0, "squares"), "forward_rows": (0, 0, "rows"), "input_grad": (0, 1, "squares"), "weight_grad": (1, 1, "columns")}
    ao, bo, bb = orders[what]
    mats = []
    for rows, cols, blocks, fmt in (((K, M) if ao else (M, K)) + ("columns" if ao else "rows", formats[0]), ((K, N) if bo else (N, K)) + (bb, formats[1])):
        pitch = (cols + 15) // 16 * 16
        q = torch.zeros(rows, pitch, dtype=torch.uint8, device="cuda")
        v = (torch.randn(rows, cols, generator=g, device="cuda") * f.LARGEST[fmt] / 5).clamp_(-f.LARGEST[fmt], f.LARGEST[fmt]).to(f.f8_type(fmt))
        q[:, :cols] = v.view(torch.uint8)
        s = (torch.rand(f.scale_shape(blocks, rows, cols), generator=g, device="cuda") + 0.5) / f.LARGEST[fmt]
        d = s.double().repeat_interleave(128, 0)
        d = d[:cols].t() if blocks == "rows" else (d[:rows] if blocks == "columns" else d[:rows].repeat_interleave(128, 1)[:, :cols])
        mats.append((q, pitch, s, v.double() * d))
    (A, lda, sa, a), (B, ldb, sb, b) = mats
    a, b = a.t() if ao else a, b if bo else b.t()
    want, total = a @ b, a.abs() @ b.abs()
    mg.mipgemm_set_tuning(force_path=2 if form == "pair" else 1)
    for kind, half, tiny in (("f32", 2.0 ** -24, 2.0 ** -149), ("bf16", 2.0 ** -8, 2.0 ** -134)):
        C = torch.full((M, N), float("nan"), dtype=torch.float32 if kind == "f32" else torch.bfloat16, device="cuda")
        mg.mipgemm_f8f8_product(mg.TYPES[kind], mg.F8_FORMATS[formats[0]], mg.F8_FORMATS[formats[1]], ao, bo, mg.F8_BLOCKS[bb], M, N, K, A, lda, sa, sa.shape[1],
                                B, ldb, sb, sb.shape[1], None, None, 0, C, N)
        assert mg.mipgemm_device_status() == mg.OK
        tol = total * (K + 8) * 2.0 ** -23 + half * want.abs() * 1.01 + tiny
        assert bool(((C.double() - want).abs() <= tol).all()), kind
