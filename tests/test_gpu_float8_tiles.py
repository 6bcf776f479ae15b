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
