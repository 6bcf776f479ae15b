"""The plain product's dense kernel, one CTA or a pair, with waits that run out in the middle of its work (more tiles than
CTAs, so that producers are stopped with stages asked for): it returns, says so once, and the next calls are exact."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture
def mg():
    from paper_2506_11728_b200 import binding
    binding.mipgemm_set_tuning()
    yield binding
    binding.mipgemm_set_tuning()


@pytest.mark.parametrize("form", ["one", "pair"])
@pytest.mark.parametrize("out", ["s32", "s8"])
@pytest.mark.parametrize("M,N,K", [(300, 416, 1024), (2500, 3000, 1300), (4096, 4096, 512)])
def test_dense_kernel(mg, M, N, K, out, form):
    import torch
    g = torch.Generator(device="cuda").manual_seed(M)
    a, b = (torch.randint(-128, 128, (r, K), device="cuda", generator=g, dtype=torch.int32).to(torch.int8) for r in (M, N))
    want = a.double() @ b.double().t()
    mg.mipgemm_set_tuning(block_n=64, split_k=1, force_path=mg.PATH_DENSE if form == "one" else mg.PATH_DENSE_PAIR)
    scale = 2.0 ** -12
    if out == "s32":
        c = torch.zeros(M, N, dtype=torch.int32, device="cuda")
        call = lambda: mg.mipgemm_s8s8s32(M, N, K, a, K, b, K, c, N, 0)
    else:
        c = torch.zeros(M, N, dtype=torch.int8, device="cuda")
        call = lambda: mg.mipgemm_s8s8s8_requant(M, N, K, a, K, b, K, c, N, scale, 0)
        want = torch.round((want.float() * scale).double()).clamp(-128, 127)
    mg.mipgemm_debug_set(1, 200_000)
    try:
        call()
        assert mg.mipgemm_device_status() == mg.ERR_TIMEOUT
        assert mg.mipgemm_device_status() == mg.OK
    finally:
        mg.mipgemm_debug_set(0, 0)
    for _ in range(2):
        c.zero_()
        call()
        assert mg.mipgemm_device_status() == mg.OK
        assert torch.equal(c.double(), want)
