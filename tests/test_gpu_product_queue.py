"""The product in its odd-staged pipelines, many calls in a row on inputs larger than the L2 and on small ones: bit-equal
results, no wait that runs out."""
import pytest

from test_gpu_layer_paths import mg  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("stages", [2, 3, 4, 0])
@pytest.mark.parametrize("M,N,K,order", [(9, 695, 4623, 0), (3893, 197, 12113, 1), (1024, 1024, 8192, 0), (2048, 6000, 9000, 1)])
def test_repeats(mg, M, N, K, order, stages):
    import torch
    mg.mipgemm_set_tuning(stages=stages)
    mg.mipgemm_debug_set(0, 50_000_000)
    try:
        g = torch.Generator(device="cuda").manual_seed(1)
        a = torch.randint(-8, 9, (K, M) if order else (M, K), device="cuda", generator=g).bfloat16()
        b = torch.randint(-128, 128, (K, N), device="cuda", generator=g, dtype=torch.int32).to(torch.int8)
        s = 2.0 ** torch.randint(-2, 3, (K,), device="cuda", generator=g).float()
        want = (a.double().t() if order else a.double()) @ (s.double()[:, None] * b.double())
        assert want.abs().max() < 2 ** 22                 # exact: integers times 1/4, in every order of the sums
        c = torch.empty(M, N, device="cuda")
        wrong = torch.zeros((), dtype=torch.int64, device="cuda")
        for _ in range(150):
            c.fill_(float("nan"))
            mg.mipgemm_bf16s8_product(0, order, M, N, K, a, a.shape[1], b, N, s, c, N)
            wrong += (c != want).sum()
        assert int(wrong) == 0
        assert mg.mipgemm_device_status() == mg.OK
    finally:
        mg.mipgemm_debug_set(0, 0)
