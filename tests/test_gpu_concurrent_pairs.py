"""Kernels that wait for tensor memory, in short pipelines and on several streams at once: two pairs of CTAs must not be able to
hold one SM's each and wait for the other's, so no two such kernels share an SM.  (Bounded by the test's own time limit.)"""
import pytest

from test_gpu_layer_paths import mg  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.timeout(120)
@pytest.mark.parametrize("stages", [2, 3, 0])
def test_pairs_of_two_streams(mg, stages):
    import torch
    mg.mipgemm_debug_set(0, 100_000_000)
    try:
        mg.mipgemm_set_tuning(block_n=256, stages=stages, split_k=1, force_path=mg.PATH_DENSE_PAIR)
        streams = [torch.cuda.Stream() for _ in range(3)]
        g = torch.Generator(device="cuda").manual_seed(1)
        a, b = (torch.randint(-8, 9, (n, 512), device="cuda", generator=g, dtype=torch.int32).to(torch.int8) for n in (700, 1024))
        d = torch.randint(-8, 9, (700, 512), device="cuda", generator=g).bfloat16()
        want_c = (a.double() @ b.double().t()).float()
        want_p = (d.double() @ b[:512].double()).float()
        outs = [[torch.zeros(700, 1024, device="cuda"), torch.zeros(700, 1024, dtype=torch.int32, device="cuda"),
                 torch.zeros(700, 512, device="cuda")] for _ in streams]
        torch.cuda.synchronize()
        for _ in range(100):
            for s, (c, ci, cp) in zip(streams, outs):
                mg.mipgemm_s8s8_linear(0, 0, 700, 1024, 512, a, 512, None, b, 512, None, None, None, 0, c, 1024, stream=s)
                mg.mipgemm_s8s8s32(700, 1024, 512, a, 512, b, 512, ci, 1024, stream=s)
                mg.mipgemm_bf16s8_product(0, 0, 700, 512, 512, d, 512, b, 512, None, cp, 512, stream=s)
        torch.cuda.synchronize()
        assert mg.mipgemm_device_status() == mg.OK
        for c, ci, cp in outs:
            assert torch.equal(c, want_c) and torch.equal(ci.float(), want_c) and torch.equal(cp, want_p)
    finally:
        mg.mipgemm_debug_set(0, 0)


@pytest.mark.timeout(120)
def test_pairs_beside_copies_and_other_kernels(mg):
    """Small pair kernels from three streams beside large copies, so that a pair's two CTAs start apart: each allocates its
    tensor memory only when both run."""
    import time
    import torch
    mg.mipgemm_set_tuning(block_n=64, force_path=mg.PATH_DENSE_PAIR)
    streams, noise = [torch.cuda.Stream() for _ in range(3)], torch.cuda.Stream()
    big = [torch.empty(1 << 28, dtype=torch.uint8, device="cuda") for _ in range(2)]
    g = torch.Generator(device="cuda").manual_seed(1)
    a, b = (torch.randint(-8, 9, (n, 2048), device="cuda", generator=g, dtype=torch.int32).to(torch.int8) for n in (84, 272))
    d = torch.randint(-8, 9, (2300, 416), device="cuda", generator=g).bfloat16()
    bp = torch.randint(-8, 9, (416, 240), device="cuda", generator=g, dtype=torch.int32).to(torch.int8)
    want_c, want_p = (a.double() @ b.double().t()).float(), (d.double() @ bp.double()).float()
    outs = [[torch.zeros(84, 272, device="cuda"), torch.zeros(2300, 240, device="cuda")] for _ in streams]
    torch.cuda.synchronize()
    start, rounds = time.time(), 0
    while time.time() - start < 5:
        rounds += 1
        with torch.cuda.stream(noise):
            for _ in range(rounds % 4):
                big[0].copy_(big[1])
        for i in range(12):
            s, (c, cp) = streams[(i * 7 + rounds) % 3], outs[(i * 7 + rounds) % 3]
            if i % 3:
                mg.mipgemm_s8s8_linear(0, 0, 84, 272, 2048, a, 2048, None, b, 2048, None, None, None, 0, c, 272, stream=s)
            else:
                mg.mipgemm_bf16s8_product(0, 0, 2300, 240, 416, d, 416, bp, 240, None, cp, 240, stream=s)
        torch.cuda.synchronize()
    assert mg.mipgemm_device_status() == mg.OK
    for c, cp in outs:
        assert torch.equal(c, want_c) and torch.equal(cp, want_p)
