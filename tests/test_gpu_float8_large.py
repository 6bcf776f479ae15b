"""Matrices of more than 2^31 elements, and calls on several streams at once."""
import numpy as np
import pytest

import float8_util as f

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mg():
    from paper_2506_11728_b200 import binding
    binding.mipgemm_set_tuning()
    return binding


M, N = 66000, 32768                    # 2.16e9 elements
ROWS = [0, 1, 32767, 65535, 65536, 65999]


@pytest.fixture(scope="module")
def x():
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    v = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    for i in range(0, M, 6000):
        v[i:i + 6000].normal_(generator=g)
    yield v
    del v
    torch.cuda.empty_cache()


def test_codes(mg, x):
    import torch
    q, c = (torch.empty(M, N, dtype=torch.uint8, device="cuda") for _ in range(2))
    s, cs = torch.empty(N // 128, M, device="cuda"), torch.empty((M + 127) // 128, N, device="cuda")
    mg.mipgemm_f8_quantize(2, 0, M, N, x, N, q, N, s, M, c, N, cs, N)
    for r in ROWS:
        want, scale = f.encode(x[r:r + 1].double().cpu().numpy(), "rows", "e4m3")
        assert np.array_equal(q[r:r + 1].view(torch.float8_e4m3fn).double().cpu().numpy(), want) and np.array_equal(s[:, r:r + 1].cpu().numpy(), scale)
    last = M // 128 * 128
    want, scale = f.encode(x[last:].double().cpu().numpy(), "columns", "e4m3")
    assert np.array_equal(c[last:].view(torch.float8_e4m3fn).double().cpu().numpy(), want) and np.array_equal(cs[-1:].cpu().numpy(), scale)
    y = torch.empty_like(x)
    mg.mipgemm_f8_dequantize(2, 0, mg.F8_BLOCKS["rows"], M, N, q, N, s, M, y, N)
    for r in ROWS:
        v = q[r].view(torch.float8_e4m3fn).float() * s[:, r].repeat_interleave(128)
        assert torch.equal(y[r], v.bfloat16())


def test_step_and_its_gradient(mg, x):
    import torch
    y, stats = torch.empty_like(x), torch.empty(M, 4, device="cuda")
    mg.mipgemm_norm_step(2, 1, 0, M, N, Z=x, ldz=N, drop=0.5, seed=11, Y=y, ldy=N, stats=stats)
    for r in ROWS:
        z = x[r].double()
        want = z * (z.square().mean() + 1e-5).rsqrt() * 2
        low = 0xFFFFFFFF
        for j in (0, 8, 16384, N - 8):
            g = r * (N // 8) + j // 8
            w = f.philox([g & low, g >> 32, 0, 0], [11, 0])
            for i in range(8):
                kept = (w[i // 2] >> (16 * (i % 2))) & 0xFFFF >= 32768
                assert abs(float(y[r, j + i]) - (float(want[j + i]) if kept else 0.0)) <= 2.0 ** -8 * abs(float(want[j + i])) * 1.01
    dw = torch.empty(N, device="cuda")
    mg.mipgemm_norm_step_grad(2, 1, 0, M, N, dY=x, lddy=N, Z=x, ldz=N, stats=stats, drop=0.5, seed=11, dZ=y, lddz=N, dpost_weight=dw)
    # dy = z here: dw = sum over rows of mask z z^; expected of half the places, twice the value
    total = torch.zeros(N, dtype=torch.float64, device="cuda")
    for i in range(0, M, 3000):
        z = x[i:i + 3000].double()
        total += (z * z * stats[i:i + 3000, 1:2].double()).sum(dim=0)
    # (66000 rows: the mask's own deviation is 1 / sqrt(66000 / 3) of the sum, six times that)
    assert float(((dw.double() - total) / total).abs().max()) < 6 * (3 / M) ** 0.5
    assert mg.mipgemm_device_status() == mg.OK


def test_product(mg, x):
    import torch
    K = 136
    a = torch.randint(-4, 5, (M, K), device="cuda").float().to(torch.float8_e4m3fn)
    b = torch.randint(-4, 5, (N, K), device="cuda").float().to(torch.float8_e4m3fn)
    c = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    mg.mipgemm_f8f8_product(2, 0, 0, 0, 0, 2, M, N, K, a, K, None, 0, b, K, None, 0, None, x, N, c, N)
    assert mg.mipgemm_device_status() == mg.OK
    for r in ROWS:
        want = (a[r].float() @ b.float().t() + x[r].float()).bfloat16()
        assert torch.equal(c[r], want)


def test_calls_on_several_streams(mg):
    """Scratch, scales and sums of calls that run beside each other are their own."""
    import torch
    shapes = [(300, 1000, 2100), (130, 520, 4100), (500, 264, 1500), (70, 700, 900)]
    work = []
    for i, (m, n, k) in enumerate(shapes):
        g = torch.Generator(device="cuda").manual_seed(i)
        a = torch.randint(-4, 5, (m, k + 3), device="cuda", generator=g).float().to(torch.float8_e4m3fn)       # (odd pitches: re-pitched)
        b = torch.randint(-4, 5, (n, k + 3), device="cuda", generator=g).float().to(torch.float8_e4m3fn)
        t = {s: torch.randn(m, n, device="cuda", generator=g) for s in ("dy", "dh", "y", "z")}
        work.append(dict(m=m, n=n, k=k, a=a, b=b, want=a[:, :k].float() @ b[:, :k].float().t(), t=t, stats=torch.rand(m, 4, device="cuda", generator=g) + 0.5,
                         c=torch.empty(m, n, device="cuda"), w=[torch.empty(n, device="cuda") for _ in range(2)], s=torch.cuda.Stream()))

    def call(v):
        m, n, k, t = v["m"], v["n"], v["k"], v["t"]
        mg.mipgemm_f8f8_product(0, 0, 0, 0, 0, 2, m, n, k, v["a"], k + 3, None, 0, v["b"], k + 3, None, 0, None, None, 0, v["c"], n)
        mg.mipgemm_norm_step_grad(0, 1, 1, m, n, dY=t["dy"], lddy=n, dH=t["dh"], lddh=n, Y=t["y"], ldy=n, Z=t["z"], ldz=n, stats=v["stats"],
                                  dpost_weight=v["w"][0], dpre_weight=v["w"][1])
    for v in work:
        call(v)
        v["sums"] = [x.clone() for x in v["w"]]
        assert torch.equal(v["c"], v["want"])
    torch.cuda.synchronize()
    for _ in range(30):
        for v in work:
            with torch.cuda.stream(v["s"]):
                v["c"].zero_()
                call(v)
    torch.cuda.synchronize()
    assert mg.mipgemm_device_status() == mg.OK
    for v in work:
        assert torch.equal(v["c"], v["want"]) and all(torch.equal(p, q) for p, q in zip(v["sums"], v["w"]))
