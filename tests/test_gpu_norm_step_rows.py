"""The step between two blocks over many rows, where blocks go on from row to row: values, statistics and codes against 64 bits, every
row."""
import numpy as np
import pytest

import float8_util as f
import layer_util as u
import test_gpu_norm_step as base

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mg():
    from paper_2506_11728_b200 import binding
    return binding


def kept(rows, cols, drop, seed, counter):
    """float8_util.kept on arrays."""
    bar, low = round(drop * 65536), np.uint64(2 ** 32 - 1)
    groups = (cols + 7) // 8
    n = np.arange(rows * groups, dtype=np.uint64)
    c = [n & low, n >> np.uint64(32), np.full_like(n, counter & 0xFFFFFFFF), np.full_like(n, counter >> 32)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), p1 & low, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    half = np.stack([(w >> np.uint64(s)) & np.uint64(0xFFFF) for w in c for s in (0, 16)], axis=1).reshape(rows, groups * 8)[:, :cols]
    return np.where(half >= bar, 1 / (1 - bar / 65536), 0.0)


def test_the_mask_on_arrays_is_the_definition():
    for rows, cols, drop, seed, counter in ((3, 17, 0.3, 5 << 40 | 77, 9), (2, 8, 0.9, 1, 1 << 33), (1, 1, 0.5, 0, 0)):
        assert np.array_equal(kept(rows, cols, drop, seed, counter), f.kept(rows, cols, drop, seed, counter))


def case(M, N, kind, post, pre, gate_rows, drop, has_x=True, has_z=True, weights=True):
    rng = np.random.default_rng([M, N, gate_rows, 31])
    c = base.case(rng, M, N, kind, post, pre, gate_rows, 0.0, x_scale=0.7, has_x=has_x, has_z=has_z, weights=weights)
    if drop:
        c.update(drop=drop, mask=kept(M, N, drop, c["seed"], c["counter"]))
    return c


# 592 rows are the fewest that go on on 148 SMs; a row of its own warps and several side by side, the last rows alone in a block
SHAPES = [(592, 8), (1500, 72), (1777, 256), (2401, 264), (700, 1001), (1203, 1024), (640, 2560), (599, 4096), (600, 4104), (593, 8192)]
MIXES = [("rms", "rms", 0, 0.1), ("layer", "layer", 3, 0.0), ("none", "rms", 1, 0.25), ("none", "layer", 0, 0.0), ("rms", "none", 100, 0.5), ("layer", "none", 0, 0.0),
         ("rms", "layer", 1 << 20, 0.3), ("layer", "rms", 0, 0.1)]


@pytest.mark.parametrize("layout", ["dense", "odd"])
@pytest.mark.parametrize("kind", u.TYPES)
@pytest.mark.parametrize("M,N", SHAPES)
def test_values_and_statistics(mg, M, N, kind, layout):
    for i, mix in enumerate(MIXES):
        if M * N > 500000 and (i + len(kind) + len(layout) + M) % 4:
            continue
        post, pre = mix[:2]
        c = case(M, N, kind, *mix, weights=i % 3 != 2)
        Y, H, stats, _, _ = base.forward(mg, c, kind, layout, M, N)
        y, h, st = f.step(c)
        sy, sh = base.sizes(c, y, h)
        base.check(Y.get(), y, sy, kind, (mix, "y"))
        if h is not None:
            base.check(H.get(), h, sh, kind, (mix, "h"))
        big = np.abs(st).copy()
        if post != "none":
            big[:, 0] += np.abs(c["z"]).mean(axis=1)
            big[:, 1] *= 1 + (np.abs(st[:, 0]) * st[:, 1]) ** 2
        if pre != "none":
            spread = np.sqrt((sy * sy).mean(axis=1))
            big[:, 2] += sy.mean(axis=1)
            big[:, 3] *= 1 + (spread * st[:, 3]) ** 2
        assert (np.abs(stats - st) <= base.arithmetic(N) * big).all(), mix


HALF = {"s8": (0.0, 0.5, 127.0), "e4m3": (2.0 ** -4, 2.0 ** -10, 448.0), "e5m2": (2.0 ** -3, 2.0 ** -17, 57344.0)}


def check_codes(mg, M, N, kind, layout, codes, post, pre, has_x, has_z):
    """Codes come from the unrounded h.  With e the error of h: a scale is the largest |h| of its block over L, off by max(e) / L and a
    rounding; a code times its scale is off by half a step -- relative for normal codes, an absolute one of the scale for subnormal
    ones and whole numbers -- and by e, the multiplier's and the scale's roundings."""
    import torch
    relative, absolute, largest = HALF[codes]
    c = case(M, N, kind, post, pre, 0, 0.0, has_x=has_x, has_z=has_z)
    Y, H, _, Q, S = base.forward(mg, c, kind, layout, M, N, codes)
    y, h, _ = f.step(c)
    sy, sh = base.sizes(c, y, h)
    base.check(Y.get(), y, sy, kind, "y")
    base.check(H.get(), h, sh, kind, "h")
    err = base.arithmetic(N) * sh
    got = Q.view.contiguous().view(torch.int8 if codes == "s8" else f.f8_type(codes)).double().cpu().numpy()
    scale = S[:, :M].double().cpu().numpy()
    assert bool((S[:, M:] == -5).all())
    if codes == "s8":
        top, off, wide = np.abs(h).max(axis=1), err.max(axis=1), np.repeat(scale.T, N, axis=1)
        scale = scale[0]
    else:
        top, off, wide = f.tops(h, "rows"), f.tops(err, "rows"), f.spread(scale, "rows", M, N)
    assert (np.abs(scale - top / largest) <= (off + 2.0 ** -23 * top) / largest).all()
    tol = 1.01 * err + relative * np.abs(h) * 1.01 + absolute * wide * 1.01 + 2.0 ** -21 * np.abs(h)
    assert (np.abs(got * wide - h) <= tol).all()
    assert (np.abs(got).max(axis=1) > 0.9 * largest).all()
    # the same codes without y and h being written
    Q2 = base.forward(mg, c, kind, layout, M, N, codes, want_y=False, want_h=False)[3]
    assert np.array_equal(Q2.get(), Q.get())


@pytest.mark.parametrize("codes", list(HALF))
@pytest.mark.parametrize("layout", ["dense", "odd"])
@pytest.mark.parametrize("kind", u.TYPES)
@pytest.mark.parametrize("M,N", SHAPES)
def test_codes(mg, M, N, kind, layout, codes):
    mixes = [("none", "rms", True, True), ("rms", "layer", True, True), ("none", "layer", True, False), ("layer", "rms", False, True)]
    for i, (post, pre, has_x, has_z) in enumerate(mixes):
        if M * N > 500000 and (i + len(kind) + len(layout) + M + len(codes)) % 4:
            continue
        check_codes(mg, M, N, kind, layout, codes, post, pre, has_x, has_z)


@pytest.mark.parametrize("codes", list(HALF))
@pytest.mark.parametrize("layout", ["dense", "odd"])
@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("M,N", [(1, 5), (9, 64), (130, 72), (33, 257), (4, 1001), (3, 4096), (2, 8200), (2, 20000)])
def test_codes_of_few_rows_from_16_bits(mg, M, N, kind, layout, codes):
    for post, pre, has_x, has_z in (("none", "rms", True, False), ("rms", "layer", True, True)):
        check_codes(mg, M, N, kind, layout, codes, post, pre, has_x, has_z)


@pytest.mark.parametrize("kind", u.TYPES)
@pytest.mark.parametrize("M,N", [(5000, 8), (1500, 72), (700, 1001), (600, 4104), (300, 16384), (40, 32768)])
def test_without_norms(mg, M, N, kind):
    """Blocks that take parts of rows, there and back."""
    import torch
    for layout, gate_rows, drop in (("dense", 7, 0.2), ("odd", 0, 0.5), ("dense", 1, 0.0)):
        c = case(M, N, kind, "none", "none", gate_rows, drop)
        Y, *_ = base.forward(mg, c, kind, layout, M, N)
        y, _, st = f.step(c)
        base.check(Y.get(), y, base.sizes(c, y, None)[0], kind, "y")
        dy = u.rounded(np.random.default_rng(5).standard_normal((M, N)), kind)
        for without in (("dX", "dgate"), ("dZ", "dgate")):                # (the forward kernel's work)
            got = base.backward(mg, c, kind, layout, M, N, y, st, dy, None, without)
            want, size = f.step_grad(c, y, st, dy, None), base.grad_sizes(c, y, st, dy, None)
            for name, ref in (("dX", "dx"), ("dZ", "dz")):
                if name in got:
                    base.check(got[name], want[ref], size[name], kind, name)


@pytest.mark.parametrize("layout", ["dense", "odd"])
@pytest.mark.parametrize("kind", u.TYPES)
@pytest.mark.parametrize("M,N", [(9001, 24), (5000, 264), (2403, 520), (1300, 1001), (1777, 2560), (1001, 4096), (700, 8192), (333, 9000), (200, 20000)])
def test_gradients(mg, M, N, kind, layout):
    """Several rows a worker: 148 SMs have two or three of up to eight rows side by side, or a cluster's share of them."""
    for i, (post, pre, gate, drop) in enumerate(MIXES):
        if M * N > 500000 and (i + len(kind) + len(layout) + M) % 4:
            continue
        c = case(M, N, kind, post, pre, gate, drop, weights=i % 3 != 2)
        base.check_grad(mg, c, kind, layout, M, N, np.random.default_rng([M, i]))
