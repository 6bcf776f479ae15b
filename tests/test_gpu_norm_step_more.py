"""The step between two blocks where its first tests do not go, against 64 bits: norms without weights."""
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


@pytest.mark.parametrize("left_out", [("post_w",), ("post_w", "post_b"), ("post_w", "post_b", "pre_w", "pre_b"), ("pre_w", "pre_b"), ("post_b",)])
@pytest.mark.parametrize("layout", ["dense", "odd"])
@pytest.mark.parametrize("M,N", [(3, 1), (7, 24), (40, 512), (20, 768), (9, 1001), (5, 4104), (3, 8200), (2, 20000)])
def test_backward_without_weights(mg, M, N, layout, left_out):
    """What a norm passes on may not hold anything in the columns behind the last one, which the next norm sums over."""
    rng = np.random.default_rng([M, N, 21])
    for kind in ("f32", "bf16"):
        for post, pre, gate in (("layer", "layer", 0), ("layer", "layer", 2), ("layer", "rms", 0), ("rms", "layer", 0), ("layer", "none", 0)):
            if M * N > 20000 and (post, pre, gate) != ("layer", "layer", 0):
                continue
            c = base.case(rng, M, N, kind, post, pre, gate, 0.0)
            for name in left_out:
                c[name] = None
            base.check_grad(mg, c, kind, layout, M, N, rng)


@pytest.mark.parametrize("layout", ["dense", "odd"])
@pytest.mark.parametrize("kind", u.TYPES)
@pytest.mark.parametrize("gate_rows", [1, 3, 1000])
@pytest.mark.parametrize("M,N", [(30, 40), (700, 24), (9, 1001), (4, 8200)])
def test_gradients_of_dropped_places_are_zero_whatever_was_there(mg, M, N, gate_rows, kind, layout):
    """Infinities and NaNs in z, the gate and the gradient, at dropped places alone: they reach nothing."""
    rng = np.random.default_rng([M, N, gate_rows, 22])
    c = base.case(rng, M, N, kind, "none", "none", gate_rows, 0.4)
    off = c["mask"] == 0
    dy = u.rounded(rng.standard_normal((M, N)), kind)
    clean = {k: np.where(off, 0, v) for k, v in (("z", c["z"]), ("dy", dy))}
    st = np.zeros((M, 4))
    for spoiled in ("z", "gate", "dy"):
        d, g = dict(c), dy
        bad = np.where(rng.random((M, N)) < 0.5, np.nan, np.where(rng.random((M, N)) < 0.5, np.inf, -np.inf))
        if spoiled == "z":
            d["z"] = np.where(off, bad, c["z"])
        elif spoiled == "dy":
            g = np.where(off, bad, dy)
        elif gate_rows == 1:
            d["gate"] = np.where(off, bad, c["gate"])
        else:
            continue
        y = f.step(dict(c, z=clean["z"]))[0]
        got = base.backward(mg, d, kind, layout, M, N, y, st, g, None, without=("dX",) if spoiled == "dy" else ())
        want, size = (fn(dict(c, z=clean["z"]), y, st, clean["dy"] if spoiled == "dy" else dy, None) for fn in (f.step_grad, base.grad_sizes))
        for name, ref in (("dX", "dx"), ("dZ", "dz"), ("dgate", "dgate")):
            if name not in got:
                continue
            extra = M * 2.0 ** -24 * size[name] if name == "dgate" else 0
            tol = base.arithmetic(N) * size[name] + extra + u.ROUND[kind] * np.abs(want[ref]) * 1.01 + u.TINY[kind]
            assert (np.abs(got[name] - want[ref]) <= tol).all(), (spoiled, name)
        assert (got["dZ"][off] == 0).all()


@pytest.mark.parametrize("N", [24, 1000, 2049, 2304, 2560, 2561, 5000, 9000])
def test_a_lent_buffer_of_the_documented_size_is_enough(mg, N):
    """8 bytes * N * (vectors wanted + 1) for each SM, whatever the row's length, with and without sums of a gate; the sums are those
    of the library's own scratch up to their order."""
    import torch
    rng = np.random.default_rng([N, 23])
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    M = 6 * sms                          # (rows for two, three or six workers on an SM, without a remainder)
    for gate_rows, vectors in ((0, 4), (M, 4), (M // 2, 4), (M, 0)):
        names = ("dpost_weight", "dpost_bias", "dpre_weight", "dpre_bias")
        c = base.case(rng, M, N, "bf16", "layer", "layer", gate_rows, 0.0)
        room = torch.empty(8 * N * (vectors + 1) * sms, dtype=torch.uint8, device="cuda")
        assert mg.mipgemm_set_workspace(room, room.numel()) == mg.OK
        try:
            base.check_grad(mg, c, "bf16", "dense", M, N, rng, without=() if vectors else names)
        finally:
            mg.mipgemm_set_workspace(None, 0)
