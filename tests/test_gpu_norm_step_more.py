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
