"""A call's plan is the one that its own arguments ask for, whatever was called on the same operands before."""
import subprocess
import sys
import os

import pytest

import layer_util as u
from test_gpu_layer_paths import mg, problem  # noqa: F401 (mg is a fixture)

pytestmark = pytest.mark.gpu


def test_plans_are_priced_for_their_activation(mg):
    """An activation with an exponential costs the epilogue twice the time of one without, and its plan is made for that: on
    the same operands the two kinds have plans of their own, activations of a kind share one."""
    if not mg.mipgemm_plan_cache_stats()[0]:
        pytest.skip("plan cache switched off")
    M, N, K = 964, 5728, 144
    p, d, G, U = problem(M, N, K)
    c = u.Matrix(M, N, "bf16")
    def misses(act):
        before = mg.mipgemm_plan_cache_stats()[2]
        mg.mipgemm_s8s8_linear(2, mg.ACTIVATIONS[act], M, N, K, p["A"].ptr, K, p["a_s"], p["W"].ptr, K, p["w_s"], None, None, 0, c.ptr, N)
        return mg.mipgemm_plan_cache_stats()[2] - before
    assert [misses(a) for a in ("none", "gelu", "relu", "silu", "gelu_tanh", "none")] == [1, 1, 0, 0, 0, 0]


CODE = """
import torch
from paper_2506_11728_b200 import binding as mg
M, N, K = 964, 5728, 144
a = torch.ones(M, K, dtype=torch.int8, device="cuda")
b = torch.ones(N, K, dtype=torch.int8, device="cuda")
c = torch.zeros(M, N, dtype=torch.bfloat16, device="cuda")
for act in %r:
    mg.mipgemm_s8s8_linear(2, mg.ACTIVATIONS[act], M, N, K, a, K, None, b, K, None, None, None, 0, c, N)
torch.cuda.synchronize()
"""


def test_the_tile_does_not_depend_on_what_was_called_before():
    def tiles(acts):
        out = subprocess.run([sys.executable, "-c", CODE % (acts,)], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                             env=dict(os.environ, MIPGEMM_LOG="1"), capture_output=True, text=True, timeout=300)
        assert out.returncode == 0, out.stderr[-2000:]
        lines = [x for x in out.stderr.splitlines() if x.startswith("mipgemm: layer")]
        return dict(zip(acts, (x.split("tile=")[1].split()[0] for x in lines)))
    assert tiles(("none", "gelu")) == tiles(("gelu", "none"))
