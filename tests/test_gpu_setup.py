"""Kernels are set up on a device when they are first needed there, also inside a graph capture."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PLAIN = """
import torch
from paper_2506_11728_b200 import binding as mg
a = torch.ones(200, 256, dtype=torch.int8, device="cuda")
c = torch.zeros(200, 200, dtype=torch.int32, device="cuda")
for M in (3, 200):
    mg.mipgemm_s8s8s32(M, 200, 256, a, 256, a, 256, c, 200)
torch.cuda.synchronize()
assert (c == 256).all()
"""
LAYER = """
y = torch.zeros(200, 200, device="cuda")
z = torch.zeros(200, 256, device="cuda")
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    mg.mipgemm_s8s8_linear(0, 0, 200, 200, 256, a, 256, None, a, 256, None, None, None, 0, y, 200)
    mg.mipgemm_bf16s8_product(0, 0, 200, 256, 200, torch.ones(200, 200, device="cuda").bfloat16(), 200, a, 256, None, z, 256)
g.replay()
torch.cuda.synchronize()
assert (y == 256).all() and (z == 200).all()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    mg.mipgemm_s8s8_linear(0, 0, 3, 200, 256, a, 256, None, a, 256, None, None, None, 0, y, 200)
y.zero_()
g.replay()
torch.cuda.synchronize()
assert (y[:3] == 256).all() and (y[3:] == 0).all()
assert mg.mipgemm_device_status() == mg.OK
"""


def stderr_of(code):
    out = subprocess.run([sys.executable, "-c", code], cwd=ROOT, env=dict(os.environ, MIPGEMM_LOG="1"), capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stderr[-2000:]
    return [line for line in out.stderr.splitlines() if line.startswith("mipgemm: set up")]


def test_plain_products_do_not_load_the_layer_operators():
    assert stderr_of(PLAIN) == []


def test_each_family_is_set_up_once_when_first_called():
    assert stderr_of(PLAIN + LAYER) == ["mipgemm: set up %s kernels" % k for k in ("dense layer", "product", "few-token layer")]
