"""Tensor memory of a CTA pair is allocated by both CTAs together: neither may issue the allocation before a cluster barrier
has shown that the other one runs.  Read from the kernels' sources."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_11728_b200", "csrc")


@pytest.mark.parametrize("name", sorted(f for f in os.listdir(CSRC) if f.endswith(".cu")))
def test_no_pair_allocates_ahead_of_its_barrier(name):
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    for m in re.finditer(r"tmem_alloc<(\w+)>", text):
        if m.group(1) == "1":
            continue
        body = text[text.rindex("__global__", 0, m.start()):m.start()]
        wait = body.rfind("cluster_wait();")
        assert wait >= 0, "%s: no cluster barrier ahead of the allocation" % name
        # the barrier is the pair form's, unconditional but for that, and nothing waits between the two
        assert re.search(r"if \(kPair\) \{\s*__syncwarp\(\);\s*cluster_arrive\(\);\s*cluster_wait\(\);\s*\}\s*if \(warp == 1\) \{\s*$", body), name


def test_pair_kernels_are_found():
    found = [f for f in os.listdir(CSRC) if f.endswith(".cu") and "tmem_alloc<kGroup>" in open(os.path.join(CSRC, f)).read()]
    assert sorted(found) == ["dense_kernel.cu", "layer_kernel.cu", "product_kernel.cu"]
