"""The product kernel's converter warps take the codes of their own use, whatever order copies land in; on the CPU."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def model(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("converter") / "model")
    cxx = shutil.which("g++") or shutil.which("c++")
    assert cxx, "no C++ compiler"
    subprocess.run([cxx, "-O2", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-o", exe, os.path.join(HERE, "converter_model.cpp")], check=True)
    return lambda *args: [int(v) for v in subprocess.run([exe, *args], check=True, capture_output=True, text=True).stdout.split()]


def test_every_use_is_converted_from_its_own_codes(model):
    for seed in ("1", "2", "3"):
        wrong, stuck, uses = model("kernel", seed)
        assert uses == 4000 * 40 and wrong == 0 and stuck == 0


def test_the_model_tells_the_other_order(model):
    """Codes first, then the free stage: a group can pass on the phase of two uses before."""
    wrong, stuck, uses = model("swapped", "1")
    assert wrong > 0
