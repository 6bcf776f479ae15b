"""Unwinding of the dense layer kernels, on the CPU: whatever is on its way when the roles stop is waited for."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def model(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("unwind") / "model")
    cxx = shutil.which("g++") or shutil.which("c++")
    assert cxx, "no C++ compiler"
    subprocess.run([cxx, "-O2", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-o", exe, os.path.join(HERE, "unwind_model.cpp")], check=True)
    return lambda *args: [int(v) for v in subprocess.run([exe, *args], check=True, capture_output=True, text=True).stdout.split()]


def test_the_wait_ends_exactly_when_nothing_is_on_its_way(model):
    for seed in ("1", "2", "3"):
        failures, uneven, trials = model("ours", seed)
        assert uneven > trials // 10          # producers did stop at different uses
        assert failures == 0


def test_the_model_tells_a_wait_that_covers_too_little(model):
    """Waiting for the uses that one producer counted, with nothing supplied, fails in many trials."""
    failures, uneven, trials = model("naive", "1")
    assert failures > trials // 10
