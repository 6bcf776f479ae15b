"""How far apart the warps of the dense 8-bit floating-point product may be, by a model of its barriers on the CPU."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
PAIR, SINGLE = ("2", "2"), ("4", "1")            # blocks in tensor memory for each half, halves


@pytest.fixture(scope="module")
def model(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("tiles") / "model")
    cxx = shutil.which("g++") or shutil.which("c++")
    assert cxx, "no C++ compiler"
    subprocess.run([cxx, "-O2", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-o", exe, os.path.join(HERE, "tile_places_model.cpp")], check=True)
    return lambda *args: [int(v) for v in subprocess.run([exe, *args], check=True, capture_output=True, text=True).stdout.split()]


@pytest.mark.parametrize("form,blocks", [(PAIR, "1"), (SINGLE, "1"), (SINGLE, "2")])
def test_the_scales_warp_is_whole_tiles_ahead_where_k_is_short(model, form, blocks):
    """So tile positions cannot come from it by a ring of four: a tile's would be that of another one when its outputs are stored."""
    moved, stuck, tiles, _ = model(*form, blocks, "4", "1")
    assert moved > 0 and stuck == 0 and tiles > 0


@pytest.mark.parametrize("form,ring", [(PAIR, "6"), (SINGLE, "10")])
def test_how_far_it_is_ahead(model, form, ring):
    """2 * depth + 1 tiles at the most."""
    for seed in ("1", "2"):
        assert model(*form, "1", ring, seed)[:2] == [0, 0]
    assert model(*form, "1", str(int(ring) - 1), "1")[0] > 0


@pytest.mark.parametrize("form,ring", [(PAIR, "8"), (SINGLE, "16")])
@pytest.mark.parametrize("blocks", ["1", "2", "3"])
def test_the_kernels_ring_is_deep_enough(model, form, ring, blocks):
    import re
    path = os.path.join(os.path.dirname(HERE), "paper_2506_11728_b200", "csrc", "float8_product_kernel.cu")
    text = re.sub(r"//[^\n]*", "", open(path).read())
    assert re.search(r"tile_places\(bool pair\) \{ return pair \? 8 : 16; \}", text) and "kTilePlaces >= 2 * kDepth + 2" in text
    assert len(re.findall(r"tile_at \+ \(tile_no & \(kTilePlaces - 1\)\)", text)) == 2          # written, read
    assert model(*form, blocks, ring, "3")[:2] == [0, 0]


@pytest.mark.parametrize("form", [PAIR, SINGLE])
@pytest.mark.parametrize("blocks", ["1", "3"])
def test_scales_are_read_before_their_place_is_given_back(model, form, blocks):
    """In front of the buffer's return, twice as many places as buffers do; behind it, the next block's scales may be there."""
    places = str(2 * int(form[0]))
    for seed in ("1", "2"):
        _, stuck, _, wrong = model(*form, blocks, "64", seed, places, "0")
        assert stuck == 0 and wrong == 0
    assert model(*form, blocks, "64", "1", places, "1")[3] > 0
    assert model(*form, blocks, "64", "1", str(int(places) - 1), "0")[3] > 0


def test_the_kernel_reads_them_so():
    """Read from the source: behind a block's return of its buffer, column scales come from registers alone."""
    import re
    path = os.path.join(os.path.dirname(HERE), "paper_2506_11728_b200", "csrc", "float8_product_kernel.cu")
    text = re.sub(r"//[^\n]*", "", open(path).read())
    assert re.search(r"scale_places\(bool pair\) \{ return pair \? 4 : 8; \}", text) and "kDepth = 4 / kHalves" in text
    block = text.split("for (int c = 0; c < kCols / 16; ++c) {")[1].split("if (++acc == kDepth)")[0]
    front, back = block.split("mbar_arrive_cluster(my_tempty")
    assert "if (kVec && last)" in front and "lds_f4(cols_at + 16u * j, b_s[j])" in front
    assert [m for m in re.findall(r"[^;{}]*lds_f4\([^;]*;", back)] == [m for m in re.findall(r"[^;{}]*if \(!last\) lds_f4\([^;]*;", back)]
    assert len(re.findall(r"lds_f4", back)) == 1 and "ld.shared" not in back
