"""The addresses of a tile's copies into LDS, for every number of keys left, in a host program."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2609_30096_amd", "csrc")


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("tile_copy") / "tile_copy")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, "-o", exe,
                    os.path.join(HERE, "tile_copy.cpp")], check=True)
    return exe


def test_no_read_past_the_last_key(program):
    """What lies past the last key is cut off by the buffer's size, which is compared with the vector offset alone."""
    r = subprocess.run([program], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout


def test_scalar_rows_of_a_partial_tile_are_found(program):
    r = subprocess.run([program, "planted"], capture_output=True, text=True, timeout=60)
    assert r.returncode == 1 and "K read past the end" in r.stdout


def test_kernel_takes_the_checked_offsets():
    """Every copy of the single-token kernel goes through tile_offset, and a scalar part stands only behind tile_whole."""
    with open(os.path.join(CSRC, "window.hip")) as f:
        src = f.read()
    body = src[src.index("void window_rows_kernel"):src.index("// ---------------------------------------------------------------- float32")]
    loads = [i for i in range(len(body)) if body.startswith("raw_ptr_buffer_load_lds(", i)]
    assert len(loads) == 4
    for i in loads:
        before, call = body[:i], body[i:body.index(";", i)]
        offset = before[before.rindex("tile_offset("):]
        if "at.scalar" in call:
            assert offset.startswith("tile_offset(true") and before.rindex("if (tile_whole(") > before.rindex("auto copy_")
        else:
            assert offset.startswith("tile_offset(false") and "at.vec, 0, 0," in call
