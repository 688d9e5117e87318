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
    """Every copy of the single-token kernel takes its address from tile_offset, that of whole tiles behind tile_whole alone."""
    with open(os.path.join(CSRC, "window.hip")) as f:
        src = f.read()
    body = src[src.index("void window_rows_kernel"):src.index("// ---------------------------------------------------------------- float32")]
    assert "raw_ptr_buffer_load" not in body and body.count("win_copy(") == body.count("win_copy_past(") == 1
    copies = [line.strip() for line in body.splitlines() if " copy(rs, " in line]
    assert len(copies) == 4 and all("tile_offset(" in line for line in copies)
    for whole, other in (copies[:2], copies[2:]):
        assert "tile_offset(true, " in whole and other == whole.replace("true", "false")
        at = [body.index(line) for line in (whole, other)]
        assert body.rindex("if (tile_whole(key0, seq.klen)) {", 0, at[0]) > body.rindex("make_buffer_rsrc", 0, at[0])
        assert body[at[0]:at[1]].count("} else {") == 1
