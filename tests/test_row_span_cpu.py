"""Where the layer norm of narrow rows loads and stores, walked through on the CPU (tests/row_span_model.cpp compiles the same header)."""
import ctypes as C
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("span") / "row_span_model.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-I" + os.path.join(ROOT, "paper_2508_06001_amd", "csrc"),
                    os.path.join(ROOT, "tests", "row_span_model.cpp"), "-o", so], check=True)
    lib = C.CDLL(so)
    lib.row_span_walk.argtypes = [C.c_int, C.c_int, C.c_long, C.c_long, C.c_int, C.c_int]
    return lib.row_span_walk


@pytest.mark.parametrize("size", [2, 4])
@pytest.mark.parametrize("lanes,groups", [(16, 16), (32, 8)])
def test_accesses_of_narrow_rows(walk, lanes, groups, size):
    rng = random.Random(lanes + size)
    for width in range(8, 8 * lanes + 1, 8):
        for left in (-5, 0, 1, 2, groups - 1, groups, groups + 1, 1 << 30):
            for stride in (width, width + 8 * rng.randrange(1, 200), 1 << 22):
                assert walk(lanes, groups, left, stride, width, size) == 0, (left, stride, width)
