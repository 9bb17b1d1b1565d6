"""The work queue of differential attention's kernels, walked through on the CPU (tests/strided_queue_model.cpp compiles the same header):
every tile of every sequence and head once, in the list's order, and dealt out once."""
import ctypes as C
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("strided") / "strided_queue_model.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Wno-unknown-pragmas",
                    "-I" + os.path.join(ROOT, "paper_2508_06001_amd", "csrc"),
                    os.path.join(ROOT, "tests", "strided_queue_model.cpp"), "-o", so], check=True)
    lib = C.CDLL(so)
    lib.strided_queue_walk.argtypes = [C.POINTER(C.c_int)] + [C.c_int] * 5

    def call(lens, H, tile, order, grid):
        return lib.strided_queue_walk((C.c_int * len(lens))(*lens), len(lens), H, tile, order, grid)

    return call


@pytest.mark.parametrize("order", [0, 1])
def test_every_tile_once(walk, order):
    rng = random.Random(7 + order)
    for _ in range(1500):
        n, top = rng.choice((1, 1, 2, 3, 7, 16, 33, 200)), rng.choice((64, 300, 1500, 6000, 40000))
        lens = [max(0, int(top ** rng.random())) for _ in range(n)]
        if rng.random() < 0.3:
            lens[rng.randrange(n)] = 0
        if rng.random() < 0.3:
            lens = [lens[0]] * n
        H, tile, grid = rng.choice((1, 2, 3, 6, 12, 24)), rng.choice((128, 256)), rng.choice((512, 256, 304, 74, 37))
        assert walk(lens, H, tile, order, grid) == 0, (lens, H, tile, order, grid)


@pytest.mark.parametrize("order", [0, 1])
def test_the_largest_bags(walk, order):
    assert walk([200] * 2048, 24, 128, order, 512) == 0
    assert walk([0] * 2047 + [5], 1, 256, order, 256) == 0
    assert walk([1 << 20], 3, 128, order, 512) == 0
    assert walk([1 << 20] + [300] * 100, 3, 128, order, 512) == 0
    assert walk([0, 0], 3, 128, order, 512) == 0
