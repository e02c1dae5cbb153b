"""The grid of the launch of an expert layer's products (dash_experts_rule.h), compiled for the host: all blocks, and fewer than 2^32 threads in each direction.
No GPU involved."""
import ctypes as C
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
SRC = r"""
#include "%s/../paper_2302_06361_amd/csrc/dash_experts_rule.h"
extern "C" void grid(long blocks, int threads, unsigned* xy) {
    const dash::BlockGrid g = dash::block_grid(blocks, threads);
    xy[0] = g.x; xy[1] = g.y;
}
"""


@pytest.fixture(scope="module")
def grid(tmp_path_factory):
    d = tmp_path_factory.mktemp("grid")
    src, so = str(d / "grid.cpp"), str(d / "grid.so")
    open(src, "w").write(SRC % HERE)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-o", so, src])
    lib = C.CDLL(so)

    def call(blocks, threads):
        xy = (C.c_uint * 2)()
        lib.grid(C.c_long(blocks), threads, xy)
        return xy[0], xy[1]
    return call


@pytest.mark.parametrize("threads", [256, 512])
def test_grids(grid, threads):
    edge = 2 ** 32 // threads
    sizes = set(range(1, 40)) | {e + d for e in (edge, 2 * edge, 5 * edge, 100 * edge, 2 ** 31 - 300) for d in range(-9, 10) if e + d < 2 ** 31}
    for blocks in sizes:
        x, y = grid(blocks, threads)
        assert x % 8 == 0 and x * threads < 2 ** 32 and 1 <= y < 65536
        assert blocks <= x * y < blocks + y * 8, (blocks, x, y)
        if blocks <= edge - 8:
            assert y == 1
