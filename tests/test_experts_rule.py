"""The choice of the tile of an expert layer's products (dash_experts_rule.h), compiled for the host.  No GPU involved."""
import ctypes as C
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
BIG, NARROW, FEW = 1, 2, 3
CHUNKS = [8, 6, 4, 3, 3, 3, 2, 2, 2, 2, 2, 2]
SRC = r"""
#include "%s/../paper_2302_06361_amd/csrc/dash_experts_rule.h"
extern "C" int tile(int forced, long rows, int experts, int M, int K, int mx4, int k, const int* chunks) {
    dash::ExpertsShape S{rows, experts, M, K, mx4 != 0, k, {}};
    for (int i = 0; i < k; i++) S.chunks[i] = chunks[i];
    return dash::experts_tile(forced, S);
}
extern "C" double tiles(int groups, long rows, int experts, int mx4, int k, const int* chunks) {
    dash::ExpertsShape S{rows, experts, 1, 1, mx4 != 0, k, {}};
    for (int i = 0; i < k; i++) S.chunks[i] = chunks[i];
    return dash::experts_tiles(S, groups);
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("rule")
    src, so = str(d / "rule.cpp"), str(d / "rule.so")
    open(src, "w").write(SRC % HERE)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-o", so, src])
    lib = C.CDLL(so)
    lib.tiles.restype = C.c_double
    return lib


def tile(lib, rows, experts, K, M, mx4, k=12, forced=0):
    return lib.tile(forced, C.c_long(rows), experts, M, K, int(mx4), k, (C.c_int * 12)(*CHUNKS))


# (rows, experts, K, M, primes): measured us with byte weights (big, narrow) and 4-bit weights (big, narrow, few)
MEASURED = [
    ((1, 1, 784, 128, 8), (12.4, 5.9), (12.9, 7.9, 7.1)), ((1, 1, 4096, 4096, 12), (36.6, 16.1), (43.4, 27.2, 25.6)),
    ((4, 1, 4096, 4096, 12), (41, 43), (47.2, 50.1, 60.2)), ((16, 1, 4096, 4096, 12), (138, 141), (148.5, 158.5, 221)),
    ((128, 1, 4096, 4096, 12), (966, 1249), (1030, 1290, 2000)), ((16, 8, 400, 120, 8), (10, 5.3), (11, 6.6, 6.3)),
    ((256, 32, 1024, 2048, 12), (336, 378), (420, 448, 687)), ((128, 16, 512, 768, 9), (43.5, 43.5), (46.7, 51.2, 82)),
    ((64, 12, 4096, 256, 12), (57, 64), (62, 72, 83)),
    ((64, 64, 1024, 1024, 12), (51, 50), (110, 81, 103)), ((64, 16, 1024, 1024, 12), (49.5, 48.3), (62.7, 60.9, 92)),
    ((2, 1, 2048, 2048, 12), (21.3, 9.7), (26, 14.4, 16.2)), ((8, 1, 256, 4096, 8), (11.05, 11.8), (19, 14.1, 23)),
    ((39, 4, 81, 29, 12), (9, 6), (9.7, 6.5, 8.0)), ((65, 4, 228, 12, 7), (10, 6), (11.0, 7.1, 8.7)), ((12, 6, 3833, 172, 9), (47, 14), (47.5, 24.3, 19.0)),
    ((256, 1, 2048, 64, 12), (74, 59), (87, 65, 79)), ((200, 8, 100, 1500, 9), (60, 86), (81, 94, 178)),
]


@pytest.mark.parametrize("shape,w8,mx4", MEASURED)
def test_choice_is_within_a_tenth_of_the_fastest(lib, shape, w8, mx4):
    rows, experts, K, M, k = shape
    for bits, times in ((False, w8), (True, mx4)):
        assert times[tile(lib, rows, experts, K, M, bits, k) - 1] <= 1.1 * min(times)


def test_forced_tiles(lib):
    for mx4 in (False, True):
        for forced in (BIG, NARROW):
            assert tile(lib, 5, 3, 100, 100, mx4, forced=forced) == forced
    assert tile(lib, 128, 1, 4096, 4096, True, forced=FEW) == FEW
    assert tile(lib, 128, 1, 4096, 4096, False, forced=FEW) == BIG       # byte weights have no such kernel


def test_every_size_gets_a_tile_of_its_format(lib):
    for rows in (1, 2, 63, 1000, 2 ** 24):
        for experts in (1, 7, 10 ** 6):
            for K in (1, 64, 5000, 2 ** 26):
                for M in (1, 129, 2 ** 20):
                    for k in (1, 2, 12):
                        assert tile(lib, rows, experts, K, M, False, k) in (BIG, NARROW)
                        assert tile(lib, rows, experts, K, M, True, k) in (BIG, NARROW, FEW)


def test_tiles_of_an_even_routing(lib):
    """what the routing makes of rows that are spread evenly"""
    chunks = (C.c_int * 12)(*CHUNKS)
    for rows, experts, k in ((1, 1, 12), (16, 8, 8), (96, 32, 9), (64, 64, 12), (1000, 10, 7)):
        r, ch = rows // experts, CHUNKS[:k]
        for groups in (4, 8, 16):
            assert lib.tiles(groups, C.c_long(rows), experts, 0, k, chunks) == experts * -(-sum(ch) * r // groups)
            assert lib.tiles(groups, C.c_long(rows), experts, 1, k, chunks) == experts * sum(-(-c * r // groups) for c in ch)
