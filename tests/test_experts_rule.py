"""The choice of the tile of an expert layer's products (dash_experts_rule.h), compiled for the host.  No GPU involved."""
import ctypes as C
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
BIG, NARROW, FEW, WIDE = 1, 2, 3, 4
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


# (rows, experts, K, M, primes): us of repeated calls with byte weights (big, narrow) and 4-bit weights (big, narrow, few, wide)
MEASURED = [
    ((1, 1, 784, 128, 8), (12.7, 5.8), (12.5, 7.7, 7.0, 10.8)),
    ((1, 1, 4096, 4096, 12), (37.4, 16.0), (43.0, 26.8, 25.2, 33.8)),
    ((4, 1, 4096, 4096, 12), (41.4, 41.5), (47.4, 50.1, 59.5, 53.6)),
    ((16, 1, 4096, 4096, 12), (130.6, 140.8), (149.0, 158.1, 228.7, 139.6)),
    ((128, 1, 4096, 4096, 12), (990.9, 1230.1), (1029.2, 1245.5, 1765.1, 1076.2)),
    ((16, 8, 400, 120, 8), (10.2, 5.2), (11.2, 6.4, 6.2, 8.7)),
    ((256, 32, 1024, 2048, 12), (325.4, 375.7), (413.7, 425.1, 667.1, 355.0)),
    ((128, 16, 512, 768, 9), (41.7, 41.8), (48.0, 50.3, 80.5, 41.2)),
    ((64, 12, 4096, 256, 12), (43.7, 43.7), (52.8, 51.8, 69.4, 54.1)),
    ((64, 64, 1024, 1024, 12), (49.2, 50.6), (108.8, 77.9, 102.1, 67.0)),
    ((64, 16, 1024, 1024, 12), (47.7, 48.0), (62.5, 59.8, 91.1, 52.8)),
    ((2, 1, 2048, 2048, 12), (22.0, 9.4), (25.5, 14.1, 16.5, 19.6)),
    ((8, 1, 256, 4096, 8), (11.3, 11.4), (18.7, 13.4, 22.7, 11.6)),
    ((39, 4, 81, 29, 12), (8.2, 4.6), (8.3, 5.1, 6.6, 6.7)),
    ((65, 4, 228, 12, 7), (8.9, 4.8), (9.5, 5.6, 7.3, 7.7)),
    ((12, 6, 3833, 172, 9), (35.6, 14.4), (45.5, 22.3, 17.1, 32.4)),
    ((256, 1, 2048, 64, 12), (73.7, 60.6), (88.7, 64.0, 76.8, 80.5)),
    ((200, 8, 100, 1500, 9), (61.5, 86.4), (79.9, 88.6, 170.9, 66.3)),
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
    for forced in (FEW, WIDE):
        assert tile(lib, 128, 1, 4096, 4096, True, forced=forced) == forced
        assert tile(lib, 128, 1, 4096, 4096, False, forced=forced) == BIG       # byte weights have no such kernel


def test_every_size_gets_a_tile_of_its_format(lib):
    for rows in (1, 2, 63, 1000, 2 ** 24):
        for experts in (1, 7, 10 ** 6):
            for K in (1, 64, 5000, 2 ** 26):
                for M in (1, 129, 2 ** 20):
                    for k in (1, 2, 12):
                        assert tile(lib, rows, experts, K, M, False, k) in (BIG, NARROW)
                        assert tile(lib, rows, experts, K, M, True, k) in (BIG, NARROW, FEW, WIDE)


def test_tiles_of_an_even_routing(lib):
    """what the routing makes of rows that are spread evenly"""
    chunks = (C.c_int * 12)(*CHUNKS)
    for rows, experts, k in ((1, 1, 12), (16, 8, 8), (96, 32, 9), (64, 64, 12), (1000, 10, 7)):
        r, ch = rows // experts, CHUNKS[:k]
        for groups in (4, 8, 16):
            assert lib.tiles(groups, C.c_long(rows), experts, 0, k, chunks) == experts * -(-sum(ch) * r // groups)
            assert lib.tiles(groups, C.c_long(rows), experts, 1, k, chunks) == experts * sum(-(-c * r // groups) for c in ch)
