"""The choice of the tile of an expert layer's products with 8-bit floating point weights (dash_experts_rule.h), and the classes of primes (dash_experts.h), compiled for
the host.  No GPU involved."""
import ctypes as C
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
BIG, NARROW, FEW, WIDE, CLASS, SMALL = 1, 2, 3, 4, 5, 6
ORDER = [BIG, WIDE, CLASS, NARROW, FEW, SMALL]
PRIMES = [2, 3, 5, 7, 11, 13, 17, 19, 23, 29, 31, 37]
CHUNKS = [8, 6, 4, 3, 3, 3, 2, 2, 2, 2, 2, 2]
SRC = r"""
#include "%s/../paper_2302_06361_amd/csrc/dash_experts_rule.h"
extern "C" int tile(int forced, long rows, int experts, int M, int K, int k, const int* chunks, int classes, const int* class_chunks) {
    dash::ExpertsShape8 S{rows, experts, M, K, k, {}, classes, {}};
    for (int i = 0; i < k; i++) S.chunks[i] = chunks[i];
    for (int i = 0; i < classes; i++) S.class_chunks[i] = class_chunks[i];
    return dash::experts_tile8(forced, S);
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("rule8")
    src, so = str(d / "rule.cpp"), str(d / "rule.so")
    open(src, "w").write(SRC % HERE)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-o", so, src])
    return C.CDLL(so)


def classes(primes):
    """the largest prime that is left and as many more as fit below 240, large ones first"""
    left, out = sorted(primes, reverse=True), []
    while left:
        m, part = 1, []
        for p in list(left):
            if m * p <= 240:
                m *= p
                part.append(p)
                left.remove(p)
        out.append(part)
    return out


def tile(lib, rows, experts, K, M, k=12, forced=0):
    cl = [sum(CHUNKS[PRIMES.index(p)] for p in part) for part in classes(PRIMES[:k])]
    return lib.tile(forced, C.c_long(rows), experts, M, K, k, (C.c_int * 12)(*CHUNKS), len(cl), (C.c_int * 16)(*cl))


# (rows, experts, K, M, primes): us of repeated calls with the tiles big, wide, class, narrow, few, small
MEASURED = [
    ((1, 1, 784, 128, 8), (13.6, 10.7, 12.1, 10.6, 11.3, 9.9)),
    ((1, 1, 4096, 4096, 12), (89.5, 50.5, 40.8, 37.6, 34.8, 37.2)),
    ((4, 1, 4096, 4096, 12), (93.4, 59.9, 61.5, 74.6, 98.2, 96.5)),
    ((16, 1, 4096, 4096, 12), (165.0, 167.3, 175.9, 250.7, 335.3, 321.9)),
    ((128, 1, 4096, 4096, 12), (1140.9, 1238.1, 1385.3, 1887.3, 2606.9, 2513.5)),
    ((16, 8, 400, 120, 8), (10.4, 9.1, 9.2, 7.9, 9.1, 8.3)),
    ((256, 32, 1024, 2048, 12), (541.7, 423.4, 452.5, 539.0, 961.9, 948.0)),
    ((128, 16, 512, 768, 9), (55.8, 45.9, 47.5, 54.5, 106.6, 103.7)),
    ((64, 12, 4096, 256, 12), (94.4, 65.0, 65.5, 76.3, 99.5, 99.9)),
    ((64, 64, 1024, 1024, 12), (327.2, 160.3, 102.9, 93.9, 166.6, 163.6)),
    ((64, 16, 1024, 1024, 12), (96.2, 66.5, 69.5, 78.1, 124.1, 122.2)),
    ((2, 1, 2048, 2048, 12), (27.0, 22.6, 23.3, 21.1, 20.4, 21.3)),
    ((8, 1, 256, 4096, 8), (19.1, 17.3, 15.3, 14.9, 26.9, 28.4)),
    ((39, 4, 81, 29, 12), (8.4, 6.7, 6.8, 5.7, 6.8, 6.2)),
    ((65, 4, 228, 12, 7), (10.0, 7.9, 7.9, 6.6, 8.0, 7.0)),
    ((12, 6, 3833, 172, 9), (46.1, 38.0, 38.3, 36.3, 32.7, 27.2)),
    ((256, 1, 2048, 64, 12), (78.7, 72.0, 70.3, 73.5, 99.4, 72.9)),
    ((200, 8, 100, 1500, 9), (90.5, 75.8, 73.5, 80.6, 219.8, 223.3)),
]


@pytest.mark.parametrize("layer,times", MEASURED)
def test_measured_layers(lib, layer, times):
    got = times[ORDER.index(tile(lib, *layer))]
    assert got <= 1.07 * min(times), (layer, got, min(times))


def test_forced_tiles(lib):
    for t in ORDER:
        assert tile(lib, 1, 1, 784, 128, forced=t) == t
    for t in (0, 7, -1):
        assert tile(lib, 128, 1, 4096, 4096, forced=t) == BIG


def test_every_size_has_a_tile(lib):
    for rows in (1, 10 ** 9):
        for experts in (1, 2 ** 24 - 2):
            for K in (1, 2 ** 26):
                for M in (1, 2 ** 31 - 1 - 255):
                    assert tile(lib, rows, experts, K, M) in ORDER


def test_classes_of_primes(tmp_path):
    """in every base: each prime once, products up to 240, the same classes as by hand"""
    src, so = str(tmp_path / "classes.cpp"), str(tmp_path / "classes.so")
    text = open(os.path.join(HERE, "..", "paper_2302_06361_amd", "csrc", "dash_experts.h")).read()
    body = text[text.index("struct PrimeClasses {"):text.index("inline RoutingView routing_view(")]
    open(src, "w").write("""
#define DASH_MAX_PRIMES 16
struct Mod { unsigned nchunk; };
struct dash_ctx { int k; int prime[16]; Mod mods[256]; };
%s
extern "C" int run(int k, const int* primes, const int* chunks, int* order, int* modulus, int* prime_first, int* chunk_first) {
    dash_ctx c = {};
    c.k = k;
    for (int i = 0; i < k; i++) { c.prime[i] = primes[i]; c.mods[primes[i]].nchunk = chunks[i]; }
    const PrimeClasses r = prime_classes(&c);
    for (int i = 0; i < 16; i++) { order[i] = r.order[i]; modulus[i] = r.modulus[i]; }
    for (int i = 0; i < 17; i++) { prime_first[i] = r.prime_first[i]; chunk_first[i] = r.chunk_first[i]; }
    return r.n;
}
""" % body)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-o", so, src])
    lib = C.CDLL(so)
    bases = [PRIMES[:k] for k in range(1, 13)] + [[2, 3, 101, 113, 127], [127], [2, 127], [113, 2, 53, 3, 47, 5], [13, 11, 7, 5, 3, 2]]
    for base in bases:
        chunks = [(i * 7) % 5 + 1 for i in range(len(base))]
        order, modulus, pf, cf = ((C.c_int * n)() for n in (16, 16, 17, 17))
        n = lib.run(len(base), (C.c_int * 16)(*base), (C.c_int * 16)(*chunks), order, modulus, pf, cf)
        want = classes(base)
        assert n == len(want)
        at = 0
        for i, part in enumerate(want):
            assert [base[order[j]] for j in range(pf[i], pf[i + 1])] == part
            m = 1
            for p in part:
                m *= p
            assert modulus[i] == m <= 240 and cf[i] == at
            at += sum(chunks[base.index(p)] for p in part)
        assert pf[n] == len(base) and cf[n] == at
