"""Which blocks of columns lie inside a row (dash_experts_rule.h), at the longest rows that 32-bit sizes name, compiled for the host.  No GPU involved."""
import ctypes as C
import os
import re
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2302_06361_amd", "csrc")
SRC = r"""
#include "%s/dash_experts_rule.h"
extern "C" int inside(int first, int n, int K) { return dash::columns_inside(first, n, K); }
"""


@pytest.fixture(scope="module")
def inside(tmp_path_factory):
    d = tmp_path_factory.mktemp("columns")
    src, so = str(d / "columns.cpp"), str(d / "columns.so")
    open(src, "w").write(SRC % CSRC)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-static-libubsan", "-shared", "-fPIC", "-o", so, src])
    return C.CDLL(so).inside


@pytest.mark.parametrize("n", [64, 128])
@pytest.mark.parametrize("K", [1, 63, 64, 65, 127, 128, 129, 4096, 2 ** 31 - 129, 2 ** 31 - 128, 2 ** 31 - 127, 2 ** 31 - 65, 2 ** 31 - 64, 2 ** 31 - 63, 2 ** 31 - 1])
def test_the_last_blocks_of_a_row(inside, n, K):
    last = (K - 1) // n * n
    for first in {0, max(last - n, 0), last}:
        assert bool(inside(first, n, K)) == (first + n <= K), first


@pytest.mark.parametrize("kernel", ["k_f8_quantise", "k_mx4_quantise"])
def test_kernels_ask_it(kernel):
    """no sum of a block's first column and its width, which may pass 31 bits, in front of the loads"""
    text = open(os.path.join(CSRC, "dash_experts.hip")).read()
    at = text.index("void %s(" % kernel)
    body = text[at:text.index("\n}\n", at)]
    assert "columns_inside(" in body and not re.search(r"\+ k(ScaleBlock|TileCols) *<=? *A\.K", body)
