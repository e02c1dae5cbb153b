"""Refusals of the 8-bit floating point weights: arguments are looked at before anything is launched.  No GPU involved."""
import ctypes as C

import pytest

from paper_2302_06361_amd import binding

EINVAL, ESIZE = -1, -2
CTX, W, S, TO = 16, 4096, 8192, 1 << 20           # (addresses that are never followed)


@pytest.fixture(scope="module")
def lib():
    return binding.lib()


def quantise(lib, ctx=CTX, w=W, dtype=0, row_stride=5, expert_stride=20, E=2, M=4, K=5, base=-10, max_scale=255, to=TO, values=None):
    return lib.dash_f8_quantise(ctx, w, dtype, row_stride, expert_stride, E, M, K, base, max_scale, to, values, None)


def prepare(lib, ctx=CTX, codes=W, row_stride=5, expert_stride=20, scales=S, E=2, M=4, K=5, to=TO):
    return lib.dash_f8_prepare(ctx, codes, row_stride, expert_stride, scales, E, M, K, to, None)


@pytest.mark.parametrize("bad", [dict(ctx=None), dict(w=None), dict(to=None), dict(to=TO + 8), dict(dtype=-1), dict(dtype=3), dict(row_stride=4), dict(expert_stride=-1),
                                 dict(E=0), dict(M=0), dict(K=0), dict(M=-3), dict(base=-65), dict(base=65), dict(max_scale=0), dict(max_scale=32768),
                                 dict(w=W + 2), dict(values=W + 1), dict(w=W + 1, dtype=1), dict(values=W + 1, dtype=2)])
def test_quantise_refuses(lib, bad):
    assert quantise(lib, **bad) == EINVAL


@pytest.mark.parametrize("bad", [dict(ctx=None), dict(codes=None), dict(scales=None), dict(scales=S + 2), dict(to=None), dict(to=TO + 4), dict(row_stride=4),
                                 dict(expert_stride=-1), dict(E=0), dict(M=0), dict(K=0)])
def test_prepare_refuses(lib, bad):
    assert prepare(lib, **bad) == EINVAL


def test_more_blocks_than_a_launch_numbers(lib):
    big = 2 ** 31 - 1
    assert quantise(lib, E=big, M=200, K=200, row_stride=200) == ESIZE
    assert prepare(lib, E=1, M=big, K=big, row_stride=big) == ESIZE
    for E in (2 ** 13, 2 ** 14, 2 ** 15, big):                # (products past 63 bits)
        assert quantise(lib, E=E, M=big, K=big, row_stride=big) == prepare(lib, E=E, M=big, K=big, row_stride=big) == ESIZE


def test_bytes(lib):
    size = lib.dash_expert_weights_bytes
    for E, M, K in ((1, 1, 1), (3, 33, 65), (2, 128, 128), (1, 129, 257), (32, 4096, 4096)):
        tiles = -(-M // 32) * -(-K // 64) * 2048
        scales = -(-M // 128) * -(-K // 128) * 4
        assert size(binding.F8, E, M, K) == E * (tiles + -(-scales // 16) * 16)
    assert size(binding.F8, 0, 1, 1) == size(binding.F8, 1, 0, 1) == size(binding.F8, 1, 1, 0) == 0
    for format in (2, 3, 5, 7, 9):
        assert size(format, 1, 1, 1) == 0


def test_f8_is_a_format_of_its_own():
    assert len({binding.W8, binding.MX4, binding.F8}) == 3
    assert "dash_f8_quantise" in binding.SYMBOLS and "dash_f8_prepare" in binding.SYMBOLS
    assert C.sizeof(binding.CLayer) == 104
