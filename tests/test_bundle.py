"""The binding's host module: a list of label tensors as a dash_labels (no GPU needed: addresses and strides of any tensor)."""
import ctypes as C
import os

import pytest
import torch


@pytest.fixture(scope="module")
def describe():
    from paper_2302_06361_amd import build
    if not os.path.exists(build.bundle_so()):
        build.build_bundle()
    from paper_2302_06361_amd._bundle import describe
    return describe


def filled(describe, tensors, n):
    from paper_2302_06361_amd.binding import CLabels
    s = CLabels()
    C.memset(C.addressof(s), 0xA5, C.sizeof(s))
    describe(tensors, C.addressof(s), n)
    return s


def test_addresses_and_strides(describe):
    whole = torch.zeros(5, 40, 16, dtype=torch.uint8)
    tensors = [whole, None, whole[:, 3:30], whole[2:], torch.zeros(1, 1, 16, dtype=torch.uint8), whole[::2]]
    s = filled(describe, tensors, 27)
    assert s.n_elem == 27
    for i in range(16):
        t = tensors[i] if i < len(tensors) else None
        assert (s.data[i] or 0) == (0 if t is None else t.data_ptr())
        assert s.chunk_stride[i] == (0 if t is None else t.stride(0))


def test_bundle_follows_its_tensors(describe):
    """nothing is kept from one call for the next: a bundle's tensors may be replaced or moved"""
    from paper_2302_06361_amd.binding import Labels
    b = Labels.__new__(Labels)
    b.n_elem, b.tensors = 4, [torch.zeros(2, 4, 16, dtype=torch.uint8)]
    first = b.c().data[0]
    b.tensors[0] = torch.zeros(2, 9, 16, dtype=torch.uint8)
    s = b.c()
    assert s.data[0] == b.tensors[0].data_ptr() != first and s.chunk_stride[0] == 144
    b.tensors[0].set_(torch.zeros(2, 5, 16, dtype=torch.uint8))
    assert b.c().data[0] == b.tensors[0].data_ptr() and b.c().chunk_stride[0] == 80


def test_refusals(describe):
    from paper_2302_06361_amd.binding import CLabels
    s = CLabels()
    at = C.addressof(s)
    t = torch.zeros(1, 1, 16, dtype=torch.uint8)
    for bad in (((t,), at, 1), ([t], at), ([3], at, 1), ([t], "x", 1), ([t], at, None)):
        with pytest.raises(TypeError):
            describe(*bad)
    with pytest.raises(IndexError):
        describe([t] * 17, at, 1)
    with pytest.raises(IndexError):
        describe([t], 0, 1)
    with pytest.raises((RuntimeError, IndexError)):
        describe([torch.zeros((), dtype=torch.uint8)], at, 1)          # no dimension to take the stride of
