"""A bundle's tensors as any sequence, and the binding without its compiled host module.  No GPU needed: addresses and strides of any tensor."""
import sys

import pytest
import torch

from paper_2302_06361_amd import binding
from paper_2302_06361_amd.binding import Labels


def bundle(tensors, n=4):
    b = Labels.__new__(Labels)
    b.n_elem, b.tensors = n, tensors
    return b


def items():
    whole = torch.zeros(5, 40, 16, dtype=torch.uint8)
    return [whole, None, whole[:, 3:30], whole[::2]]


def check(s, want, n=4):
    assert s.n_elem == n
    for i in range(16):
        t = want[i] if i < len(want) else None
        assert (s.data[i] or 0) == (0 if t is None else t.data_ptr())
        assert s.chunk_stride[i] == (0 if t is None else t.stride(0))


class Sequence:
    def __init__(self, items):
        self.items = items

    def __len__(self):
        return len(self.items)

    def __getitem__(self, i):
        return self.items[i]


SEQUENCES = {"list": list, "tuple": tuple, "list type": lambda t: type("Tensors", (list,), {})(t), "own": Sequence, "values": lambda t: dict(enumerate(t)).values(),
             "parameters": lambda t: [None if x is None else torch.nn.Parameter(x, requires_grad=False) for x in t]}


@pytest.mark.parametrize("kind", list(SEQUENCES))
def test_any_sequence_of_tensors(kind):
    t = items()
    b = bundle(SEQUENCES[kind](t))
    for _ in range(2):
        check(b.c(), t)


@pytest.mark.parametrize("kind", list(SEQUENCES))
def test_without_the_host_module(kind, monkeypatch):
    """the library alone is enough: addresses are then asked for one by one"""
    monkeypatch.setitem(sys.modules, "paper_2302_06361_amd._bundle", None)       # (an import of it fails)
    monkeypatch.setattr(binding, "_describe", binding._describe_first)
    t = items()
    b = bundle(SEQUENCES[kind](t))
    for _ in range(2):
        check(b.c(), t)
    with pytest.raises(IndexError):
        bundle([t[0]] * 17).c()
