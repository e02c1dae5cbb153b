"""A router's attributes and the descriptor that the library reads stay the same thing.  No GPU involved."""
import numpy as np
import pytest
import torch

from paper_2302_06361_amd import DashError, Router


def test_another_bias():
    """as a bias that balances experts is replaced between calls: the descriptor has the new one's address, not that of memory that may have gone"""
    r = Router(8, 2, bias=torch.zeros(8))
    for b in (torch.ones(8), torch.zeros(64)[8:16]):
        r.bias = b
        assert r.bias is b and r.c.bias == b.data_ptr()
    for bad in (torch.zeros(7), torch.zeros(16)[::2], torch.zeros(8).double()):
        with pytest.raises(DashError, match="bias"):
            r.bias = bad
        assert r.bias is b and r.c.bias == b.data_ptr()
    r.bias = None
    assert r.bias is None and r.c.bias is None


@pytest.mark.parametrize("name", ["n_experts", "top_k", "c"])
def test_sizes_stay(name):
    """outputs are made for the attributes, written by the descriptor"""
    r = Router(8, 2)
    with pytest.raises(DashError):
        setattr(r, name, 1)
    assert (r.n_experts, r.top_k) == (r.c.n_experts, r.c.top_k) == (8, 2)


@pytest.mark.parametrize("name", ["n_experts", "top_k", "score", "groups", "top_groups", "group_score", "gate_bits"])
def test_integers_that_the_descriptor_does_not_hold(name):
    """refused, not cut off"""
    good = dict(n_experts=8, top_k=2, score=0, groups=1, top_groups=1, group_score=0, gate_bits=8)
    for bad in (2 ** 32 + good[name], -2 ** 32 + good[name], 2 ** 31, good[name] + 0.5):
        with pytest.raises(DashError, match=name):
            Router(**dict(good, **{name: bad}))
    for same in (np.int64(good[name]), np.uint8(good[name]), float(good[name])):
        r = Router(**dict(good, **{name: same}))
        assert (r.c.n_experts, r.c.top_k, r.c.score, r.c.n_groups, r.c.top_groups, r.c.group_score, r.c.gate_bits) == tuple(good.values())
