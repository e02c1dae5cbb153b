"""A router's attributes and the descriptor that the library reads stay the same thing.  No GPU involved."""
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
