"""The tensors that a choice of experts is written to, which the library reads by address: what does not hold the choice is refused where it is put in.  No GPU involved."""
import pytest
import torch

from paper_2302_06361_amd import Choice, DashError


class Host:
    device = torch.device("cpu")


def made():
    return Choice(Host(), 5, 2)


@pytest.mark.parametrize("name,dtype", [("experts", torch.int32), ("gates", torch.int32), ("weights", torch.float32)])
def test_replaced_tensors(name, dtype):
    c = made()
    part = torch.zeros(64, dtype=dtype)[7:17].view(5, 2)
    setattr(c, name, part)
    assert getattr(c, name) is part
    for bad in (torch.zeros(4, 2, dtype=dtype), torch.zeros(5, 3, dtype=dtype), torch.zeros(2, 5, dtype=dtype).t(), torch.zeros(5, 4, dtype=dtype)[:, ::2], torch.zeros(1, 2, dtype=dtype).expand(5, 2),
                torch.zeros(5, 2, dtype=torch.int64), torch.zeros(5, 2, dtype=torch.int16), torch.zeros(5, 2, dtype=torch.float32 if dtype == torch.int32 else torch.int32),
                torch.zeros(5, 2, dtype=dtype, device="meta"), None, [0] * 10):
        with pytest.raises(DashError, match=name):
            setattr(c, name, bad)
    assert getattr(c, name) is part


@pytest.mark.parametrize("name", ["n", "top_k", "device"])
def test_sizes_stay(name):
    c = made()
    with pytest.raises(DashError):
        setattr(c, name, 1000)
    assert (c.n, c.top_k, c.device) == (5, 2, Host.device)
