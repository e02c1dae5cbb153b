"""What a network takes of a router: logits, bias and the rows that take part.  No GPU involved: what reaches the choice is looked at."""
import numpy as np
import pytest
import torch

from paper_2302_06361_amd import network


class Recorder:
    """stands in for the context: keeps what a choice is made from"""
    device = torch.device("cpu")

    def choose(self, router, logits, valid=None, out=None):
        self.router, self.logits, self.valid = router, logits, valid
        return out


def routed(**router):
    ctx = Recorder()
    network._Routed(dict(dict(logits=np.zeros((6, 4)), top_k=2), **router), 2, ctx, 3, "experts").part(2, 3)
    return ctx


@pytest.mark.parametrize("values", [[0, 1, 2, 0, 255, 0], [0, 256, 512, 0, -256, 0], [0, 2 ** 40, 1, 0, -1, 0], [0.0, 0.25, 1e-30, 0.0, -0.5, 0.0], [False, True, True, False, True, False]])
def test_rows_that_take_part(values):
    """whatever is not zero takes part, of any type"""
    for given in (values, np.array(values)):
        got = routed(valid=given).valid
        assert got.itemsize == 1 and (got != 0).tolist() == [bool(v) for v in values[2:5]]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16, torch.float64, torch.int64])
def test_logits_as_tensors(dtype):
    """the three types that a choice reads as they are, others as float32; a copy: a change after the network was made does not tear its layers apart"""
    wide = torch.arange(-12, 36).reshape(6, 8).to(dtype)
    for given in (wide[:, :4], wide[:, :4].contiguous(), wide[:, ::2], wide[:, :4].clone().requires_grad_() if dtype.is_floating_point else wide[:, 4:]):
        want = given.detach()[2:5].to(dtype if dtype in (torch.float32, torch.bfloat16, torch.float16) else torch.float32).clone()
        got = routed(logits=given).logits
        assert got.dtype == want.dtype and torch.equal(got, want) and got.is_contiguous()
        ctx = Recorder()
        r = network._Routed(dict(logits=given, top_k=2), 2, ctx, 3, "experts")
        with torch.no_grad():
            given += 1
        r.part(2, 3)
        assert torch.equal(ctx.logits, want)


@pytest.mark.parametrize("dtype", [np.float32, np.float64, np.int32, np.float16])
def test_logits_as_arrays(dtype):
    a = np.arange(-12, 36).reshape(6, 8).astype(dtype)
    for given in (a[:, :4], a[:, ::2], np.asfortranarray(a[:, 4:]), a[:, :4].tolist()):
        got = routed(logits=given).logits
        assert got.dtype == torch.float32 and (got.numpy() == np.asarray(given)[2:5]).all()


def test_bias_and_valid_as_tensors():
    for dtype in (torch.float32, torch.float64, torch.bfloat16):
        b = torch.arange(8).to(dtype)[::2]
        r = routed(bias=b).router
        assert r.bias.dtype == torch.float32 and r.bias.is_contiguous() and r.bias.tolist() == [0, 2, 4, 6] and r.c.bias == r.bias.data_ptr()
    for dtype in (torch.uint8, torch.bool, torch.int64, torch.float32):
        v = torch.tensor([1, 1, 0, 1, 0, 1]).to(dtype)
        got = routed(valid=v).valid
        assert got.itemsize == 1 and got.tolist() == [0, 1, 0]
