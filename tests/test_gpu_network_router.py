"""GPU: networks whose router's logits are on the device already, in the types that a choice reads"""
import numpy as np
import pytest
import torch

import workloads
from test_gpu_routed_network import as_plain
from test_gpu_experts import plain

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_logits_on_the_device(dtype):
    from paper_2302_06361_amd import Context, GarbledNetwork
    net = workloads.mixture(k=12, f8=True, router=dict(valid=np.array([1, 0, 1, 1], np.uint8)))
    router = next(L["router"] for L in net["layers"] if "router" in L)
    logits = torch.from_numpy(router["logits"]).to(dtype)
    want = dict(net, layers=[dict(L, router=dict(L["router"], logits=logits.float().numpy())) if "router" in L else L for L in net["layers"]])
    given = dict(net, layers=[dict(L, router=dict(L["router"], logits=logits.cuda(), valid=torch.tensor([1, 0, 1, 1]).cuda())) if "router" in L else L for L in net["layers"]])
    ctx = Context(net["primes"], net["seed"], net["digits"])
    gn = GarbledNetwork(ctx, given)
    gn.garble()
    gn.encode(torch.as_tensor(net["x"]).to(ctx.device))
    gn.evaluate()
    values, valid = gn.decode()
    assert valid.all() and (values.cpu().numpy() == plain(as_plain(want))).all()
