"""GPU: expert layers at the ends of their ranges: calls of no rows, launches of more threads than one direction of a grid holds."""
import numpy as np
import pytest
import torch

import workloads
from gpu_util import SEED

pytestmark = pytest.mark.gpu


def context(primes, **kw):
    from paper_2302_06361_amd import Context
    return Context(primes, SEED, (2, 6), **kw)


def test_calls_of_no_rows():
    """empty parts of bundles and empty gates have no address; a dense layer of no batch elements does nothing either"""
    from paper_2302_06361_amd import COMBINE, DENSE, EXPERTS, Labels, Layer
    ctx = context(workloads.PRIMES[:3])
    whole = Labels(ctx, 40, zero=True)
    empty = whole.slice(7, 7)
    assert all(t.data_ptr() == 0 for t in empty.tensors)
    W = ctx.weights8_prepare(torch.zeros(2, 8, 10, dtype=torch.int8, device=ctx.device))
    one = ctx.weights8_prepare(torch.zeros(1, 8, 10, dtype=torch.int8, device=ctx.device))
    ids = torch.zeros(0, dtype=torch.int32, device=ctx.device)
    gates = torch.zeros(0, 2, dtype=torch.int32, device=ctx.device)
    layers = [Layer(DENSE, 1, 0, in_c=10, out_c=8, weights=ctx.weights_prepare(np.zeros((8, 10), np.int32))),
              Layer(EXPERTS, 1, 0, top_k=1, weights=W, routing=ctx.route(ids, 2)), Layer(EXPERTS, 1, 0, top_k=3, weights=one),
              Layer(COMBINE, 1, 0, in_c=5, top_k=2, gates=gates)]
    for lay in layers:
        ctx.garble_layer(lay, empty, empty)
        ctx.eval_layer(lay, empty, None, empty)
        ctx.eval_layer(lay, whole, None, whole)
    torch.cuda.synchronize()
    assert all((t == 0).all() for t in whole.tensors)
