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


@pytest.fixture(autouse=True)
def memory_goes_back():
    yield
    torch.cuda.empty_cache()


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


# Launches of 2^32 threads and more; what they read and write is small or the same over and over, so that a plain form of it is at hand.
def need(bytes):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < bytes + 2 ** 33:
        pytest.skip("not enough device memory")


def bundle(ctx, tensor):
    from paper_2302_06361_amd import Labels
    b = Labels.__new__(Labels)
    b.ctx, b.n_elem, b.tensors = ctx, tensor.shape[1], [tensor]
    return b


@pytest.mark.parametrize("fmt,tile", [("w8", "rule"), ("w8", "narrow"), ("mx4", "rule"), ("mx4", "big"), ("mx4", "narrow"), ("mx4", "few"), ("mx4", "wide")])
@pytest.mark.parametrize("routed", [False, True])
def test_products_of_very_many_rows(fmt, tile, routed, monkeypatch):
    """one input, one output, labels of one digit: a tile for every 4, 8 or 16 rows"""
    from paper_2302_06361_amd import EXPERTS, Layer
    monkeypatch.setenv("DASH_EXPERTS_TILE", tile)
    ctx = context([5], lam=[1])
    n = 2 ** 24 + 5 if routed else 2 ** 27 + 5             # (a routing numbers groups and tiles in 31 bits: 33 million rows at most here)
    need(48 * n)
    x = torch.zeros((1, n, 16), dtype=torch.uint8, device=ctx.device)
    x[0, :, 0] = torch.randint(0, 5, (n,), dtype=torch.uint8, device=ctx.device)
    y = torch.full_like(x, 0xA5)
    if fmt == "w8":
        W, ints = ctx.weights8_prepare(torch.tensor([[[2]], [[-1]]], dtype=torch.int8, device=ctx.device)[:1 + routed]), (2, 4)
    else:
        W, ints = ctx.mx4_quantise(torch.tensor([[[1.5]], [[-2.0]]], device=ctx.device)[:1 + routed], base=0), (3, 1)
    R, ids = None, torch.zeros(n, dtype=torch.int32, device=ctx.device)
    if routed:
        ids = torch.randint(-1, 2, (n,), dtype=torch.int32, device=ctx.device)
        R = ctx.route(ids, 2)
    ctx.eval_layer(Layer(EXPERTS, 1, n, top_k=1, weights=W, routing=R), bundle(ctx, x), None, bundle(ctx, y))
    torch.cuda.synchronize()
    factor = torch.tensor([0, ints[0], ints[1]], dtype=torch.uint8, device=ctx.device)[ids + 1]
    x[0, :, 0] = x[0, :, 0] * factor % 5
    assert torch.equal(x, y)


def every_matrix_is(data, one):
    """data: matrices one after the other, each the bytes of `one`"""
    whole = data.view(-1, one.numel())
    return all(bool((whole[i:i + 2 ** 20] == one).all()) for i in range(0, whole.shape[0], 2 ** 20))


def test_quantisation_of_very_many_tiles():
    ctx = context([5])
    E = 2 ** 24 + 3
    need(1088 * E)
    w = torch.randn(1, 32, 64, device=ctx.device)
    one = ctx.mx4_quantise(w, -6, 8).data.clone()
    assert one.numel() == 1088 and one.any()
    assert every_matrix_is(ctx.mx4_quantise(w.expand(E, 32, 64), -6, 8).data, one)


def test_bytes_of_very_many_tiles():
    ctx = context([5])
    E = 2 ** 25 + 3
    need(2048 * E)
    w = torch.randint(-128, 128, (1, 32, 64), dtype=torch.int8, device=ctx.device)
    one = ctx.weights8_prepare(w).data.clone()
    assert one.numel() == 2048 and one.any()
    assert every_matrix_is(ctx.weights8_prepare(w.expand(E, 32, 64)).data, one)


def test_weighted_sums_of_very_many_values():
    from paper_2302_06361_amd import COMBINE, Layer
    ctx = context([2], lam=[128])
    n = 2 ** 29 + 3
    need(2 * 128 * n + 4 * n)
    x = torch.empty((8, n, 16), dtype=torch.uint8, device=ctx.device)
    for ch in x:
        ch.random_(0, 2)
    y = torch.full_like(x, 0xA5)
    gates = torch.randint(-2, 2, (n, 1), dtype=torch.int32, device=ctx.device)
    ctx.eval_layer(Layer(COMBINE, 1, n, in_c=1, top_k=1, gates=gates), bundle(ctx, x), None, bundle(ctx, y))
    torch.cuda.synchronize()
    for at in range(0, n, 2 ** 26):
        part = slice(at, at + 2 ** 26)
        odd = (gates[part] & 1).to(torch.uint8)
        for ch in range(8):
            assert torch.equal(y[ch, part], x[ch, part] * odd), (ch, at)
