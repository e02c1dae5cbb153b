"""GPU: expert layers with 8-bit floating point weights at the ends of their ranges: calls of no rows, launches of more threads than one direction of a grid holds,
sums that pass 31 bits, values written over the weights, other streams, the entry point without allocations."""
import numpy as np
import pytest
import torch

import f8_ref
import workloads
from test_gpu_experts import P127
from test_gpu_experts_edges import bundle, context, every_matrix_is, memory_goes_back, need      # noqa: F401 (a fixture among them)

pytestmark = pytest.mark.gpu
TILES = ["rule", "big", "narrow", "few", "wide", "class", "small"]


def weights(ctx, E, M, K, seed=1):
    g = np.random.default_rng(seed)
    codes, S = g.integers(0, 256, (E, M, K)), g.integers(-300, 300, (E, f8_ref.blocks(M), f8_ref.blocks(K)))
    return ctx.f8_prepare(torch.from_numpy(codes.astype(np.uint8)).to(ctx.device), torch.from_numpy(S.astype(np.int32)).to(ctx.device))


def random_labels(ctx, n, seed=3):
    from paper_2302_06361_amd import Labels
    labels = Labels(ctx, n, zero=True)
    g = torch.Generator(device=ctx.device)
    g.manual_seed(seed)
    for t, p in zip(labels.tensors, ctx.primes):
        lam = ctx.lam(p)
        for ch in range(t.shape[0]):
            d = min(16, lam - 16 * ch)
            t[ch, :, :d] = torch.randint(0, p, (n, d), dtype=torch.uint8, device=ctx.device, generator=g)
    return labels


@pytest.mark.parametrize("tile", TILES)
def test_calls_of_no_rows(tile, monkeypatch):
    from paper_2302_06361_amd import EXPERTS, Labels, Layer
    monkeypatch.setenv("DASH_EXPERTS_TILE", tile)
    ctx = context(workloads.PRIMES[:3])
    whole = Labels(ctx, 40, zero=True)
    empty = whole.slice(7, 7)
    ids = torch.zeros(0, dtype=torch.int32, device=ctx.device)
    for lay in (Layer(EXPERTS, 1, 0, top_k=1, weights=weights(ctx, 2, 8, 10), routing=ctx.route(ids, 2)), Layer(EXPERTS, 1, 0, top_k=3, weights=weights(ctx, 1, 8, 10))):
        ctx.garble_layer(lay, empty, empty)
        ctx.eval_layer(lay, empty, None, empty)
        ctx.eval_layer(lay, whole, None, whole)
    torch.cuda.synchronize()
    assert all((t == 0).all() for t in whole.tensors)


@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("routed", [False, True])
def test_products_of_very_many_rows(tile, routed, monkeypatch):
    """one input, one output, labels of one digit: a tile for every 8, 16 or 32 rows"""
    from paper_2302_06361_amd import EXPERTS, Layer
    monkeypatch.setenv("DASH_EXPERTS_TILE", tile)
    ctx = context([5], lam=[1])
    n = 2 ** 24 + 5 if routed else 2 ** 27 + 5
    need(48 * n)
    x = torch.zeros((1, n, 16), dtype=torch.uint8, device=ctx.device)
    x[0, :, 0] = torch.randint(0, 5, (n,), dtype=torch.uint8, device=ctx.device)
    y = torch.full_like(x, 0xA5)
    # 2^-9 and -2^-9: the codes 1 and 129, integers 1 and -1, times 2 and 3
    W = ctx.f8_prepare(torch.tensor([[[1]], [[129]]], dtype=torch.uint8, device=ctx.device)[:1 + routed], torch.tensor([[[2]], [[3]]], dtype=torch.int32, device=ctx.device)[:1 + routed])
    R, ids = None, torch.zeros(n, dtype=torch.int32, device=ctx.device)
    if routed:
        ids = torch.randint(-1, 2, (n,), dtype=torch.int32, device=ctx.device)
        R = ctx.route(ids, 2)
    ctx.eval_layer(Layer(EXPERTS, 1, n, top_k=1, weights=W, routing=R), bundle(ctx, x), None, bundle(ctx, y))
    torch.cuda.synchronize()
    factor = torch.tensor([0, 2, 5 - 3], dtype=torch.uint8, device=ctx.device)[ids + 1]
    x[0, :, 0] = x[0, :, 0] * factor % 5
    assert torch.equal(x, y)


def test_quantisation_of_very_many_blocks():
    ctx = context([5])
    E = 2 ** 23 + 3                         # (512 threads each)
    need(2064 * E)
    w = torch.randn(1, 32, 64, device=ctx.device)
    one = ctx.f8_quantise(w, -6, 8).data.clone()
    assert one.numel() == 2064 and one.any()
    one[2052:] = 0
    data = ctx.f8_quantise(w.expand(E, 32, 64), -6, 8).data
    data.view(E, 2064)[:, 2052:] = 0        # (what pads the scales is not written)
    assert every_matrix_is(data, one)


def test_codes_of_very_many_tiles():
    ctx = context([5])
    E = 2 ** 25 + 3
    need(2064 * E + 4 * E)
    codes = torch.randint(0, 127, (1, 32, 64), dtype=torch.uint8, device=ctx.device)
    one = ctx.f8_prepare(codes, torch.full((1, 1, 1), 77, dtype=torch.int32, device=ctx.device)).data.clone()
    assert one.numel() == 2064 and one.any()
    one[2052:] = 0
    data = ctx.f8_prepare(codes.expand(E, 32, 64), torch.full((E, 1, 1), 77, dtype=torch.int32, device=ctx.device)).data
    data.view(E, 2064)[:, 2052:] = 0
    assert every_matrix_is(data, one)


@pytest.mark.parametrize("primes,K", [(P127, (2 ** 31 - 1 - 126) // (256 * 126)), (workloads.PRIMES[:12], (2 ** 31 - 1 - 36) // (256 * 36))])
def test_sums_of_31_bits(primes, K):
    """the longest reductions that a prime allows: labels of p - 1, weights whose residues modulo a class are the largest; one input more is refused"""
    from paper_2302_06361_amd import DashError, EXPERTS, Labels, Layer
    ctx = context(primes)
    codes = torch.full((1, 2, K), 0x7E, dtype=torch.uint8, device=ctx.device)
    codes[0, 1] += 128
    blocks = f8_ref.blocks(K)
    S = torch.randint(1, 2 ** 15, (1, 1, blocks), dtype=torch.int32, device=ctx.device)
    lay = Layer(EXPERTS, 1, 1, top_k=1, weights=ctx.f8_prepare(codes, S))
    src, dst = Labels(ctx, K, zero=True), Labels(ctx, 2)
    for t, p in zip(src.tensors, ctx.primes):
        for ch in range(t.shape[0]):
            t[ch, :, :min(16, ctx.lam(p) - 16 * ch)] = p - 1
    ctx.garble_layer(lay, src, dst)
    total = sum(512 * 448 * int(s) * min(128, K - 128 * i) for i, s in enumerate(S.flatten().tolist()))
    for i, p in enumerate(ctx.primes):
        got = dst.to_numpy(i)
        assert (got[0] == total * (p - 1) % p).all() and (got[1] == -total * (p - 1) % p).all(), p
    long = Layer(EXPERTS, 1, 1, top_k=1, weights=ctx.f8_prepare(torch.zeros(1, 2, K + 1, dtype=torch.uint8, device=ctx.device),
                                                                torch.ones(1, 1, f8_ref.blocks(K + 1), dtype=torch.int32, device=ctx.device)))
    with pytest.raises(DashError):
        ctx.garble_layer(long, Labels(ctx, K + 1), dst)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_values_over_the_weights(dtype):
    ctx = context([5])
    w = torch.randn(2, 140, 300, device=ctx.device).to(dtype)
    values = torch.empty_like(w)
    want = ctx.f8_quantise(w, -9, 255, values=values)
    got = ctx.f8_quantise(w, -9, 255, values=w)
    torch.cuda.synchronize()
    assert torch.equal(w, values)
    a, b = (f8_ref.unpack(x.data.cpu().numpy(), 2, 140, 300) for x in (want, got))
    assert (a[0] == b[0]).all() and (a[1] == b[1]).all()


@pytest.mark.parametrize("tile", TILES)
def test_other_streams(tile, monkeypatch):
    """quantisation, routing and products on a stream of their own, two such streams at once, as one stream after the other"""
    from paper_2302_06361_amd import EXPERTS, Labels, Layer
    monkeypatch.setenv("DASH_EXPERTS_TILE", tile)
    ctx = context(workloads.PRIMES[:8])
    n, E, M, K = 37, 4, 150, 400
    w = [torch.randn(E, M, K, device=ctx.device) for _ in range(2)]
    ids = [torch.randint(-1, E, (n,), dtype=torch.int32, device=ctx.device) for _ in range(2)]
    src = [random_labels(ctx, n * K, 5 + i) for i in range(2)]

    def run(i, dst):
        ctx.eval_layer(Layer(EXPERTS, 1, n, top_k=1, weights=ctx.f8_quantise(w[i], -9), routing=ctx.route(ids[i], E)), src[i], None, dst)

    want, got = ([Labels(ctx, n * M) for _ in range(2)] for _ in range(2))
    for i in range(2):
        run(i, want[i])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                run(i, got[i])
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a.tensors, b.tensors))


def test_without_allocations():
    from paper_2302_06361_amd import EXPERTS, Labels, Layer
    ctx = context(workloads.PRIMES[:8])
    n, E, M, K = 9, 3, 140, 200
    lay = Layer(EXPERTS, 1, n, top_k=1, weights=weights(ctx, E, M, K), routing=ctx.route(torch.arange(n, dtype=torch.int32, device=ctx.device) % E, E))
    src = random_labels(ctx, n * K)
    a, b = Labels(ctx, n * M), Labels(ctx, n * M)
    ctx.eval_layer(lay, src, None, a)
    ctx.eval_layer_noalloc(lay, src, None, b)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) and x.any() for x, y in zip(a.tensors, b.tensors))


def test_binding_refuses():
    from paper_2302_06361_amd import DashError
    ctx = context([5])
    w = torch.randn(2, 40, 70, device=ctx.device)
    codes, S = torch.zeros(2, 40, 70, dtype=torch.uint8, device=ctx.device), torch.ones(2, 1, 1, dtype=torch.int32, device=ctx.device)
    other = ctx.f8_quantise(torch.randn(2, 40, 80, device=ctx.device), -9)
    bytes_ = ctx.weights8_prepare(torch.zeros(2, 40, 70, dtype=torch.int8, device=ctx.device))
    for call in (lambda: ctx.f8_quantise(w, -9, out=other), lambda: ctx.f8_quantise(w, -9, out=bytes_), lambda: ctx.f8_prepare(codes, S, out=bytes_),
                 lambda: ctx.f8_quantise(w.transpose(1, 2), -9), lambda: ctx.f8_quantise(w.double(), -9), lambda: ctx.f8_quantise(w.cpu(), -9),
                 lambda: ctx.f8_quantise(w, -9, values=torch.empty(2, 40, 71, device=ctx.device)), lambda: ctx.f8_quantise(w, -9, values=w.bfloat16()),
                 lambda: ctx.f8_quantise(w, -65), lambda: ctx.f8_quantise(w, -9, 0), lambda: ctx.f8_prepare(w, S), lambda: ctx.f8_prepare(codes, S.float()),
                 lambda: ctx.f8_prepare(codes, S[:1]), lambda: ctx.f8_prepare(codes, S.cpu()), lambda: ctx.f8_prepare(codes, torch.ones(2, 1, 2, dtype=torch.int32, device=ctx.device)[:, :, ::2])):
        with pytest.raises(DashError):
            call()
