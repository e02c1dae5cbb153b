"""GPU parity: the choice of experts from a router's logits against a plain 64-bit reference.  Experts and gates are integers and have to be equal;
weights are rounded once to float32: off by at most half a step of it, 2^-24 of the value (2^-150 where it is subnormal), and what 64 bits
leave (1e-12)."""
import numpy as np
import pytest
import torch

import choose_ref
import workloads
from test_gpu_experts import context

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def ctx():
    return context(workloads.PRIMES[:8])


def guarded(t, ctx, value):
    """a contiguous tensor of t's size in the middle of a longer one"""
    whole = torch.full((t.numel() + 64,), value, dtype=t.dtype, device=ctx.device)
    return whole, whole[32:32 + t.numel()].view(t.shape)


def check(ctx, logits, top_k, dtype="f32", pad=0, valid=None, bias=None, sigmoid=False, groups=1, top_groups=1, pair=False, **kw):
    """logits float64 [n][E], rounded to the type first; a slice of a wider tensor if pad"""
    from paper_2302_06361_amd import GROUP_MAX, GROUP_PAIR, SIGMOID, SOFTMAX, Choice, Router
    t = torch.from_numpy(np.asarray(logits, np.float64)).to(TYPES[dtype])
    n, E = t.shape
    wide = torch.full((n, E + pad), 9.0, dtype=t.dtype)
    wide[:, :E] = t
    b = None if bias is None else torch.from_numpy(bias.astype(np.float32)).to(ctx.device)
    router = Router(E, top_k, score=SIGMOID if sigmoid else SOFTMAX, bias=b, groups=groups, top_groups=top_groups, group_score=GROUP_PAIR if pair else GROUP_MAX, **kw)
    out = Choice(ctx, n, top_k)
    all_e, out.experts = guarded(out.experts, ctx, -77)
    all_g, out.gates = guarded(out.gates, ctx, -77)
    all_w, out.weights = guarded(out.weights, ctx, -77.0)
    v = None if valid is None else torch.from_numpy(valid).to(ctx.device)
    got = ctx.choose(router, wide.to(ctx.device)[:, :E], valid=v, out=out)
    torch.cuda.synchronize()
    assert got is out
    experts, gates, weights = choose_ref.choose(t.double().numpy(), top_k, sigmoid, None if bias is None else bias.astype(np.float32), groups, top_groups, pair,
                                                valid=valid, **kw)
    bad = np.argwhere(out.experts.cpu().numpy() != experts)
    assert bad.size == 0, (len(bad), bad[:3], out.experts.cpu().numpy()[bad[0][0]], experts[bad[0][0]])
    assert (out.gates.cpu().numpy() == gates).all()
    w = out.weights.cpu().double().numpy()
    assert (np.abs(w - weights) <= weights * (2.0 ** -24 + 1e-12) + 2.0 ** -150).all()
    for whole in (all_e, all_g, all_w):
        assert (whole[:32] == -77).all() and (whole[-32:] == -77).all(), "around the output"
    again = ctx.choose(router, wide.to(ctx.device)[:, :E], valid=v)
    assert torch.equal(again.experts, out.experts) and torch.equal(again.gates, out.gates) and torch.equal(again.weights, out.weights)
    return out


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("E", [1, 2, 7, 8, 15, 16, 17, 31, 32, 33, 64, 65, 100, 128, 129, 160, 250, 256, 257, 400, 512, 513, 1000, 1024])
def test_numbers_of_experts(ctx, E, dtype):
    g = np.random.default_rng(E)
    for top_k, sigmoid, bias, renormalise in ((1, False, False, True), (min(E, 2), True, False, False), (min(E, 8), False, True, False), (min(E, 6), True, True, True)):
        check(ctx, 2 * g.standard_normal((19, E)), top_k, dtype, pad=E % 3, bias=0.1 * g.standard_normal(E) if bias else None, sigmoid=sigmoid,
              renormalise=renormalise, scale=2.5, gate_bits=12)


@pytest.mark.parametrize("n", [1, 2, 3, 15, 16, 17, 63, 64, 65, 1000])
def test_numbers_of_rows(ctx, n):
    g = np.random.default_rng(n)
    for E in (8, 60, 256, 700):
        check(ctx, g.standard_normal((n, E)), 4, "bf16", bias=0.1 * g.standard_normal(E))
        check(ctx, g.standard_normal((n, E)), 4, "f32", valid=g.integers(0, 2, n).astype(np.uint8))


def test_no_rows(ctx):
    from paper_2302_06361_amd import Router
    out = ctx.choose(Router(8, 2), torch.empty((0, 8), device=ctx.device))
    assert out.experts.shape == (0, 2)


@pytest.mark.parametrize("E,top_k", [(1, 1), (5, 5), (16, 16), (17, 17), (32, 32), (40, 32), (256, 32), (1024, 31)])
def test_many_chosen(ctx, E, top_k):
    g = np.random.default_rng(E + top_k)
    check(ctx, g.standard_normal((21, E)), top_k, "f32", bias=0.2 * g.standard_normal(E), sigmoid=True)
    check(ctx, g.standard_normal((21, E)), top_k, "f16")


@pytest.mark.parametrize("E,groups,top_groups,top_k", [(8, 2, 1, 3), (8, 8, 3, 3), (160, 8, 3, 6), (256, 8, 4, 8), (60, 20, 7, 10), (64, 64, 10, 5), (1024, 16, 5, 12),
                                                       (640, 64, 1, 9), (36, 3, 2, 24), (256, 8, 8, 8), (300, 2, 1, 32)])
@pytest.mark.parametrize("pair", [False, True])
def test_groups(ctx, E, groups, top_groups, top_k, pair):
    g = np.random.default_rng(E + groups + top_k)
    for sigmoid, bias in ((False, False), (True, False), (False, True), (True, True)):
        check(ctx, 1.5 * g.standard_normal((35, E)), top_k, "bf16" if bias else "f32", bias=0.1 * g.standard_normal(E) if bias else None, sigmoid=sigmoid,
              groups=groups, top_groups=top_groups, pair=pair, renormalise=sigmoid)


@pytest.mark.parametrize("pair", [False, True])
@pytest.mark.parametrize("groups", [1, 4])
def test_ties(ctx, groups, pair):
    """few different logits: the lower number of expert and of group"""
    g = np.random.default_rng(groups)
    for E in (8, 64, 256, 520):
        for bias in (None, np.zeros(E), 0.25 * g.integers(0, 2, E)):
            check(ctx, g.integers(0, 3, (40, E)), 8 // groups, "bf16", bias=bias, groups=groups, top_groups=max(1, groups // 2), pair=pair)
        check(ctx, np.zeros((5, E)), 8 // groups, "f16", groups=groups, top_groups=max(1, groups // 2), pair=pair, sigmoid=True)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("groups", [1, 8])
def test_masks(ctx, sigmoid, bias, groups):
    """logits of -infinity: few left, fewer than are wanted, none; groups of nothing; numbers that are none, infinities"""
    g = np.random.default_rng(3)
    for E in (16, 64, 256):
        l = g.standard_normal((60, E))
        l[:20][g.random((20, E)) < 0.9] = -np.inf
        l[20] = -np.inf
        l[21, :] = np.nan
        l[22, 3] = 0.5
        l[22, np.arange(E) != 3] = -np.inf
        l[23, 5] = np.inf
        l[24, [1, 7, 9]] = np.inf
        l[25, ::2] = np.nan
        l[26, : E // 2] = -np.inf
        l[27] = np.inf
        b = 0.1 * g.standard_normal(E)
        check(ctx, l, 2, "f32", bias=b if bias else None, sigmoid=sigmoid, groups=groups, top_groups=groups // 2 or 1, pair=groups > 1 and bias, renormalise=not bias)
        check(ctx, l, E // groups, "bf16", bias=b if bias else None, sigmoid=sigmoid, groups=groups, top_groups=1, pair=groups > 1) if E // groups <= 32 else None
        if bias:
            for v in (-np.inf, np.inf, np.nan):
                b2 = b.copy()
                b2[[0, 5, E - 1]] = v
                b2[E // 2:E // 2 + 4] = v
                check(ctx, l, 2, "f32", bias=b2, sigmoid=sigmoid, groups=groups, top_groups=groups // 2 or 1)


def test_logits_of_the_lowest_value(ctx):
    """masks by the type's lowest number: chosen last, weight zero"""
    g = np.random.default_rng(8)
    for dtype, low in (("f32", -3.4028234663852886e38), ("bf16", float(torch.finfo(torch.bfloat16).min)), ("f16", -65504.0)):
        l = g.standard_normal((30, 16))
        l[g.random((30, 16)) < 0.8] = low
        l[3] = low
        for sigmoid in (False, True):
            check(ctx, l, 4, dtype, sigmoid=sigmoid)
            check(ctx, l, 4, dtype, sigmoid=sigmoid, bias=g.standard_normal(16))


def test_far_logits(ctx):
    """scores that 64 bits hold as zero, or as one; a sum of chosen scores that is zero"""
    g = np.random.default_rng(9)
    for size in (30.0, 300.0, 3000.0, 1e30):
        for sigmoid in (False, True):
            for renormalise in (False, True):
                check(ctx, size * g.standard_normal((40, 24)), 5, "f32", sigmoid=sigmoid, renormalise=renormalise)
                check(ctx, -size * np.abs(g.standard_normal((40, 24))), 5, "bf16", sigmoid=sigmoid, renormalise=renormalise, bias=g.standard_normal(24))


@pytest.mark.parametrize("gate_bits,scale", [(0, 1.0), (0, 1000.0), (8, 0.001), (20, 1.0), (30, 1.0), (20, 1024.0)])
def test_gates(ctx, gate_bits, scale):
    g = np.random.default_rng(gate_bits)
    for renormalise in (False, True):
        check(ctx, g.standard_normal((300, 32)), 6, "f32", renormalise=renormalise, gate_bits=gate_bits, scale=scale)
    # weights of exactly one half, three quarters ...
    check(ctx, np.zeros((3, 64)), 4, "f32", renormalise=False, gate_bits=5)
    check(ctx, np.zeros((3, 64)), 32, "f32", renormalise=True, gate_bits=4)


def test_many_rows(ctx):
    g = np.random.default_rng(12)
    check(ctx, 1.5 * g.standard_normal((5000, 64)), 6, "bf16", bias=0.05 * g.standard_normal(64), sigmoid=True, groups=8, top_groups=3, pair=True, scale=2.5, gate_bits=12)


@pytest.mark.parametrize("n,E", [(2048, 72), (2049, 72), (1024, 128), (2049, 128), (1024, 136), (1025, 256), (8192, 200), (8193, 256), (2048, 264), (2049, 512), (2049, 400)])
def test_lanes_of_a_row(ctx, n, E):
    """the kernels by rows and experts: plain, with a bias, in groups, with both, of rows with ties, masks and nothing at all among others"""
    g = np.random.default_rng(n + E)
    rows = 1.5 * g.standard_normal((97, E))
    rows[5] = -np.inf
    rows[6, 3:] = -np.inf
    rows[7] = 0.5
    rows[8] = np.round(rows[8])
    rows[9, ::3] = np.nan
    rows[10, E // 2:] = np.inf
    l = np.resize(rows, (n, E))
    b = np.round(0.1 * g.standard_normal(E), 2)
    check(ctx, l, 6, "bf16")
    check(ctx, l, 6, "f32", bias=b)
    check(ctx, l, 6, "f16", bias=b, sigmoid=True, groups=8, top_groups=3, pair=True)
    check(ctx, l, 6, "f32", groups=8, top_groups=3, pair=True, renormalise=False)
    check(ctx, l, 6, "bf16", sigmoid=True, groups=4, top_groups=1)


def test_another_stream_and_a_graph(ctx):
    from paper_2302_06361_amd import Choice, Router
    g = np.random.default_rng(13)
    l = torch.from_numpy(g.standard_normal((100, 64))).float().to(ctx.device)
    router = Router(64, 4, groups=8, top_groups=3)
    want = ctx.choose(router, l)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ctx.choose(router, l)
    side.synchronize()
    assert torch.equal(got.experts, want.experts) and torch.equal(got.gates, want.gates)
    out = Choice(ctx, 100, 4)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.choose(router, l, out=out)
    for i in range(4):
        l.copy_(torch.from_numpy(g.standard_normal((100, 64))).float())
        want = ctx.choose(router, l)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.experts, want.experts) and torch.equal(out.gates, want.gates) and torch.equal(out.weights, want.weights)
