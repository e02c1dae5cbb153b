"""GPU parity: expert layers on LabelTensors (4-bit and 8-bit weights, products by expert, weighted sums, routing) through the C
ABI against plain 64-bit references.  All results are integers and have to be equal."""
import numpy as np
import pytest
import torch

import experts_ref as ref
import workloads
from gpu_util import SEED

pytestmark = pytest.mark.gpu

P127 = [2, 3, 101, 113, 127]


def context(primes, **kw):
    from paper_2302_06361_amd import Context
    return Context(primes, SEED, (2, 6), **kw)


def draw_labels(g, ctx, n, top=False):
    """host labels [n][lambda] per residue; top: every digit p - 1"""
    return [np.full((n, ctx.lam(p)), p - 1, np.uint8) if top else g.integers(0, p, (n, ctx.lam(p))).astype(np.uint8) for p in ctx.primes]


def upload(ctx, x, pad=(0, 0)):
    """a bundle of the labels, a slice of a longer one if pad"""
    from paper_2302_06361_amd import Labels
    n = x[0].shape[0]
    whole = Labels(ctx, n + sum(pad), zero=True)
    part = whole.slice(pad[0], pad[0] + n)
    for i, a in enumerate(x):
        part.from_numpy(i, a)
    return part


def weights(g, ctx, fmt, E, M, K, max_shift=9, extreme=False):
    """-> (ExpertWeights, integers [E][M][K])"""
    if fmt == "w8":
        w = np.full((E, M, K), -128, np.int8) if extreme else g.integers(-128, 128, (E, M, K)).astype(np.int8)
        return ctx.weights8_prepare(torch.from_numpy(w).to(ctx.device)), w.astype(np.int64)
    codes = g.integers(0, 16, (E, M, K))
    shifts = g.integers(0, max_shift + 1, (E, M, (K + 31) // 32))
    val = ref.E2M1[codes & 7] * np.where(codes & 8, -1, 1) * np.exp2(np.repeat(shifts, 32, -1)[:, :, :K] - 120.0)
    W = ctx.mx4_quantise(torch.from_numpy(val.astype(np.float32)).to(ctx.device), base=-120, max_shift=255)
    return W, ref.mx4_integers(codes, shifts)


def run_experts(ctx, fmt, E, top_k, route, K, M, seed, bias=False, garble=False, pad=(0, 0), routed=True, top=False, **kw):
    from paper_2302_06361_amd import EXPERTS, Labels, Layer
    g = np.random.default_rng(seed)
    n = len(route)
    x = draw_labels(g, ctx, n // top_k * K, top)
    W, ints = weights(g, ctx, fmt, E, M, K, extreme=top, **kw)
    b = g.integers(-2 ** 31, 2 ** 31, (E, M)).astype(np.int32) if bias else None
    R = ctx.route(torch.tensor(route, dtype=torch.int32, device=ctx.device), E) if routed else None
    lay = Layer(EXPERTS, 3, n, top_k=top_k, weights=W, routing=R, bias=torch.from_numpy(b).to(ctx.device) if bias else None)
    assert ctx.layer_sizes(lay) == (M, 0, 0)
    src = upload(ctx, x, pad)
    whole = Labels(ctx, n * M + sum(pad))
    for t in whole.tensors:
        t.fill_(0xA5)
    dst = whole.slice(pad[0], pad[0] + n * M)
    (ctx.garble_layer if garble else lambda l, i, o: ctx.eval_layer(l, i, None, o))(lay, src, dst)
    torch.cuda.synchronize()
    for i, p in enumerate(ctx.primes):
        lam = ctx.lam(p)
        one = ctx.one(i, 0 if garble else 1)
        want = ref.experts(x[i].reshape(n // top_k, K, lam), ints, route, top_k, p, b, one).reshape(n * M, lam)
        got = dst.to_numpy(i)
        bad = np.argwhere(got != want)
        assert bad.size == 0, "p = %d: %d of %d digits differ, first at %s (row %d, output %d)" % (p, len(bad), got.size, bad[0], bad[0][0] // M, bad[0][0] % M)
        assert dst.pad_is_zero(i)
        if sum(pad):
            t = whole.tensors[i]
            assert (t[:, :pad[0]] == 0xA5).all() and (t[:, pad[0] + n * M:] == 0xA5).all(), "bytes around the output were written"


FORMATS = ["w8", "mx4"]


@pytest.fixture(params=["rule", "big", "narrow", "few", "wide"])
def tile(request, monkeypatch):
    """the tile that the layer's sizes ask for, and each tile forced"""
    monkeypatch.setenv("DASH_EXPERTS_TILE", request.param)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("K", [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 200, 257, 400])
def test_experts_reduction_lengths(fmt, K, tile):
    ctx = context(workloads.PRIMES[:8])
    run_experts(ctx, fmt, 3, 1, [2, 0, 2, 1, 2], K, 37, K, bias=K % 2 == 0, garble=K % 3 == 0)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M", [1, 2, 31, 32, 33, 64, 127, 128, 129, 255, 257])
def test_experts_output_counts(fmt, M, tile):
    ctx = context(workloads.PRIMES[:12])
    run_experts(ctx, fmt, 2, 1, [1, 0, 1], 70, M, M, bias=M % 2 == 1, garble=M % 3 == 0)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("route,E", [([0], 1), ([-1], 1), ([4], 7), ([-1, -1, -1], 2), ([0] * 9, 3), ([2] * 65, 3), (list(range(40)), 40),
                                     ([5, -1, 0, 7, 2 ** 31 - 1, -2 ** 31, 5, 3], 8), ([i * i % 11 for i in range(130)], 11)])
def test_experts_routes(fmt, route, E, tile):
    """one row, rows of no expert, experts of no rows, one expert for all, an expert a row, numbers out of range"""
    ctx = context(workloads.PRIMES[:8])
    run_experts(ctx, fmt, E, 1, route, 65, 40, len(route) + E, bias=True)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("top_k", [2, 3, 8])
def test_experts_several_rows_per_input(fmt, top_k, tile):
    ctx = context(workloads.PRIMES[:9])
    g = np.random.default_rng(top_k)
    run_experts(ctx, fmt, 5, top_k, g.integers(-1, 5, 7 * top_k).tolist(), 100, 33, top_k, bias=True)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n", [1, 2, 3, 7, 16, 17, 100])
def test_dense_without_routing(fmt, n, tile):
    """one expert, no routing: a dense layer; single rows and more than a tile of them"""
    ctx = context(workloads.PRIMES[:12])
    run_experts(ctx, fmt, 1, 1, [0] * n, 130, 70, n, bias=n % 2 == 1, garble=n % 3 == 0, routed=False)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows,E,M,K", [(40, 2, 300, 200), (96, 1, 256, 320), (33, 3, 513, 129), (64, 1, 700, 64)])
def test_experts_many_tiles(fmt, rows, E, M, K, tile):
    """more rows and outputs than a tile of any kernel holds"""
    ctx = context(workloads.PRIMES[:12])
    g = np.random.default_rng(rows)
    run_experts(ctx, fmt, E, 1, g.integers(0, E, rows).tolist(), K, M, rows, bias=rows % 2 == 0)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("k", [1, 2, 5, 7])
def test_experts_small_bases(fmt, k, tile):
    ctx = context(workloads.PRIMES[:k])
    run_experts(ctx, fmt, 2, 1, [0, 1, 1], 90, 50, 70 + k, bias=True)


@pytest.mark.parametrize("fmt", FORMATS)
def test_experts_floor_rule_and_given_lengths(fmt, tile):
    from paper_2302_06361_amd import LAMBDA_FLOOR
    run_experts(context(workloads.PRIMES[:12], rule=LAMBDA_FLOOR), fmt, 2, 1, [0, 1, 1], 90, 50, 80, bias=True)
    run_experts(context(workloads.PRIMES[:5], lam=[1, 128, 16, 17, 33]), fmt, 2, 1, [0, 1, 1] * 7, 90, 50, 81, bias=True)


@pytest.mark.parametrize("fmt", FORMATS)
def test_experts_large_primes_and_extreme_values(fmt, tile):
    """primes up to 127; weights of -128 on labels of p - 1; reductions whose sums pass 2^24"""
    ctx = context(P127)
    run_experts(ctx, fmt, 2, 1, [0, 1, -1, 1], 700, 33, 90, bias=True)
    run_experts(ctx, fmt, 1, 1, [0], 5000, 33, 91, bias=True, top=True, routed=False)
    run_experts(context(workloads.PRIMES[:12]), fmt, 1, 1, [0] * 3, 13000, 5, 92, routed=False, top=True)


@pytest.mark.parametrize("fmt", FORMATS)
def test_experts_long_reductions(fmt, tile):
    """more than a thousand stages, an odd end"""
    ctx = context(workloads.PRIMES[:8])
    run_experts(ctx, fmt, 1, 1, [0, 0], 70001, 5, 99, routed=False)
    run_experts(ctx, fmt, 2, 1, [1], 9000, 130, 100, bias=True)


@pytest.mark.parametrize("fmt", FORMATS)
def test_experts_many_rows_and_many_experts(fmt, tile):
    """more experts than rows; more tiles of rows than blocks on the device; rows of no expert among them"""
    ctx = context(workloads.PRIMES[:8])
    g = np.random.default_rng(11)
    run_experts(ctx, fmt, 700, 1, g.integers(0, 700, 60).tolist(), 20, 9, 101)
    run_experts(ctx, fmt, 7, 1, g.integers(-1, 7, 4000).tolist(), 8, 3, 102, bias=True)
    run_experts(ctx, fmt, 1, 1, [0] * 3000, 70, 2, 103, routed=False)


@pytest.mark.parametrize("fmt", FORMATS)
def test_experts_one_output_bundle_for_two_contexts_in_turn(fmt):
    """calls of different sizes one after the other leave nothing behind for the next"""
    a, b = context(workloads.PRIMES[:12]), context(workloads.PRIMES[:5])
    for i, (K, M) in enumerate(((300, 260), (33, 5), (64, 129), (1, 1))):
        run_experts(a, fmt, 3, 1, [i % 3, 2, 0], K, M, 104 + i)
        run_experts(b, fmt, 2, 2, [1, 0], K, M, 110 + i, bias=True)


def test_mx4_shifts_over_their_whole_range(tile):
    ctx = context(workloads.PRIMES[:12])
    run_experts(ctx, "mx4", 2, 1, [0, 1, 1, 0], 512, 64, 93, max_shift=236)
    run_experts(context(P127), "mx4", 2, 1, [0, 1, 1, 0], 300, 64, 94, max_shift=236)


@pytest.mark.parametrize("fmt", FORMATS)
def test_experts_slices_of_longer_bundles(fmt, tile):
    """bundles whose chunks lie further apart than their elements: nothing around the output is touched"""
    ctx = context(workloads.PRIMES[:8])
    run_experts(ctx, fmt, 3, 1, [2, 0, 2, 1, 2], 100, 37, 95, pad=(5, 3))
    run_experts(ctx, fmt, 1, 1, [0] * 20, 64, 260, 96, pad=(1, 0), routed=False)


@pytest.mark.parametrize("fmt", FORMATS)
def test_experts_offsets_past_32_bits(fmt, tile):
    """chunks 640 MB apart: the last chunk of the two-digit residue starts past 4 GB"""
    ctx = context([2, 3])
    run_experts(ctx, fmt, 2, 1, [1, 0, -1], 70, 40, 97, pad=(40_000_000, 0))


@pytest.mark.parametrize("fmt", FORMATS)
def test_experts_on_another_stream(fmt, tile):
    ctx = context(workloads.PRIMES[:8])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run_experts(ctx, fmt, 3, 2, [2, 0, 2, 1, 2, 1], 100, 37, 98, bias=True)


def test_layers_in_a_graph():
    """routing, both products and the weighted sum captured once; every replay on new inputs equals the eager calls"""
    from paper_2302_06361_amd import COMBINE, EXPERTS, Labels, Layer
    ctx = context(workloads.PRIMES[:8])
    g = np.random.default_rng(5)
    E, T, k, K, M = 5, 6, 2, 64, 48
    W1, _ = weights(g, ctx, "mx4", E, M, K)
    W2, _ = weights(g, ctx, "w8", E, K, M)
    ids = torch.zeros(T * k, dtype=torch.int32, device=ctx.device)
    gates = torch.zeros(T, k, dtype=torch.int32, device=ctx.device)
    src, mid, out, res = Labels(ctx, T * K), Labels(ctx, T * k * M), Labels(ctx, T * k * K), Labels(ctx, T * K)
    R = ctx.route(ids, E)
    l1 = Layer(EXPERTS, 1, T * k, top_k=k, weights=W1, routing=R)
    l2 = Layer(EXPERTS, 2, T * k, top_k=1, weights=W2, routing=R)
    l3 = Layer(COMBINE, 3, T, in_c=K, top_k=k, gates=gates)

    def step():
        ctx.route(ids, E, out=R)
        ctx.eval_layer(l1, src, None, mid)
        ctx.eval_layer(l2, mid, None, out)
        ctx.eval_layer(l3, out, None, res)

    def fill(seed):
        h = np.random.default_rng(seed)
        ids.copy_(torch.from_numpy(h.integers(-1, E, T * k).astype(np.int32)))
        gates.copy_(torch.from_numpy(h.integers(-9, 9, (T, k)).astype(np.int32)))
        for i, a in enumerate(draw_labels(h, ctx, T * K)):
            src.from_numpy(i, a)
    fill(0)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(4):
        fill(seed)
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in res.tensors]
        for t in res.tensors + out.tensors + mid.tensors:
            t.fill_(0x77)
        graph.replay()
        torch.cuda.synchronize()
        for i in range(ctx.k):
            assert torch.equal(res.tensors[i], want[i]), (seed, i)


# ---- routing ----
@pytest.mark.parametrize("n,E", [(0, 1), (1, 1), (1, 300), (63, 4), (64, 4), (65, 4), (1000, 7), (5000, 1), (777, 1025)])
def test_route(n, E):
    ctx = context(workloads.PRIMES[:3])
    ids = np.random.default_rng(n + E).integers(-2, E + 2, n).astype(np.int32)
    R = ctx.route(torch.from_numpy(ids).to(ctx.device), E)
    assert (R.c.n, R.c.n_experts) == (n, E)
    key = np.where((ids < 0) | (ids >= E), E, ids)
    raw = R.data.cpu().numpy()
    offsets = raw[:4 * (E + 2)].view(np.int32)
    assert (offsets == np.concatenate([[0], np.cumsum(np.bincount(key, minlength=E + 1))])).all()
    at = (4 * (E + 2) + 63) // 64 * 64
    assert (raw[at:at + 4 * n].view(np.int32) == np.argsort(key, kind="stable")).all()


# ---- quantisation ----
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def run_quantise(w, base, max_shift):
    """w: tensor [E][M][K] on the device; codes, shifts and values against the reference"""
    ctx = context(workloads.PRIMES[:3])
    E, M, K = w.shape
    values = torch.full((E, M, K), 77.0, dtype=w.dtype, device=w.device)
    W = ctx.mx4_quantise(w, base, max_shift, values=values)
    W2 = ctx.mx4_quantise(w, base, max_shift)
    torch.cuda.synchronize()
    codes, shifts, vals = ref.quantise(w.double().cpu().numpy(), base, max_shift)
    got_codes, got_shifts, rest = ref.mx4_unpack(W.data.cpu().numpy(), E, M, K)
    assert (got_shifts == shifts).all()
    assert (got_codes == codes).all()
    assert rest, "codes past the matrix are not zero"
    # the values are exact in their type (two significant bits), but for float16 outside its range
    want = torch.from_numpy(vals).to(w.dtype)
    assert torch.equal(values.cpu(), want)
    assert torch.equal(W.data, W2.data)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 1, 31), (2, 3, 32), (1, 33, 33), (3, 5, 64), (1, 32, 65), (2, 31, 130), (1, 70, 257)])
def test_quantise_shapes(dtype, shape):
    g = torch.Generator().manual_seed(shape[2])
    w = torch.randn(shape, generator=g) * torch.exp2(3 * torch.randn(shape[0], shape[1], 1, generator=g) - 4)
    run_quantise(w.to(DTYPES[dtype]).cuda(), -8, 12)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("cut", [(0, 64), (1, 65), (3, 100), (8, 72), (0, 97)])
def test_quantise_strided(dtype, cut):
    """columns of a wider matrix, every other matrix"""
    g = torch.Generator().manual_seed(3)
    w = torch.randn(6, 40, 113, generator=g).to(DTYPES[dtype]).cuda()[::2, :, cut[0]:cut[1]]
    run_quantise(w, -6, 8)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_quantise_ties_and_steps(dtype):
    """every multiple of 1/16 up to 8 and both neighbours of it, at several exponents: all ties of the grid"""
    a = torch.arange(-128, 129, dtype=torch.float32) / 16
    w = torch.cat([a, torch.nextafter(a, torch.tensor(9.0)), torch.nextafter(a, torch.tensor(-9.0))])
    w = torch.stack([w * 2.0 ** e for e in (-7, -3, 0, 2)])[None]
    lead = torch.full((1, 4, 1), 0.0)
    for e, r in zip((-7, -3, 0, 2), range(4)):
        lead[0, r, 0] = 4.0 * 2.0 ** e
    blocks = [torch.cat([lead, w[:, :, i:i + 31]], 2) for i in range(0, w.shape[2] - 31, 31)]     # every block holds a 4: shared exponent 0
    run_quantise(torch.cat(blocks, 2).to(DTYPES[dtype]).cuda(), -7, 255)


def test_quantise_special_values():
    """zeros, signed zeros, NaN, infinities, subnormal numbers, the largest and the smallest; exponents clipped at both ends"""
    inf, nan = float("inf"), float("nan")
    rows = [[0.0] * 40, [-0.0, 1e-45, -1e-45] + [0.0] * 37, [nan] * 40, [nan, 1.0, -3.0] + [0.5] * 37, [inf, 1e30, -inf] + [1.0] * 37,
            [3.4e38, -3.4e38] + [1e38] * 38, [1e-38, 2e-38, -1.2e-38] + [1e-39] * 37, [2.0 ** -126] * 20 + [2.0 ** 127] * 20]
    w = torch.tensor(rows, dtype=torch.float32)[None].cuda()
    for base, max_shift in ((-126, 255), (-126, 0), (0, 0), (125, 255), (-20, 30)):
        run_quantise(w, base, max_shift)
    run_quantise(torch.tensor([[[65504.0, -65504.0, 6e-8, inf, nan] + [1.0] * 30]], dtype=torch.float16, device="cuda"), -24, 30)


def test_weights8_tiles():
    ctx = context(workloads.PRIMES[:3])
    for E, M, K in ((1, 1, 1), (2, 33, 65), (3, 70, 130)):
        w = torch.randint(-128, 128, (E + 1, M, K + 3), dtype=torch.int8, device=ctx.device)[1:, :, 2:K + 2]
        full = ref.w8_unpack(ctx.weights8_prepare(w).data.cpu().numpy(), E, M, K)
        assert (full[:, :M, :K] == w.cpu().numpy()).all()
        full[:, :M, :K] = 0
        assert not full.any()


# ---- weighted sums ----
@pytest.mark.parametrize("T,top_k,V", [(1, 1, 1), (1, 2, 84), (3, 1, 65), (5, 3, 33), (2, 8, 100), (1, 9, 257), (70, 4, 5), (2, 100, 7)])
def test_combine(T, top_k, V):
    from paper_2302_06361_amd import COMBINE, Labels, Layer
    for primes in (workloads.PRIMES[:12], P127):
        ctx = context(primes)
        g = np.random.default_rng(T * 100 + top_k + V)
        gates = g.integers(-2 ** 31, 2 ** 31, (T, top_k)).astype(np.int32)
        gates.flat[0] = -2 ** 31
        for top in (False, True):
            x = draw_labels(g, ctx, T * top_k * V, top)
            if top:
                gates = np.full((T, top_k), -1, np.int32)
            src, pad = upload(ctx, x, (2, 1)), (3, 2)
            whole = Labels(ctx, T * V + sum(pad))
            for t in whole.tensors:
                t.fill_(0xA5)
            dst = whole.slice(pad[0], pad[0] + T * V)
            ctx.garble_layer(Layer(COMBINE, 1, T, in_c=V, top_k=top_k, gates=torch.from_numpy(gates).to(ctx.device)), src, dst)
            torch.cuda.synchronize()
            for i, p in enumerate(ctx.primes):
                want = ref.combine(x[i].reshape(T, top_k, V, -1), gates, p).reshape(T * V, -1)
                assert (dst.to_numpy(i) == want).all(), (p, top)
                assert dst.pad_is_zero(i)
                assert (whole.tensors[i][:, :pad[0]] == 0xA5).all() and (whole.tensors[i][:, pad[0] + T * V:] == 0xA5).all()


def test_combine_offsets_past_32_bits():
    from paper_2302_06361_amd import COMBINE, Layer
    ctx = context([2, 3])
    g = np.random.default_rng(8)
    x = draw_labels(g, ctx, 2 * 2 * 30)
    src = upload(ctx, x, (40_000_000, 0))
    dst = upload(ctx, draw_labels(g, ctx, 2 * 30), (40_000_000, 0))
    gates = np.array([[1, -5], [0, 3]], np.int32)
    ctx.eval_layer(Layer(COMBINE, 1, 2, in_c=30, top_k=2, gates=torch.from_numpy(gates).to(ctx.device)), src, None, dst)
    torch.cuda.synchronize()
    for i, p in enumerate(ctx.primes):
        assert (dst.to_numpy(i) == ref.combine(x[i].reshape(2, 2, 30, -1), gates, p).reshape(60, -1)).all()


# ---- whole network ----
@pytest.mark.parametrize("mx4", [True, False])
def test_mixture_network(mx4):
    """Gb, En, Ev, De of a mixture of experts: decoded outputs equal the plain integers; whole batch and batch chunks, one process"""
    from paper_2302_06361_amd import Context, GarbledNetwork, StreamedNetwork
    net = workloads.mixture(mx4=mx4)
    batch = net["batch"]
    want = plain(net)
    ctx = Context(net["primes"], net["seed"], net["digits"])
    gn = GarbledNetwork(ctx, net)
    gn.garble()
    gn.encode(torch.as_tensor(net["x"]).to(ctx.device))
    gn.evaluate()
    values, valid = gn.decode()
    assert valid.all() and (values.cpu().numpy() == want).all()
    n_in, n_out = net["n_in"], gn.n_out
    sn = StreamedNetwork(ctx, net, batch=2)
    for base in range(0, batch, 2):
        sn.batch_base = base
        sn.rebase()
        v, ok = sn.run(torch.as_tensor(net["x"][base * n_in:(base + 2) * n_in]).to(ctx.device))
        assert ok.all() and (v.cpu().numpy() == want[base * n_out:(base + 2) * n_out]).all(), base


def plain(net):
    """the network on integers"""
    P, batch = int(np.prod(np.array(net["primes"], object))), net["batch"]
    x = net["x"].astype(object).reshape(batch, -1)
    for L in net["layers"]:
        if L["kind"] == "conv":
            x = x @ L["W"].reshape(L["out_c"], -1).T.astype(object)
        elif L["kind"] == "relu":
            x = np.where(x > 0, x, 0)
        elif L["kind"] == "scale":
            for _ in range(L["repeat"]):
                x = -(-x // 2)                                 # each halving rounds up
        elif L["kind"] == "experts":
            if L.get("base") is None:
                W = L["W"].astype(object)
            else:
                codes, shifts, _ = ref.quantise(L["W"].astype(np.float64), L["base"], L["max_shift"])
                W = ref.mx4_integers(codes, shifts)
            x = x.reshape(batch * L["rows"] // L["top_k"], -1)
            rows = []
            for r, e in enumerate(L["route"]):
                y = np.zeros(W.shape[1], object)
                if e >= 0:
                    y = W[e] @ x[r // L["top_k"]] + (L["bias"][e].astype(object) if L.get("bias") is not None else 0)
                rows.append(y)
            x = np.array(rows, object).reshape(batch, -1)
        elif L["kind"] == "combine":
            x = (x.reshape(batch, L["top_k"], L["V"]) * L["gates"].astype(object)[:, :, None]).sum(1)
        assert np.abs(x).max() < P // 2, "the workload leaves the range of its primes"
    return x.reshape(-1).astype(np.int64)


# ---- refusals ----
def test_refusals():
    from paper_2302_06361_amd import COMBINE, EXPERTS, DashError, ExpertWeights, Labels, Layer, W8, MX4
    ctx, other = context(workloads.PRIMES[:3]), context(workloads.PRIMES[:3])
    dev = ctx.device
    w = torch.zeros(2, 8, 40, dtype=torch.int8, device=dev)
    W = ctx.weights8_prepare(w)
    ids = torch.zeros(4, dtype=torch.int32, device=dev)
    R = ctx.route(ids, 2)
    x, y = Labels(ctx, 4 * 40, zero=True), Labels(ctx, 4 * 8, zero=True)

    def refused(lay, i=x, o=y, what="bad argument|invalid|inconsistent|size not supported"):
        with pytest.raises(DashError):
            ctx.eval_layer(lay, i, None, o)
    ok = Layer(EXPERTS, 1, 4, top_k=1, weights=W, routing=R)
    ctx.eval_layer(ok, x, None, y)
    refused(Layer(EXPERTS, 1, 4, top_k=1, weights=W))                                   # two experts, no routing
    refused(Layer(EXPERTS, 1, 3, top_k=1, weights=W, routing=R))                        # rows are not the routing's
    refused(Layer(EXPERTS, 1, 4, top_k=0, weights=W, routing=R))
    refused(Layer(EXPERTS, 1, 4, top_k=3, weights=W, routing=R))                        # 4 rows are not a multiple of 3
    refused(Layer(EXPERTS, 1, 4, top_k=1, weights=W, routing=ctx.route(ids, 3)))        # another number of experts
    refused(Layer(EXPERTS, 1, 4, top_k=1, weights=W, routing=other.route(ids, 2)))      # a routing of another context
    bad = Layer(EXPERTS, 1, 4, top_k=1, weights=W, routing=R)
    bad.c.weight_format = 2
    refused(bad)
    bad = Layer(EXPERTS, 1, 4, top_k=1, weights=W, routing=R)
    bad.c.weights += 8                                                                  # not 16-byte aligned
    refused(bad)
    bad = Layer(EXPERTS, 1, 4, top_k=1, weights=W, routing=R)
    bad.c.weights = 0
    refused(bad)
    refused(ok, Labels(ctx, 4 * 40 - 1), y)                                             # bundles too short
    refused(ok, x, Labels(ctx, 4 * 8 - 1))
    refused(ok, Labels(ctx, 4 * 40, only=(0, 1)), y)                                    # a residue is missing
    with pytest.raises(DashError):                                                      # sums would pass 32 bits
        big = context([2, 127])
        huge = ExpertWeights(big, W8, 1, 1, 70000)
        big.eval_layer(Layer(EXPERTS, 1, 1, top_k=1, weights=huge), Labels(big, 70000), None, Labels(big, 1))
    gates = torch.zeros(2, 2, dtype=torch.int32, device=dev)
    ctx.eval_layer(Layer(COMBINE, 1, 2, in_c=8, top_k=2, gates=gates), y, None, Labels(ctx, 16))
    refused(Layer(COMBINE, 1, 2, in_c=8, top_k=2), y, Labels(ctx, 16))                  # no gates
    refused(Layer(COMBINE, 1, 2, in_c=8, top_k=0, gates=gates), y, Labels(ctx, 16))
    refused(Layer(COMBINE, 1, 2, in_c=0, top_k=2, gates=gates), y, Labels(ctx, 16))
    refused(Layer(COMBINE, 1, 2, in_c=8, top_k=2, gates=gates), y, Labels(ctx, 15))
    refused(Layer(COMBINE, 1, 2, in_c=9, top_k=2, gates=gates), y, Labels(ctx, 18))
    refused(Layer(COMBINE, 1, 1, in_c=1, top_k=1025, gates=gates), Labels(ctx, 1025), Labels(ctx, 1))
    f = torch.zeros(2, 8, 40, device=dev)
    for bad in (dict(base=-127), dict(base=126), dict(base=0, max_shift=-1), dict(base=0, max_shift=256)):
        with pytest.raises(DashError):
            ctx.mx4_quantise(f, **bad)
    for bad in (f.double(), f.cpu(), f.transpose(1, 2), f[:, :0], f[0, 0]):
        with pytest.raises(DashError):
            ctx.mx4_quantise(bad, 0)
    with pytest.raises(DashError):
        ctx.mx4_quantise(f, 0, values=f.half())
    with pytest.raises(DashError):
        ctx.mx4_quantise(f, 0, out=W)
    with pytest.raises(DashError):
        ctx.weights8_prepare(f)
    with pytest.raises(DashError):
        ctx.weights8_prepare(w[:, :4], out=W)
    with pytest.raises(DashError):
        ExpertWeights(ctx, 5, 1, 1, 1)
    with pytest.raises(DashError):
        ctx.route(ids.long(), 2)
    with pytest.raises(DashError):
        ctx.route(ids, 0)
    with pytest.raises(DashError):
        ctx.route(torch.zeros(400, dtype=torch.int32, device=dev), 2, out=R)
    # no rows: nothing to do
    ctx.eval_layer(Layer(EXPERTS, 1, 0, top_k=1, weights=W, routing=ctx.route(ids[:0], 2)), x, None, y)
    ctx.eval_layer(Layer(COMBINE, 1, 0, in_c=8, top_k=2, gates=gates), x, None, y)
    torch.cuda.synchronize()
