"""Choice of experts, routing, products with 8-bit floating point weights and weighted sums together, as a network uses them: decoded outputs
equal the plain integers."""
import numpy as np
import pytest
import torch

import choose_ref
import f8_ref
import workloads
from test_gpu_experts import context, draw_labels, plain, upload
import experts_ref as ref

pytestmark = pytest.mark.gpu


def as_plain(net):
    """the same network with the experts, gates and weights that the references choose, as integers"""
    layers = []
    for L in net["layers"]:
        L = dict(L)
        if "router" in L:
            r = dict(L["router"])
            logits = r.pop("logits").astype(np.float64)
            r["sigmoid"] = bool(r.pop("score", 0))
            experts, gates, _ = choose_ref.choose(logits, **r)
            L["route"], L["gates"] = experts.reshape(-1), gates
        if L["kind"] == "experts" and "scales" in L:
            L["W"] = f8_ref.integers(L["codes"], L["scales"])
        elif L["kind"] == "experts" and "max_scale" in L:
            codes, scales, _ = f8_ref.quantise(L["W"].astype(np.float64), L["base"], L["max_scale"])
            L["W"], L["base"] = f8_ref.integers(codes, scales), None
        layers.append(L)
    return dict(net, layers=layers)


def run(net):
    from paper_2302_06361_amd import Context, GarbledNetwork, StreamedNetwork
    want, batch = plain(as_plain(net)), net["batch"]
    half = int(np.prod(np.array(net["primes"], object))) // 2
    assert max(abs(int(v)) for v in want) < half and len(set(want.tolist())) > 5
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


@pytest.mark.parametrize("router", [dict(), dict(score=1, bias=np.linspace(-0.2, 0.2, 4).astype(np.float32), scale=2.5), dict(valid=np.array([1, 0, 1, 1], np.uint8))])
def test_8_bit_floats_and_a_router(router):
    run(workloads.mixture(k=12, f8=True, router=router))


def test_8_bit_floats_without_a_router():
    run(workloads.mixture(k=12, f8=True))


def test_a_router_for_other_weights():
    run(workloads.mixture(k=12, mx4=False, router=dict()))


def test_codes_and_scales():
    net = workloads.mixture(k=12, f8=True, router=dict())
    g = np.random.default_rng(4)
    for L in net["layers"]:
        if L["kind"] == "experts":
            E, M, K = L.pop("W").shape
            L["base"] = L.pop("max_scale")
            L["codes"] = (g.integers(0, 256, (E, M, K)) & 0xBF).astype(np.uint8)           # (magnitudes below 2)
            L["scales"] = g.integers(1, 40, (E, f8_ref.blocks(M), f8_ref.blocks(K))).astype(np.int32)
            L["base"] = None
    run(net)


def test_in_a_graph():
    """logits change between replays: choice, routing, products and weighted sum follow"""
    from paper_2302_06361_amd import COMBINE, EXPERTS, Choice, Labels, Layer, Router
    ctx = context(workloads.PRIMES[:8])
    g = np.random.default_rng(6)
    T, E, K, M, k = 9, 6, 140, 70, 2
    codes, S = g.integers(0, 256, (E, M, K)), g.integers(1, 255, (E, 1, 2))
    W = ctx.f8_prepare(torch.from_numpy(codes.astype(np.uint8)).to(ctx.device), torch.from_numpy(S.astype(np.int32)).to(ctx.device))
    x = draw_labels(g, ctx, T * K)
    src, mid, dst = upload(ctx, x), Labels(ctx, T * k * M), Labels(ctx, T * M)
    logits = torch.zeros(T, E, device=ctx.device)
    router, choice = Router(E, k, gate_bits=10), Choice(ctx, T, k)
    routing = ctx.route(torch.zeros(T * k, dtype=torch.int32, device=ctx.device), E)
    products, join = Layer(EXPERTS, 1, T * k, top_k=k, weights=W, routing=routing), Layer(COMBINE, 2, T, in_c=M, top_k=k, gates=choice.gates)

    def step():
        ctx.choose(router, logits, out=choice)
        ctx.route(choice.experts, E, out=routing)
        ctx.eval_layer(products, src, None, mid)
        ctx.eval_layer(join, mid, None, dst)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    ints = f8_ref.integers(codes, S)
    for i in range(4):
        new = g.standard_normal((T, E)).astype(np.float32)
        new[i, i:] = -np.inf
        logits.copy_(torch.from_numpy(new))
        graph.replay()
        torch.cuda.synchronize()
        experts, gates, _ = choose_ref.choose(new.astype(np.float64), k, gate_bits=10)
        assert (choice.experts.cpu().numpy() == experts).all() and (choice.gates.cpu().numpy() == gates).all()
        for j, p in enumerate(ctx.primes):
            lam = ctx.lam(p)
            y = ref.experts(x[j].reshape(T, K, lam), ints, experts.reshape(-1).tolist(), k, p)
            want = ref.combine(y.reshape(T, k, M, lam), gates, p)
            assert (dst.to_numpy(j) == want.reshape(T * M, lam)).all(), (i, p)


@pytest.mark.parametrize("net", [dict(), dict(router=dict()), dict(k=12, f8=True, router=dict())])
def test_memory_goes_back_with_the_network(net):
    """at once, not with the next collection of cycles"""
    import gc
    from paper_2302_06361_amd import Context, GarbledNetwork
    net = workloads.mixture(**net)
    ctx = Context(net["primes"], net["seed"], net["digits"])
    gc.collect()
    gc.disable()
    try:
        before = torch.cuda.memory_allocated()
        gn = GarbledNetwork(ctx, net)
        assert torch.cuda.memory_allocated() > before
        del gn
        assert torch.cuda.memory_allocated() == before
    finally:
        gc.enable()
