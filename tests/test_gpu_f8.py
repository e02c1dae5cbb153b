"""GPU parity: expert layers with 8-bit floating point weights (e4m3, an integer scale for every 128 x 128) through the C ABI against plain
64-bit references.  Codes, scales and labels are integers and have to be equal; values are products of 4 and 15 significant bits, rounded once."""
import numpy as np
import pytest
import torch

import experts_ref as ref
import f8_ref
import workloads
from test_gpu_experts import P127, context, draw_labels, upload

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def run_f8(ctx, E, top_k, route, K, M, seed, bias=False, garble=False, pad=(0, 0), routed=True, top=False, scales=255):
    from paper_2302_06361_amd import EXPERTS, Labels, Layer
    g = np.random.default_rng(seed)
    n = len(route)
    x = draw_labels(g, ctx, n // top_k * K, top)
    codes = g.integers(0, 256, (E, M, K))
    S = g.integers(0, scales + 1, (E, f8_ref.blocks(M), f8_ref.blocks(K))) if scales >= 0 else g.integers(-2 ** 31, 2 ** 31, (E, f8_ref.blocks(M), f8_ref.blocks(K)))
    W = ctx.f8_prepare(torch.from_numpy(codes.astype(np.uint8)).to(ctx.device), torch.from_numpy(S.astype(np.int32)).to(ctx.device))
    ints = f8_ref.integers(codes, S)
    b = g.integers(-2 ** 31, 2 ** 31, (E, M)).astype(np.int32) if bias else None
    R = ctx.route(torch.tensor(route, dtype=torch.int32, device=ctx.device), E) if routed else None
    lay = Layer(EXPERTS, 3, n, top_k=top_k, weights=W, routing=R, bias=torch.from_numpy(b).to(ctx.device) if bias else None)
    assert ctx.layer_sizes(lay)[:2] == (M, 0)
    src = upload(ctx, x, pad)
    whole = Labels(ctx, n * M + sum(pad))
    for t in whole.tensors:
        t.fill_(0xA5)
    dst = whole.slice(pad[0], pad[0] + n * M)
    (ctx.garble_layer if garble else lambda l, i, o: ctx.eval_layer(l, i, None, o))(lay, src, dst)
    torch.cuda.synchronize()
    for i, p in enumerate(ctx.primes):
        lam = ctx.lam(p)
        want = ref.experts(x[i].reshape(n // top_k, K, lam), ints, route, top_k, p, b, ctx.one(i, 0 if garble else 1)).reshape(n * M, lam)
        got = dst.to_numpy(i)
        bad = np.argwhere(got != want)
        assert bad.size == 0, "p = %d: %d of %d digits differ, first at %s (row %d, output %d)" % (p, len(bad), got.size, bad[0], bad[0][0] // M, bad[0][0] % M)
        assert dst.pad_is_zero(i)
        if sum(pad):
            t = whole.tensors[i]
            assert (t[:, :pad[0]] == 0xA5).all() and (t[:, pad[0] + n * M:] == 0xA5).all(), "bytes around the output were written"


# ---- weights ----
def check_quantised(ctx, w, base, max_scale, dtype, pad=0):
    """w float64 [E][M][K], rounded to the type first; a slice of a wider tensor if pad"""
    t = torch.from_numpy(w).to(TYPES[dtype])
    E, M, K = w.shape
    wide = torch.full((E, M + (1 if pad else 0), K + pad), 77.0, dtype=TYPES[dtype])
    wide[:, :M, :K] = t
    wide = wide.to(ctx.device)
    values = torch.full((E, M, K), 55.0, dtype=TYPES[dtype], device=ctx.device)
    W = ctx.f8_quantise(wide[:, :M, :K], base, max_scale, values=values)
    torch.cuda.synchronize()
    codes, S, v = f8_ref.quantise(t.double().numpy(), base, max_scale)
    got, scales, rest = f8_ref.unpack(W.data.cpu().numpy(), E, M, K)
    assert (scales == S).all(), np.argwhere(scales != S)[:4]
    assert (got == codes).all(), (np.argwhere(got != codes)[:4], got[got != codes][:4], codes[got != codes][:4])
    assert rest, "codes past the end of the matrix"
    want = torch.from_numpy(v).to(TYPES[dtype])
    assert torch.equal(values.cpu(), want)
    again = ctx.f8_quantise(wide[:, :M, :K], base, max_scale)
    torch.cuda.synchronize()
    got, scales, _ = f8_ref.unpack(again.data.cpu().numpy(), E, M, K)
    assert (got == codes).all() and (scales == S).all()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("E,M,K", [(1, 1, 1), (1, 10, 128), (2, 31, 33), (1, 32, 64), (3, 127, 129), (1, 128, 128), (2, 129, 127), (1, 300, 65), (1, 5, 1030), (2, 257, 260)])
def test_quantise_sizes(dtype, E, M, K):
    g = np.random.default_rng(E * 7 + M + K)
    ctx = context(workloads.PRIMES[:8])
    w = g.standard_normal((E, M, K)) * np.exp2(2 * g.standard_normal((E, M, 1)) - 5)
    for pad in (0, 3):
        check_quantised(ctx, w, -14, 255, dtype, pad)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("base,max_scale", [(-18, 1), (-18, 32767), (-8, 255), (-64, 255), (64, 32767), (0, 1)])
def test_quantise_ranges(dtype, base, max_scale):
    g = np.random.default_rng(100 + base + max_scale)
    ctx = context(workloads.PRIMES[:8])
    check_quantised(ctx, g.standard_normal((2, 70, 300)) * np.exp2(3 * g.standard_normal((2, 70, 1))), base, max_scale, dtype)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_quantise_borders(dtype):
    """the middle of every two values and its neighbours in the type, under scales that are no powers of two"""
    ctx = context(workloads.PRIMES[:8])
    mid = np.concatenate([(f8_ref.E4M3[1:] + f8_ref.E4M3[:-1]) / 2, f8_ref.E4M3])
    w = np.zeros((4, 128, 512))
    for e, S in enumerate((1, 3, 7, 11)):
        v = torch.from_numpy(np.concatenate([mid, -mid]) * S).to(TYPES[dtype])
        up, down = torch.nextafter(v, torch.full_like(v, 1e4)), torch.nextafter(v, torch.full_like(v, -1e4))
        row = np.clip(torch.cat([v, up, down]).double().numpy(), -448 * S, 448 * S)
        for b in range(4):
            part = np.resize(np.roll(row, 100 * b), 127 * 128)
            w[e, 1:, 128 * b:128 * b + 128] = part.reshape(127, 128)
            w[e, 0, 128 * b] = 448 * S
    codes, S, _ = f8_ref.quantise(torch.from_numpy(w).to(TYPES[dtype]).double().numpy(), 0, 255)
    assert sorted(set(S.reshape(-1))) == [1, 3, 7, 11]
    check_quantised(ctx, w, 0, 255, dtype)


def test_quantise_scales_at_their_steps():
    """largest magnitudes at, just below and just above 448 S 2^base, S over its whole range"""
    ctx = context(workloads.PRIMES[:8])
    S = np.array([1, 2, 3, 5, 17, 255, 256, 1000, 4095, 16383, 32766, 32767], np.float32)
    for base in (-14, 0, 9):
        a = (448 * S * np.float32(2.0 ** base)).astype(np.float32)
        tops = np.concatenate([a, np.nextafter(a, np.float32(0)), np.nextafter(a, np.float32(np.inf))])
        w = np.zeros((len(tops), 3, 5))
        w[:, 1, 2] = tops
        w[:, 2, 4] = tops / 3
        check_quantised(ctx, w, base, 32767, "f32")


@pytest.mark.parametrize("dtype", list(TYPES))
def test_quantise_what_is_no_number(dtype):
    """NaN as 0, infinities as the largest float32, zeros without a sign, a block of zeros, subnormal numbers"""
    ctx = context(workloads.PRIMES[:8])
    g = np.random.default_rng(5)
    w = g.standard_normal((1, 200, 300))
    w[0, 3, 4] = np.nan
    w[0, 3, 5] = -0.0
    w[0, 150, 10] = np.inf
    w[0, 150, 200] = -np.inf
    w[0, :128, 256:] = 0
    w[0, 128:, 256:] = 1e-42
    w[0, 130, 290] = np.nan
    check_quantised(ctx, w, -10, 255, dtype)
    check_quantised(ctx, np.full((1, 3, 3), np.nan), -10, 255, dtype)
    check_quantised(ctx, np.full((1, 3, 3), -1e-30), 64, 255, dtype)


@pytest.mark.parametrize("E,M,K,pad", [(1, 1, 1, 0), (2, 33, 65, 5), (3, 129, 257, 0), (1, 128, 128, 1), (2, 100, 1030, 2)])
def test_prepare(E, M, K, pad):
    """codes stay as they are, those of no number become zeros; rows at any address"""
    ctx = context(workloads.PRIMES[:8])
    g = np.random.default_rng(M + K)
    codes = g.integers(0, 256, (E, M, K + pad)).astype(np.uint8)
    S = g.integers(-2 ** 31, 2 ** 31, (E, f8_ref.blocks(M), f8_ref.blocks(K))).astype(np.int32)
    t = torch.from_numpy(codes).to(ctx.device)[:, :, pad:]
    W = ctx.f8_prepare(t.view(torch.float8_e4m3fn) if pad == 0 else t, torch.from_numpy(S).to(ctx.device))
    torch.cuda.synchronize()
    got, scales, rest = f8_ref.unpack(W.data.cpu().numpy(), E, M, K)
    want = np.where(codes & 127 == 127, 0, codes)[:, :, pad:]
    assert (got == want).all() and (scales == S).all() and rest


# ---- products ----
@pytest.fixture(params=["rule", "big", "narrow", "few", "wide", "class", "small"])
def tile(request, monkeypatch):
    """the tile that the layer's sizes ask for, and each tile forced"""
    monkeypatch.setenv("DASH_EXPERTS_TILE", request.param)


@pytest.mark.parametrize("K", [1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 191, 192, 193, 255, 256, 257, 400, 640])
def test_reduction_lengths(K, tile):
    """stages of 64, scales of 128, slots in turn"""
    run_f8(context(workloads.PRIMES[:8]), 3, 1, [2, 0, 2, 1, 2], K, 37, K, bias=K % 2 == 0, garble=K % 3 == 0)


@pytest.mark.parametrize("M", [1, 2, 31, 32, 33, 64, 127, 128, 129, 255, 256, 257, 400])
def test_output_counts(M, tile):
    run_f8(context(workloads.PRIMES[:12]), 2, 1, [1, 0, 1], 150, M, M, bias=M % 2 == 1, garble=M % 3 == 0)


@pytest.mark.parametrize("route,E", [([0], 1), ([-1], 1), ([4], 7), ([-1, -1, -1], 2), ([0] * 9, 3), ([2] * 65, 3), (list(range(40)), 40),
                                     ([5, -1, 0, 7, 2 ** 31 - 1, -2 ** 31, 5, 3], 8), ([i * i % 11 for i in range(130)], 11)])
def test_routes(route, E, tile):
    run_f8(context(workloads.PRIMES[:8]), E, 1, route, 65, 40, len(route) + E, bias=True)


@pytest.mark.parametrize("top_k", [2, 3, 8])
def test_several_rows_per_input(top_k, tile):
    g = np.random.default_rng(top_k)
    run_f8(context(workloads.PRIMES[:9]), 5, top_k, g.integers(-1, 5, 7 * top_k).tolist(), 140, 133, top_k, bias=True)


@pytest.mark.parametrize("n", [1, 2, 3, 7, 16, 17, 33, 100])
def test_dense_without_routing(n, tile):
    run_f8(context(workloads.PRIMES[:12]), 1, 1, [0] * n, 200, 150, n, bias=n % 2 == 1, garble=n % 3 == 0, routed=False)


@pytest.mark.parametrize("rows,E,M,K", [(40, 2, 300, 200), (96, 1, 256, 320), (33, 3, 513, 129), (64, 1, 700, 64), (300, 1, 260, 300)])
def test_many_tiles(rows, E, M, K, tile):
    g = np.random.default_rng(rows)
    run_f8(context(workloads.PRIMES[:12]), E, 1, g.integers(0, E, rows).tolist(), K, M, rows, bias=rows % 2 == 0)


@pytest.mark.parametrize("k", [1, 2, 5, 7])
def test_small_bases(k, tile):
    run_f8(context(workloads.PRIMES[:k]), 2, 1, [0, 1, 1], 190, 50, 70 + k, bias=True)


def test_floor_rule_and_given_lengths(tile):
    from paper_2302_06361_amd import LAMBDA_FLOOR
    run_f8(context(workloads.PRIMES[:12], rule=LAMBDA_FLOOR), 2, 1, [0, 1, 1], 190, 50, 80, bias=True)
    run_f8(context(workloads.PRIMES[:5], lam=[1, 128, 16, 17, 33]), 2, 1, [0, 1, 1] * 7, 190, 50, 81, bias=True)


def test_scales_of_any_value(tile):
    """the whole range of 32 bits, multiples of the primes and zero among them, and 1"""
    run_f8(context(workloads.PRIMES[:12]), 2, 1, [0, 1, 1], 700, 300, 82, bias=True, scales=-1)
    run_f8(context(workloads.PRIMES[:12]), 2, 1, [0, 1, 1], 700, 300, 83, scales=0)
    run_f8(context(P127), 2, 1, [0, 1, -1, 1], 700, 140, 84, bias=True, scales=-1)


def test_large_primes_and_extreme_values(tile):
    """primes up to 127, labels of p - 1; reductions whose sums pass 2^24"""
    run_f8(context(P127), 1, 1, [0], 5000, 33, 91, bias=True, top=True, routed=False)
    run_f8(context(workloads.PRIMES[:12]), 1, 1, [0] * 3, 13000, 5, 92, routed=False, top=True)


def test_long_reductions(tile):
    run_f8(context(workloads.PRIMES[:8]), 1, 1, [0, 0], 30001, 5, 99, routed=False)
    run_f8(context(workloads.PRIMES[:8]), 2, 1, [1], 9000, 130, 100, bias=True)


def test_many_rows_and_many_experts(tile):
    ctx = context(workloads.PRIMES[:8])
    g = np.random.default_rng(11)
    run_f8(ctx, 300, 1, g.integers(0, 300, 60).tolist(), 20, 9, 101)
    run_f8(ctx, 7, 1, g.integers(-1, 7, 4000).tolist(), 8, 3, 102, bias=True)
    run_f8(ctx, 1, 1, [0] * 3000, 70, 2, 103, routed=False)


def test_slices_of_longer_bundles(tile):
    ctx = context(workloads.PRIMES[:8])
    run_f8(ctx, 3, 1, [2, 0, 2, 1, 2], 200, 37, 95, pad=(5, 3))
    run_f8(ctx, 1, 1, [0] * 20, 64, 260, 96, pad=(1, 0), routed=False)


def test_one_output_bundle_for_two_contexts_in_turn():
    """calls of different sizes one after the other leave nothing behind for the next"""
    a, b = context(workloads.PRIMES[:12]), context(workloads.PRIMES[:5])
    for i, (K, M) in enumerate(((300, 260), (33, 5), (64, 129), (1, 1))):
        run_f8(a, 3, 1, [i % 3, 2, 0], K, M, 104 + i)
        run_f8(b, 2, 2, [1, 0], K, M, 110 + i, bias=True)
