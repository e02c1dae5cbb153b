"""GPU: gates whose weight lies in the middle of two integers go to the even one.  Equal scores share as integers do, whatever the scores are: of k of them each weight is
scale / k, so that the gate follows in whole numbers (Python's fractions); there is nothing to be tolerant of."""
from fractions import Fraction

import numpy as np
import pytest
import torch

import workloads
from test_gpu_experts import context

pytestmark = pytest.mark.gpu
MIDDLES = [0.5, 1.5, 2.5, 3.5, 6.5, 1000.5, 123456.5, 2.0 ** 20 + 0.5]


@pytest.fixture(scope="module")
def ctx():
    return context(workloads.PRIMES[:8])


def gate(scale, gate_bits, shares):
    return round(Fraction(float(np.float32(scale))) * 2 ** gate_bits / shares)         # (ties to the even)


def cases(shares):
    """(scale, gate_bits) with weights in the middle of two gates, and one to either side of it by a step of the scale's float32"""
    out = []
    for h in MIDDLES:
        for bits in (0, 1, 7):
            scale = np.float32(shares * h / 2 ** bits)
            if float(scale) != shares * h / 2 ** bits or float(scale) * 2 ** bits > 2 ** 30:
                continue
            out += [(float(s), bits) for s in (scale, np.nextafter(scale, np.float32(0)), np.nextafter(scale, np.float32(np.inf)))]
    return out


def check(ctx, logits, top_k, shares, bias=None, **kw):
    """every gate of an expert is that of `shares` equal scores"""
    from paper_2302_06361_amd import Router
    for scale, bits in cases(shares):
        got = ctx.choose(Router(logits.shape[1], top_k, bias=bias, scale=scale, gate_bits=bits, **kw), logits)
        want = torch.where(got.experts >= 0, gate(scale, bits, shares), 0).to(torch.int32)
        bad = (got.gates != want).any(1).nonzero()
        assert bad.numel() == 0, (scale, bits, len(bad), got.gates[bad[0]].tolist(), want[bad[0]].tolist(), logits[bad[0], :4].tolist())
        assert (got.experts[:, :min(shares, top_k)] >= 0).all()


def rows(n, E, dtype=torch.float32, seed=0):
    """equal logits in every row, of another size in each"""
    g = np.random.default_rng(seed)
    return torch.from_numpy(4 * g.standard_normal((n, 1))).to(dtype).expand(n, E).contiguous().cuda()


@pytest.mark.parametrize("top_k", [1, 2, 3, 4, 5, 6, 7, 8, 11, 16, 17, 24, 29, 32])
@pytest.mark.parametrize("E", [32, 64, 200, 400, 1000])
def test_chosen_of_equal_scores(ctx, top_k, E):
    from paper_2302_06361_amd import SIGMOID
    check(ctx, rows(300, E, seed=top_k), top_k, top_k, score=SIGMOID)
    # softmax: beside a larger logit that a bias forbids, so that the chosen exponentials are no ones
    l, b = rows(300, E, seed=top_k + 1), torch.zeros(E, device="cuda")
    if E > top_k:
        l[:, E // 2] += torch.rand(300, device="cuda") * 5
        b[E // 2] = -np.inf
    check(ctx, l, top_k, top_k, bias=b)
    check(ctx, rows(300, E, seed=top_k + 2), top_k, top_k, bias=torch.zeros(E, device="cuda"), score=SIGMOID)


@pytest.mark.parametrize("left", [1, 2, 3, 5, 7, 8])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_few_left_by_a_mask(ctx, left, dtype):
    from paper_2302_06361_amd import SIGMOID, SOFTMAX
    l = rows(300, 60, dtype, left)
    keep = torch.zeros(300, 60, dtype=torch.bool)
    for r in range(300):
        keep[r, np.random.default_rng(r).choice(60, left, replace=False)] = True
    l[~keep.cuda()] = -np.inf
    for score in (SOFTMAX, SIGMOID):
        check(ctx, l, 8, left, score=score)


@pytest.mark.parametrize("groups,top_groups", [(8, 3), (4, 1)])
@pytest.mark.parametrize("E", [64, 256, 512])
def test_groups_of_equal_scores(ctx, E, groups, top_groups):
    from paper_2302_06361_amd import GROUP_PAIR, SIGMOID
    for top_k in (3, 6, 7):
        check(ctx, rows(65, E, seed=top_k), top_k, top_k, groups=groups, top_groups=top_groups, group_score=GROUP_PAIR, score=SIGMOID)
        check(ctx, rows(65, E, seed=top_k), top_k, top_k, groups=groups, top_groups=top_groups, group_score=GROUP_PAIR, bias=torch.zeros(E, device="cuda"))


@pytest.mark.parametrize("shares", [1, 2, 3, 5, 6, 7, 10, 49, 60, 100, 160, 250])
def test_softmax_of_equal_logits(ctx, shares):
    """not renormalised: the scores of a row of equal logits are its experts' equal shares"""
    l = rows(300, 256, seed=shares)
    l[:, shares:] = -np.inf
    check(ctx, l, 4, shares, renormalise=False)
    check(ctx, l, 4, shares, renormalise=False, bias=torch.zeros(256, device="cuda"))


def test_sigmoid_of_zero(ctx):
    """not renormalised: one half each"""
    from paper_2302_06361_amd import SIGMOID
    check(ctx, torch.zeros(7, 20, device="cuda"), 4, 2, renormalise=False, score=SIGMOID)


@pytest.mark.parametrize("x", [-1.0, -300.0, -689.0])
def test_small_scores_under_large_scales(ctx, x):
    """the smallest scores that count, whose inverses the scale would take past 64 bits"""
    from paper_2302_06361_amd import SIGMOID, Router
    l = torch.full((3, 8), x, device="cuda")
    for top_k in (1, 2, 4):
        got = ctx.choose(Router(8, top_k, score=SIGMOID, scale=2.0 ** 30, gate_bits=0), l)
        assert (got.gates == 2 ** 30 // top_k).all() and (got.weights == 2.0 ** 30 / top_k).all()


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renormalise", [False, True])
def test_gates_next_to_a_middle(ctx, sigmoid, renormalise):
    """millions of gates of 30 bits, some so near to a middle that the remainder decides (2^-18), but farther than 64 bits leave open: the sum, quotient and products of the
    reference and the scores are off by less than 2^-49 of a gate of up to 2^30, 2^-19"""
    from paper_2302_06361_amd import SIGMOID, SOFTMAX, Router
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    l = 1.5 * torch.randn((500000, 16), device="cuda", generator=g)
    got = ctx.choose(Router(16, 8, score=SIGMOID if sigmoid else SOFTMAX, renormalise=renormalise, gate_bits=30), l)
    d = l.double()
    s = 1 / (1 + torch.exp(-d)) if sigmoid else torch.exp(d - d.amax(1, keepdim=True))
    chosen = s.gather(1, got.experts.long())
    t = chosen / (chosen.sum(1, keepdim=True) if renormalise else 1 if sigmoid else s.sum(1, keepdim=True)) * 2.0 ** 30
    off = (t - t.floor() - 0.5).abs()
    assert int(((off > 2.0 ** -19) & (off < 2.0 ** -18)).sum()) >= 5
    wrong = (got.gates.double() != torch.round(t)) & (off > 2.0 ** -19)
    assert not wrong.any(), (int(wrong.sum()), t[wrong][:3].tolist())
