"""GPU: sums of products with 8-bit floats at both ends of the range that 31 bits hold: the longest reductions that the largest prime allows, labels of p - 1 and one weight all over,
whose residue is the largest modulo a prime, or the largest or smallest modulo a class of primes."""
import pytest
import torch

import f8_ref
import workloads
from test_experts_rule8 import classes
from test_gpu_experts import P127
from test_gpu_experts_edges import context, memory_goes_back      # noqa: F401 (a fixture)
from test_gpu_f8_edges import TILES

pytestmark = pytest.mark.gpu


def moduli(primes):
    out = []
    for c in classes(list(primes)):
        m = 1
        for p in c:
            m *= p
        out.append(m)
    return out


@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("primes", [P127, workloads.PRIMES[:12], [2, 127]])
@pytest.mark.parametrize("bias", [False, True])
def test_residues_of_one_sign(tile, primes, bias, monkeypatch):
    from paper_2302_06361_amd import EXPERTS, Labels, Layer
    monkeypatch.setenv("DASH_EXPERTS_TILE", tile)
    ctx = context(primes)
    K = (2 ** 31 - 1 - (max(primes) - 1)) // (256 * (max(primes) - 1))
    # code 1 is 2^-9, the integer 1: the weight is the scale; code 129 its negative
    codes = torch.tensor([1, 129], dtype=torch.uint8, device=ctx.device).view(1, 2, 1).expand(1, 2, K).contiguous()
    src, dst = Labels(ctx, K, zero=True), Labels(ctx, 2)
    for t, p in zip(src.tensors, ctx.primes):
        for ch in range(t.shape[0]):
            t[ch, :, :min(16, ctx.lam(p) - 16 * ch)] = p - 1
    b = torch.tensor([2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device=ctx.device) if bias else None
    scales = {p - 1 for p in primes} | {m // 2 for m in moduli(primes)} | {m // 2 + 1 for m in moduli(primes)} | {2 ** 31 - 1, -2 ** 31}
    for S in sorted(scales):
        W = ctx.f8_prepare(codes, torch.full((1, 1, f8_ref.blocks(K)), S, dtype=torch.int32, device=ctx.device))
        ctx.eval_layer(Layer(EXPERTS, 1, 1, top_k=1, weights=W, bias=b), src, None, dst)
        for i, p in enumerate(ctx.primes):
            got, one = dst.to_numpy(i), ctx.one(i, 1).astype(int) if bias else 0
            for j, (sign, add) in enumerate(((1, 2 ** 31 - 1), (-1, -2 ** 31))):
                assert (got[j] == (sign * S * K * (p - 1) + (add * one if bias else 0)) % p).all(), (S, p, j)
