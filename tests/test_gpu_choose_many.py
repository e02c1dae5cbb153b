"""GPU: choices of more rows than the blocks of one launch hold (2^24 - 1 blocks of 256 threads, 16, 32 or 64 of them a row).  All logits are zero but around the border between launches and
at the ends, so that the choice of every row is at hand: expert 0, or the largest of a row that was drawn."""
import pytest
import torch

import workloads
from test_gpu_experts import context
from test_gpu_experts_edges import memory_goes_back, need      # noqa: F401 (a fixture among them)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lanes,E", [(16, 2), (32, 257), (64, 513)])
def test_rows_of_two_launches(lanes, E):
    from paper_2302_06361_amd import Router
    ctx = context(workloads.PRIMES[:3])
    border = (256 // lanes) * (2 ** 24 - 1)
    n = border + 1000
    need(2 * n * E + 12 * n + 2 ** 28)
    logits = torch.zeros((n, E), dtype=torch.bfloat16, device=ctx.device)
    drawn = torch.cat([torch.arange(40), torch.arange(border - 40, border + 40), torch.arange(n - 40, n)]).to(ctx.device)
    g = torch.Generator(device=ctx.device)
    g.manual_seed(lanes)
    logits[drawn] = 1 + torch.rand((len(drawn), E), device=ctx.device, generator=g).to(torch.bfloat16)
    got = ctx.choose(Router(E, 1, gate_bits=5), logits)
    torch.cuda.synchronize()
    at = torch.arange(E, device=ctx.device)
    x = logits[drawn]
    want = torch.where(x == x.amax(1, keepdim=True), at, E).amin(1)             # (the first of the largest)
    assert torch.equal(got.experts[drawn, 0], want.to(torch.int32))
    got.experts[drawn] = 0
    for first in range(0, n, 2 ** 26):
        part = slice(first, first + 2 ** 26)
        assert (got.experts[part] == 0).all() and (got.gates[part] == 32).all() and (got.weights[part] == 1).all()
