"""GPU: quantisation of the longest rows that 32-bit sizes name.  Blocks do not see each other, so that the last ones are those of a short row with the same end; what lies behind a
row would make the last scales and shifts larger."""
import pytest
import torch

from test_gpu_experts_edges import context, memory_goes_back, need      # noqa: F401 (a fixture among them)

pytestmark = pytest.mark.gpu
SPARE = 256


def long_row(ctx, K):
    """[1][1][K] float16, and large numbers behind it"""
    whole = torch.empty(K + SPARE, dtype=torch.float16, device=ctx.device)
    for at in range(0, K, 2 ** 28):
        whole[at:min(at + 2 ** 28, K)].normal_()
    whole[K:] = 60000.0
    return whole, whole[:K].view(1, 1, K)


@pytest.mark.parametrize("K", [2 ** 31 - 1, 2 ** 31 - 128])
def test_8_bit_floats(K):
    ctx = context([5])
    tiles = -(-K // 64)
    need(2 * K + 2048 * tiles + 4 * -(-K // 128))
    whole, w = long_row(ctx, K)
    got = ctx.f8_quantise(w, -9).data
    first = (K - 1) // 128 * 128 - 128
    short = ctx.f8_quantise(w[:, :, first:].contiguous(), -9).data
    n = -(-(K - first) // 64)
    torch.cuda.synchronize()
    assert torch.equal(got[(tiles - n) * 2048:tiles * 2048], short[:n * 2048])
    scales = got[tiles * 2048:][:4 * -(-K // 128)].view(torch.int32)
    want = short[n * 2048:][:4 * -(-(K - first) // 128)].view(torch.int32)
    assert torch.equal(scales[-want.numel():], want)
    assert (whole[K:] == 60000.0).all()


@pytest.mark.parametrize("K", [2 ** 31 - 1, 2 ** 31 - 64])
def test_4_bit_floats(K):
    ctx = context([5])
    tiles = -(-K // 64)
    need(2 * K + 1088 * tiles)
    whole, w = long_row(ctx, K)
    got = ctx.mx4_quantise(w, -9).data
    first = (K - 1) // 64 * 64 - 64
    short = ctx.mx4_quantise(w[:, :, first:].contiguous(), -9).data
    torch.cuda.synchronize()
    assert torch.equal(got[(tiles - 2) * 1088:], short) and short.any()
    assert (whole[K:] == 60000.0).all()


@pytest.mark.parametrize("format", ["w8", "mx4", "f8"])
@pytest.mark.parametrize("M", [2 ** 31 - 1, 2 ** 31 - 255])
def test_more_outputs_than_blocks_of_them_end_in_31_bits(format, M):
    """the blocks of 256 outputs that a layer is cut into are counted in 32 bits"""
    from paper_2302_06361_amd import EXPERTS, F8, MX4, W8, Labels, Layer, binding
    ctx = context([5], lam=[1])
    some = torch.zeros(4096, dtype=torch.uint8, device=ctx.device)
    lay = Layer(EXPERTS, 1, 1, in_c=1, out_c=M, top_k=1, n_experts=1, weights=some)
    lay.c.weight_format = dict(w8=W8, mx4=MX4, f8=F8)[format]
    src, dst = Labels(ctx, 1, zero=True), Labels(ctx, 1, zero=True)     # (a bundle of one label: nothing is launched for it in any case)
    with pytest.raises(binding.DashError, match=r"\(-2\)"):
        ctx.garble_layer(lay, src, dst)
