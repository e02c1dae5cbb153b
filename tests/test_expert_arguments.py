"""Arguments of expert layers: orders and types of the arrays that a layer keeps by address.  No GPU involved."""
import numpy as np
import pytest
import torch

from paper_2302_06361_amd import COMBINE, DENSE, EXPERTS, DashError, Layer, network
from test_network_types import Recorder


class Weights(Recorder):
    """keeps what a layer is prepared from and looks at its order as the context does"""

    def weights8_prepare(self, w):
        assert w.stride(2) == 1 or w.shape[2] == 1
        self.weights = w
        return w

    mx4_quantise = lambda self, w, base, max_shift: self.weights8_prepare(w)


def build(**layer):
    ctx = Weights()
    lays, *_ = network.build_layers(ctx, dict(n_in=3, layers=[dict(dict(kind="experts", id=1, rows=1, top_k=1), **layer)]), 1, 0)
    return ctx, lays[0]


W = np.arange(-12, 12).reshape(2, 4, 3)
ORDERS = {"rows": lambda a: np.ascontiguousarray(a), "columns": lambda a: np.asfortranarray(a), "every other": lambda a: np.repeat(a, 2, -1)[..., ::2],
          "backwards": lambda a: a[..., ::-1].copy()[..., ::-1], "axes swapped": lambda a: np.ascontiguousarray(np.swapaxes(a, -1, -2)).swapaxes(-1, -2)}


@pytest.mark.parametrize("order", list(ORDERS))
def test_weights_of_any_order(order):
    for dtype, more in ((np.int8, {}), (np.int64, {}), (np.float32, dict(base=-2, max_shift=2)), (np.float64, dict(base=-2, max_shift=2))):
        given = ORDERS[order](W.astype(dtype))
        ctx, _ = build(W=given, **more)
        assert (ctx.weights.numpy() == W).all()


@pytest.mark.parametrize("order", list(ORDERS))
def test_bias_of_any_order(order):
    """a layer reads its bias at bias[e * out_c + j]"""
    for dtype in (np.int32, np.int64):
        bias = np.arange(8).reshape(2, 4).astype(dtype)
        _, lay = build(W=W, bias=ORDERS[order](bias))
        kept = [t for t in lay.keep if t.data_ptr() == lay.c.bias]
        assert len(kept) == 1 and kept[0].is_contiguous() and kept[0].dtype == torch.int32 and (kept[0].numpy() == bias).all()


def test_tensors_that_a_layer_cannot_read():
    t = torch.zeros(4, 6, dtype=torch.int32)
    for kind, name in ((EXPERTS, "bias"), (COMBINE, "gates")):
        for bad in (t.t(), t[:, ::2], t[:, 1:], t.long(), t.float(), t.short()):
            with pytest.raises(DashError, match=name):
                Layer(kind, 1, 4, **{name: bad})
        for good in (t, t[1:], t.reshape(-1), t[:, :0], None):
            assert (getattr(Layer(kind, 1, 4, **{name: good}).c, name) or 0) == (0 if good is None else good.data_ptr())
    # dense layers as before
    assert Layer(DENSE, 1, 4, bias=t[0, ::2]).c.bias == t.data_ptr()


def expert_weights(format, E, M, K):
    from paper_2302_06361_amd import ExpertWeights
    w = ExpertWeights.__new__(ExpertWeights)
    w.format, w.n_experts, w.out_c, w.K, w.data = format, E, M, K, torch.zeros(16, dtype=torch.uint8)
    return w


def test_bias_has_an_entry_for_every_expert_and_output():
    """the products read n_experts * out_c of them"""
    W = expert_weights(0, 3, 5, 7)
    for n in (15, 16):
        b = torch.zeros(n, dtype=torch.int32)
        for kw in (dict(weights=W, bias=b), dict(bias=b, weights=W)):
            assert Layer(EXPERTS, 1, 2, top_k=1, **kw).c.bias == b.data_ptr()
    for n in (0, 5, 14):
        b = torch.zeros(n, dtype=torch.int32)
        for kw in (dict(weights=W, bias=b), dict(bias=b, weights=W)):
            with pytest.raises(DashError, match="bias"):
                Layer(EXPERTS, 1, 2, top_k=1, **kw)
    assert not Layer(EXPERTS, 1, 2, top_k=1, weights=W, bias=None).c.bias


def test_expert_weights_belong_to_expert_layers():
    """a dense layer reads its weights as residues, k bytes a weight, past the end of these"""
    from paper_2302_06361_amd import CONV2D, RELU
    for kind in (DENSE, CONV2D, COMBINE, RELU):
        for format in (0, 1):
            with pytest.raises(DashError, match="EXPERTS"):
                Layer(kind, 1, 2, weights=expert_weights(format, 1, 5, 7))
    assert Layer(EXPERTS, 1, 2, top_k=1, weights=expert_weights(1, 1, 5, 7)).c.weight_format == 1
