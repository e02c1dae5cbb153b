"""Expert layers of the network format: integers that do not fit the type that the library takes them in are refused, not wrapped.  No GPU
involved: what build_layers hands to the context is looked at."""
import numpy as np
import pytest
import torch

import workloads
from paper_2302_06361_amd import network


class Recorder:
    """stands in for the context: keeps the weights that a layer is prepared from"""
    device = torch.device("cpu")

    def weights8_prepare(self, w):
        self.weights = w
        return w

    def layer_sizes(self, layer):
        return 1, 0, 0


def build(**changes):
    ctx = Recorder()
    layer = dict(kind="experts", id=1, rows=1, top_k=1, W=[[[1, -2]]])
    layer.update(changes)
    lays, *_ = network.build_layers(ctx, dict(n_in=2, layers=[layer]), 1, 0)
    return ctx, lays[0]


@pytest.mark.parametrize("dtype", [np.int8, np.int16, np.int64, np.float32, np.float64, object])
def test_weights_that_fit(dtype):
    W = np.array([[[-128, 127, 0], [5, -1, 100]]], dtype)
    ctx, _ = build(W=W)
    assert ctx.weights.dtype == torch.int8 and (ctx.weights.numpy() == W.astype(np.int64)).all()
    assert (build(W=W.tolist())[0].weights.numpy() == W.astype(np.int64)).all()


@pytest.mark.parametrize("value", [128, -129, 200, 300, 2 ** 40, 0.7, -127.5, float("nan"), float("inf"), 2 ** 70])
def test_weights_that_do_not_fit(value):
    """integers past a byte; floats whose `base` was forgotten"""
    for W in ([[[1, value]]], np.array([[[1, value]]])):
        with pytest.raises(ValueError, match="W"):
            build(W=W)


@pytest.mark.parametrize("value", [2 ** 31, -2 ** 31 - 1, 2 ** 32 + 1, 0.5])
def test_bias_route_and_gates_that_do_not_fit(value):
    for v in ([value], np.array([value])):
        with pytest.raises(ValueError, match="bias"):
            build(bias=v)
        with pytest.raises(ValueError, match="route"):
            build(route=v)
        with pytest.raises(ValueError, match="gates"):
            network.build_layers(Recorder(), dict(n_in=2, layers=[dict(kind="combine", id=1, rows=1, top_k=1, V=2, gates=v)]), 1, 0)


def test_extremes_of_route_and_gates():
    for v in (2 ** 31 - 1, -2 ** 31, -1, 0):
        assert network._PerBatch([v], 1, Recorder(), "gates").part(0, 1).tolist() == [v]


@pytest.mark.parametrize("mx4", [True, False])
def test_the_mixture_is_of_its_types(mx4):
    for L in workloads.mixture(mx4=mx4)["layers"]:
        if L["kind"] == "experts" and not mx4:
            assert (network._integers(L["W"], np.int8, "W") == L["W"]).all()
        for key in ("bias", "route", "gates"):
            if L.get(key) is not None and L["kind"] in ("experts", "combine"):
                assert (network._integers(L[key], np.int32, key) == L[key]).all()
