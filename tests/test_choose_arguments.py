"""Refusals of the choice of experts: arguments are looked at before anything is launched.  No GPU involved."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2302_06361_amd import DashError, Router, binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, EINVAL, ESIZE = 0, -1, -2
CTX, L, TO = 16, 4096, 1 << 20           # (addresses that are never followed)


def choose(ctx=CTX, logits=L, dtype=0, stride=64, n=5, valid=None, experts=TO, gates=TO, weights=TO, router=True, **kw):
    r = dict(n_experts=64, top_k=4, score=0, n_groups=8, top_groups=3, group_score=0, renormalise=1, gate_bits=8, scale=1.0, bias=None)
    r.update(kw)
    c = binding.CRouter(**r)
    return binding.lib().dash_choose(ctx, C.byref(c) if router else None, logits, dtype, stride, n, valid, experts, gates, weights, None)


@pytest.mark.parametrize("bad", [dict(ctx=None), dict(router=False), dict(logits=None), dict(experts=None), dict(dtype=3), dict(dtype=-1), dict(n=-1), dict(stride=63), dict(stride=-64),
                                 dict(n_experts=0), dict(n_experts=63), dict(top_k=0), dict(top_k=25), dict(n_groups=0), dict(n_groups=7), dict(top_groups=0),
                                 dict(top_groups=9), dict(score=2), dict(score=-1), dict(group_score=2), dict(gate_bits=-1), dict(gate_bits=31), dict(scale=0.0),
                                 dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=5e6), dict(gate_bits=30, scale=1.5),
                                 dict(logits=L + 2), dict(logits=L + 1, dtype=1), dict(experts=TO + 2), dict(gates=TO + 1), dict(weights=TO + 2), dict(bias=L + 2)])
def test_refuses(bad):
    assert choose(**bad) == EINVAL


@pytest.mark.parametrize("big", [dict(n_experts=1032, stride=2000), dict(top_k=33, n_experts=512, stride=512), dict(n_experts=520, n_groups=65, stride=520, top_groups=10)])
def test_sizes(big):
    assert choose(**big) == ESIZE


def test_no_rows():
    """nothing is launched, nothing looked at"""
    assert choose(n=0) == OK and choose(n=0, logits=None, experts=None, gates=None, weights=None, stride=0) == OK
    assert choose(n=0, top_k=0) == EINVAL


def test_header(tmp_path):
    names = [f[0] for f in binding.CRouter._fields_]
    src = tmp_path / "t.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "dash.h"\nint main(void) { printf("%%d", (int)sizeof(dash_router)); %s return 0; }\n' %
                   " ".join('printf(" %%d", (int)offsetof(dash_router, %s));' % n for n in names))
    subprocess.check_call(["gcc", "-std=c11", "-Wall", "-Wextra", "-Wpedantic", "-Werror", "-I", os.path.join(ROOT, "include"), "-o", str(tmp_path / "t"), str(src)])
    out = [int(v) for v in subprocess.check_output([str(tmp_path / "t")]).split()]
    assert out[0] == C.sizeof(binding.CRouter) and out[1:] == [getattr(binding.CRouter, n).offset for n in names]


def test_router_bias():
    b = torch.zeros(64)
    assert Router(64, 4, bias=b).c.bias == b.data_ptr()
    for bad in (b.double(), b[:63], torch.zeros(128)[::2], b.half()):
        with pytest.raises(DashError, match="bias"):
            Router(64, 4, bias=bad)


class Plain:
    """a context without a GPU: the binding's own checks"""
    def __init__(self):
        self.device, self.h, self._types, self.L = torch.device("cpu"), 16, None, self
        self._float_types = lambda: binding.Context._float_types(self)
        self.calls = 0

    def dash_choose(self, *a):
        self.calls += 1
        return 0


def test_binding_refuses(monkeypatch):
    monkeypatch.setattr(binding, "_stream", lambda: None)
    ctx, r = Plain(), Router(8, 2)
    call = lambda *a, **k: binding.Context.choose(ctx, *a, **k)
    good = torch.zeros(5, 8)
    assert call(r, good).experts.shape == (5, 2) and call(r, torch.zeros(5, 10)[:, :8]).gates.dtype == torch.int32
    assert call(r, good[:1].expand(1, 8)).n == 1 and call(r, good, valid=torch.ones(5, dtype=torch.bool)).n == 5
    calls = ctx.calls
    for bad in (torch.zeros(5, 9), torch.zeros(8), torch.zeros(5, 16)[:, ::2], good.double(), good.long(), good[:1].expand(5, 8), torch.zeros(8, 5).t()):
        with pytest.raises(DashError, match="logits"):
            call(r, bad)
    for bad in (torch.ones(4, dtype=torch.uint8), torch.ones(5), torch.ones(10, dtype=torch.uint8)[::2]):
        with pytest.raises(DashError, match="valid"):
            call(r, good, valid=bad)
    for out in (binding.Choice(ctx, 4, 2), binding.Choice(ctx, 5, 3)):
        with pytest.raises(DashError, match="out"):
            call(r, good, out=out)
    assert ctx.calls == calls


def test_network_refuses_routers_of_another_size():
    import numpy as np
    from paper_2302_06361_amd import network
    from test_expert_arguments import Weights
    ctx = Weights()
    ctx.choose = ctx.route = lambda *a, **k: None
    ctx.weights8_prepare = lambda w: type("W", (), dict(n_experts=3, data_ptr=lambda: 16))
    ctx.device = torch.device("cpu")
    layer = dict(kind="experts", id=1, rows=2, top_k=2, W=np.zeros((3, 4, 3), np.int8), router=dict(logits=np.zeros((5, 3)), top_k=1))
    with pytest.raises(ValueError, match="top_k"):
        network.build_layers(ctx, dict(n_in=3, layers=[layer]), 5, 0)
    layer["router"] = dict(logits=np.zeros((5, 4)), top_k=2)
    with pytest.raises(ValueError, match="experts"):
        network.build_layers(ctx, dict(n_in=3, layers=[layer]), 5, 0)
    layer["router"] = dict(logits=np.zeros((5, 3)), top_k=2)
    with pytest.raises(ValueError, match="logits"):
        network.build_layers(ctx, dict(n_in=3, layers=[layer]), 6, 0)
