"""dash_layer keeps its size and the places of its fields: dash_garble_layers and dash_eval_layers read arrays of it, so that a program compiled
before expert layers were added goes on working.  No GPU involved."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2302_06361_amd import COMBINE, EXPERTS, Layer, binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Before(C.Structure):
    """the descriptor of layers without experts"""
    _fields_ = [("kind", C.c_int32), ("layer_id", C.c_int32), ("elem_base", C.c_int64), ("n_elem", C.c_int64),
                ("in_h", C.c_int32), ("in_w", C.c_int32), ("in_c", C.c_int32), ("out_c", C.c_int32),
                ("kh", C.c_int32), ("kw", C.c_int32), ("stride", C.c_int32), ("pad", C.c_int32),
                ("weights", C.c_void_p), ("bias", C.c_void_p), ("repeat", C.c_int32),
                ("p_index", C.c_int32), ("q_index", C.c_int32), ("phi", C.c_void_p), ("phi_stride", C.c_int64)]


NEW = ["top_k", "n_experts", "weight_format", "routing", "gates"]


def test_binding():
    assert C.sizeof(binding.CLayer) == C.sizeof(Before) == 104
    for name, _ in Before._fields_:
        assert getattr(binding.CLayer, name).offset == getattr(Before, name).offset, name


@pytest.mark.parametrize("compiler", [["gcc"], ["gcc", "-std=c11", "-Wall", "-Wextra", "-Wpedantic", "-Werror"], ["g++", "-x", "c++", "-std=c++11", "-Wall", "-Werror"]])
def test_header(compiler, tmp_path):
    names = [n for n, _ in Before._fields_] + NEW
    src = tmp_path / "t.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "dash.h"\nint main(void) { printf("%%d", (int)sizeof(dash_layer)); %s return 0; }\n' %
                   " ".join('printf(" %%d", (int)offsetof(dash_layer, %s));' % n for n in names))
    subprocess.check_call(compiler + ["-I", os.path.join(ROOT, "include"), "-o", str(tmp_path / "t"), str(src)])
    out = [int(v) for v in subprocess.check_output([str(tmp_path / "t")]).split()]
    assert out[0] == C.sizeof(Before)
    for name, at in zip(names, out[1:]):
        assert at == getattr(binding.CLayer if name in NEW else Before, name).offset, name


def test_fields_of_expert_layers_are_apart():
    """those that one kind of layer reads together"""
    lay = Layer(EXPERTS, 1, 6, in_c=7, out_c=9, top_k=2, n_experts=3, weight_format=1)
    lay.c.weights, lay.c.bias, lay.c.routing = 16, 32, 48
    c = lay.c
    assert (c.n_elem, c.in_c, c.out_c, c.top_k, c.n_experts, c.weight_format, c.weights, c.bias, c.routing) == (6, 7, 9, 2, 3, 1, 16, 32, 48)
    lay = Layer(COMBINE, 1, 6, in_c=7, top_k=2)
    lay.c.gates = 64
    assert (lay.c.n_elem, lay.c.in_c, lay.c.top_k, lay.c.gates) == (6, 7, 2, 64)
