"""Wait states in front of the loads of the products with 8-bit floating point weights, as test_asm_load_waits.py has them for the other formats, and no
register spilled (a spilled descriptor comes back through a vector register).  No GPU involved."""
import os
import re
import subprocess

import pytest

from paper_2302_06361_amd import build
from test_asm_load_waits import STATES, violations
from test_asm_waits import HIPCC


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("asm") / "f8.s")
    r = subprocess.run([HIPCC] + build.FLAGS + ["--cuda-device-only", "-S", os.path.join(build.CSRC, "dash_experts_f8.hip"), "-o", out], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    return open(out).read()


def test_loads(assembly):
    kernels = dict(re.findall(r"^(_Z\S*k_experts_mfma\S*):(.*?)^\s*\.section", assembly, re.S | re.M))
    assert len(kernels) >= 3
    for name, body in kernels.items():
        assert violations(body) == [], name
        loads = [b for b in re.findall(r";;#ASMSTART\n(.*?);;#ASMEND", body, re.S) if "buffer_load" in b]
        assert len(loads) >= 15, name
        for block in loads:
            lines = [line.strip() for line in block.strip().splitlines()]
            at = next(i for i, line in enumerate(lines) if line.startswith("buffer_load"))
            assert sum(int(line.split()[1], 0) + 1 if line.startswith("s_nop") else 1 for line in lines[:at]) >= STATES, block


def test_nothing_is_spilled(assembly):
    counts = re.findall(r"\.vgpr_spill_count:\s*(\d+)", assembly)
    assert counts and set(counts) == {"0"}
