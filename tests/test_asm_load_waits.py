"""Wait states in front of the expert layers' loads: a scalar register that a vector instruction writes (a v_readlane of a spilled
descriptor among them) may be read by a vector-memory instruction five wait states later at the earliest.  The compiler sees to that in
its own code, but not in front of a load in inline assembly.  The kernels' assembly as it is built, over all ways through it.  No GPU involved."""
import os
import re
import subprocess

import pytest

from paper_2302_06361_amd import build
from test_asm_waits import HIPCC, scalars

STATES = 5
MEMORY = ("buffer_", "global_", "flat_", "scratch_")


def parse(assembly):
    """-> instructions (line number, operation, operands, text) and the index that every label stands in front of"""
    code, labels = [], {}
    for number, line in enumerate(assembly.splitlines(), 1):
        text = line.split(";")[0].strip()
        label = re.match(r"([\w.$]+):", text)
        if label:
            labels[label.group(1)] = len(code)
        elif text and not text.startswith((".", "#")):
            op, _, rest = text.partition(" ")
            code.append((number, op, [o.strip() for o in re.split(r",(?![^\[]*\])", rest)], text))
    return code, labels


def step(instruction, age):
    """(ages after it, whether it reads a scalar too soon); ages: scalar register -> wait states since a vector instruction wrote it, below STATES"""
    _, op, operands, _ = instruction
    bad, steps, written = False, 1, set()
    if op == "s_nop":
        steps = int(operands[0], 0) + 1
    elif op.startswith(MEMORY):
        # (a buffer's last operand carries the scalar offset and the flags, separated by blanks)
        read = set().union(*[scalars(word) for o in operands for word in o.split()])
        bad = any(r in age for r in read)
    elif op.startswith("v_"):
        dests = 2 if "_co_" in op or op.startswith(("v_mad_u64", "v_mad_i64", "v_div_scale")) else 1
        written = set().union(*[scalars(o) for o in operands[:dests]])
    else:
        # what a scalar instruction writes is no vector result any more
        age = {r: a for r, a in age.items() if not (op.startswith("s_") and operands and r in scalars(operands[0]))}
    age = {r: a + steps for r, a in age.items() if a + steps < STATES}
    age.update({r: 0 for r in written})
    return age, bad


def violations(assembly):
    """(line, text) of memory instructions that read a scalar register too soon, over every edge between instructions"""
    code, labels = parse(assembly)
    starts, work, bad = {}, [(0, {})] + [(i, {}) for i in set(labels.values())], set()
    while work:
        i, age = work.pop()
        while i < len(code):
            seen = starts.get(i)
            if seen is not None:
                merged = {r: min(seen.get(r, STATES), age.get(r, STATES)) for r in set(seen) | set(age)}
                if merged == seen:
                    break
                age = merged
            starts[i] = age
            number, op, operands, text = code[i]
            age, wrong = step(code[i], age)
            if wrong:
                bad.add((number, text))
            if op.startswith(("s_branch", "s_cbranch")) and operands[-1] in labels:
                work.append((labels[operands[-1]], age))
            if op in ("s_branch", "s_endpgm", "s_setpc_b64"):
                break
            i += 1
    return sorted(bad)


def test_the_check_itself():
    load = "v_readlane_b32 s7, v200, 3\n%sbuffer_load_dwordx4 v1, s[4:7], 0 offen offset:1024 lds\n"
    assert violations(load % "") and violations(load % "s_add_u32 m0, s0, 0x400\ns_nop 2\n")
    assert not violations(load % "s_add_u32 m0, s0, 0x400\ns_nop 3\n")
    assert not violations(load % "s_mov_b32 s7, 0x20000\n") and violations(load % "s_mov_b32 s8, 0x20000\n")
    assert violations("v_readfirstlane_b32 s9, v2\nbuffer_store_dword v1, v2, s[4:7], s9 offen\n")
    assert violations("v_cmp_eq_u32_e64 s[8:9], v1, v2\nglobal_load_dword v1, v2, s[8:9]\n")
    assert not violations("v_readlane_b32 s7, v200, 3\nbuffer_load_dwordx4 v1, s[8:11], 0 offen lds\n")
    # round a loop, and over a branch
    assert violations(".L1:\nbuffer_load_dword v1, s[4:7], 0 offen lds\ns_nop 1\nv_readlane_b32 s4, v9, 1\ns_cbranch_scc1 .L1\ns_endpgm\n")
    assert violations("v_readlane_b32 s4, v9, 1\ns_branch .L2\n.L1:\ns_nop 4\n.L2:\nbuffer_load_dword v1, s[4:7], 0 offen lds\ns_endpgm\n")
    assert not violations("v_readlane_b32 s4, v9, 1\ns_cbranch_scc1 .L2\ns_endpgm\n.L2:\ns_nop 3\nbuffer_load_dword v1, s[4:7], 0 offen lds\ns_endpgm\n")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("asm") / "experts.s")
    r = subprocess.run([HIPCC] + build.FLAGS + ["--cuda-device-only", "-S", os.path.join(build.CSRC, "dash_experts_gemm.hip"), "-o", out], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    return dict(re.findall(r"^(_Z\S*k_experts_mfma\S*):(.*?)^\s*\.section", open(out).read(), re.S | re.M))


def test_descriptors_are_there_when_a_load_reads_them(kernels):
    assert len(kernels) == 6
    for name, body in kernels.items():
        assert len(re.findall(r"buffer_load_dword\S* .* lds", body)) >= 20, name          # (the loads are there)
        assert violations(body) == [], name


def test_every_load_in_assembly_waits_by_itself(kernels):
    """whatever stands in front of it: the assembly block of a load brings five wait states of its own"""
    for name, body in kernels.items():
        blocks = re.findall(r";;#ASMSTART\n(.*?);;#ASMEND", body, re.S)
        loads = [b for b in blocks if "buffer_load" in b]
        assert len(loads) >= 20, name
        for block in loads:
            lines = [line.strip() for line in block.strip().splitlines()]
            at = [i for i, line in enumerate(lines) if line.startswith("buffer_load")]
            assert len(at) == 1
            states = sum(int(line.split()[1], 0) + 1 if line.startswith("s_nop") else 1 for line in lines[:at[0]])
            assert states >= STATES, block
