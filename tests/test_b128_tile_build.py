"""The tile kernels of e4m3 blocks of 128 (gemm_b128_tile.hip) issue their MFMAs as inline assembly, which hides them from the compiler's hazard handling.
What the padding there relies on is read off a build with the library's flags, along every path through the branches: no vector instruction writes an operand,
scales among them, right in front of an MFMA, none touches an accumulator before its MFMA is through, and nothing is spilled, as a spilled accumulator would be read
without that wait."""
import os
import re
import subprocess

import pytest

from paper_2303_06182_amd import build
from test_ring_hazards import READ_WAIT, RESULT_WAIT, registers, wait_states


def program(text):
    """[(mnemonic, operands)] in order, and the place of each label; modifiers behind the last operand are left out."""
    prog, labels = [], {}
    for line in text.splitlines():
        line = line.split(";")[0].strip()
        m = re.match(r"(\.?[\w$.]+):$", line)
        if m:
            labels[m[1]] = len(prog)
        elif line and not line.startswith("."):
            name, _, rest = line.partition(" ")
            rest = re.sub(r"\s+\w+:(\[[^]]*\]|\S+).*$", "", rest.strip())
            prog.append((name, [o.strip() for o in rest.split(",")] if rest else []))
    return prog, labels


def following(prog, labels, at):
    name, ops = prog[at]
    if name == "s_endpgm":
        return []
    if name == "s_branch":
        return [labels[ops[0]]]
    return [at + 1] + ([labels[ops[0]]] if name.startswith("s_cbranch") else [])


def reached(prog, labels, start, states):
    """Instructions that may be issued fewer than `states` wait states behind instruction `start`."""
    waited, todo = {}, [(i, 0) for i in following(prog, labels, start)]
    while todo:
        at, n = todo.pop()
        if n >= states or at >= len(prog) or waited.get(at, states) <= n:
            continue
        waited[at] = n
        todo += [(i, n + wait_states(prog[at])) for i in following(prog, labels, at)]
    return sorted(waited)


def hazards(text):
    """(MFMAs looked at, descriptions of the hazards found)"""
    prog, labels = program(text)
    found, n = [], 0
    mfma = lambda i: i[0].startswith("v_mfma")
    for at, (name, ops) in enumerate(prog):
        if mfma((name,)):
            n += 1
            result = registers(ops[0])
            assert len(result) >= 4, ops
            for i in reached(prog, labels, at, RESULT_WAIT):
                other = prog[i]
                touched = other[1][1:3] if mfma(other) else other[1]
                if set().union(*map(registers, touched)) & result:
                    found.append("%s behind %s" % (other, ops))
        elif name.startswith("v_") and ops:
            written = set().union(*map(registers, ops[:2] if "swap" in name else ops[:1]))
            for i in reached(prog, labels, at, READ_WAIT) if written else []:
                if mfma(prog[i]) and set().union(*map(registers, prog[i][1][1:])) & written:
                    found.append("%s in front of %s" % ((name, ops), prog[i][1]))
    return n, found


def test_the_check_finds_what_it_is_for():
    scaled = "\tv_mfma_scale_f32_32x32x64_f8f6f4 v[0:15], v[16:23], v[24:31], v[0:15], v32, v33 op_sel_hi:[0,0,0]\n"
    for operand in (16, 31, 0, 32, 33):
        assert hazards("\tv_mov_b32_e32 v%d, v40\n\ts_nop 0\n" % operand + scaled)[1], operand
        assert hazards("\tv_mov_b32_e32 v%d, v40\n\ts_nop 1\n" % operand + scaled) == (1, [])
    assert hazards(scaled + "\ts_nop 15\n\tscratch_store_dword off, v15, off\n")[1]
    assert hazards(scaled + "\ts_nop 15\n\ts_nop 15\n\tscratch_store_dword off, v15, off\n") == (1, [])
    # round a loop, either way
    assert hazards(".LBB0_1:\n" + scaled + "\tv_mov_b32_e32 v33, v40\n\ts_cbranch_scc1 .LBB0_1\n\ts_endpgm\n")[1]
    assert hazards(".LBB0_1:\n\tv_mov_b32_e32 v50, v3\n\ts_nop 3\n" + scaled + "\ts_cbranch_scc1 .LBB0_1\n\ts_endpgm\n")[1]
    assert hazards(scaled + "\ts_branch .LBB0_2\n\tv_mov_b32_e32 v50, v3\n.LBB0_2:\n\ts_endpgm\n") == (1, [])


@pytest.fixture(scope="module")
def built(tmp_path_factory):
    out = tmp_path_factory.mktemp("b128") / "tile.s"
    cmd = [build._hipcc(), *build.HIPCC_FLAGS, "--cuda-device-only", "-S", "-Rpass-analysis=kernel-resource-usage", os.path.join(build.CSRC, "gemm_b128_tile.hip"),
           "-o", str(out)]
    r = subprocess.run(cmd, check=True, capture_output=True, text=True)
    return out.read_text(), r.stderr


def test_no_hazard_in_the_tile_kernels(built):
    n, found = hazards(built[0])
    assert n > 500 and not found, found[:5]


def test_no_spill_in_the_tile_kernels(built):
    assert built[1].count("Function Name: ") >= 6 and build.spilled_kernels(built[1]) == []
    assert "scratch_" not in built[0]
    assert "gemm_b128_tile.hip" in build.NO_SPILL_SOURCES
