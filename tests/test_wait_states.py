"""Waits between dependent instructions of the attention's kernels, in the assembly that hipcc
makes of csrc/attention4.hip, on the CPU.

gfx950 does not hold an instruction back for two kinds of results; the program has to leave
room (the compiler does so by itself, but does not look into inline assembly):
  a vector instruction's, which a matrix instruction reads   2 wait states between them
  a transcendental's, which a vector instruction reads       1
An instruction is one wait state, s_nop n is n + 1."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2608_01653_amd import build

pytestmark = pytest.mark.skipif(shutil.which(build.HIPCC) is None, reason="needs hipcc")
TRANSCENDENTAL = re.compile(r"v_(exp|log|rcp|rsq|sqrt|sin|cos)_")
REGISTERS = re.compile(r"\bv(?:\[(\d+):(\d+)\]|(\d+)\b)")


def registers(operand):
    out = set()
    for first, last, one in REGISTERS.findall(operand):
        out |= {int(one)} if one else set(range(int(first), int(last) + 1))
    return out


def instruction(line):
    """(name, registers written, registers read) of a line of assembly; None if it has none."""
    text = line.split(";")[0].strip()
    if not text or text.startswith((".", "/")) or text.endswith(":"):
        return None
    name, _, rest = text.partition(" ")
    operands = rest.split(",")
    if not name.startswith("v_") or name.startswith("v_cmp"):
        return name, set(), registers(rest)
    read = registers(",".join(operands[1:]))
    if "_swap_" in name or "_fmac_" in name or "mixhi" in name:
        read |= registers(operands[0])
    written = registers(operands[0]) | (registers(operands[1]) if "_swap_" in name else set())
    return name, written, read


def short_waits(lines):
    """[(line number, line, the line whose result it reads too soon)]"""
    found, recent = [], []      # recent: the last instructions, newest first, of one run of code
    for at, line in enumerate(lines):
        one = instruction(line)
        if one is None:
            continue            # (a label: what falls through to it still counts)
        name, written, read = one
        vector, matrix = name.startswith("v_"), name.startswith("v_mfma")
        states = 0
        for text, before, wrote, length in recent:
            need = 2 if matrix and not before.startswith("v_mfma") else 0
            if vector and TRANSCENDENTAL.match(before):
                need = max(need, 1)
            if states < need and wrote & read:
                found.append((at + 1, line.strip(), text))
            states += length
        length = int(line.split("s_nop")[1].split(";")[0]) + 1 if name == "s_nop" else 1
        recent = [(line.strip(), name, written, length)] + recent[:3]
        if name in ("s_branch", "s_endpgm", "s_setpc_b64"):
            recent = []
    return found


def test_the_rule_itself():
    head = ["v_fma_mixhi_f16 v5, v1, v2, 0"]
    mfma = "v_mfma_f32_16x16x32_f16 a[0:3], v[8:11], v[4:7], a[0:3]"
    assert short_waits(head + [mfma]) and short_waits(head + ["s_mov_b32 s1, 0", mfma])
    assert short_waits(head + [".LBB0_1:", "; %bb.2:", mfma])
    assert not short_waits(head + ["s_nop 1", mfma]) and not short_waits(head + ["v_mov_b32_e32 v20, v21", "s_mov_b32 s1, 0", mfma])
    assert not short_waits(["v_fma_mixhi_f16 v12, v1, v2, 0", mfma])
    assert short_waits(["v_exp_f32_e32 v1, v2", "v_mul_f32_e32 v3, v1, v1"])
    assert not short_waits(["v_exp_f32_e32 v1, v2", "s_nop 0", "v_mul_f32_e32 v3, v1, v1"])
    assert not short_waits(["v_exp_f32_e32 v1, v2", "v_mul_f32_e32 v3, v2, v2", "v_mul_f32_e32 v3, v1, v1"])


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    """The lines of every part of attention4.hip."""
    folder = tmp_path_factory.mktemp("assembly")
    flags = [f for f in build.FLAGS if f not in ("-fPIC", "-shared")]

    def part(k):
        to = str(folder / f"part{k}.s")
        subprocess.run([build.HIPCC, *flags, f"-DHATQ_ATTENTION_PART={k}", "--cuda-device-only", "-S", os.path.join(build.CSRC, "attention4.hip"),
                        "-o", to], check=True, capture_output=True, timeout=600)
        with open(to) as f:
            return f.read().splitlines()
    with ThreadPoolExecutor(build.ATTENTION_PARTS) as pool:
        return dict(zip(range(1, build.ATTENTION_PARTS + 1), pool.map(part, range(1, build.ATTENTION_PARTS + 1))))


@pytest.mark.parametrize("part", range(1, build.ATTENTION_PARTS + 1))
def test_attention(assembly, part):
    lines = assembly[part]
    assert sum("v_mfma" in line for line in lines) > 100
    found = short_waits(lines)
    assert not found, "\n".join(f"line {at}: {line}   reads too soon   {before}" for at, line, before in found[:8])
