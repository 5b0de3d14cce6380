"""The tiles' matrix instructions are written out (csrc/gemm_tile_dev.h), so the
wait states around them are this code's own business.  What it counts on in the
built kernels: no operand of a matrix instruction is written by a vector
instruction within the two before it, the sums stay where they are from one to
the next, and nothing else reads a sum until it has settled."""
import glob
import os
import re
import shutil
import subprocess

import pytest

from paper_2303_00158_amd import gnn

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
KERNEL = re.compile(r"act_(tile|tile_part|dw|da)_kernel")
WAIT = 18  # states from a matrix instruction to a vector instruction that reads its result


def regs(operand):
    """The registers of an operand: a[4:7] is a4 to a7."""
    m = re.match(r"^([av])\[(\d+):(\d+)\]$", operand)
    if m:
        return {m[1] + str(i) for i in range(int(m[2]), int(m[3]) + 1)}
    return {operand} if re.match(r"^[av]\d+$", operand) else set()


def parse(line):
    name, _, rest = line.split("//")[0].strip().partition(" ")
    return name, [o.strip().split(" ")[0] for o in rest.split(",")] if rest else []


def touched(instruction):
    return set().union(*(regs(x) for x in instruction[1])) if instruction[1] else set()


def faults(code):
    """What is wrong with a kernel's instructions, in words."""
    found = []
    at = [i for i, (n, _) in enumerate(code) if n.startswith("v_mfma")]
    sums = set().union(*(regs(code[i][1][0]) for i in at))
    fragments = set().union(*(regs(code[i][1][1]) | regs(code[i][1][2]) for i in at))
    if sums & fragments:
        found.append("sums and fragments share registers")
    for i in at:
        name, ops = code[i]
        if ops[0] != ops[3]:
            found.append(f"{i}: {name} is not in place")
        for n, o in code[max(0, i - 2):i]:
            if not n.startswith("v_") or n.startswith("v_mfma") or not o:
                continue
            wrote = regs(o[0]) | (regs(o[1]) if "swap" in n else set())
            if wrote & touched(code[i]):
                found.append(f"{i}: {n} {o} just before {name} reads it")
        states = 0
        for n, o in code[i + 1:i + 1 + WAIT]:
            if states >= WAIT or n in ("s_branch", "s_endpgm"):
                break
            if not n.startswith("v_mfma") and regs(ops[0]) & touched((n, o)):
                found.append(f"{i}: {n} touches {ops[0]} {states} states after {name}")
            states += int(o[0]) + 1 if n == "s_nop" else 1
    for n, o in code[at[0]:at[-1]]:
        if not n.startswith("v_mfma") and sums & touched((n, o)):
            found.append(f"{n} {o} among the products")
    return found


def kernels(text):
    name, code = None, {}
    for line in text.splitlines():
        m = re.match(r"^[0-9a-f]+ <(\S+)>:", line)
        if m:
            name = m[1]
        elif name and KERNEL.search(name) and line.startswith("\t"):
            code.setdefault(name, []).append(parse(line))
    return code


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler")
def test_matrix_instructions_of_the_built_tiles(tmp_path):
    shutil.copy(gnn.LIB_PATH, tmp_path / "libgnn.so")
    subprocess.run([OBJDUMP, "--offloading", str(tmp_path / "libgnn.so")], check=True, capture_output=True, cwd=tmp_path)
    seen = 0
    for path in glob.glob(str(tmp_path / "*gfx950*")):
        with open(path, "rb") as f:
            if not KERNEL.search(f.read().decode("latin-1")):
                continue
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", path], check=True, capture_output=True, text=True).stdout
        for name, code in kernels(text).items():
            assert any(n.startswith("v_mfma") for n, _ in code), name
            assert not faults(code), (name, faults(code)[:5])
            seen += 1
    assert seen >= 40


def test_what_is_found():
    good = ["ds_read_b128 v[0:3], v9", "v_mov_b32_e32 v20, v21", "v_mfma_f32_16x16x32_bf16 a[0:3], v[0:3], v[4:7], a[0:3]",
            "s_nop 15", "s_nop 15", "v_accvgpr_read_b32 v8, a0"]
    assert faults([parse(x) for x in good]) == []
    for at, line in ((1, "v_mov_b32_e32 v4, v21"), (0, "v_accvgpr_write_b32 a3, v1"),
                     (2, "v_mfma_f32_16x16x32_bf16 a[0:3], v[0:3], v[4:7], a[4:7]")):
        assert faults([parse(x) for x in good[:at] + [line] + good[at + 1:]]), line
    assert faults([parse(x) for x in good[:4] + good[5:]])
    assert faults([parse(x) for x in good[:3] + ["v_add_f32_e32 v1, a1, v2"]])
