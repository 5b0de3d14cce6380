"""The built kernels of the loss over many classes hold to what the tiles'
matrix instructions count on (tests/test_tile_code.py)."""
import glob
import os
import re
import shutil
import subprocess

import pytest

from paper_2303_00158_amd import gnn
from tests.test_tile_code import OBJDUMP, faults, parse

KERNEL = re.compile(r"class_(product|sums_tile|dz_tile)_kernel")


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
        name, code = None, {}
        for line in text.splitlines():
            m = re.match(r"^[0-9a-f]+ <(\S+)>:", line)
            if m:
                name = m[1]
            elif name and KERNEL.search(name) and line.startswith("\t"):
                code.setdefault(name, []).append(parse(line))
        for name, instructions in code.items():
            assert any(n.startswith("v_mfma") for n, _ in instructions), name
            assert not faults(instructions), (name, faults(instructions)[:5])
            seen += 1
    assert seen >= 20
