"""The tiles' matrix instructions are written out (csrc/gemm_tile_dev.h), so the
compiler does not know how long their results take.  Whatever it does with a
sum has to depend on the wait behind the last product, not merely stand behind
it: in the compiler's intermediate code nothing but the products themselves and
the wait's own statements may use a product's result."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"


def unsettled(text):
    """Lines that use a product's result without the wait between."""
    body = text[text.index("@tile_sums("):]
    lines = body[:body.index("\n}")].splitlines()
    sums = {m[1] for m in (re.match(r"\s*(%\w+) = .*asm sideeffect \"v_mfma", x) for x in lines) if m}
    assert sums, "no products"
    while True:  # through the joins of control flow
        more = {m[1] for m in (re.match(r"\s*(%\w+) = phi ", x) for x in lines)
                if m and m[1] not in sums and sums & set(re.findall(r"%\w+", m.string.split("phi", 1)[1]))}
        if not more:
            break
        sums |= more
    waited, found = False, []
    for x in lines:
        if re.match(r"^\w+:", x):  # a block's label: its wait is its own
            waited = False
        waited |= '"s_nop 15' in x
        used = sums & set(re.findall(r"%\w+", x.split(" = ", 1)[-1]))
        tied = waited and re.search(r'asm sideeffect "", "=a,0"', x)
        if used and " phi " not in x and '"v_mfma' not in x and not tied:
            found.append(x.strip())
    return found


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
def test_sums_are_used_behind_the_wait(tmp_path):
    out = str(tmp_path / "tile_sums.ll")
    subprocess.run([HIPCC, "--offload-arch=gfx950", "--offload-device-only", "-S", "-emit-llvm", "-O3", "-std=c++17", "-w",
                    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                    "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2303_00158_amd", "csrc"),
                    os.path.join(ROOT, "tests", "host", "tile_sums.hip"), "-o", out], check=True, capture_output=True)
    with open(out) as f:
        assert unsettled(f.read()) == []
