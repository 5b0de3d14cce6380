"""Rows of the distillation loss at the border of what a shape holds in
registers: on the CPU which thread takes which class, on the GPU the loss and
its gradient, at every place of a row in its 128-byte line."""
import os
import shutil
import subprocess

import pytest
import torch

from paper_2303_00158_amd import gnn
from tests.test_distill import BF16, DEV, F32, bounds, check, formula, inputs, within

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
# threads to a row and elements to a thread, in the order they are tried
SHAPES = [(16, 8), (64, 8), (64, 16), (64, 32), (64, 64), (256, 32), (256, 64), (512, 64), (1024, 64)]


def longest(dt):
    """Each shape's longest row: its vectors and one more (the row's end) less
    the part of the first line that may lie before the row."""
    ve, line = (8, 64) if dt == BF16 else (4, 32)
    shapes = SHAPES + ([(1024, 128)] if dt == BF16 else [])
    return [((t, e), t * (e + ve) - line) for t, e in shapes]


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("distill") / "distill_rows")
    subprocess.run([HIPCC, "--offload-arch=gfx950", "--offload-host-only", "-std=c++17", "-O2", "-w",
                    "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2303_00158_amd", "csrc"),
                    os.path.join(ROOT, "tests", "host", "distill_rows.hip"), "-o", exe], check=True, capture_output=True)

    def run(rows):
        text = "\n".join(" ".join(map(str, r)) for r in rows)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True, timeout=110).stdout
        return [tuple(int(x) for x in line.split()) for line in out.splitlines()]
    return run


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
@pytest.mark.parametrize("dt", [F32, BF16])
def test_every_class_is_taken_once(host, dt):
    top = longest(dt)[-1][1]
    counts = set(range(1, 2700))
    for _, c in longest(dt):
        counts |= {x for x in range(c - 70, c + 71) if c < 20_000 or abs(x - c) % 7 < 2}
    rows = [(int(dt == BF16), c, k) for c in sorted(counts) for k in (5,) if c <= top]
    rows += [(int(dt == BF16), c, k) for c in (8, 200, 224, 960, 992, top) for k in (113, 455, gnn.GNN_MAX_TOP)]
    got = host(rows)
    assert len(got) == len(rows)
    wrong = [r[1:] for r, (t, _, bad) in zip(rows, got) if t == 0 or bad]
    assert not wrong, f"{len(wrong)} class counts, {wrong[:3]} to {wrong[-1]}"


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
@pytest.mark.parametrize("dt", [F32, BF16])
def test_the_borders_are_these(host, dt):
    """The sizes that the GPU test takes are the borders of the shapes."""
    t = int(dt == BF16)
    assert [g[:2] for g in host([(t, c, 5) for _, c in longest(dt)])] == [s for s, _ in longest(dt)]
    after = [s for s, _ in longest(dt)][1:] + [(0, 0)]
    assert [g[:2] for g in host([(t, c + 1, 5) for _, c in longest(dt)])] == after


def border_sizes(dt):
    sizes = {200, 224, 225, 992, 993, 1504, 1505, 2528, 4576}
    for _, c in longest(dt):
        sizes |= {c, c + 1}
    return sorted(sizes)


@pytest.mark.gpu
@pytest.mark.parametrize("dt, c", [(dt, c) for dt in (F32, BF16) for c in border_sizes(dt)])
def test_loss_and_gradient_at_the_borders(dt, c):
    """Rows enough for every place in a line; from 32,768 classes on, enough of
    them to stay whole."""
    b = 65 if c <= 5000 else 17 if c < 32_768 else 129
    z, t, idx, labels = inputs(c, b, c, 7, dt, dt)
    _, rows, g = check(z, t, idx, 2.0, 0.7, labels)
    over, loss, r2 = z.clone(), torch.empty(1, device=DEV), torch.empty(b, device=DEV)
    gnn.distill_topk(over, t, idx, 2.0, over, loss, r2, alpha=0.7, labels=labels.to(DEV))
    assert torch.equal(over, g) and torch.equal(r2, rows)


@pytest.mark.gpu
@pytest.mark.parametrize("off", [1, 31, 32, 33, 63])
@pytest.mark.parametrize("dt, c", [(F32, 160), (F32, 736), (BF16, 192), (BF16, 193), (BF16, 224), (BF16, 961),
                                   (BF16, 1472), (BF16, 10_177), (BF16, 18_369)])
def test_borders_off_the_line(dt, c, off):
    z, t, idx, labels = inputs(c + off, 9, c, 6, dt, dt)
    buf = torch.empty(z.numel() + 64, dtype=dt, device=DEV)
    moved = buf[off:off + z.numel()].view(z.shape)
    moved.copy_(z)
    g, loss = torch.full_like(z, 7.0), torch.empty(1, device=DEV)
    gnn.distill_topk(moved, t, idx, 2.0, g, loss, None, alpha=0.5, labels=labels.to(DEV))
    _, _, want = formula(z, t, idx, 2.0, 0.5, labels)
    within(g, want, bounds(z, t, idx, 2.0, 0.5, labels, None, dt)[1], "gradient")
