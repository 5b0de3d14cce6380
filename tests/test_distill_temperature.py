"""The temperatures that the distillation loss takes: those whose square and
whose reciprocal are in fp32's range with room for the logits."""
import pytest
import torch

from paper_2303_00158_amd import gnn
from tests.test_distill import BF16, DEV, F32, check, inputs


def status(temp):
    """gnn_distill_topk's status for a call whose workspace is too small, which
    ends on the host either way."""
    fake = 1 << 24
    return gnn.lib().gnn_distill_topk(fake, 0, 4, 10, fake, 0, fake, 3, temp, 1.0, None, None, None, fake + 4096, 0, None,
                                      fake, fake, 8, None)


@pytest.mark.parametrize("temp", [1e-45, 1e-39, 1.2e-38, 1e-30, 9.9e-19, 1.1e18, 2e19, 3e38])
def test_temperatures_out_of_range_are_refused(temp):
    assert status(temp) == gnn.GNN_EINVAL and b"temperature" in gnn.lib().gnn_last_error()


@pytest.mark.parametrize("temp", [2e-18, 1e-6, 1.0, 1e6, 9e17])
def test_temperatures_in_range_are_taken(temp):
    assert status(temp) == gnn.GNN_ESIZE  # the workspace is the next thing looked at


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("c", [47, 3000, 100_000])
@pytest.mark.parametrize("temp", [2e-18, 1e-3, 30.0, 9e17])
def test_far_temperatures(c, temp, dt):
    """The gradient and the loss stay within their bounds, which grow with the
    square of a high temperature: there the loss is the difference of nearly
    equal logarithms, times that square."""
    z, t, idx, _ = inputs(c, 6, c, 5, dt, dt, pad=False)
    loss, rows, g = check(z, t, idx, temp)
    assert loss.isfinite().all() and rows.isfinite().all() and g.isfinite().all()
