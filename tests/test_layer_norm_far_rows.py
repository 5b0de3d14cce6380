"""Layer norm's gradients of rows so far from zero that mean x rstd is past
fp32's range, though every value and every gradient is within it."""
import pytest
import torch

from paper_2303_00158_amd import gnn

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("weights", [True, False])
@pytest.mark.parametrize("f", [7, 32, 40, 100, 200, 300, 600, 1024, 1100, 2500, 5001, 9000, 20_000, 40_000])
def test_constant_rows_far_from_zero(f, weights, dt):
    """x = 2^80 throughout and eps = 2^-100: mean 2^80 and rstd 2^50, whose
    product overflows, h = 0, d_x = rstd (q - mean q), dgamma = 0.  Two such
    rows stand among ordinary ones."""
    gen = torch.Generator().manual_seed(f)
    rows, eps = 5, 2.0 ** -100
    x = torch.randn((rows, f), generator=gen)
    x[1], x[4] = 2.0 ** 80, -2.0 ** 80
    x = x.to(dt).to(DEV)
    g = torch.randn((rows, f), generator=gen).to(dt).to(DEV)
    gamma = torch.randn(f, generator=gen).to(DEV) if weights else None
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    gnn.layer_norm_fwd(x, gamma, None, y, eps, mean, rstd)
    assert mean[1] == 2.0 ** 80 and mean[4] == -2.0 ** 80 and (rstd[[1, 4]] == 2.0 ** 50).all() and not y[[1, 4]].any()
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty(f, device=DEV), torch.empty(f, device=DEV)
    gnn.layer_norm_bwd(g, x, gamma, mean, rstd, dx, dgamma, dbeta)
    assert dx.isfinite().all() and dgamma.isfinite().all() and dbeta.isfinite().all()
    q = g[[1, 4]].double() * (gamma.double() if weights else 1.0)
    want = 2.0 ** 50 * (q - q.mean(1, keepdim=True))
    # q is rounded once; a sum of its f values takes at most 64 additions of a
    # thread, 6 and 16 of the tree; the mean, the difference and the product
    # with rstd one each
    off = 2.0 ** 50 * U * (3 * q.abs() + 92 * q.abs().mean(1, keepdim=True)) + (torch.finfo(dt).eps / 2 + 2 * U) * want.abs()
    assert ((dx[[1, 4]].double() - want).abs() <= off).all()
    # the constant rows add nothing to dgamma: it is the ordinary rows'
    here = [0, 2, 3]
    alone, none = torch.empty(f, device=DEV), torch.empty(f, device=DEV)
    gnn.layer_norm_bwd(g[here].contiguous(), x[here].contiguous(), gamma, mean[here].contiguous(),
                       rstd[here].contiguous(), None, alone, none)
    h = (x[here].double() - mean[here].double()[:, None]) * rstd[here].double()[:, None]
    near = (g[here].double() * h).abs().sum(0) * 16 * U  # rounded at most eight times on each side
    assert ((dgamma - alone).double().abs() <= near).all()
