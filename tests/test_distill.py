"""The loss against a teacher's top logits, and its gradient, against the
formulas in 64 bits."""
import math

import pytest
import torch

from paper_2303_00158_amd import gnn

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


def half_step(dt):
    return torch.finfo(dt).eps / 2


def formula(z, t, idx, temp, alpha, labels=None, scale=None):
    """(loss, row losses, gradient) in 64 bits, row by row."""
    b, c = z.shape
    z, t, idx = z.double().cpu(), t.double().cpu(), idx.cpu()
    s = torch.full((b,), 1.0 / max(b, 1), dtype=torch.float64) if scale is None else scale.double().cpu()
    rows, grad = torch.zeros(b, dtype=torch.float64), torch.zeros((b, c), dtype=torch.float64)
    for i in range(b):
        if s[i] == 0:
            continue
        here = (idx[i] >= 0) & (idx[i] < c) & (t[i] != -math.inf)
        if alpha > 0 and here.any():
            p, at = torch.softmax(t[i][here] / temp, 0), idx[i][here]
            logp, logq = torch.log_softmax(t[i][here] / temp, 0), torch.log_softmax(z[i] / temp, 0)
            some = p > 0
            rows[i] += alpha * temp ** 2 * (p[some] * (logp[some] - logq[at][some])).sum()
            grad[i] += alpha * temp * (logq.exp() - torch.zeros(c, dtype=torch.float64).index_add_(0, at, p))
        if alpha < 1 and labels is not None and 0 <= labels[i] < c:
            logq = torch.log_softmax(z[i], 0)
            rows[i] -= (1 - alpha) * logq[labels[i]]
            grad[i] += (1 - alpha) * logq.exp()
            grad[i, labels[i]] -= 1 - alpha
        grad[i] *= s[i]
    return (rows * s).sum(), rows, grad


def bounds(z, t, idx, temp, alpha, labels, scale, g_dt):
    """How far the row losses and the gradient may be off.  With x the largest
    distance (in units of the exponent) of a logit from its row's maximum, an
    exponential is off by 2 U x (its argument's roundings) and 4 U (its own,
    at most two steps), a sum of them by its additions' roundings (a thread's
    serial part, at most c / 64 and 1,100, then the tree) and a quotient by
    2 U more: e below, relative.  A logarithm's argument gives that error
    absolutely."""
    b, c = z.shape
    z64, t64 = z.double().cpu(), t.double().cpu()
    inv = max(1.0, 1.0 / temp)

    def spread(x):
        x = torch.where(x.abs() == math.inf, math.nan, x)
        top = torch.nan_to_num(x, nan=-math.inf).max(1).values
        low = torch.nan_to_num(x, nan=math.inf).min(1).values
        return torch.nan_to_num(top - low, nan=0.0, posinf=0.0, neginf=0.0)
    x = (spread(z64) + spread(t64)) * inv
    n = min(c // 64 + 1, 1100) + 24
    e = ((4 * x + 12 + n) * U)[:, None]
    _, rows, grad = formula(z, t, idx, temp, alpha, labels, scale)
    one = torch.full((b, c), 1.0)
    s = (torch.full((b,), 1.0 / max(b, 1)) if scale is None else scale.cpu()).double().abs()[:, None]
    # every probability in the gradient's terms is relatively exact to e; the
    # subtracted shares are those of the listed classes and the label
    top = torch.zeros((b, c), dtype=torch.float64)
    for i in range(b):
        here = (idx[i].cpu() >= 0) & (idx[i].cpu() < c) & (t64[i] != -math.inf)
        if here.any():
            top[i].index_add_(0, idx[i].cpu()[here], torch.softmax(t64[i][here] / temp, 0))
        if labels is not None and 0 <= labels[i] < c:
            top[i, labels[i]] += 1
    parts = s * (alpha * temp * (torch.softmax(torch.nan_to_num(z64 / temp, nan=0.0), 1) + top)
                 + (1 - alpha) * (torch.softmax(torch.nan_to_num(z64, nan=0.0), 1) + top))
    e_grad = 1.02 * (e * parts + 4 * U * parts) + half_step(g_dt) * grad.abs() * 1.02 + 1e-37 * one
    # log p and log q: errors of their arguments and sums, times T^2, weighted
    # by probabilities that add up to 1; the k-term sum over them
    lg = x + math.log(max(c, 2)) + 1
    e_row = (e[:, 0] * 2 + (idx.shape[1] / 64 + 20) * U) * (lg + 1) * max(temp * temp, 1.0) + 4 * U * rows.abs() + 1e-30
    return e_row, e_grad


def within(got, want, bound, what):
    got = got.double().cpu()
    off = (got - want).abs()
    bad = ~((off <= bound) | (got == want) | (got.isnan() & want.isnan()))
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, most {float((off / bound).max()):.3g} times the bound"


def inputs(seed, b, c, k, zdt=F32, tdt=F32, pad=True):
    gen = torch.Generator().manual_seed(seed)
    z = (torch.randn((b, c), generator=gen) * 2).to(zdt).to(DEV)
    t = (torch.randn((b, k), generator=gen) * 3).to(tdt)
    idx = torch.stack([torch.randperm(c, generator=gen)[torch.arange(k) % c] for _ in range(b)]) if b else torch.zeros((0, k), dtype=torch.int64)
    if pad:  # rows of every length, one of them empty
        n = torch.arange(b) % (k + 1)
        idx[(torch.arange(k)[None, :] >= n[:, None]) & (torch.arange(b)[:, None] % 3 == 0)] = -1
    labels = torch.randint(0, c, (b,), generator=gen)
    return z, t.to(DEV), idx.to(DEV), labels


def call(z, t, idx, temp, alpha=1.0, labels=None, scale=None, gdt=None, **kw):
    b, c = z.shape
    g = torch.full((b, c), 7.0, dtype=gdt or z.dtype, device=DEV)
    loss, rows = torch.full((1,), 7.0, device=DEV), torch.full((b,), 7.0, device=DEV)
    gnn.distill_topk(z, t, idx, temp, g, loss, rows, alpha=alpha, labels=labels.to(DEV) if labels is not None else None,
                     row_scale=scale, **kw)
    return loss, rows, g


def check(z, t, idx, temp, alpha=1.0, labels=None, scale=None, gdt=None, **kw):
    loss, rows, g = call(z, t, idx, temp, alpha, labels, scale, gdt, **kw)
    w_loss, w_rows, w_g = formula(z, t, idx, temp, alpha, labels, scale)
    e_rows, e_g = bounds(z, t, idx, temp, alpha, labels, scale, g.dtype)
    within(rows, w_rows, e_rows, "row losses")
    within(g, w_g, e_g, "gradient")
    s = torch.full((z.shape[0],), 1.0 / max(z.shape[0], 1)) if scale is None else scale.cpu()
    e_loss = (s.double().abs() * e_rows).sum() + (z.shape[0] / 256 + 16) * U * (s.double().abs() * w_rows.abs()).sum()
    within(loss, w_loss[None], e_loss[None] + 1e-37, "loss")
    return loss, rows, g


SIZES = [(1, 1, 1), (3, 2, 2), (5, 7, 3), (64, 47, 8), (33, 172, 5), (16, 255, 16), (9, 256, 4), (7, 1000, 64), (5, 1023, 33), (4, 1025, 100), (6, 2049, 10),
         (3, 4096, 128), (4, 8191, 7), (2, 10_000, 256), (3, 16_385, 64), (2, 32_768, 20), (1, 50_001, 64), (3, 65_537, 1000),
         (2, 131_072, 64), (1, 200_003, 1024), (1, 1 << 20, 3), (300, 3000, 6), (700, 10, 3),
         # long lists over few classes, every shape's longest row and the next one
         (40, 30, 112), (40, 30, 113), (9, 250, 454), (9, 250, 455), (3, 12, 1024), (20, 248, 9), (20, 249, 9), (9, 1016, 5),
         (9, 1017, 5), (6, 1528, 5), (6, 1529, 5), (3, 6136, 5), (3, 6145, 5), (2, 10_232, 5), (2, 18_433, 3), (130, 8192, 4),
         (140, 36_856, 3), (140, 36_865, 3), (129, 69_628, 3), (129, 73_725, 3), (129, 139_256, 3), (129, 139_257, 3), (2, 139_300, 3)]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("b, c, k", SIZES)
def test_loss_and_gradient(b, c, k, dt):
    z, t, idx, _ = inputs(b + c, b, c, k, dt, dt)
    check(z, t, idx, 1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("temp, alpha", [(2.0, 0.7), (1.0, 0.5), (4.0, 1.0), (0.5, 0.9), (3.0, 0.0)])
@pytest.mark.parametrize("b, c, k", [(64, 47, 8), (7, 1000, 64), (5, 4099, 33), (3, 65_537, 100), (2, 150_000, 64)])
def test_temperature_and_labels(b, c, k, temp, alpha, dt):
    z, t, idx, labels = inputs(b * c + k, b, c, k, dt, dt)
    labels[::3] = -1  # rows without a label
    labels[1::5] = c
    check(z, t, idx, temp, alpha, labels)


@pytest.mark.gpu
@pytest.mark.parametrize("b, c, k", [(9, 300, 8), (3, 40_000, 9)])
@pytest.mark.parametrize("zdt, tdt, gdt", [(F32, BF16, F32), (BF16, F32, F32), (F32, F32, BF16), (BF16, BF16, F32)])
def test_mixed_types(b, c, k, zdt, tdt, gdt):
    z, t, idx, labels = inputs(c, b, c, k, zdt, tdt)
    check(z, t, idx, 2.0, 0.5, labels, gdt=gdt)


@pytest.mark.gpu
@pytest.mark.parametrize("c", [50, 5000, 70_001])
def test_alpha_zero_is_the_cross_entropy(c):
    """With alpha = 0 the loss and gradient are those of softmax_ce."""
    z, t, idx, labels = inputs(c, 12, c, 4)
    loss, _, g = call(z, t, idx, 5.0, 0.0, labels)
    w_loss, w_g = torch.empty(1, device=DEV), torch.empty_like(g)
    if c <= gnn.GNN_MAX_DIM:
        gnn.softmax_ce(z, labels.to(DEV), None, w_g, w_loss)
    else:
        w_loss, _, w_g = (x.float().to(DEV) for x in formula(z, t, idx, 5.0, 0.0, labels))
    e_rows, e_g = bounds(z, t, idx, 5.0, 0.0, labels, None, F32)
    within(g, w_g.double().cpu(), 2 * e_g, "gradient")
    within(loss.view(1), w_loss.double().cpu().view(1), 2 * e_rows.mean()[None], "loss")


@pytest.mark.gpu
@pytest.mark.parametrize("c", [40, 3000, 100_000])
def test_the_same_class_twice(c):
    """Each entry of a class listed more than once counts."""
    z, t, idx, labels = inputs(c, 6, c, 12, pad=False)
    idx[0, :] = 5
    idx[1, 3], idx[1, 7], idx[1, 11] = idx[1, 0], idx[1, 0], idx[1, 0]
    idx[2, 1::2] = idx[2, 0::2]
    labels[3] = idx[3, 4].item()
    check(z, t, idx, 2.0, 0.6, labels)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("c", [60, 4000, 90_001])
def test_masked_values(c, dt):
    """Absent entries whose values are NaN or infinite, teacher values of
    -infinity and the type's lowest, rows with no entry, logits of -infinity."""
    z, t, idx, labels = inputs(c, 8, c, 6, dt, dt, pad=False)
    t[0, 2], idx[0, 2] = float("nan"), -1
    t[0, 3], idx[0, 3] = float("inf"), c
    t[0, 4], idx[0, 4] = 3.0, -(1 << 40)
    t[1, 1:] = -math.inf
    t[2, 3:] = torch.finfo(dt).min
    t[3] = -math.inf                # no entry at all
    idx[4] = -1                     # and none either
    z[5, ::2] = -math.inf           # classes masked out
    idx[5] = torch.arange(6) * 2 + 1
    labels[5] = 1
    z[6, idx[6, 0]] = -math.inf     # a listed class without probability: an infinite loss
    labels[6] = -1
    loss, rows, g = check(z, t, idx, 2.0, 0.5, labels)
    assert rows[6] == math.inf and g[6].isfinite().all() and loss.item() == math.inf
    assert torch.equal(rows[3:5] > 0, torch.tensor([True, True], device=DEV))  # their labels remain
    _, rows, g = check(z[:5], t[:5], idx[:5], 2.0)
    assert (rows[3:5] == 0).all() and (g[3:5] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("c", [60, 4000, 90_001])
def test_bad_rows_stay_alone(c):
    z, t, idx, labels = inputs(c, 6, c, 5, pad=False)
    z[0, c // 2], z[2, 0], z[4] = float("nan"), float("inf"), -math.inf
    scale = torch.full((6,), 0.5, device=DEV)
    loss, rows, g = call(z, t, idx, 1.0, 0.5, labels, scale)
    assert rows[[0, 2, 4]].isnan().all() and loss.isnan().all() and g[0].isnan().all()
    want = formula(z[1::2], t[1::2], idx[1::2], 1.0, 0.5, labels[1::2], scale[1::2])
    e_rows, e_g = bounds(z[1::2], t[1::2], idx[1::2], 1.0, 0.5, labels[1::2], scale[1::2], F32)
    within(rows[1::2], want[1], e_rows, "row losses")
    within(g[1::2], want[2], e_g, "gradient")
    # rows of scale 0 are not read
    scale[::2] = 0
    loss, rows, g = call(z, t, idx, 1.0, 0.5, labels, scale)
    assert (rows[::2] == 0).all() and (g[::2] == 0).all() and loss.isfinite().all()
    within(g[1::2], want[2], e_g, "gradient")


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("b, c, k", [(20, 47, 4), (9, 3001, 20), (5, 30_003, 64), (3, 131_073, 100), (1, 262_144, 9)])
def test_scales_in_place_and_loss_alone(b, c, k, dt):
    z, t, idx, labels = inputs(b + c, b, c, k, dt, dt)
    scale = torch.rand(b, device=DEV) * (torch.arange(b, device=DEV) % 4 != 1)
    loss, rows, g = check(z, t, idx, 2.0, 0.8, labels, scale)
    # the loss without the gradient, and the gradient over the logits
    l2, r2 = torch.empty((), device=DEV), torch.empty(b, device=DEV)
    gnn.distill_topk(z, t, idx, 2.0, None, l2, r2, alpha=0.8, labels=labels.to(DEV), row_scale=scale)
    assert torch.equal(l2, loss[0]) and torch.equal(r2, rows)
    over = z.clone()
    gnn.distill_topk(over, t, idx, 2.0, over, l2, None, alpha=0.8, labels=labels.to(DEV), row_scale=scale)
    assert torch.equal(over, g) and torch.equal(l2, loss[0])


@pytest.mark.gpu
@pytest.mark.parametrize("off", [1, 2, 3, 7])
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("c", [47, 2048, 4097, 70_000])
def test_any_alignment_of_the_element(c, dt, off):
    z, t, idx, labels = inputs(c + off, 5, c, 9, dt, dt)

    def moved(x):
        buf = torch.empty(x.numel() + 64, dtype=x.dtype, device=DEV)
        v = buf[off:off + x.numel()].view(x.shape)
        v.copy_(x)
        return v
    zz, g = moved(z), moved(torch.zeros_like(z))
    loss = torch.empty(1, device=DEV)
    gnn.distill_topk(zz, moved(t), moved(idx), 2.0, g, loss, None, alpha=0.5, labels=moved(labels.to(DEV)))
    _, _, want = formula(z, t, idx, 2.0, 0.5, labels)
    within(g, want, bounds(z, t, idx, 2.0, 0.5, labels, None, dt)[1], "gradient")
    assert torch.equal(zz, z)


@pytest.mark.gpu
def test_targets_pick_the_labels():
    z, t, idx, _ = inputs(4, 6, 30, 4)
    labels = torch.randint(0, 30, (100,))
    targets = torch.tensor([99, 0, 5, 5, 17, 42])
    loss, rows, g = call(z, t, idx, 1.0, 0.5, labels, targets=targets.to(DEV))
    want = call(z, t, idx, 1.0, 0.5, labels[targets])
    assert torch.equal(loss, want[0]) and torch.equal(rows, want[1]) and torch.equal(g, want[2])


@pytest.mark.gpu
@pytest.mark.parametrize("c, temp, alpha", [(25, 2.0, 1.0), (25, 1.0, 0.3), (5000, 3.0, 0.6)])
def test_gradient_against_differences(c, temp, alpha):
    z, t, idx, labels = inputs(c, 5, c, 8)
    _, _, g = call(z, t, idx, temp, alpha, labels)
    v = torch.randn(5, c, generator=torch.Generator().manual_seed(1), dtype=torch.float64)
    step = 1e-4
    up, down = (formula(z.double().cpu() + h * v, t, idx, temp, alpha, labels)[0] for h in (step, -step))
    slope = float((up - down) / (2 * step))
    # the products are of size temp / 5 at most in sum, each within 1e-5; the
    # difference's own error is a third derivative (below 10) times step^2
    assert abs(float((g.double().cpu() * v).sum()) - slope) <= 1e-5 * temp * max(1.0, abs(slope)) + 1e-6


@pytest.mark.gpu
def test_no_rows():
    loss = torch.full((1,), 3.0, device=DEV)
    gnn.distill_topk(torch.empty((0, 9), device=DEV), torch.empty((0, 2), device=DEV),
                     torch.empty((0, 2), dtype=torch.int64, device=DEV), 1.0, torch.empty((0, 9), device=DEV), loss)
    assert loss.item() == 0.0


@pytest.mark.gpu
@pytest.mark.parametrize("b, c, k", [(200, 300, 8), (3, 100_000, 64)])
def test_captured_and_on_another_stream(b, c, k):
    z, t, idx, labels = inputs(7, b, c, k, BF16)
    labels = labels.to(DEV)

    def buffers():
        return torch.zeros_like(z), torch.zeros(1, device=DEV), torch.zeros(b, device=DEV)

    def go(o, **kw):
        gnn.distill_topk(z, t, idx, 2.0, o[0], o[1], o[2], alpha=0.5, labels=labels, **kw)
    eager, replayed, side = buffers(), buffers(), buffers()
    go(replayed)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(replayed)
    stream = torch.cuda.Stream()
    for seed in range(4):
        z.copy_(inputs(50 + seed, b, c, k, BF16)[0])
        go(eager)
        graph.replay()
        stream.wait_stream(torch.cuda.current_stream())
        go(side, stream=stream)
        torch.cuda.synchronize()
        for x, y, w in zip(eager, replayed, side):
            assert torch.equal(x, y) and torch.equal(x, w)


@pytest.mark.gpu
def test_offsets_past_32_bits():
    b, c = 2100, 1 << 20
    z = torch.zeros((b, c), dtype=BF16, device=DEV)
    z[-2:, 7] = 3.0
    t, idx = torch.zeros((b, 1), device=DEV), torch.full((b, 1), 7, dtype=torch.int64, device=DEV)
    scale = torch.zeros(b, device=DEV)
    scale[-2:] = 1.0
    loss, rows, g = call(z, t, idx, 1.0, 1.0, None, scale)
    want = formula(z[-2:], t[-2:], idx[-2:], 1.0, 1.0, None, scale[-2:])
    e_rows, e_g = bounds(z[-2:], t[-2:], idx[-2:], 1.0, 1.0, None, scale[-2:], BF16)
    within(rows[-2:], want[1], e_rows, "row losses")
    within(g[-2:], want[2], e_g, "gradient")
    assert (rows[:-2] == 0).all() and not g[0].any() and not g[-3].any()


def test_refusals_on_the_host():
    lib = gnn.lib()
    fake, inval, unsup = 1 << 24, gnn.GNN_EINVAL, gnn.GNN_EUNSUPPORTED
    args = [fake, 0, 4, 10, fake, 0, fake, 3, 1.0, 1.0, None, None, None, fake + 4096, 0, None, fake, fake, 1 << 20, None]

    def f(**kw):
        a = list(args)
        for k, v in kw.items():
            a[int(k[1:])] = v
        return lib.gnn_distill_topk(*a)
    for at in (0, 4, 6, 16, 17):
        assert f(**{f"_{at}": None}) == inval
    for at in (1, 5, 14):
        assert f(**{f"_{at}": gnn.GNN_F16}) == unsup
    assert f(_2=-1) == inval and f(_2=1 << 40) == inval
    assert f(_3=0) == inval and f(_3=gnn.GNN_MAX_CLASSES + 1) == inval
    assert f(_7=0) == inval and f(_7=gnn.GNN_MAX_TOP + 1) == inval
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        assert f(_8=bad) == inval
    for bad in (-0.1, 1.1, float("nan")):
        assert f(_9=bad) == inval
    for at in (0, 4, 6, 13, 16, 17):
        assert f(**{f"_{at}": fake + 2}) == inval
    assert f(_13=fake, _14=gnn.GNN_BF16) == inval and b"same dtype" in lib.gnn_last_error()
    assert f(_18=8) == gnn.GNN_ESIZE
    nb = gnn._sz()
    assert lib.gnn_distill_topk_workspace_size(4, 0, 1, gnn.ctypes.byref(nb)) == inval
    assert lib.gnn_distill_topk_workspace_size(4, 5, 1, None) == inval
    assert lib.gnn_distill_topk_workspace_size(4, 5, 1, gnn.ctypes.byref(nb)) == gnn.GNN_OK


@pytest.mark.gpu
def test_refusals_of_the_binding():
    z, t, idx, labels = inputs(1, 4, 10, 3)
    loss, g = torch.empty(1, device=DEV), torch.empty_like(z)
    for bad in (lambda: gnn.distill_topk(z[0], t, idx, 1.0, g, loss), lambda: gnn.distill_topk(z, t[:3], idx, 1.0, g, loss),
                lambda: gnn.distill_topk(z, t, idx.int(), 1.0, g, loss),
                lambda: gnn.distill_topk(z, t, idx[:, :2], 1.0, g, loss),
                lambda: gnn.distill_topk(z.half(), t, idx, 1.0, g, loss),
                lambda: gnn.distill_topk(z, t, idx, 1.0, g.t(), loss),
                lambda: gnn.distill_topk(z, t, idx, 1.0, g, loss.double()),
                lambda: gnn.distill_topk(z, t, idx, 1.0, g, loss, labels=labels),
                lambda: gnn.distill_topk(z, t, idx, 1.0, g, loss, labels=labels[:2].to(DEV)),
                lambda: gnn.distill_topk(z.cpu(), t, idx, 1.0, g, loss)):
        with pytest.raises(ValueError):
            bad()
    for kw in (dict(temperature=0.0), dict(temperature=1.0, alpha=2.0)):
        with pytest.raises(gnn.GnnError):
            gnn.distill_topk(z, t, idx, g_out=g, loss_out=loss, **kw)
