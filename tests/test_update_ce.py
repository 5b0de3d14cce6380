"""The softmax cross-entropy of an update with many classes, and its gradients,
against the formulas in 64 bits."""
import ctypes
import math

import pytest
import torch

from paper_2303_00158_amd import gnn

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24  # half a step of fp32, relative


def half_step(dt):
    return torch.finfo(dt).eps / 2


def rand(gen, *shape, dtype=F32, scale=1.0):
    return (torch.randn(shape, generator=gen) * scale).to(dtype).to(DEV)


def misaligned(t, off):
    """t's values at an address `off` elements past an aligned one."""
    buf = torch.empty(t.numel() + 64, dtype=t.dtype, device=t.device)
    v = buf[off:off + t.numel()].view(t.shape)
    v.copy_(t)
    return v


def product_off(x, y, n):
    """How far a sum of n products of x (m x n) and y (n x q) may be off in
    fp32, in any order."""
    return (n + 4) * U * (x.abs() @ y.abs())


def exact(a, wt, bias, labels, scale, gemm):
    """(loss, row losses, dwt, db, d_a) in 64 bits, and how far each may be off
    before its own rounding."""
    b, c = a.shape[0], wt.shape[0]
    if gemm == gnn.GNN_BF16:
        a, wt = a.to(BF16), wt.to(BF16)
    s = torch.full((b,), 1.0 / max(b, 1), device=DEV) if scale is None else scale
    live = (labels >= 0) & (labels < c) & (s != 0)
    s = torch.where(live, s, 0.0).double()
    y = torch.where(live, labels, 0)
    a = torch.where(live[:, None], a.double(), 0.0)
    wt = wt.double()
    z = a @ wt.t()
    e_z = product_off(a, wt.t(), a.shape[1])
    if bias is not None:
        z = z + bias.double()
        e_z = e_z + U * torch.where(z.isfinite(), z.abs(), 0.0)
    top = z.amax(1, keepdim=True)
    far = torch.where(z.isfinite(), (z - top).abs(), 0.0)
    ez = torch.exp(z - top)
    total = ez.sum(1, keepdim=True)
    p = ez / total
    # an exponential's argument (its rounding, and what it was made of) and its own error; the sum's additions;
    # the logarithm; the sum of the two
    lse = top + torch.log(total)
    adds = 2 * math.ceil(c / 256) + 40
    e_lse = (p * (e_z + U * (3 * far + 6))).sum(1, keepdim=True) + (adds + 4) * U + 2 * U * (lse.abs() + top.abs())
    z_y = z.gather(1, y[:, None])
    row = torch.where(live, (lse - z_y)[:, 0], 0.0)
    e_row = torch.where(live, (e_lse + e_z.gather(1, y[:, None]) + U * (lse - z_y).abs())[:, 0], 0.0) * 1.01
    loss = (row * s).sum()
    e_loss = (e_row * s.abs()).sum() + (b / 256 + 40) * U * (row * s).abs().sum()
    e_p = p * (e_z + e_lse + U * (3 * (z - lse).abs().nan_to_num(0.0, 0.0, 0.0) + 8))
    hot = torch.zeros_like(p).scatter_(1, y[:, None], live.double()[:, None])
    dz = s[:, None] * (p - hot)
    dz[~live] = 0.0
    e_dz = s.abs()[:, None] * (e_p + 2 * U * (p - hot).abs()) + 1e-37
    e_dz[~live] = 0.0
    db = dz.sum(0)
    e_db = e_dz.sum(0) + (b + 2) * U * dz.abs().sum(0)
    if gemm == gnn.GNN_BF16:
        e_dz = e_dz + half_step(BF16) * (dz.abs() + e_dz)
    dwt, d_a = dz.t() @ a, dz @ wt
    e_dwt = e_dz.t() @ a.abs() + product_off(dz.t(), a, b)
    e_da = e_dz @ wt.abs() + product_off(dz, wt, c)
    return (loss, row, dwt, db, d_a), (e_loss, e_row, e_dwt * 1.02, e_db * 1.01, e_da * 1.02)


def within(got, want, off, what):
    got = got.double().reshape(want.shape)
    bound = off + half_step(F32) * 2 * want.abs() + 1e-36
    same = (got == want) | (got.isnan() & want.isnan())
    bad = ~(((got - want).abs() <= bound) | same)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, most {float(((got - want).abs() / bound)[bad].max()):.3g} times the bound"


def check(outs, want, offs):
    for name, got, w, off in zip(("loss", "row_loss", "dwt", "db", "d_a"), outs, want, offs):
        if got is not None:
            within(got, w, off + half_step(got.dtype) * (w.abs() + off) * 1.01, name)


def call(a, wt, bias, labels, gemm, gdt=None, dwdt=None, scale=None, grads=True, off=0, **kw):
    b, k = a.shape
    c = wt.shape[0]
    gdt, dwdt = gdt or (BF16 if gemm == gnn.GNN_BF16 else F32), dwdt or (BF16 if gemm == gnn.GNN_BF16 else F32)

    def full(*shape, dt=F32):
        return misaligned(torch.full(shape, 7.0, dtype=dt, device=DEV), off)
    loss, row = full(1), full(b)
    dwt, db, d_a = (full(c, k, dt=dwdt), full(c), full(b, k, dt=gdt)) if grads else (None, None, None)
    assert gnn.update_ce(a, wt, bias, labels, loss, gemm, row_loss=row, d_a=d_a, dwt=dwt, db=db, row_scale=scale, **kw) is loss
    return loss, row, dwt, db, d_a


def problem(gen, b, k, c, adt=F32, wdt=F32, off=0):
    wt = rand(gen, c, k, scale=1 / math.sqrt(k))
    labels = torch.randint(0, c, (b,), generator=gen).to(DEV)
    a = rand(gen, b, k) + 3 * wt[labels]
    return misaligned(a.to(adt), off), misaligned(wt.to(wdt), off), misaligned(rand(gen, c, scale=0.3), off), labels


SIZES = [(1, 1, 1), (1, 1, 2), (2, 3, 3), (5, 2, 47), (1, 64, 1000), (47, 31, 63), (64, 64, 64), (65, 100, 65), (100, 8, 257), (255, 33, 172),
         (257, 256, 47), (1024, 256, 47), (300, 602, 256), (129, 1024, 1000), (33, 100, 4099), (7, 520, 32_003), (1461, 64, 153), (600, 257, 1025),
         (1, 4096, 3001), (3000, 16, 20), (20_000, 8, 5), (40, 5000, 10), (2, 100, 131_072), (1023, 24, 2049), (1024, 24, 2049), (3, 40, 2048)]


@pytest.mark.gpu
@pytest.mark.parametrize("gemm", [gnn.GNN_F32, gnn.GNN_BF16])
@pytest.mark.parametrize("b, k, c", SIZES)
def test_loss_and_gradients(b, k, c, gemm):
    gen = torch.Generator().manual_seed(b + 7 * k + 31 * c)
    dt = BF16 if gemm == gnn.GNN_BF16 else F32
    a, wt, bias, labels = problem(gen, b, k, c, dt, dt)
    want, offs = exact(a, wt, bias, labels, None, gemm)
    check(call(a, wt, bias, labels, gemm), want, offs)
    check(call(a, wt, bias, labels, gemm, grads=False), want, offs)


@pytest.mark.gpu
@pytest.mark.parametrize("gemm", [gnn.GNN_F32, gnn.GNN_BF16])
@pytest.mark.parametrize("b, k, c", [(8200, 40, 17_000), (100_000, 24, 1500), (600_001, 8, 520), (3000, 72, 50_000),
                                     (1500, 1536, 9000), (20_000, 1541, 14_000), (70_000, 1536, 2000)])
def test_several_pieces(b, k, c, gemm):
    gen = torch.Generator().manual_seed(b)
    dt = BF16 if gemm == gnn.GNN_BF16 else F32
    a, wt, bias, labels = problem(gen, b, k, c, dt, dt)
    labels[:3] = torch.tensor([0, c - 1, -1], device=DEV)
    want, offs = exact(a, wt, bias, labels, None, gemm)
    check(call(a, wt, bias, labels, gemm), want, offs)
    check(call(a, wt, bias, labels, gemm, grads=False), want, offs)


@pytest.mark.gpu
@pytest.mark.parametrize("adt", [F32, BF16])
@pytest.mark.parametrize("wdt", [F32, BF16])
@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("gemm, gdt, dwdt", [(gnn.GNN_F32, F32, F32), (gnn.GNN_BF16, F32, F32), (gnn.GNN_BF16, BF16, F32),
                                            (gnn.GNN_BF16, F32, BF16)])
@pytest.mark.parametrize("b, k, c", [(77, 64, 300), (130, 100, 47), (66, 13, 1001)])
def test_types_and_alignments(b, k, c, gemm, gdt, dwdt, off, wdt, adt):
    gen = torch.Generator().manual_seed(k)
    a, wt, bias, labels = problem(gen, b, k, c, adt, wdt, off)
    want, offs = exact(a, wt, bias, labels, None, gemm)
    check(call(a, wt, bias, labels, gemm, gdt, dwdt, off=off), want, offs)
    check(call(a, wt, bias, labels, gemm, grads=False), want, offs)


@pytest.mark.gpu
@pytest.mark.parametrize("gemm", [gnn.GNN_F32, gnn.GNN_BF16])
@pytest.mark.parametrize("b, k, c", [(100, 64, 300), (300, 40, 2000)])
def test_rows_that_take_no_part(b, k, c, gemm):
    gen = torch.Generator().manual_seed(b)
    dt = BF16 if gemm == gnn.GNN_BF16 else F32
    a, wt, bias, labels = problem(gen, b, k, c, dt, dt)
    scale = torch.rand(b, generator=gen).to(DEV) - 0.2
    scale[::7] = 0.0
    labels[3::11] = torch.tensor([-1, c, 2 ** 50, -2 ** 60], device=DEV).repeat(b)[:len(labels[3::11])]
    dead = (scale == 0) | (labels < 0) | (labels >= c)
    want, offs = exact(a, wt, bias, labels, scale, gemm)
    a[dead] = torch.tensor([math.nan, math.inf, -math.inf, 1e38], device=DEV).to(dt).repeat(b)[:int(dead.sum())][:, None]
    outs = call(a, wt, bias, labels, gemm, scale=scale)
    check(outs, want, offs)
    assert (outs[1][dead] == 0).all() and (outs[4][dead] == 0).all()
    check(call(a, wt, bias, labels, gemm, scale=scale, grads=False), want, offs)
    # each gradient alone
    for name, i in (("dwt", 2), ("db", 3), ("d_a", 4)):
        out = torch.full_like(outs[i], 7.0)
        gnn.update_ce(a, wt, bias, labels, outs[0], gemm, row_scale=scale, **{name: out})
        assert torch.equal(out, outs[i]), name
    # in place of the activations
    again = a.clone()
    gnn.update_ce(again, wt, bias, labels, outs[0], gemm, d_a=again, row_scale=scale)
    assert torch.equal(again, outs[4])
    # nobody takes part
    outs = call(a, wt, bias, torch.full_like(labels, -1), gemm, scale=scale)
    assert all((x == 0).all() for x in outs)


@pytest.mark.gpu
@pytest.mark.parametrize("gemm", [gnn.GNN_F32, gnn.GNN_BF16])
def test_labels_of_targets(gemm):
    gen = torch.Generator().manual_seed(2)
    a, wt, bias, _ = problem(gen, 90, 32, 50)
    every, targets = torch.randint(0, 50, (1000,), generator=gen).to(DEV), torch.randperm(1000, generator=gen)[:90].to(DEV)
    want, offs = exact(a, wt, bias, every[targets], None, gemm)
    check(call(a, wt, bias, every, gemm, targets=targets), want, offs)


@pytest.mark.gpu
@pytest.mark.parametrize("gemm", [gnn.GNN_F32, gnn.GNN_BF16])
def test_no_rows_and_no_bias(gemm):
    gen = torch.Generator().manual_seed(3)
    a, wt, bias, labels = problem(gen, 70, 48, 333)
    want, offs = exact(a, wt, None, labels, None, gemm)
    check(call(a, wt, None, labels, gemm), want, offs)
    outs = call(a[:0], wt, bias, labels[:0], gemm)
    assert (outs[0] == 0).all() and (outs[2] == 0).all() and (outs[3] == 0).all()
    a, wt, bias, labels = problem(gen, 0, 48, 5000)
    outs = call(a, wt, bias, labels, gemm)
    assert (outs[0] == 0).all() and (outs[2] == 0).all() and (outs[3] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("gemm", [gnn.GNN_F32, gnn.GNN_BF16])
@pytest.mark.parametrize("c", [40, 700])
def test_large_logits_and_classes_that_are_shut(c, gemm):
    gen = torch.Generator().manual_seed(c)
    dt = BF16 if gemm == gnn.GNN_BF16 else F32
    a, wt, bias, labels = problem(gen, 150, 24, c, dt, dt)
    bias = bias * 1000 + 5000
    bias[::3] = -math.inf
    labels = labels // 3 * 3 + 1  # classes that are open
    labels.clamp_(max=(c - 2) // 3 * 3 + 1)
    want, offs = exact(a, wt, bias, labels, None, gemm)
    outs = call(a, wt, bias, labels, gemm)
    check(outs, want, offs)
    assert (outs[3][::3] == 0).all() and (outs[2][::3] == 0).all()
    # a label that is shut: an infinite loss, and a gradient that is not
    labels[5] = 3
    want, offs = exact(a, wt, bias, labels, None, gemm)
    outs = call(a, wt, bias, labels, gemm)
    assert outs[0].isinf().all() and outs[1][5] == math.inf and outs[1].isfinite().sum() == 149
    check((None, None) + outs[2:], want, offs)
    # no class is open, or one is infinite: that is no number
    for value in (-math.inf, math.inf, math.nan):
        bad = torch.full_like(bias, -math.inf)
        bad[7] = value
        assert call(a, wt, bad, labels, gemm)[1].isnan().all()
    # a row's own
    a[9, 0] = math.inf
    outs = call(a, wt, bias, torch.where(torch.arange(150, device=DEV) == 5, -1, labels), gemm)
    others = torch.arange(150, device=DEV) != 9
    assert outs[1][9].isnan() and outs[1][others].isfinite().all() and outs[4][others].isfinite().all()


@pytest.mark.gpu
@pytest.mark.parametrize("b, k, c", [(6, 5, 9), (70, 20, 300)])
def test_gradients_against_differences(b, k, c):
    gen = torch.Generator().manual_seed(4)
    a, wt, bias, labels = problem(gen, b, k, c)
    scale = torch.rand(b, generator=gen).to(DEV) + 0.5
    outs = call(a, wt, bias, labels, gnn.GNN_F32, scale=scale)
    (_, offs) = exact(a, wt, bias, labels, scale, gnn.GNN_F32)
    h = 2.0 ** -5
    for got, x, other in ((outs[4], a, wt), (outs[2], wt, a), (outs[3], bias, torch.ones(1, device=DEV))):
        for at in ((0,) * x.dim(), tuple(n - 1 for n in x.shape), tuple(n // 2 for n in x.shape)):
            ends = []
            for sign in (1, -1):
                y = x.clone()
                y[at] += sign * h
                args = [y if t is x else t for t in (a, wt, bias)]
                ends.append((float(call(*args, labels, gnn.GNN_F32, scale=scale, grads=False)[0]), float(y[at])))
            slope = (ends[0][0] - ends[1][0]) / (ends[0][1] - ends[1][1])
            # the third derivative of a log sum exp along a direction of size d is at most d^3; a difference's own error
            d = float(other.abs().max())
            bound = float(scale.sum()) * d ** 3 * h * h / 6 + 2 * float(offs[0]) / (2 * h) + 1e-4 * abs(slope)
            assert abs(slope - float(got[at])) <= bound, (at, slope, float(got[at]), bound)


@pytest.mark.gpu
@pytest.mark.parametrize("gemm", [gnn.GNN_F32, gnn.GNN_BF16])
@pytest.mark.parametrize("b, k, c", [(200, 64, 900), (9000, 16, 16_000)])
def test_the_same_bits_again_also_from_a_graph_on_another_stream(b, k, c, gemm):
    gen = torch.Generator().manual_seed(1)
    dt = BF16 if gemm == gnn.GNN_BF16 else F32
    a, wt, bias, labels = problem(gen, b, k, c, dt, dt)
    first = call(a, wt, bias, labels, gemm)
    ws = gnn.update_ce_workspace(a, wt, gemm)
    ws.fill_(0xff)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        second = call(a, wt, bias, labels, gemm, ws=ws)
    stream.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(first, second))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        gnn.update_ce(a, wt, bias, labels, second[0], gemm, row_loss=second[1], dwt=second[2], db=second[3], d_a=second[4], ws=ws)
    for n in range(3):
        labels.copy_(labels.roll(1))
        bias.neg_()
        first = call(a, wt, bias, labels, gemm)
        ws.fill_(n)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(first, second)), n


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """2.2e9 weights: the first, the last and the rows around 2^31 values against 64 bits."""
    b, k, c = 3, 2200, 1_000_003
    gen = torch.Generator(device=DEV).manual_seed(1)
    wt = torch.empty((c, k), dtype=BF16, device=DEV)
    for at in range(0, c, 100_000):
        wt[at:at + 100_000] = torch.randn((min(100_000, c - at), k), generator=gen, device=DEV) / math.sqrt(k)
    a = torch.randn((b, k), generator=gen, device=DEV).to(BF16)
    labels = torch.tensor([0, c - 1, 976_128], device=DEV)  # row 976,128 has value 2^31
    loss, row, dwt, db = torch.empty(1, device=DEV), torch.empty(b, device=DEV), torch.empty_like(wt), torch.empty(c, device=DEV)
    d_a = torch.empty((b, k), device=DEV)
    gnn.update_ce(a, wt, None, labels, loss, gnn.GNN_BF16, row_loss=row, d_a=d_a, dwt=dwt, db=db)
    z = torch.cat([a.double() @ wt[at:at + 100_000].double().t() for at in range(0, c, 100_000)], 1)
    lse = torch.logsumexp(z, 1)
    want = lse - z.gather(1, labels[:, None])[:, 0]
    # logits are off by (k + 4) U of their terms' sizes (about 28 for the normal ones here), the sum by its additions
    off = (k + 4) * U * float((a.double().abs() @ wt[:1000].double().abs().t()).max()) * 1.5
    assert ((row.double() - want).abs() <= 2 * off + (2 * math.ceil(c / 256) + 60) * U).all()
    dz = torch.exp(z - lse[:, None])
    dz[torch.arange(b, device=DEV), labels] -= 1
    dz /= b
    e = 2 * off + (2 * math.ceil(c / 256) + 100) * U
    assert ((db.double() - dz.sum(0)).abs() <= e * dz.abs().sum(0) + 1e-30).all()
    for at in (0, 1, 976_127, 976_128, 976_129, c - 2, c - 1):
        w = dz[:, at] @ a.double()
        assert ((dwt[at].double() - w).abs() <= (dz[:, at].abs() @ a.double().abs()) * (e + 2.0 ** -8 * 1.1) + w.abs() * 2.0 ** -8 * 1.1).all(), at
    w, size = torch.zeros((b, k), dtype=torch.float64, device=DEV), torch.zeros((b, k), dtype=torch.float64, device=DEV)
    for at in range(0, c, 100_000):
        w += dz[:, at:at + 100_000] @ wt[at:at + 100_000].double()
        size += dz[:, at:at + 100_000].abs() @ wt[at:at + 100_000].double().abs()
    assert ((d_a.double() - w).abs() <= size * (e + 2.0 ** -8 * 1.1 + (c + 4) * U)).all()


# --- refusals ---------------------------------------------------------------

BUF = ctypes.create_string_buffer(1 << 16)
P = (ctypes.addressof(BUF) + 255) // 256 * 256  # any address: a refused call reads nothing


@pytest.mark.parametrize("change, code, what", [
    (dict(adt=2), gnn.GNN_EUNSUPPORTED, "dtypes"), (dict(wdt=3), gnn.GNN_EUNSUPPORTED, "dtypes"),
    (dict(gdt=2), gnn.GNN_EUNSUPPORTED, "dtypes"), (dict(dwdt=-1), gnn.GNN_EUNSUPPORTED, "dtypes"),
    (dict(gemm=2), gnn.GNN_EUNSUPPORTED, "dtypes"), (dict(gdt=1), gnn.GNN_EUNSUPPORTED, "GNN_F32 products"),
    (dict(dwdt=1), gnn.GNN_EUNSUPPORTED, "GNN_F32 products"),
    (dict(b=-1), gnn.GNN_EINVAL, "bad b"), (dict(b=1 << 24), gnn.GNN_EINVAL, "bad b"), (dict(k=0), gnn.GNN_EINVAL, "k out"),
    (dict(k=65_537), gnn.GNN_EINVAL, "k out"), (dict(c=0), gnn.GNN_EINVAL, "c out"),
    (dict(c=(1 << 20) + 1), gnn.GNN_EINVAL, "c out"), (dict(a=None), gnn.GNN_EINVAL, "NULL"), (dict(wt=None), gnn.GNN_EINVAL, "NULL"),
    (dict(labels=None), gnn.GNN_EINVAL, "NULL"), (dict(loss=None), gnn.GNN_EINVAL, "NULL"),
    (dict(dwt=P + 1024), gnn.GNN_EINVAL, "dwt must"), (dict(dwt=P), gnn.GNN_EINVAL, "dwt must"), (dict(dwt=P + 2048), gnn.GNN_EINVAL, "dwt must"),
    (dict(d_a=P + 1024), gnn.GNN_EINVAL, "d_a must"), (dict(d_a=P, adt=1), gnn.GNN_EINVAL, "d_a must"),
    (dict(a=P + 2), gnn.GNN_EINVAL, "misaligned"), (dict(wt=P + 1026), gnn.GNN_EINVAL, "misaligned"),
    (dict(bias=P + 1), gnn.GNN_EINVAL, "misaligned"), (dict(labels=P + 4), gnn.GNN_EINVAL, "misaligned"),
    (dict(targets=P + 4), gnn.GNN_EINVAL, "misaligned"), (dict(scale=P + 2), gnn.GNN_EINVAL, "misaligned"),
    (dict(row=P + 2), gnn.GNN_EINVAL, "misaligned"), (dict(db=P + 2), gnn.GNN_EINVAL, "misaligned"),
    (dict(ws=None), gnn.GNN_EINVAL, "ws"), (dict(ws=P + 128), gnn.GNN_EINVAL, "ws"), (dict(bytes=1000), gnn.GNN_ESIZE, "workspace"),
])
def test_refusals(change, code, what):
    a = dict(a=P, adt=0, b=4, k=8, wt=P + 1024, wdt=0, bias=None, c=10, labels=P, targets=None, scale=None, gemm=0, row=None, loss=P + 4096,
             d_a=P + 2048, gdt=0, dwt=P + 3200, dwdt=0, db=None, ws=P, bytes=1 << 40) | change
    got = gnn.lib().gnn_update_ce(*a.values(), None)
    assert got == code and what in gnn.lib().gnn_last_error().decode()


def test_workspace_sizes():
    def size(*args):
        nb = ctypes.c_size_t()
        assert gnn.lib().gnn_update_ce_workspace_size(*args, ctypes.byref(nb)) == gnn.GNN_OK
        return nb.value
    # a piece, not the whole: 100,000 rows of 1,000,000 classes would have 400 GB of logits
    assert size(100_000, 256, 1_000_000, gnn.GNN_BF16, 1) < 4 << 30
    assert 0 < size(0, 8, 10, gnn.GNN_F32, 1) <= size(10, 8, 10, gnn.GNN_F32, 1)
    for gemm in (gnn.GNN_F32, gnn.GNN_BF16):  # no rows and a long reduction over the classes
        assert size(0, 8, 100_000, gemm, 1) > 0
    assert size(1000, 64, 500, gnn.GNN_F32, 0) <= size(1000, 64, 500, gnn.GNN_F32, 1)
    assert gnn.lib().gnn_update_ce_workspace_size(1, 8, 10, 0, 1, None) == gnn.GNN_EINVAL
    nb = ctypes.c_size_t()
    assert gnn.lib().gnn_update_ce_workspace_size(1, 8, 10, 3, 1, ctypes.byref(nb)) == gnn.GNN_EUNSUPPORTED
    assert gnn.lib().gnn_update_ce_workspace_size(1, 8, 0, 0, 1, ctypes.byref(nb)) == gnn.GNN_EINVAL


def test_the_binding_refuses_what_is_not_on_a_gpu():
    with pytest.raises(ValueError, match="GPU"):
        gnn.update_ce(torch.zeros(3, 8), torch.zeros(4, 8), None, torch.zeros(3, dtype=torch.int64), torch.zeros(1), gnn.GNN_F32)


@pytest.mark.gpu
def test_the_binding_refuses_wrong_tensors():
    a, wt, y, loss = torch.zeros((3, 8), device=DEV), torch.zeros((4, 8), device=DEV), torch.zeros(3, dtype=torch.int64, device=DEV), torch.zeros(1, device=DEV)
    for bad in (dict(a=a.half()), dict(wt=wt[:, :4]), dict(wt=wt.t()), dict(bias=a[0]), dict(labels=y.int()), dict(labels=y[:2]),
                dict(loss_out=loss.double()), dict(row_loss=loss), dict(d_a=wt), dict(dwt=a), dict(db=a[0]), dict(row_scale=loss),
                dict(targets=y[:1]), dict(ws=a), dict(labels=y.cpu())):
        args = dict(a=a, wt=wt, bias=None, labels=y, loss_out=loss, gemm_dtype=gnn.GNN_F32) | bad
        with pytest.raises(ValueError):
            gnn.update_ce(**args)
    with pytest.raises(gnn.GnnError, match="workspace"):
        gnn.update_ce(a, wt, None, y, loss, gnn.GNN_F32, ws=torch.empty(256, dtype=torch.uint8, device=DEV))
