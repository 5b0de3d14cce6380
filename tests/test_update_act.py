"""The update with an activation and a residual, forward and backward, against
the formulas in 64 bits."""
import math

import pytest
import torch

from paper_2303_00158_amd import gnn

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
ACTS = {"none": gnn.GNN_ACT_NONE, "relu": gnn.GNN_ACT_RELU, "gelu": gnn.GNN_ACT_GELU,
        "gelu_tanh": gnn.GNN_ACT_GELU_TANH, "silu": gnn.GNN_ACT_SILU}


def half_step(dt):
    return torch.finfo(dt).eps / 2


def act64(z, name):
    if name == "relu":
        return z.clamp(min=0)
    if name == "gelu":
        return z * torch.special.ndtr(z)
    if name == "gelu_tanh":
        # (1 + tanh u) / 2 = sigmoid(2 u); the sum itself is 0 in 64 bits from u = -19 on
        return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def slope64(z, name):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = torch.sigmoid(z)
        return s + z * s * (1 - s)
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (z + 0.044715 * z ** 3))
    return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)


def act_error(z, name):
    """The activation's own error: the normal distribution's is 7.5e-8 by its
    formula and 4 U by its roundings; a sigmoid's argument x has 4 roundings,
    its exponential and quotient 8 U."""
    if name == "gelu":
        return z.abs() * (7.5e-8 + 4 * U)
    if name in ("gelu_tanh", "silu"):
        x = (2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3) if name == "gelu_tanh" else z).abs().clamp(max=90)
        return act64(z, name).abs() * (4 * x + 8) * U + z.abs() * 2.0 ** -126
    return torch.zeros_like(z)


def operands(a_self, a_nbr, w, wt, gemm):
    """A and W in 64 bits as the products read them."""
    a = a_self if a_nbr is None else torch.cat([a_self, a_nbr], 1)
    if gemm == gnn.GNN_F32:
        return a.double(), w.double()
    return a.bfloat16().double(), (wt.t() if wt is not None else w.bfloat16()).double()


def within(got, want, bound, what):
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, most {float((off / bound).max()):.3g} times the bound"


def check_forward(o, a, w, bias, residual, name, odt, rows=None):
    n = a.shape[0] if rows is None else rows
    z = a[:n] @ w
    size = a[:n].abs() @ w.abs()
    if bias is not None:
        z, size = z + bias.double(), size + bias.double().abs()
    e_z = (w.shape[0] + 4) * U * size
    y = act64(z, name)
    out = y + residual[:n].double() if residual is not None else y
    # the steepest slope of these activations is below 1.13
    e_out = 1.13 * e_z + act_error(z, name) + 2 * U * (y.abs() + out.abs())
    within(o["out"][:n], out, 1.01 * (e_out + half_step(odt) * (out.abs() + e_out)) + 1e-37, "out")
    if o["z"] is not None:
        within(o["z"][:n], z, 1.01 * (e_z + half_step(odt) * (z.abs() + e_z)) + 1e-37, "z")


def check_backward(o, a, w, z, g, name, gemm, gdt, dwdt, rows=None):
    n = a.shape[0] if rows is None else rows
    a, z, g = a[:n], z[:n].double() if z is not None else None, g[:n].double()
    d = g * slope64(z, name) if z is not None else g
    # a slope is within 1e-6: the activation's error above, and its own
    # exponential's, which is off by z^2 / 2 U where it is exp(-z^2 / 2)
    e_d = g.abs() * (0.0 if name in ("none", "relu") else 1e-6) + 2 * U * d.abs()
    e_op = e_d + (half_step(BF16) * (d.abs() + e_d) if gemm == gnn.GNN_BF16 else 0.0)
    db, e_db = d.sum(0), e_d.sum(0) + (n + 4) * U * d.abs().sum(0)
    dw, e_dw = a.t() @ d, a.t().abs() @ e_op + (n + 4) * U * (a.t().abs() @ (d.abs() + e_op))
    within(o["dw"], dw, 1.01 * (e_dw + half_step(dwdt) * (dw.abs() + e_dw)) + 1e-37, "dw")
    if o["db"] is not None:
        within(o["db"], db, 1.01 * e_db + 1e-37, "db")
    if o["d_a"] is not None:
        da, e_da = d @ w.t(), e_op @ w.t().abs() + (w.shape[1] + 4) * U * ((d.abs() + e_op) @ w.t().abs())
        within(o["d_a"][:n], da, 1.01 * (e_da + half_step(gdt) * (da.abs() + e_da)) + 1e-37, "d_a")


def rand(gen, *shape, dtype=F32, scale=1.0):
    return (torch.randn(shape, generator=gen) * scale).to(dtype).to(DEV)


def forward(a_self, a_nbr, w, wt, bias, name, gemm, odt, residual=None, keep=True, **kw):
    rows = a_self.shape[0]
    n = w.shape[1] if w is not None else wt.shape[0]
    o = {"out": torch.full((rows, n), 7.0, dtype=odt, device=DEV),
         "z": torch.full((rows, n), 7.0, dtype=odt, device=DEV) if keep else None}
    got = gnn.update_fwd_act(a_self, a_nbr, w, bias, o["out"], ACTS[name], gemm, residual=residual, z=o["z"], wt=wt, **kw)
    assert got is o["out"]
    return o


def backward(a_self, a_nbr, w, wt, z, g, name, gemm, dwdt, input_grad=True, bias_grad=True, **kw):
    rows, K = a_self.shape[0], a_self.shape[1] * (1 if a_nbr is None else 2)
    n = g.shape[1]
    o = {"dw": torch.full((K, n), 7.0, dtype=dwdt, device=DEV), "db": torch.full((n,), 7.0, device=DEV) if bias_grad else None,
         "d_a": torch.full((rows, K), 7.0, dtype=g.dtype, device=DEV) if input_grad else None}
    gnn.update_bwd_act(a_self, a_nbr, w, z, g, o["dw"], o["db"], o["d_a"], ACTS[name], gemm, wt=wt, **kw)
    return o


# rows, K, n_out: about each tile, chunk and vector width; few rows and many
SIZES = [(1, 1, 1), (1, 8, 16), (2, 7, 3), (1, 100, 47), (1, 4096, 512), (1, 1000, 1001), (3, 257, 129), (8, 512, 256), (15, 64, 64), (16, 96, 100),
         (17, 128, 72), (31, 33, 31), (32, 1024, 1024), (33, 200, 256), (48, 520, 264), (63, 100, 65), (64, 640, 320), (65, 72, 200), (100, 2056, 136),
         (127, 31, 8), (128, 256, 128), (129, 40, 1000), (200, 1001, 777), (255, 64, 257), (256, 512, 512), (257, 1536, 520),
         (300, 36, 24), (511, 1024, 255), (513, 260, 768), (1000, 602, 256), (1461, 64, 47), (1500, 24, 1025), (2049, 512, 640),
         (2100, 1032, 1032), (4097, 200, 256), (9000, 128, 72), (70_000, 8, 4)]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("name", list(ACTS))
@pytest.mark.parametrize("m, k, n", SIZES)
def test_forward(m, k, n, name, dt):
    gen = torch.Generator().manual_seed(m + 3 * k + 5 * n)
    a, w, bias = rand(gen, m, k, dtype=dt), rand(gen, k, n, scale=2 / math.sqrt(k)), rand(gen, n, scale=0.3)
    residual = rand(gen, m, n, dtype=dt)
    gemm = gnn.GNN_BF16 if dt == BF16 else gnn.GNN_F32
    wt = w.t().contiguous().bfloat16() if dt == BF16 else None
    a64, w64 = operands(a, None, w, wt, gemm)
    o = forward(a, None, w, wt, bias, name, gemm, dt, residual)
    check_forward(o, a64, w64, bias, residual, name, dt)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("name", list(ACTS))
@pytest.mark.parametrize("m, k, n", SIZES)
def test_backward(m, k, n, name, dt):
    gen = torch.Generator().manual_seed(m + 5 * k + 3 * n)
    a, w = rand(gen, m, k, dtype=dt), rand(gen, k, n, scale=1 / math.sqrt(k))
    z, g = rand(gen, m, n, dtype=dt, scale=1.5), rand(gen, m, n, dtype=dt)
    gemm = gnn.GNN_BF16 if dt == BF16 else gnn.GNN_F32
    wt = w.t().contiguous().bfloat16() if dt == BF16 else None
    a64, w64 = operands(a, None, w, wt, gemm)
    check_backward(backward(a, None, w, wt, z, g, name, gemm, dt), a64, w64, z, g, name, gemm, dt, dt)


# halves of A, types that differ, weights from either form, with and without
# each optional operand
FORMS = [(40, 32, 48), (65, 100, 47), (130, 33, 129), (300, 256, 512), (700, 512, 264), (1, 64, 96), (20, 300, 200),
         (1300, 768, 1024)]


@pytest.mark.gpu
@pytest.mark.parametrize("gemm, adt, odt, dwdt, form", [
    (gnn.GNN_F32, F32, F32, F32, "w"), (gnn.GNN_F32, BF16, F32, F32, "w"), (gnn.GNN_F32, F32, BF16, F32, "w"),
    (gnn.GNN_BF16, BF16, BF16, F32, "both"), (gnn.GNN_BF16, BF16, F32, F32, "wt"), (gnn.GNN_BF16, F32, BF16, BF16, "wt"),
    (gnn.GNN_BF16, F32, F32, BF16, "w"), (gnn.GNN_BF16, BF16, BF16, BF16, "w")])
@pytest.mark.parametrize("two", [False, True])
@pytest.mark.parametrize("m, k, n", FORMS)
def test_forms(m, k, n, two, gemm, adt, odt, dwdt, form):
    gen = torch.Generator().manual_seed(m + k + n)
    a, b = rand(gen, m, k, dtype=adt), rand(gen, m, k, dtype=adt) if two else None
    K = 2 * k if two else k
    w0 = rand(gen, K, n, scale=1 / math.sqrt(K))
    w = w0 if form != "wt" else None
    wt = w0.t().contiguous().bfloat16() if form != "w" else None
    bias, residual = (rand(gen, n), rand(gen, m, n, dtype=odt)) if m % 2 else (None, None)
    a64, w64 = operands(a, b, w, wt, gemm)
    o = forward(a, b, w, wt, bias, "silu", gemm, odt, residual, keep=bool(m % 4))
    check_forward(o, a64, w64, bias, residual, "silu", odt)
    gdt = odt if gemm == gnn.GNN_BF16 else F32
    z, g = rand(gen, m, n, dtype=odt), rand(gen, m, n, dtype=gdt)
    o = backward(a, b, w, wt, z, g, "silu", gemm, dwdt, input_grad=bool(m % 3), bias_grad=bool(m % 4))
    check_backward(o, a64, w64, z, g, "silu", gemm, gdt, dwdt)
    # no activation: z is not needed
    o = backward(a, b, w, wt, None, g, "none", gemm, dwdt)
    check_backward(o, a64, w64, None, g, "none", gemm, gdt, dwdt)


# few rows and columns over long reductions, which are split; splits that begin in
# one half of A and end in the other
@pytest.mark.gpu
@pytest.mark.parametrize("live", [False, True])
@pytest.mark.parametrize("two", [False, True])
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("m, k, n", [(130, 1088, 256), (100, 1024, 72), (129, 1100, 130), (65, 64, 4160), (100, 1031, 47), (300, 72, 2049),
                                     (70, 2176, 1001)])
def test_split_reductions(m, k, n, dt, two, live):
    gen = torch.Generator().manual_seed(m + k + n)
    gemm = gnn.GNN_BF16 if dt == BF16 else gnn.GNN_F32
    a, b = rand(gen, m, k, dtype=dt), rand(gen, m, k, dtype=dt) if two else None
    K = 2 * k if two else k
    w, bias, res = rand(gen, K, n, scale=1 / math.sqrt(K)), rand(gen, n), rand(gen, m, n, dtype=dt)
    z, g = rand(gen, m, n, dtype=dt), rand(gen, m, n, dtype=dt)
    wt = w.t().contiguous().bfloat16() if dt == BF16 else None
    rows = m - 30 if live else m
    kw = {"m_dev": torch.tensor([rows], device=DEV)} if live else {}
    a64, w64 = operands(a, b, w, wt, gemm)
    o = forward(a, b, w, wt, bias, "gelu", gemm, dt, res, **kw)
    check_forward(o, a64, w64, bias, res, "gelu", dt, rows)
    assert (o["out"][rows:] == 7).all() and (o["z"][rows:] == 7).all()
    o = backward(a, b, w, wt, z, g, "gelu", gemm, dt, **kw)
    check_backward(o, a64, w64, z, g, "gelu", gemm, dt, dt, rows)
    assert (o["d_a"][rows:] == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("off", [1, 2, 4, 5])
@pytest.mark.parametrize("m, k, n", [(5, 64, 64), (70, 128, 256), (300, 512, 512), (33, 100, 47)])
def test_any_alignment_of_the_element(m, k, n, off, dt):
    gen = torch.Generator().manual_seed(m + off)
    gemm = gnn.GNN_BF16 if dt == BF16 else gnn.GNN_F32

    def moved(t, by=off):
        buf = torch.full((t.numel() + 64,), 3.0, dtype=t.dtype, device=DEV)
        v = buf[by:by + t.numel()].view(t.shape)
        v.copy_(t)
        return v
    a, w, bias = rand(gen, m, k, dtype=dt), rand(gen, k, n, scale=1 / math.sqrt(k)), rand(gen, n)
    res, z, g = (rand(gen, m, n, dtype=dt) for _ in range(3))
    wt = moved(w.t().contiguous().bfloat16(), 4 * off) if dt == BF16 else None  # the shadow keeps 8 bytes
    a64, w64 = operands(a, None, w, wt, gemm)
    o = {"out": moved(res), "z": moved(res)}
    gnn.update_fwd_act(moved(a), None, moved(w), moved(bias), o["out"], ACTS["gelu"], gemm, residual=moved(res), z=o["z"], wt=wt)
    check_forward(o, a64, w64, bias, res, "gelu", dt)
    o = {"dw": moved(torch.zeros((k, n), dtype=dt, device=DEV)), "db": moved(bias), "d_a": moved(a)}
    gnn.update_bwd_act(moved(a), None, moved(w), moved(z), moved(g), o["dw"], o["db"], o["d_a"], ACTS["gelu"], gemm, wt=wt)
    check_backward(o, a64, w64, z, g, "gelu", gemm, dt, dt)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("rows, live, k, n", [(40, 0, 64, 32), (40, 1, 64, 32), (64, 17, 100, 47), (600, 300, 256, 512),
                                              (2000, 1025, 512, 768), (30, 30, 128, 64), (30, 99, 128, 64), (300, -3, 64, 64)])
def test_device_row_count(rows, live, k, n, dt):
    """Rows at or past the device count are not written and change nothing,
    whatever they hold; a count above the capacity is the capacity."""
    gen = torch.Generator().manual_seed(rows + live)
    gemm = gnn.GNN_BF16 if dt == BF16 else gnn.GNN_F32
    m = max(0, min(rows, live))
    a, res, z, g = (rand(gen, rows, c, dtype=dt) for c in (k, n, n, n))
    for t in (a, res, z, g):
        t[m:] = float("nan")
    w, bias = rand(gen, k, n, scale=1 / math.sqrt(k)), rand(gen, n)
    wt = w.t().contiguous().bfloat16() if dt == BF16 else None
    a64, w64 = operands(a, None, w, wt, gemm)
    m_dev = torch.tensor([live], device=DEV)
    o = forward(a, None, w, wt, bias, "relu", gemm, dt, res, m_dev=m_dev)
    assert (o["out"][m:] == 7).all() and (o["z"][m:] == 7).all()
    check_forward(o, a64, w64, bias, res, "relu", dt, m)
    o = backward(a, None, w, wt, z, g, "gelu_tanh", gemm, dt, m_dev=m_dev)
    assert (o["d_a"][m:] == 7).all()
    check_backward(o, a64, w64, z, g, "gelu_tanh", gemm, dt, dt, m)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, BF16])
def test_no_rows(dt):
    gemm = gnn.GNN_BF16 if dt == BF16 else gnn.GNN_F32
    a, w = torch.empty((0, 24), dtype=dt, device=DEV), torch.ones((24, 9), device=DEV)
    assert forward(a, None, w, None, None, "gelu", gemm, dt)["out"].shape == (0, 9)
    none = torch.empty((0, 9), dtype=dt, device=DEV)
    o = backward(a, None, w, None, none, none, "gelu", gemm, dt)
    assert (o["dw"] == 0).all() and (o["db"] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("m, k, n", [(1, 256, 128), (70, 100, 47), (500, 512, 512)])
def test_residual_in_place(m, k, n, dt):
    gen = torch.Generator().manual_seed(m)
    gemm = gnn.GNN_BF16 if dt == BF16 else gnn.GNN_F32
    a, w, res = rand(gen, m, k, dtype=dt), rand(gen, k, n), rand(gen, m, n, dtype=dt)
    o = forward(a, None, w, None, None, "silu", gemm, dt, res)
    over = res.clone()
    gnn.update_fwd_act(a, None, w, None, over, ACTS["silu"], gemm, residual=over)
    assert torch.equal(over, o["out"])


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("m, k, n", [(1, 4096, 512), (64, 256, 200), (33, 4096, 512), (64, 1032, 777), (32, 1032, 777), (70, 1024, 256), (129, 4160, 65), (600, 512, 513), (9000, 256, 260)])
def test_residual_in_place_of_the_tiles(m, k, n, dt):
    """The output's type apart from the products': few rows, split reductions, tiles."""
    gen = torch.Generator().manual_seed(m)
    a, wt, res = rand(gen, m, k, dtype=BF16), rand(gen, n, k, dtype=BF16, scale=1 / math.sqrt(k)), rand(gen, m, n, dtype=dt)
    o = forward(a, None, None, wt, None, "gelu", gnn.GNN_BF16, dt, res)
    check_forward(o, a.double(), wt.t().double(), None, res, "gelu", dt)
    over = res.clone()
    gnn.update_fwd_act(a, None, None, None, over, ACTS["gelu"], gnn.GNN_BF16, residual=over, wt=wt)
    assert torch.equal(over, o["out"])


@pytest.mark.gpu
def test_two_captured_calls_share_a_workspace():
    """Two graphs with one workspace, replayed in turn: nothing is kept in it."""
    gen = torch.Generator().manual_seed(4)
    sizes, calls = [(70, 2048, 200), (300, 520, 777)], []
    ws = torch.empty(1 << 26, dtype=torch.uint8, device=DEV)
    for m, k, n in sizes:
        a, z, g = (rand(gen, m, c, dtype=BF16) for c in (k, n, n))
        w = rand(gen, k, n, scale=1 / math.sqrt(k))
        wt = w.t().contiguous().bfloat16()
        out = [torch.zeros((m, n), dtype=BF16, device=DEV), torch.zeros((k, n), device=DEV), torch.zeros(n, device=DEV),
               torch.zeros((m, k), dtype=BF16, device=DEV)]

        def go(a=a, z=z, g=g, w=w, wt=wt, out=out):
            gnn.update_fwd_act(a, None, w, None, out[0], ACTS["silu"], gnn.GNN_BF16, wt=wt, ws=ws)
            gnn.update_bwd_act(a, None, w, z, g, *out[1:], ACTS["silu"], gnn.GNN_BF16, wt=wt, ws=ws)
        go()
        want = [t.clone() for t in out]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            go()
        calls.append((graph, out, want, go))  # go keeps the graph's operands
    for _ in range(3):
        for graph, out, *_ in calls:
            for t in out:
                t.fill_(7)
            graph.replay()
        ws.fill_(255)  # NaN in any type
        torch.cuda.synchronize()
        for _, out, want, _ in calls:
            for t, v in zip(out, want):
                assert torch.equal(t, v)


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(ACTS))
def test_activations_far_out(name):
    """Z over the whole range, through a product that is exact: no NaN where
    the formula has none, and the tails go to their limits."""
    zs = torch.cat([torch.linspace(-12, 12, 4001), torch.tensor([0.0, 30, -30, 88, -88, 1e4, -1e4, 1e18, -1e18, 1e30, -1e30])])
    zs = zs.to(DEV)[:, None]
    one = torch.ones((1, 1), device=DEV)
    o = forward(zs, None, one, None, None, name, gnn.GNN_F32, F32)
    z = zs.double()
    want = torch.where(z.abs() > 1e4, z.clamp(min=0) if name != "none" else z, act64(z.clamp(-1e4, 1e4), name))
    bound = torch.where(z.abs() > 1e4, 4 * U * z.abs(), act_error(z.clamp(-1e4, 1e4), name) + 4 * U * want.abs()) + 1e-30
    within(o["out"], want, bound, name)
    # act'(z) through db: one row a column
    n = zs.shape[0]
    g = torch.ones((1, n), device=DEV)
    b = backward(one, None, torch.ones((1, n), device=DEV), None, zs.view(1, n), g, name, gnn.GNN_F32, F32, input_grad=False)
    want = torch.where(z.abs() > 1e4, (z > 0).double() if name != "none" else torch.ones_like(z), slope64(z.clamp(-1e4, 1e4), name))
    within(b["db"].view(n, 1), want, torch.full_like(want, 1e-6), name + "'")


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, BF16])
def test_bad_rows_stay_alone(dt):
    gen = torch.Generator().manual_seed(9)
    gemm = gnn.GNN_BF16 if dt == BF16 else gnn.GNN_F32
    for m, k, n in ((9, 72, 40), (300, 520, 520)):
        a, w = rand(gen, m, k, dtype=dt), rand(gen, k, n, scale=0.1)
        clean = forward(a, None, w, None, None, "none", gemm, dt)["out"]
        a[3, k - 1], a[5, 0] = float("nan"), float("inf")
        out = forward(a, None, w, None, None, "none", gemm, dt)["out"]
        assert out[3].isnan().all() and not out[5].isfinite().any()
        keep = [i for i in range(m) if i not in (3, 5)]
        assert torch.equal(out[keep], clean[keep])


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(ACTS))
def test_gradients_against_differences(name):
    gen = torch.Generator().manual_seed(3)
    m, k, n = 14, 10, 12
    a, w, bias, g = rand(gen, m, k), rand(gen, k, n), rand(gen, n), rand(gen, m, n)
    o = forward(a, None, w, None, bias, name, gnn.GNN_F32, F32)
    b = backward(a, None, w, None, o["z"], g, name, gnn.GNN_F32, F32)
    h = 1e-5
    if name == "relu":  # no difference across the kink
        assert o["z"].abs().min() > 20 * h
    for key, t in (("d_a", a), ("dw", w), ("db", bias)):
        v = rand(gen, *t.shape).double()

        def loss(s):
            x = {"d_a": a.double(), "dw": w.double(), "db": bias.double()}
            x[key] = x[key] + s * v
            return (g.double() * act64(x["d_a"] @ x["dw"] + x["db"], name)).sum()
        want = float((loss(h) - loss(-h)) / (2 * h))
        # sums of some hundred products of unit size, each within 1e-6 of its
        # terms' sizes; the difference's own error goes by h^2 and 1e-16 / h
        assert abs(float((b[key].double() * v).sum()) - want) <= 2e-5 * max(1.0, abs(want)) + 1e-4 * 1e-1


@pytest.mark.gpu
@pytest.mark.parametrize("m, k, n", [(1, 512, 256), (60, 256, 256), (700, 512, 512), (300, 100, 47)])
def test_captured_and_on_another_stream(m, k, n):
    gen = torch.Generator().manual_seed(8)
    a, z, g, res = (rand(gen, m, c, dtype=BF16) for c in (k, n, n, n))
    w, bias = rand(gen, k, n, scale=1 / math.sqrt(k)), rand(gen, n)
    wt = w.t().contiguous().bfloat16()

    def buffers():
        return [torch.zeros((m, n), dtype=BF16, device=DEV), torch.zeros((m, n), dtype=BF16, device=DEV),
                torch.zeros((k, n), device=DEV), torch.zeros(n, device=DEV), torch.zeros((m, k), dtype=BF16, device=DEV)]

    def both(o, **kw):
        gnn.update_fwd_act(a, None, w, bias, o[0], ACTS["gelu"], gnn.GNN_BF16, residual=res, z=o[1], wt=wt, **kw)
        gnn.update_bwd_act(a, None, w, o[1], g, o[2], o[3], o[4], ACTS["gelu"], gnn.GNN_BF16, wt=wt, **kw)
    eager, replayed, side = buffers(), buffers(), buffers()
    both(replayed)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(replayed)
    stream = torch.cuda.Stream()
    for _ in range(4):
        a.copy_(rand(gen, m, k, dtype=BF16))
        g.copy_(rand(gen, m, n, dtype=BF16))
        both(eager)
        graph.replay()
        stream.wait_stream(torch.cuda.current_stream())
        both(side, stream=stream)
        torch.cuda.synchronize()
        for x, y, v in zip(eager, replayed, side):
            assert torch.equal(x, y) and torch.equal(x, v)


@pytest.mark.gpu
def test_relu_agrees_with_update_fwd():
    """ReLU without a residual agrees with gnn_update_fwd on the same operands."""
    gen = torch.Generator().manual_seed(2)
    for m, k, n in ((100, 128, 64), (600, 512, 512)):
        a, w, bias = rand(gen, m, k, dtype=BF16), rand(gen, k, n, scale=1 / math.sqrt(k)), rand(gen, n)
        wt = w.t().contiguous().bfloat16()
        out = torch.empty((m, n), dtype=BF16, device=DEV)
        gnn.update_fwd(a, None, w, bias, out, True, gnn.GNN_BF16, wt=wt)
        o = forward(a, None, w, wt, bias, "relu", gnn.GNN_BF16, BF16, keep=False)
        size = a.double().abs() @ wt.double().t().abs() + bias.double().abs()
        # both within their sums' roundings of Z, and a rounding to bf16 each
        within(o["out"], out.double(), 2 * (k + 4) * U * size + 4 * half_step(BF16) * out.double().abs() + 1e-37, "out")


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """The last rows of activations and outputs of more than 2^31 elements."""
    m, k, n = 135_000, 16_384, 16
    a = torch.zeros((m, k), dtype=BF16, device=DEV)
    gen = torch.Generator().manual_seed(1)
    a[-3:] = rand(gen, 3, k, dtype=BF16)
    wt = rand(gen, n, k, dtype=BF16, scale=0.01)
    o = forward(a, None, None, wt, None, "none", gnn.GNN_BF16, BF16)
    a64, w64 = a[-3:].double(), wt.t().double()
    check_forward({k_: v[-3:] for k_, v in o.items()}, a64, w64, None, None, "none", BF16)
    assert (o["out"][:-3] == 0).all()
    g = torch.zeros((m, n), dtype=BF16, device=DEV)
    g[-3:] = rand(gen, 3, n, dtype=BF16)
    b = backward(a, None, None, wt, None, g, "none", gnn.GNN_BF16, BF16)
    check_backward({"dw": b["dw"], "db": b["db"], "d_a": b["d_a"][-3:]}, a64, w64, None, g[-3:], "none", gnn.GNN_BF16,
                   BF16, BF16)
    assert (b["d_a"][:-3] == 0).all()


def test_refusals_on_the_host():
    lib = gnn.lib()
    fake, inval, unsup = 1 << 24, gnn.GNN_EINVAL, gnn.GNN_EUNSUPPORTED
    big = 1 << 40
    fwd = [fake, None, 1, 64, None, 8, fake, None, None, 32, 0, None, None, 1, fake + 4096, 1, fake, big, None]

    def f(**kw):
        a = list(fwd)
        for k, v in kw.items():
            a[int(k[1:])] = v
        return lib.gnn_update_fwd_act(*a)
    assert f(_0=None) == inval and f(_6=None) == inval and f(_14=None) == inval
    assert f(_2=2) == unsup and f(_13=2) == unsup and f(_15=9) == unsup
    assert f(_3=0) == inval and f(_9=gnn.GNN_MAX_DIM + 1) == inval and f(_5=-1) == inval and f(_5=1 << 40) == inval
    assert f(_10=-1) == inval and f(_10=5) == inval and b"activation" in lib.gnn_last_error()
    assert f(_0=fake + 1) == inval and f(_6=fake + 2) == inval and f(_7=fake + 4) == inval and f(_8=fake + 2) == inval
    assert f(_11=fake + 1) == inval and f(_12=fake + 1) == inval and f(_4=fake + 4) == inval
    assert f(_6=None, _7=fake, _13=0) == inval   # a shadow alone with fp32 products
    assert f(_12=fake + 4096) == inval           # z over out
    assert f(_11=fake + 512, _12=fake + 512) == inval
    assert f(_14=fake) == inval                  # out over A
    bwd = [fake, None, 1, 64, None, 8, fake, None, fake, 1, fake, 1, 32, 2, 1, fake + 4096, 1, None, None, fake, big, None]

    def b(**kw):
        a = list(bwd)
        for k, v in kw.items():
            a[int(k[1:])] = v
        return lib.gnn_update_bwd_act(*a)
    assert b(_0=None) == inval and b(_8=None) == inval and b(_10=None) == inval and b(_15=None) == inval
    assert b(_6=None, _18=fake + 8192) == inval  # d_a without weights
    assert b(_9=2) == unsup and b(_11=2) == unsup and b(_16=2) == unsup and b(_14=2) == unsup
    assert b(_14=0) == unsup and b"GNN_F32" in lib.gnn_last_error()
    assert b(_13=7) == inval and b(_15=fake + 4097) == inval and b(_18=fake) == inval
    assert b(_19=None) == inval and b(_19=fake + 64) == inval and b(_20=16) == gnn.GNN_ESIZE
    nb = gnn._sz()
    ref = gnn.ctypes.byref(nb)
    assert lib.gnn_update_fwd_act_workspace_size(1, 0, 0, 8, 8, 1, 1, ref) == inval
    assert lib.gnn_update_fwd_act_workspace_size(2, 8, 0, 8, 8, 1, 1, ref) == unsup
    assert lib.gnn_update_fwd_act_workspace_size(1, 8, 0, 8, 8, 1, 1, None) == inval
    assert lib.gnn_update_bwd_act_workspace_size(1, 8, 0, 8, -1, 1, 1, 1, 1, ref) == inval
    assert lib.gnn_update_bwd_act_workspace_size(1, 8, 0, 8, 8, 3, 1, 1, 1, ref) == unsup


@pytest.mark.gpu
def test_refusals_of_the_binding():
    a, w, out = torch.zeros((4, 8), device=DEV), torch.zeros((8, 6), device=DEV), torch.zeros((4, 6), device=DEV)
    wt, f32, bf = torch.zeros((6, 8), dtype=BF16, device=DEV), gnn.GNN_F32, gnn.GNN_BF16
    for bad in (lambda: gnn.update_fwd_act(a, None, w.t(), None, out, 0, f32),
                lambda: gnn.update_fwd_act(a, None, w[:7], None, out, 0, f32),
                lambda: gnn.update_fwd_act(a, a.bfloat16(), w, None, out, 0, f32),
                lambda: gnn.update_fwd_act(a, a, w, None, out, 0, f32),           # K doubles
                lambda: gnn.update_fwd_act(a, None, None, None, out, 0, f32, wt=wt),
                lambda: gnn.update_fwd_act(a, None, w, None, out, 0, bf, wt=wt.t()),
                lambda: gnn.update_fwd_act(a, None, w, None, out[:3], 0, f32),
                lambda: gnn.update_fwd_act(a, None, w, None, out, 0, f32, residual=out.bfloat16()),
                lambda: gnn.update_fwd_act(a, None, w, None, out, 0, f32, z=out.bfloat16()),
                lambda: gnn.update_fwd_act(a, None, w, out[0, :5], out, 0, f32),
                lambda: gnn.update_fwd_act(a[:, ::2], None, w[:4], None, out, 0, f32),
                lambda: gnn.update_fwd_act(a.cpu(), None, w, None, out, 0, f32),
                lambda: gnn.update_bwd_act(a, None, w, out, out, w.half(), None, None, 1, f32),
                lambda: gnn.update_bwd_act(a, None, w, out, out, w.clone(), None, a.bfloat16(), 1, f32),
                lambda: gnn.update_bwd_act(a, None, None, out, out, w.clone(), None, torch.empty_like(a), 1, f32)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: gnn.update_fwd_act(a, None, w, None, out, 9, f32),
                lambda: gnn.update_bwd_act(a, None, w, None, out, w.clone(), None, None, 1, f32),
                lambda: gnn.update_bwd_act(a, None, w, out, out, w.bfloat16(), None, None, 1, f32)):
        with pytest.raises(gnn.GnnError):
            bad()
