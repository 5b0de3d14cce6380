"""A trained table of rows: its lookup and gradient, the loss over its many
classes, and the step of the optimizer: what a pass through each costs.

Each case is one call of one operator, as a training or serving program makes
it.  A table holds a row for each vertex, token or class; rows that the inputs
name are looked up, the same or another table's rows score the outputs, and an
AdamW step moves the table and the layers between.  Sizes are those of the
repository's models (2.4M vertices, hidden width 256, 47 classes, 1,024
targets, 26,624 rows of a mini-batch) and generic ones up to the largest tables
that one card trains.

  listed()          the fixed cases
  draw(rng)         one more case of the same ranges
  prepare(case, s)  the inputs a program holds before the call, from seed s
  run(state)        one pass; returns its outputs
  work(case)        bytes and operations a pass cannot do without
  exact(case, s)    run()'s result in 64 bits

Operators, for rows i:

  embed_fwd  out_i = scale table[ids_i], 0 where ids_i is outside the table
  embed_bwd  d_table_v = sum over the i with ids_i = v of scale g_i, in place of
             what the table of gradients held or added to it
  ce         z = a wt^T + bias; row_i = log sum exp z_i - z_i[label_i];
             loss = sum_i s_i row_i; with dz = s (softmax(z) - onehot(label)):
             dwt = dz^T a, db = sum_i dz, da = dz wt; rows whose label is
             negative are absent
  adamw      m = b1 m + (1 - b1) g, v = b2 v + (1 - b2) g^2,
             w = w (1 - lr decay) - lr m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps)
             over all tensors of a model.  States in 8 bits: m and sqrt(v) are
             e4m3 values times one scale for each 256 elements of a tensor, the
             largest of them at 448, rounded up or down by chance: with h = mix(
             key ^ (element / 2)) the four 16-bit parts of h, in their order,
             are for m and sqrt(v) of the even element and of the odd one, key =
             mix(mix(mix(seed) ^ t) ^ tensor), mix the output function of
             SplitMix64 (without its increment)

Where the matrix products run in bf16, dz is rounded to bf16 as their operand
and the gradients that are summed from it are kept in bf16 too.
"""
import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
BETA1, BETA2, EPS, LR, DECAY = 0.9, 0.999, 1e-8, 1e-3, 0.01
GROUP = 256      # elements of a tensor that share a scale
TOP = 448.0      # the largest e4m3 value
SEED = 1234      # of the optimizer's rounding


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # a serving program looks up the one token it goes on from
        dict(name="embed-fwd-1-32000x4096", op="embed_fwd", ids=1, rows=32_000, dim=4096, dtype="bf16", law="zipf",
             pad=False),
        # the distinct vertices of a mini-batch, trained features of 2.4M vertices
        dict(name="embed-fwd-26624-2449029x256-f32", op="embed_fwd", ids=26_624, rows=2_449_029, dim=256, dtype="f32",
             law="distinct", pad=False),
        # a large batch of tokens with padding
        dict(name="embed-fwd-131072-100003x4096", op="embed_fwd", ids=131_072, rows=100_003, dim=4096, dtype="bf16",
             law="zipf", pad=True),
        # a training step's tokens, added to a gradient that the output side left
        dict(name="embed-bwd-8192-32000x1024", op="embed_bwd", ids=8192, rows=32_000, dim=1024, dtype="bf16",
             law="zipf", pad=True, add=True),
        # small odd tables, fp32
        dict(name="embed-bwd-1461-5003x100-f32", op="embed_bwd", ids=1461, rows=5003, dim=100, dtype="f32",
             law="zipf", pad=False, add=False),
        # a large batch, frequent tokens by the thousands
        dict(name="embed-bwd-262144-131072x2048", op="embed_bwd", ids=262_144, rows=131_072, dim=2048, dtype="bf16",
             law="zipf", pad=True, add=False),
        # the score of one answer
        dict(name="ce-1x4096x32000", op="ce", rows=1, k=4096, c=32_000, dtype="bf16", grads=False, pad=False),
        # a mini-batch's targets, the last layer of the small fp32 model
        dict(name="ce-1024x256x47-f32", op="ce", rows=1024, k=256, c=47, dtype="f32", grads=True, pad=False),
        # many classes, an odd number of them, rows that pad the batch
        dict(name="ce-4096x2048x100003", op="ce", rows=4096, k=2048, c=100_003, dtype="bf16", grads=True, pad=True),
        # the optimizer of the two-layer model: four small tensors
        dict(name="adamw-2layer-f32", op="adamw", blocks=1, f=200, hidden=256, classes=47, state="f32", dtype="f32",
             shadow=False, step=7),
        # 12 wide residual blocks, 73 tensors, with bf16 shadows
        dict(name="adamw-73x100m-f32", op="adamw", blocks=12, f=1024, hidden=4096, classes=1, state="f32", dtype="bf16",
             shadow=True, step=100),
        # a large table and a few blocks, states in 8 bits
        dict(name="adamw-table-8bit", op="adamw", blocks=4, f=1024, hidden=4096, classes=100_003, state="8bit",
             dtype="bf16", shadow=True, step=1000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed_fwd", "embed_bwd", "embed_bwd", "ce", "ce", "ce", "adamw", "adamw"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op in ("embed_fwd", "embed_bwd"):
        dim = rng.choice([64, 100, 128, 256, 768, 1024, 4096, _log(rng, 16, 8192)])
        rows = _log(rng, 1000, min(2_449_029, (1 << 28) // dim))
        ids = _log(rng, 1, min(262_144, (1 << 29) // dim))
        law = rng.choice(["zipf", "zipf", "distinct"])
        case = dict(op=op, ids=min(ids, rows) if law == "distinct" else ids, rows=rows, dim=dim, dtype=dtype, law=law,
                    pad=rng.random() < 0.5)
        return case if op == "embed_fwd" else dict(case, add=rng.random() < 0.4)
    if op == "ce":
        # fp32 products are those of small models
        k = rng.choice([64, 100, 256, 512, 1024, _log(rng, 16, 4096 if dtype == "bf16" else 512)])
        c = rng.choice([8, 47, 172, 1000, 32_000, 131_072, _log(rng, 100, 131_072)])
        most = (1 << 39 if dtype == "bf16" else 1 << 33) // (k * c)
        rows = _log(rng, 1, max(2, min(16_384, most, (1 << 29) // c)))
        return dict(op=op, rows=rows, k=k, c=c, dtype=dtype, grads=rng.random() < 0.8, pad=rng.random() < 0.5)
    return dict(op=op, blocks=rng.randint(1, 12), f=_log(rng, 16, 1024), hidden=_log(rng, 16, 4096),
                classes=_log(rng, 1, 100_000), state=rng.choice(["f32", "8bit"]), dtype=dtype,
                shadow=rng.random() < 0.5, step=_log(rng, 1, 10_000))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _randn(g, *shape, dtype=torch.float32, scale=1.0, shift=0.0):
    return (torch.randn(shape, generator=g, device=DEVICE).mul_(scale).add_(shift)).to(dtype)


def _uniform(g, *shape):
    return torch.rand(shape, generator=g, device=DEVICE)


def _ids(case, g):
    """Row ids: distinct ones, or ranks whose frequency falls as 1 / rank, in
    a random order of the table; of padded batches one in sixteen is absent."""
    n, rows = case["ids"], case["rows"]
    order = torch.randperm(rows, generator=g, device=DEVICE)
    if case["law"] == "distinct":
        ids = order[:n].clone()
    else:
        rank = torch.exp(_uniform(g, n).double() * math.log(rows + 1)).long() - 1
        ids = order[rank.clamp(0, rows - 1)]
    if case["pad"]:
        ids[torch.arange(n, device=DEVICE) % 16 == 15] = -1
    return ids


def _shapes(case):
    """The tensors of a model: a table, then blocks of a norm, a widening layer
    and a narrowing one."""
    f, h = case["f"], case["hidden"]
    return [(case["classes"], f)] + [(f,), (f,), (f, h), (h,), (h, f), (f,)] * case["blocks"]


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(int(seed))
    op, dt = case["op"], DTYPES[case["dtype"]]
    s = {"case": case}
    if op == "embed_fwd":
        s["table"] = _randn(g, case["rows"], case["dim"], dtype=dt)
        s["ids"] = _ids(case, g)
        s["out"] = torch.empty((case["ids"], case["dim"]), dtype=dt, device=DEVICE)
        return s
    if op == "embed_bwd":
        s["ids"] = _ids(case, g)
        s["g"] = _randn(g, case["ids"], case["dim"], dtype=dt)
        shape = (case["rows"], case["dim"])
        s["d_table"] = _randn(g, *shape, dtype=dt) if case["add"] else torch.empty(shape, dtype=dt, device=DEVICE)
        return s
    if op == "ce":
        rows, k, c = case["rows"], case["k"], case["c"]
        wt = _randn(g, c, k, scale=1.0 / math.sqrt(k))
        s["labels"] = torch.randint(0, c, (rows,), generator=g, device=DEVICE)
        # a model that has learnt something: the label's score is above the others'
        s["a"] = _randn(g, rows, k).add_(wt[s["labels"]], alpha=4.0).to(dt)
        s["wt"], s["bias"] = wt.to(dt), _randn(g, c, scale=0.1)
        s["scale"] = None
        if case["pad"]:
            live = torch.arange(rows, device=DEVICE) % 16 != 15
            s["labels"] = torch.where(live, s["labels"], -1)
            s["scale"] = live.float() / live.sum()
        empty = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=DEVICE)  # noqa: E731
        s["loss"], s["row_loss"] = empty(1), empty(rows)
        if case["grads"]:
            s.update(dwt=empty(c, k, dtype=dt), db=empty(c), d_a=empty(rows, k, dtype=dt))
        return s
    # every tensor starts at a whole group of one long buffer, zeros between
    shapes = _shapes(case)
    sizes = [math.prod(x) for x in shapes]
    groups = [-(-n // GROUP) for n in sizes]
    total = sum(groups) * GROUP
    count = torch.tensor(groups, device=DEVICE)
    first = torch.cumsum(count, 0) - count
    owner = torch.repeat_interleave(torch.arange(len(sizes), device=DEVICE), count)
    begin = (torch.arange(sum(groups), device=DEVICE) - first[owner]) * GROUP  # the group's first element in its tensor
    there = begin[:, None] + torch.arange(GROUP, device=DEVICE) < torch.tensor(sizes, device=DEVICE)[owner][:, None]
    there = there.reshape(-1)
    s["w"] = _randn(g, total, scale=0.05).mul_(there)
    # gradients of a tensor differ by orders of magnitude
    s["g"] = _randn(g, total, scale=1e-2).mul_(torch.exp(_randn(g, total))).mul_(there).to(dt)
    m = _randn(g, total, scale=3e-3).mul_(there)
    r = _randn(g, total, scale=1e-2).abs_().add_(1e-4).mul_(there)
    s["shapes"], s["sizes"] = shapes, sizes
    s["starts"] = [int(x) * GROUP for x in first.tolist()]
    # tables and matrices decay, vectors do not
    s["decays"] = [DECAY if len(x) == 2 else 0.0 for x in shapes]
    s["owner"], s["begin"] = owner, begin
    s["decay"] = torch.tensor(s["decays"], device=DEVICE)[owner][:, None]
    s["shadow"] = torch.zeros(total, dtype=torch.bfloat16, device=DEVICE) if case["shadow"] else None
    if case["state"] == "f32":
        return dict(s, m=m, v=r.square_())
    for name, x in (("m", m), ("v", r)):
        x = x.reshape(-1, GROUP)
        scale = x.abs().amax(1, keepdim=True) / TOP
        s[name + "_scale"] = scale.reshape(-1)
        s[name] = (x / scale).reshape(-1).to(torch.float8_e4m3fn)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    if own:
        return _kernels(s)
    return _plain(s)


def _kernels(s):
    """The calls a user makes."""
    from paper_2303_00158_amd import gnn
    case = s["case"]
    op = case["op"]
    if op == "embed_fwd":
        gnn.embed_fwd(s["table"], s["ids"], s["out"], math.sqrt(case["dim"]))
        return (s["out"],)
    if op == "embed_bwd":
        if "ws" not in s:
            s["ws"] = gnn.embed_bwd_workspace(case["ids"], case["rows"], case["dim"], DEVICE)
        gnn.embed_bwd(s["g"], s["ids"], s["d_table"], math.sqrt(case["dim"]), accumulate=case["add"], ws=s["ws"])
        return (s["d_table"],)
    if op == "ce":
        gemm = gnn.GNN_BF16 if case["dtype"] == "bf16" else gnn.GNN_F32
        if "ws" not in s:
            s["ws"] = gnn.update_ce_workspace(s["a"], s["wt"], gemm, grads=case["grads"])
        gnn.update_ce(s["a"], s["wt"], s["bias"], s["labels"], s["loss"], gemm, row_loss=s["row_loss"],
                      d_a=s.get("d_a"), dwt=s.get("dwt"), db=s.get("db"), row_scale=s["scale"], ws=s["ws"])
        return (s["loss"], s["row_loss"]) + ((s["dwt"], s["db"], s["d_a"]) if case["grads"] else ())
    if "opt" not in s:
        def each(x):
            return [x[at:at + n] for at, n in zip(s["starts"], s["sizes"])]

        def scales(x):
            return [x[at // GROUP:at // GROUP - (-n // GROUP)] for at, n in zip(s["starts"], s["sizes"])]
        eight = case["state"] == "8bit"
        s["opt"] = gnn.AdamW(each(s["w"]), each(s["g"]), weight_decay=s["decays"], betas=(BETA1, BETA2), eps=EPS,
                             state_dtype=torch.float8_e4m3fn if eight else torch.float32, m=each(s["m"]),
                             v=each(s["v"]), m_scale=scales(s["m_scale"]) if eight else None,
                             v_scale=scales(s["v_scale"]) if eight else None,
                             shadows=each(s["shadow"]) if case["shadow"] else None, seed=SEED)
    s["opt"].step(LR, case["step"])
    return _state(s)


def _state(s):
    names = ["w", "m", "v"] + (["m_scale", "v_scale"] if s["case"]["state"] == "8bit" else [])
    return {n: s[n] for n in names + (["shadow"] if s["case"]["shadow"] else [])}


def _plain(s):
    """The operators from elementary operations in 32 bits."""
    case = s["case"]
    op = case["op"]
    if op in ("embed_fwd", "embed_bwd"):
        scale, there, at = math.sqrt(case["dim"]), (s["ids"] >= 0)[:, None], s["ids"].clamp(min=0)
        if op == "embed_fwd":
            return (torch.where(there, s["table"][at].float() * scale, 0.0).to(s["table"].dtype),)
        rows = torch.where(there, s["g"].float() * scale, 0.0)
        if not case["add"]:
            total = torch.zeros(s["d_table"].shape, dtype=torch.float32, device=DEVICE).index_add_(0, at, rows)
            return (total.to(s["g"].dtype),)
        s["d_table"].copy_(s["d_table"].float().index_add_(0, at, rows))
        return (s["d_table"],)
    if op == "ce":
        a, wt, rows = s["a"].float(), s["wt"].float(), case["rows"]
        z = (a @ wt.t()).add_(s["bias"])
        there, at = s["labels"] >= 0, s["labels"].clamp(min=0)[:, None]
        top = z.amax(1, keepdim=True)
        lse = top + torch.log(torch.exp(z - top).sum(1, keepdim=True))
        row = torch.where(there, (lse - z.gather(1, at))[:, 0], 0.0)
        weight = torch.full_like(row, 1.0 / rows) if s["scale"] is None else s["scale"]
        loss = (row * weight).sum()[None]
        if not case["grads"]:
            return loss, row
        weight = torch.where(there, weight, 0.0)[:, None]
        dz = torch.exp(z.sub_(lse)).scatter_add_(1, at, torch.full_like(weight, -1.0)).mul_(weight)
        return loss, row, (dz.t() @ a).to(s["a"].dtype), dz.sum(0), (dz @ wt).to(s["a"].dtype)
    t, eight = case["step"], case["state"] == "8bit"
    w, g = s["w"].view(-1, GROUP), s["g"].view(-1, GROUP).float()
    m, v = s["m"].view(-1, GROUP).float(), s["v"].view(-1, GROUP).float()
    if eight:
        m = m * s["m_scale"][:, None]
        v = torch.square(v * s["v_scale"][:, None])
    m = BETA1 * m + (1.0 - BETA1) * g
    v = BETA2 * v + (1.0 - BETA2) * (g * g)
    root = torch.sqrt(v)
    step = m / (root / math.sqrt(1.0 - BETA2 ** t) + EPS)
    w.copy_(w * (1.0 - LR * s["decay"].double()).float() - step * (LR / (1.0 - BETA1 ** t)))
    if s["shadow"] is not None:
        s["shadow"].copy_(s["w"])
    if eight:
        chance = _chance(s)
        _round8(m, chance[:, :, 0::2], s["m"], s["m_scale"])
        _round8(root, chance[:, :, 1::2], s["v"], s["v_scale"])
    else:
        s["m"].view(-1, GROUP).copy_(m)
        s["v"].view(-1, GROUP).copy_(v)
    return _state(s)


def _signed(x):
    return x - (1 << 64) if x >> 63 else x


def _mix(x):
    """The output function of SplitMix64, of an integer or of int64 values."""
    one, two = 0xBF58476D1CE4E5B9, 0x94D049BB133111EB
    if isinstance(x, int):
        x = ((x ^ (x >> 30)) * one) % (1 << 64)
        x = ((x ^ (x >> 27)) * two) % (1 << 64)
        return x ^ (x >> 31)
    x = (x ^ ((x >> 30) & ((1 << 34) - 1))) * _signed(one)
    x = (x ^ ((x >> 27) & ((1 << 37) - 1))) * _signed(two)
    return x ^ ((x >> 31) & ((1 << 33) - 1))


def _chance(s):
    """Four numbers in (0, 1) for each pair of elements: m and sqrt(v) of the
    even one, m and sqrt(v) of the odd one."""
    key = _signed(_mix(_mix(SEED) ^ s["case"]["step"]))
    key = _mix(s["owner"] ^ key)
    pair = (s["begin"] // 2)[:, None] + torch.arange(GROUP // 2, device=DEVICE)
    h = _mix(key[:, None] ^ pair)
    parts = (h[:, :, None] >> torch.tensor([0, 16, 32, 48], device=DEVICE)) & 0xffff
    return (parts.float() + 0.5) * 2.0 ** -16


def _round8(x, chance, codes, scales):
    """x in groups as e4m3 codes and scales, rounded by chance."""
    scale = x.abs().amax(1, keepdim=True) / TOP
    inverse = torch.where(scale >= torch.finfo(torch.float32).tiny, 1.0 / scale, 0.0)
    t = x.abs() * inverse
    # values are whole multiples of 2^e, eight to sixteen of them above the smallest e
    e = ((t.view(torch.int32) >> 23) - 130).clamp(min=-9)
    q = torch.floor(t * torch.exp2(-e.float()) + chance.reshape(x.shape))
    code = (((e + 9) << 3) + q.int()).clamp(max=126)
    code = code + torch.where(torch.signbit(x), 128, 0)
    codes.view(torch.uint8).view(-1, GROUP).copy_(code)
    scales.copy_(torch.where(inverse > 0, scale, 0.0)[:, 0])


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    op, e = case["op"], SIZE[case["dtype"]]
    if op in ("embed_fwd", "embed_bwd"):
        n, rows, dim = case["ids"], case["rows"], case["dim"]
        live = n - n // 16 if case["pad"] else n
        # distinct rows that the ids name: of ranks by 1 / rank, each has 1 - (1 - p)^n
        named = live
        if case["law"] == "zipf":
            whole, named, r = math.log(rows + 1), 0.0, 1
            while r <= rows:  # ranks in runs that double
                end = min(rows, 2 * r - 1)
                named += (end - r + 1) * -math.expm1(live * math.log1p(-math.log1p(1.0 / (0.5 * (r + end))) / whole))
                r = end + 1
        if op == "embed_fwd":
            return {"bytes": (named + n) * dim * e + 8 * n, "flops": live * dim}
        return {"bytes": live * dim * e + (2 * named if case["add"] else rows) * dim * e + 8 * n, "flops": 2 * live * dim}
    if op == "ce":
        m, k, c = case["rows"], case["k"], case["c"]
        once = (m * k + c * k) * e + 4 * c + 12 * m
        return {"bytes": 2 * once if case["grads"] else once, "flops": 2 * m * k * c * (3 if case["grads"] else 1)}
    n = sum(math.prod(x) for x in _shapes(case))
    each = 8 + e + (16 if case["state"] == "f32" else 4 + 16 / GROUP) + 2 * case["shadow"]
    return {"bytes": n * each, "flops": 14 * n}


# ---------------------------------------------------------------------------
# in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "embed_fwd":
        # the table with a row of zeros behind it for what is absent
        at = torch.remainder(s["ids"], case["rows"] + 1)
        out = torch.zeros((case["ids"], case["dim"]), dtype=torch.float64, device=DEVICE)
        there = torch.nonzero(at < case["rows"])[:, 0]
        out[there] = torch.index_select(s["table"], 0, at[there]).double()
        return (out.mul_(case["dim"] ** 0.5),)
    if op == "embed_bwd":
        there = torch.nonzero(s["ids"] >= 0)[:, 0]
        ids, order = torch.sort(s["ids"][there], stable=True)
        rows, run_of = torch.unique_consecutive(ids, return_inverse=True)
        sums = torch.zeros((rows.numel(), case["dim"]), dtype=torch.float64, device=DEVICE)
        sums.index_put_((run_of,), s["g"][there[order]].double(), accumulate=True)
        total = s["d_table"].double() if case["add"] else torch.zeros(s["d_table"].shape, dtype=torch.float64, device=DEVICE)
        total[rows] += sums.mul_(case["dim"] ** 0.5)
        return (total,)
    if op == "ce":
        a, wt = s["a"].double(), s["wt"].double()
        logp = torch.log_softmax(torch.addmm(s["bias"].double(), a, wt.t()), dim=1)
        live = torch.nonzero(s["labels"] >= 0)[:, 0]
        weight = torch.full((case["rows"],), 1.0 / case["rows"], dtype=torch.float64, device=DEVICE)
        if case["pad"]:
            weight = s["scale"].double()
        row = torch.zeros_like(weight)
        row[live] = -logp[live, s["labels"][live]]
        loss = torch.dot(row, weight)[None]
        if not case["grads"]:
            return loss, row
        dz = logp.exp_()
        dz[live, s["labels"][live]] -= 1.0
        dz[s["labels"] < 0] = 0.0
        dz *= weight[:, None]
        return loss, row, torch.mm(dz.t(), a), dz.sum(0), torch.mm(dz, wt)
    t = case["step"]

    def up(name):
        x = s[name].double().view(-1, GROUP)
        return x if case["state"] == "f32" else x * s[name + "_scale"].double()[:, None]
    g = s["g"].double().view(-1, GROUP)
    m = torch.lerp(g, up("m"), BETA1)
    v = torch.lerp(g.square(), up("v") if case["state"] == "f32" else up("v").square(), BETA2)
    w = s["w"].double().view(-1, GROUP)
    moved = LR * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + EPS)
    w = (w - LR * s["decay"].double() * w - moved).reshape(-1)
    got = {"w": w}
    if case["shadow"]:
        got["shadow"] = w
    if case["state"] == "f32":
        return dict(got, m=m.reshape(-1), v=v.reshape(-1))
    chance = _chance(s).double()
    for name, x, u in (("m", m, chance[:, :, 0::2]), ("v", v.sqrt(), chance[:, :, 1::2])):
        largest = x.abs().amax(1)
        got[name + "_scale"] = largest / TOP
        y = torch.nan_to_num(x.abs() * (TOP / largest)[:, None])
        # the distance of neighbouring e4m3 values around y
        ulp = torch.exp2(torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - 3)
        y = (torch.floor(y / ulp + u.reshape(x.shape)) * ulp).clamp(max=TOP)
        got[name] = torch.copysign(y, x).reshape(-1)
    return got
