"""Layer normalisation, the update with activation and residual, and the
distillation loss: what a pass through each costs.

Each case is one call of one operator, forward or backward, as a training or
serving program makes it.  Widths and row counts are those of the repository's
models (hidden width 256, the 768-feature model's 1,536 x 1,024 layer, 47
classes, 1,024 targets, 26,624 rows of a mini-batch) and generic ones up to the
largest layers and class counts that one card trains.

  listed()          the fixed cases
  draw(rng)         one more case of the same ranges
  prepare(case, s)  the inputs a program holds before the call, from seed s
  run(state)        one pass; returns its outputs
  work(case)        bytes and operations a pass cannot do without
  exact(case, s)    run()'s result in 64 bits

Operators, for rows i and columns j (act: none, relu, gelu, gelu_tanh, silu):

  ln_fwd    mu_i, r_i = mean and 1 / sqrt(variance + eps) of x_i;
            y = gamma (x - mu) r + beta
  ln_bwd    from g = dLoss/dy:  q = gamma g, h = (x - mu) r,
            dx = r (q - mean(q) - h mean(q h)) + residual gradient,
            dgamma = sum_i g h, dbeta = sum_i g
  act_fwd   z = a w + b, out = act(z) + residual; z is kept for the backward
  act_bwd   dz = g act'(z), dw = a^T dz, db = sum_i dz, da = dz w^T
  distill   p_i = softmax of the teacher's top entries over T, s = row scale:
            soft_i = T^2 sum_e p_ie (log p_ie - log softmax(z_i / T)[idx_ie]),
            hard_i = -log softmax(z_i)[label_i],
            loss = sum_i s_i (alpha soft_i + (1 - alpha) hard_i) and dLoss/dz;
            entries with a negative index and rows with a negative label are
            absent

Where the matrix products run in bf16, the weights are read from their bf16
shadow and a weight gradient that was summed from rounded products is kept in
bf16 too.
"""
import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
EPS = 1e-5
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # a serving program normalises the one row it answers with
        dict(name="ln-fwd-1x4096", op="ln_fwd", rows=1, f=4096, dtype="bf16"),
        # the rows of an ordinary mini-batch at the hidden width, fp32 model
        dict(name="ln-fwd-26624x256-f32", op="ln_fwd", rows=26_624, f=256, dtype="f32"),
        # a large batch of wide rows
        dict(name="ln-fwd-32768x8192", op="ln_fwd", rows=32_768, f=8192, dtype="bf16"),
        # a training step of an fp32 model whose width is no multiple of anything
        dict(name="ln-bwd-7585x1001-f32", op="ln_bwd", rows=7585, f=1001, dtype="f32", residual=False),
        # a residual block of a wide model: the skip's gradient is added on the way
        dict(name="ln-bwd-16384x4096", op="ln_bwd", rows=16_384, f=4096, dtype="bf16", residual=True),
        # one row through a square layer: the weights' bytes and latency
        dict(name="act-fwd-1x4096x4096", op="act_fwd", rows=1, k=4096, n=4096, act="silu", dtype="bf16",
             residual=True, keep=False),
        # the wide layer of the 768-feature model with a residual, for training
        dict(name="act-fwd-26624x1536x1024", op="act_fwd", rows=26_624, k=1536, n=1024, act="gelu", dtype="bf16",
             residual=True, keep=True),
        # the largest layer
        dict(name="act-fwd-16384x4096x8192", op="act_fwd", rows=16_384, k=4096, n=8192, act="gelu_tanh", dtype="bf16",
             residual=False, keep=True),
        # a small fp32 model's layer backwards: launches and latency
        dict(name="act-bwd-1461x64x47-f32", op="act_bwd", rows=1461, k=64, n=47, act="silu", dtype="f32"),
        # a wide layer backwards
        dict(name="act-bwd-8192x4096x4096", op="act_bwd", rows=8192, k=4096, n=4096, act="gelu", dtype="bf16"),
        # a mini-batch's targets and classes, a teacher of eight entries, labels beside it
        dict(name="distill-1024x47-f32", op="distill", rows=1024, c=47, top=8, dtype="f32", temp=2.0, alpha=0.7,
             scaled=False),
        # a large class count that is odd, rows padded to a rectangle
        dict(name="distill-4096x100003", op="distill", rows=4096, c=100_003, top=64, dtype="bf16", temp=1.0,
             alpha=1.0, scaled=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["ln_fwd", "ln_bwd", "act_fwd", "act_fwd", "act_bwd", "distill"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op in ("ln_fwd", "ln_bwd"):
        f = rng.choice([64, 100, 128, 256, 602, 768, 1024, 4096, _log(rng, 16, 16_384)])
        rows = _log(rng, 1, min(65_536, (1 << 28) // f))
        case = dict(op=op, rows=rows, f=f, dtype=dtype)
        return case if op == "ln_fwd" else dict(case, residual=rng.random() < 0.6)
    if op == "distill":
        c = rng.choice([8, 47, 153, 172, 1000, 32_000, 131_072, _log(rng, 100, 200_000)])
        return dict(op=op, rows=_log(rng, 1, min(16_384, 400_000_000 // c)), c=c, top=_log(rng, 1, min(c, 128)),
                    dtype=dtype, temp=rng.choice([1.0, 2.0, 4.0]), alpha=rng.choice([1.0, 0.5, 0.9]),
                    scaled=rng.random() < 0.4)
    # fp32 products are those of small models
    top = 8192 if dtype == "bf16" else 1024
    k, n = (rng.choice([64, 100, 256, 512, 1024, _log(rng, 16, top)] + ([4096] if dtype == "bf16" else []))
            for _ in range(2))
    most = (1 << 39 if dtype == "bf16" else 1 << 35) // (k * n * (1 if op == "act_fwd" else 2))
    case = dict(op=op, rows=_log(rng, 1, max(2, min(32_768, most))), k=k, n=n, act=rng.choice(ACTS), dtype=dtype)
    return dict(case, residual=rng.random() < 0.5, keep=rng.random() < 0.6) if op == "act_fwd" else case


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _randn(g, *shape, dtype=torch.float32, scale=1.0, shift=0.0):
    return (torch.randn(shape, generator=g, device=DEVICE).mul_(scale).add_(shift)).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(int(seed))
    op, rows, dt = case["op"], case["rows"], DTYPES[case["dtype"]]
    empty = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=DEVICE)  # noqa: E731
    s = {"case": case}
    if op in ("ln_fwd", "ln_bwd"):
        f = case["f"]
        # a residual stream: rows of different size, off zero
        x = torch.randn((rows, f), generator=g, device=DEVICE)
        x.mul_(torch.rand((rows, 1), generator=g, device=DEVICE).mul_(2.0).add_(0.5)).add_(_randn(g, rows, 1, scale=0.5))
        s["x"] = x.to(dt)
        s["gamma"], s["beta"] = _randn(g, f, scale=0.1, shift=1.0), _randn(g, f, scale=0.1)
        if op == "ln_fwd":
            return dict(s, y=empty(rows, f, dtype=dt), mean=empty(rows), rstd=empty(rows))
        x = s["x"].double()
        var, mu = torch.var_mean(x, dim=1, unbiased=False)
        s["mean"], s["rstd"] = mu.float(), (var + EPS).rsqrt().float()
        s["g"] = _randn(g, rows, f, dtype=dt, scale=1e-2)
        s["d_res"] = _randn(g, rows, f, dtype=dt, scale=1e-2) if case["residual"] else None
        return dict(s, d_x=empty(rows, f, dtype=dt), dgamma=empty(f), dbeta=empty(f))
    if op in ("act_fwd", "act_bwd"):
        k, n = case["k"], case["n"]
        s["a"] = _randn(g, rows, k, dtype=dt)
        s["w"] = _randn(g, k, n, scale=1.0 / math.sqrt(k))
        s["wt"] = s["w"].t().contiguous().bfloat16() if case["dtype"] == "bf16" else None
        if op == "act_fwd":
            s["bias"] = _randn(g, n, scale=0.1)
            s["residual"] = _randn(g, rows, n, dtype=dt) if case["residual"] else None
            return dict(s, out=empty(rows, n, dtype=dt), z=empty(rows, n, dtype=dt) if case["keep"] else None)
        s["z"] = _randn(g, rows, n, dtype=dt)
        s["g"] = _randn(g, rows, n, dtype=dt, scale=1e-2)
        return dict(s, dw=empty(k, n, dtype=dt), db=empty(n), d_a=empty(rows, k, dtype=dt))
    c, top = case["c"], case["top"]
    teacher = _randn(g, rows, c, scale=2.0)
    val, idx = torch.topk(teacher, top, dim=1)
    # a student that agrees with its teacher in part
    s["logits"] = teacher.mul_(0.6).add_(torch.randn((rows, c), generator=g, device=DEVICE)).to(dt)
    s["teacher"], s["idx"] = val.to(dt), idx
    # some rows have fewer entries than the table is wide
    few = torch.randint(1, top + 1, (rows, 1), generator=g, device=DEVICE)
    some = torch.rand((rows, 1), generator=g, device=DEVICE) < 0.25
    s["idx"][some & (torch.arange(top, device=DEVICE)[None, :] >= few)] = -1
    s["labels"] = torch.randint(0, c, (rows,), generator=g, device=DEVICE) if case["alpha"] < 1.0 else None
    s["scale"] = None
    if case["scaled"]:
        # one row in sixteen is padding; the others share the weight
        live = (torch.arange(rows, device=DEVICE) % 16 != 15).float()
        s["scale"] = live / live.sum()
    return dict(s, g_out=empty(rows, c, dtype=dt), loss=empty(1), row_loss=empty(rows))


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
    if op == "ln_fwd":
        gnn.layer_norm_fwd(s["x"], s["gamma"], s["beta"], s["y"], EPS, s["mean"], s["rstd"])
        return s["y"], s["mean"], s["rstd"]
    if op == "ln_bwd":
        if "ws" not in s:
            s["ws"] = gnn.layer_norm_bwd_workspace(case["f"], case["rows"], DEVICE)
        gnn.layer_norm_bwd(s["g"], s["x"], s["gamma"], s["mean"], s["rstd"], s["d_x"], s["dgamma"], s["dbeta"],
                           s["d_res"], ws=s["ws"])
        return s["d_x"], s["dgamma"], s["dbeta"]
    if op == "distill":
        if "ws" not in s:
            s["ws"] = gnn.distill_topk_workspace(case["rows"], case["c"], case["top"], DEVICE)
        gnn.distill_topk(s["logits"], s["teacher"], s["idx"], case["temp"], s["g_out"], s["loss"], s["row_loss"],
                         alpha=case["alpha"], labels=s["labels"], row_scale=s["scale"], ws=s["ws"])
        return s["loss"], s["row_loss"], s["g_out"]
    gemm = gnn.GNN_BF16 if case["dtype"] == "bf16" else gnn.GNN_F32
    act = ACTS.index(case["act"])
    if op == "act_fwd":
        if "ws" not in s:
            s["ws"] = gnn.update_fwd_act_workspace(s["a"], None, case["n"], gemm, s["wt"] is not None)
        gnn.update_fwd_act(s["a"], None, s["w"], s["bias"], s["out"], act, gemm, residual=s["residual"], z=s["z"],
                           wt=s["wt"], ws=s["ws"])
        return (s["out"], s["z"]) if case["keep"] else (s["out"],)
    if "ws" not in s:
        s["ws"] = gnn.update_bwd_act_workspace(s["a"], None, case["n"], gemm, s["wt"] is not None, s["g"].dtype,
                                               s["dw"].dtype)
    gnn.update_bwd_act(s["a"], None, s["w"], s["z"], s["g"], s["dw"], s["db"], s["d_a"], act, gemm, wt=s["wt"],
                       ws=s["ws"])
    return s["dw"], s["db"], s["d_a"]


def _phi(z):
    return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "gelu":
        return z * _phi(z)
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _slope(z, act):
    """act'(z)"""
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return _phi(z) + z * torch.exp(-0.5 * z * z) * math.sqrt(0.5 / math.pi)
    if act == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 0.134145 * z * z)
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-z))
        return p * (1.0 + z * (1.0 - p))
    return torch.ones_like(z)


def _plain(s):
    """The operators from elementary operations in 32 bits."""
    case = s["case"]
    op = case["op"]
    if op == "ln_fwd":
        x = s["x"].float()
        mean = x.mean(1, keepdim=True)
        d = x - mean
        rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
        y = (d * rstd * s["gamma"] + s["beta"]).to(s["x"].dtype)
        return y, mean[:, 0], rstd[:, 0]
    if op == "ln_bwd":
        x, g, rstd = s["x"].float(), s["g"].float(), s["rstd"][:, None]
        h = (x - s["mean"][:, None]) * rstd
        q = g * s["gamma"]
        dx = rstd * (q - q.mean(1, keepdim=True) - h * (q * h).mean(1, keepdim=True))
        if case["residual"]:
            dx = dx + s["d_res"].float()
        return dx.to(s["x"].dtype), (g * h).sum(0), g.sum(0)
    if op == "act_fwd":
        w = s["w"] if s["wt"] is None else s["wt"].float().t()
        z = s["a"].float() @ w + s["bias"]
        out = _act(z, case["act"])
        if case["residual"]:
            out = out + s["residual"].float()
        out = out.to(s["a"].dtype)
        return (out, z.to(s["a"].dtype)) if case["keep"] else (out,)
    if op == "act_bwd":
        w = s["w"].t() if s["wt"] is None else s["wt"].float()
        dz = s["g"].float() * _slope(s["z"].float(), case["act"])
        return (s["a"].float().t() @ dz).to(s["a"].dtype), dz.sum(0), (dz @ w).to(s["a"].dtype)
    z, temp, alpha = s["logits"].float(), case["temp"], case["alpha"]
    rows = case["rows"]
    there = s["idx"] >= 0
    at = s["idx"].clamp(min=0)
    t = torch.where(there, s["teacher"].float() / temp, -math.inf)
    logp = torch.where(there, t - torch.logsumexp(t, 1, keepdim=True), 0.0)
    p = torch.where(there, torch.exp(logp), 0.0)
    y = z / temp
    logq = y - torch.logsumexp(y, 1, keepdim=True)
    row = (temp * temp * alpha) * (p * (logp - logq.gather(1, at))).sum(1)
    g = torch.exp(logq).scatter_add_(1, at, -p).mul_(alpha * temp)
    if s["labels"] is not None:
        logq = z - torch.logsumexp(z, 1, keepdim=True)
        label = s["labels"][:, None]
        row = row - (1.0 - alpha) * logq.gather(1, label)[:, 0]
        g = g + torch.exp(logq).scatter_add_(1, label, torch.full_like(label, -1.0, dtype=torch.float32)) * (1.0 - alpha)
    if s["scale"] is None:
        return row.sum()[None] / rows, row, (g / rows).to(s["logits"].dtype)
    row = torch.where(s["scale"] != 0, row, 0.0)
    return (row * s["scale"]).sum()[None], row, (g * s["scale"][:, None]).to(s["logits"].dtype)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    op, m, e = case["op"], case["rows"], SIZE[case["dtype"]]
    if op == "ln_fwd":
        f = case["f"]
        return {"bytes": 2 * m * f * e + 8 * f + 8 * m, "flops": 8 * m * f}
    if op == "ln_bwd":
        f = case["f"]
        return {"bytes": (4 if case["residual"] else 3) * m * f * e + 12 * f + 8 * m, "flops": 14 * m * f}
    if op == "distill":
        c, top = case["c"], case["top"]
        live = m - m // 16 if case["scaled"] else m
        terms = 2 if case["alpha"] < 1.0 and case["temp"] != 1.0 else 1
        return {"bytes": (live + m) * c * e + live * top * (8 + e) + m * (4 + 4 * case["scaled"]) + 4,
                "flops": live * c * 5 * terms}
    k, n = case["k"], case["n"]
    if op == "act_fwd":
        return {"bytes": m * k * e + k * n * e + 4 * n + m * n * e * (1 + case["residual"] + case["keep"]),
                "flops": 2 * m * k * n}
    return {"bytes": 2 * m * k * e + 2 * k * n * e + 4 * n + 2 * m * n * e, "flops": 4 * m * k * n}


# ---------------------------------------------------------------------------
# in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    up = lambda name: s[name].double()  # noqa: E731
    if op == "ln_fwd":
        x = up("x")
        var, mu = torch.var_mean(x, dim=1, unbiased=False)
        x = (x - mu[:, None]).div_((var + EPS).sqrt()[:, None])
        return x.mul_(up("gamma")).add_(up("beta")), mu, (var + EPS).rsqrt()
    if op == "ln_bwd":
        # the Jacobian of the normalised row: (1 - (1 1^T + h h^T) / f) r
        f, g = case["f"], up("g")
        h = (up("x") - up("mean")[:, None]) * up("rstd")[:, None]
        dgamma, dbeta = torch.mul(g, h).sum(0), g.sum(0)
        q = g.mul_(up("gamma"))
        dx = q - (q.sum(1)[:, None] + h * torch.mul(q, h).sum(1)[:, None]) / f
        dx = dx * up("rstd")[:, None]
        return dx + up("d_res") if case["residual"] else dx, dgamma, dbeta
    if op in ("act_fwd", "act_bwd"):
        w = up("w") if s["wt"] is None else up("wt").t()
        z = torch.addmm(up("bias"), up("a"), w) if op == "act_fwd" else up("z")
        z.requires_grad_(op == "act_bwd")
        if case["act"] == "relu":
            y = z.clamp(min=0)
        elif case["act"] == "gelu":
            y = z * torch.special.ndtr(z)
        elif case["act"] == "gelu_tanh":
            # (1 + tanh u) / 2 = 1 / (1 + exp(-2 u))
            y = z * torch.sigmoid(math.sqrt(8.0 / math.pi) * (z + 0.044715 * z.pow(3)))
        elif case["act"] == "silu":
            y = z * torch.sigmoid(z)
        else:
            y = z * 1.0
        if op == "act_fwd":
            y = y + up("residual") if case["residual"] else y
            return (y, z) if case["keep"] else (y,)
        y.backward(up("g"))
        dz = z.grad
        return torch.mm(up("a").t(), dz), dz.sum(0), torch.mm(dz, w.t())
    z, t, temp, alpha = up("logits"), up("teacher"), case["temp"], case["alpha"]
    rows, c = z.shape
    there = s["idx"] >= 0
    share = torch.softmax(torch.where(there, t / temp, -math.inf), dim=1)
    target = torch.zeros_like(z).scatter_add_(1, s["idx"].clamp(min=0), share)
    scale = up("scale") if case["scaled"] else torch.full((rows,), 1.0 / rows, dtype=torch.float64, device=DEVICE)
    logq = torch.log_softmax(z / temp, dim=1)
    row = alpha * temp * temp * (torch.special.entr(share).neg().sum(1) - torch.mul(target, logq).sum(1))
    g = logq.exp_().sub_(target).mul_(alpha * temp)
    del target, logq
    if s["labels"] is not None:
        logq = torch.log_softmax(z, dim=1)
        row = row - (1.0 - alpha) * logq[torch.arange(rows, device=DEVICE), s["labels"]]
        logq.exp_()
        logq[torch.arange(rows, device=DEVICE), s["labels"]] -= 1.0
        g = g.add_(logq, alpha=1.0 - alpha)
    row = torch.where(scale != 0, row, 0.0)
    return torch.dot(row, scale)[None], row, g.mul_(scale[:, None])
