"""A run of the operators together: rows of a trained table through a residual
block, scored against the same table, and every tensor moved by AdamW; its
gradients against automatic differentiation in 64 bits."""
import math

import pytest
import torch

from paper_2303_00158_amd import gnn

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
EPS = 1e-5


class Model:
    """ids -> scale table[ids] -> x + gelu(norm(x) W1 + b1) W2 -> norm -> logits against the table -> loss."""

    def __init__(self, rows, vocab, f, hidden, dt, state=F32):
        gen = torch.Generator().manual_seed(rows + f)
        self.dt, self.rows, self.f, self.scale = dt, rows, f, math.sqrt(f)
        self.gemm = gnn.GNN_BF16 if dt == BF16 else gnn.GNN_F32

        def rand(*shape, scale=1.0, shift=0.0):
            return (torch.randn(shape, generator=gen) * scale + shift).to(DEV)
        self.ids = torch.randint(0, vocab, (rows,), generator=gen).to(DEV)
        self.labels = torch.randint(0, vocab, (rows,), generator=gen).to(DEV)
        self.ids[:rows // 3] = 1  # a frequent one
        self.labels[::5] = -1     # padding
        self.ids[::5] = -1
        live = self.labels >= 0
        self.weight = live.float() / live.sum()
        self.p = {"table": rand(vocab, f, scale=1 / math.sqrt(f)), "gamma1": rand(f, scale=0.1, shift=1.0), "beta1": rand(f, scale=0.1),
                  "w1": rand(f, hidden, scale=1 / math.sqrt(f)), "b1": rand(hidden, scale=0.1),
                  "w2": rand(hidden, f, scale=1 / math.sqrt(hidden)), "b2": rand(f, scale=0.1),
                  "gamma2": rand(f, scale=0.1, shift=1.0), "beta2": rand(f, scale=0.1), "bias": rand(vocab, scale=0.1)}
        # what the bf16 products round is kept in bf16
        self.d = {k: torch.zeros_like(v, dtype=dt if v.dim() == 2 else F32) for k, v in self.p.items()}
        self.table16 = self.p["table"].to(BF16)  # the table's shadow has its layout
        self.wt = {k: self.p[k].t().contiguous().to(BF16) if dt == BF16 else None for k in ("w1", "w2")}

        def buf(*shape, t=dt):
            return torch.zeros(shape, dtype=t, device=DEV)
        self.x, self.n1, self.y, self.n2, self.dy, self.dn, self.dx = (buf(rows, f) for _ in range(7))
        self.z, self.h, self.dh = (buf(rows, hidden) for _ in range(3))
        self.stats = [buf(rows, t=F32) for _ in range(4)]
        self.loss, self.row_loss = buf(1, t=F32), buf(rows, t=F32)
        names = list(self.p)
        self.opt = gnn.AdamW([self.p[k] for k in names], [self.d[k] for k in names], [0.01 if self.p[k].dim() == 2 else 0.0 for k in names],
                             state_dtype=state, shadows=[self.table16 if k == "table" else None for k in names], seed=5)

    def table(self):
        return self.table16 if self.dt == BF16 else self.p["table"]

    def gradients(self):
        p, d, wt, gemm, table = self.p, self.d, self.wt, self.gemm, self.table()
        none, gelu = gnn.GNN_ACT_NONE, gnn.GNN_ACT_GELU
        gnn.embed_fwd(table, self.ids, self.x, self.scale)
        gnn.layer_norm_fwd(self.x, p["gamma1"], p["beta1"], self.n1, EPS, self.stats[0], self.stats[1])
        gnn.update_fwd_act(self.n1, None, p["w1"], p["b1"], self.h, gelu, gemm, z=self.z, wt=wt["w1"])
        gnn.update_fwd_act(self.h, None, p["w2"], p["b2"], self.y, none, gemm, residual=self.x, wt=wt["w2"])
        gnn.layer_norm_fwd(self.y, p["gamma2"], p["beta2"], self.n2, EPS, self.stats[2], self.stats[3])
        gnn.update_ce(self.n2, table, p["bias"], self.labels, self.loss, gemm, row_loss=self.row_loss, d_a=self.dn, dwt=d["table"],
                      db=d["bias"], row_scale=self.weight)
        gnn.layer_norm_bwd(self.dn, self.y, p["gamma2"], self.stats[2], self.stats[3], self.dy, d["gamma2"], d["beta2"])
        gnn.update_bwd_act(self.h, None, p["w2"], None, self.dy, d["w2"], d["b2"], self.dh, none, gemm, wt=wt["w2"])
        gnn.update_bwd_act(self.n1, None, p["w1"], self.z, self.dh, d["w1"], d["b1"], self.dn, gelu, gemm, wt=wt["w1"])
        gnn.layer_norm_bwd(self.dn, self.x, p["gamma1"], self.stats[0], self.stats[1], self.dx, d["gamma1"], d["beta1"], d_res=self.dy)
        # the table's second gradient, onto the first
        gnn.embed_bwd(self.dx, self.ids, d["table"], self.scale, accumulate=True)

    def step(self, **kw):
        self.gradients()
        self.opt.step(**kw)
        for k, v in self.wt.items():
            if v is not None:
                v.copy_(self.p[k].t())

    def exact(self):
        p = {k: v.double().requires_grad_() for k, v in self.p.items()}
        there = self.ids >= 0
        x = torch.where(there[:, None], p["table"][self.ids.clamp(min=0)], 0.0) * self.scale

        def norm(v, gamma, beta):
            c = v - v.mean(1, keepdim=True)
            return c / (c.square().mean(1, keepdim=True) + EPS).sqrt() * gamma + beta
        z = norm(x, p["gamma1"], p["beta1"]) @ p["w1"] + p["b1"]
        y = x + (z * torch.special.ndtr(z)) @ p["w2"] + p["b2"]
        logp = torch.log_softmax(norm(y, p["gamma2"], p["beta2"]) @ p["table"].t() + p["bias"], 1)
        live = self.labels >= 0
        loss = -(logp.gather(1, self.labels.clamp(min=0)[:, None])[:, 0] * self.weight.double())[live].sum()
        loss.backward()
        return {"loss": loss.detach()[None], **{k: v.grad for k, v in p.items()}}


def tolerance(m):
    """Relative to a tensor's norm.  The longest path has 18 tensors between its ends, the
    table's copy among them: in bf16 each is rounded by at most 2^-8 of its values; in fp32 a
    product over K terms is off by at most (K + 4) 2^-24 of their sizes.  Norms and widths here
    keep every factor's gain about 1."""
    most = max([m.rows] + [max(v.shape) for v in m.p.values()])
    return 18 * (2.0 ** -8 if m.dt == BF16 else most * 2.0 ** -24)


CASES = [(1, 10, 32, 64), (70, 47, 96, 200), (333, 1000, 128, 512), (1000, 5003, 256, 1024)]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("state", [F32, torch.float8_e4m3fn])
@pytest.mark.parametrize("rows, vocab, f, hidden", CASES)
def test_gradients_of_a_model_with_a_tied_table(rows, vocab, f, hidden, state, dt):
    m = Model(rows, vocab, f, hidden, dt, state)
    if rows == 1:
        m.ids[0], m.labels[0], m.weight[0] = 3, 4, 1.0
    for t in range(3):
        before = {k: v.clone() for k, v in m.p.items()}
        want = m.exact()
        m.step(lr=1e-3)
        for k, w in want.items():
            got = m.loss if k == "loss" else m.d[k]
            off = float((got.double() - w).norm() / w.norm())
            assert off <= tolerance(m), f"{k}, step {t}: {off:.3g}"
        for k, v in m.p.items():
            assert v.isfinite().all() and not torch.equal(v, before[k]), k
        assert torch.equal(m.table16, m.p["table"].to(BF16))


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("state", [F32, torch.float8_e4m3fn])
def test_a_captured_step_repeats_the_eager_one(state, dt):
    eager, other = (Model(300, 500, 128, 512, dt, state) for _ in range(2))
    t, t2 = torch.ones(1, dtype=torch.int64, device=DEV), torch.ones(1, dtype=torch.int64, device=DEV)
    for m, n in ((eager, t), (other, t2)):
        m.step(lr=1e-3, step_dev=n)
        n.add_(1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        other.step(lr=1e-3, step_dev=t2)
        t2.add_(1)
    for k in range(4):
        eager.step(lr=1e-3, step_dev=t)
        t.add_(1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(eager.loss, other.loss), k
        for name in eager.p:
            assert torch.equal(eager.p[name], other.p[name]) and torch.equal(eager.d[name], other.d[name]), (k, name)
        eager.ids.copy_(eager.ids.roll(1))
        other.ids.copy_(other.ids.roll(1))


@pytest.mark.gpu
def test_two_calls_at_once_with_workspaces_of_their_own():
    made = [Model(300, 700, 64, 128, F32) for _ in range(3)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        made[0].step(lr=1e-3)
        for m, s in zip(made[1:], streams):
            with torch.cuda.stream(s):
                m.step(lr=1e-3)
    torch.cuda.synchronize()
    for m in made[1:]:
        for name in m.p:
            assert torch.equal(m.p[name], made[0].p[name]), name
