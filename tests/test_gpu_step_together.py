"""The operators around the compressed layers run together, as a training
step of a small transformer block uses them: lookup, pre-norm, two TTM layers,
post-norm with gate and residual, loss gradient, the whole way back, and
clipping; eagerly, on another stream and as a replayed graph.  The expected
gradients are those of the same step in fp64.

Tolerance of the step: fp32 throughout, sums of at most 300 tokens and 96
products; the eight operators in a row each add at most a few hundred half
steps of fp32 of the magnitudes that they join (the bounds of their own
tests), 1e-4 of the largest entry in all, as for a TTM layer alone.
"""
import numpy as np
import pytest

from oracle import block_norm as ON
from oracle import dense_embed as OE
from oracle import grad_clip as OG
from oracle import ttm as OT
from paper_2405_14377_amd import comera as C
from paper_2405_14377_amd import workloads as wl
from tests.gpu_util import rel_err

pytestmark = pytest.mark.gpu

V, E, B, EPS, SCALE, RES, BRANCH, MAX = 500, 60, 300, 1e-5, 7.5, 0.9, 0.6, 0.5
N, M, R = (3, 4, 5), (4, 5, 6), (1, 5, 4, 1)          # 60 -> 120 and back


class Step:
    """Parameters, buffers and plans of the step, and the step itself."""

    def __init__(self, seed):
        import torch
        rng = np.random.default_rng(seed)
        self.np = {}

        def par(name, x):
            self.np[name] = np.asarray(x, np.float32)
            return torch.from_numpy(self.np[name]).cuda()

        up, down = wl.TTMLayerShape("up", N, M, R), wl.TTMLayerShape("down", M, N, R)
        self.T = par("T", 0.2 * rng.standard_normal((V, E)))
        self.w = {k: par(k, 1 + 0.2 * rng.standard_normal(E)) for k in ("w1", "wp", "w2", "gate")}
        self.bias = {k: par(k, 0.2 * rng.standard_normal(E)) for k in ("b1", "bp", "b2")}
        self.G = [[par(f"G{i}{k}", 0.5 * c) for k, c in enumerate(wl.random_cores(rng, s))]
                  for i, s in enumerate((up, down))]
        self.plans = [C.TTMPlan(s.n, s.m, s.r, batch=B) for s in (up, down)]

        def buf(*shape):
            return torch.full(shape, float("nan"), device="cuda")

        self.ids = torch.zeros(B, dtype=torch.int64, device="cuda")
        self.dout = buf(B, E)
        self.X, self.H, self.Xn, self.out = (buf(B, E) for _ in range(4))
        self.A, self.dA = buf(B, 120), buf(B, 120)
        self.F, self.dF, self.dH, self.dXn, self.dX = (buf(B, E) for _ in range(5))
        self.grads = {k: torch.empty_like(v) for k, v in (("T", self.T), *self.w.items(), *self.bias.items())}
        self.dG = [[torch.empty_like(g) for g in gs] for gs in self.G]
        self.names = list(self.grads) + [f"G{i}{k}" for i in range(2) for k in range(3)]
        every = list(self.grads.values()) + self.dG[0] + self.dG[1]
        self.clipped = [torch.empty_like(g) for g in every]
        self.plan = C.GradPlan(every, self.clipped)
        self.norm, self.flag = buf(1), torch.zeros(1, dtype=torch.int32, device="cuda")
        self.es = C.dense_embed_shape(V, E)
        self.first = C.block_norm_shape(E, pre=C.NORM_LAYER, eps=EPS)
        self.second = C.block_norm_shape(E, post=C.NORM_RMS, pre=C.NORM_LAYER, gate=C.GATE_CHANNEL, eps=EPS,
                                         res_scale=RES, branch_scale=BRANCH)
        sizes = [C.comera_dense_embed_workspace_bytes(self.es, B), C.comera_block_norm_workspace_bytes(self.second, B),
                 self.plan.workspace_bytes] + [p.workspace_bytes for p in self.plans]
        self.ws = torch.empty(max(sizes), dtype=torch.uint8, device="cuda")     # one for all: nothing carries over

    def run(self):
        w, b, g, ws = self.w, self.bias, self.grads, self.ws
        C.comera_dense_embed_forward(self.es, self.ids, B, self.T, SCALE, self.X, self.flag)
        C.comera_block_norm_forward(self.first, B, self.X, None, None, None, None, w["w1"], b["b1"], None, self.H)
        C.comera_ttm_forward(self.plans[0].handle, B, self.H, self.G[0], None, self.A, ws)
        C.comera_ttm_forward(self.plans[1].handle, B, self.A, self.G[1], None, self.F, ws)
        C.comera_block_norm_forward(self.second, B, self.X, self.F, w["wp"], b["bp"], w["gate"], w["w2"], b["b2"],
                                    self.Xn, self.out)
        C.comera_block_norm_backward(self.second, B, self.Xn, self.F, w["wp"], b["bp"], w["gate"], w["w2"], None,
                                     self.dout, self.dXn, self.dF, g["gate"], g["wp"], g["bp"], g["w2"], g["b2"], ws)
        C.comera_ttm_backward(self.plans[1].handle, B, self.A, self.dF, self.G[1], None, self.dA, self.dG[1], ws)
        C.comera_ttm_backward(self.plans[0].handle, B, self.H, self.dA, self.G[0], None, self.dH, self.dG[0], ws)
        C.comera_block_norm_backward(self.first, B, self.X, None, None, None, None, w["w1"], self.dXn, self.dH,
                                     self.dX, None, None, None, None, g["w1"], g["b1"], ws)
        C.comera_dense_embed_backward(self.es, self.ids, B, self.dX, SCALE, 0, g["T"], ws, self.flag)
        C.comera_grad_clip(self.plan.handle, 1.0, MAX, self.norm, self.flag, ws)

    def results(self):
        import torch
        return [self.out, self.norm] + [torch.clone(x) for x in self.clipped]

    def inputs(self, seed):
        import torch
        rng = np.random.default_rng(seed)
        ids = rng.integers(0, V, B)
        ids[rng.random(B) < 0.2] = 0              # padding
        ids[rng.random(B) < 0.2] = 7
        dout = rng.standard_normal((B, E)).astype(np.float32)
        self.ids.copy_(torch.from_numpy(ids))
        self.dout.copy_(torch.from_numpy(dout))
        return ids, dout.astype(np.float64)

    def oracle(self, ids, dout):
        p = {k: v.astype(np.float64) for k, v in self.np.items()}
        Gs = [[p[f"G{i}{k}"] for k in range(3)] for i in range(2)]
        X = OE.forward(ids, p["T"], SCALE)
        _, H = ON.forward(X, None, "none", None, None, None, "layer", p["w1"], p["b1"], EPS, 1, 1)
        A = OT.forward_dense(H, Gs[0], None)
        F = OT.forward_dense(A, Gs[1], None)
        Xn, out = ON.forward(X, F, "rms", p["wp"], p["bp"], p["gate"], "layer", p["w2"], p["b2"], EPS, RES, BRANCH)
        d2 = ON.backward(Xn, F, "rms", p["wp"], p["bp"], p["gate"], "layer", p["w2"], None, dout, EPS, RES, BRANCH)
        dA, dG1 = OT.backward_dense(A, d2["dF"], Gs[1], None)
        dH, dG0 = OT.backward_dense(H, dA, Gs[0], None)
        d1 = ON.backward(X, None, "none", None, None, None, "layer", p["w1"], d2["dX"], dH, EPS, 1, 1)
        dT = OE.backward(ids, d1["dX"], V, SCALE, 0)
        got = {"T": dT, "w1": d1["dpre_w"], "b1": d1["dpre_b"], "wp": d2["dpost_w"], "bp": d2["dpost_b"],
               "w2": d2["dpre_w"], "b2": d2["dpre_b"], "gate": d2["dgate"],
               **{f"G{i}{k}": (dG0, dG1)[i][k] for i in range(2) for k in range(3)}}
        norm, clipped = OG.clip([got[k] for k in self.names], 1.0, MAX)
        return out, norm, clipped


def _check(step, ids, dout):
    out, norm, clipped = step.oracle(ids, dout)
    assert rel_err(step.out.cpu().numpy(), out) <= 1e-4
    assert step.norm.item() == pytest.approx(norm, rel=1e-4) and step.flag.item() == 0
    for name, g, r in zip(step.names, step.clipped, clipped):
        assert rel_err(g.cpu().numpy(), r) <= 1e-4, name


def test_step_matches_the_oracle():
    step = Step(1)
    for seed in (11, 12):
        ids, dout = step.inputs(seed)
        step.run()
        _check(step, ids, dout)


def test_step_on_another_stream():
    import torch
    step = Step(2)
    ids, dout = step.inputs(21)
    step.run()
    want = step.results()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for x in step.clipped:
        x.fill_(float("nan"))
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step.run()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(step.results(), want))


def test_two_captured_steps_with_a_workspace_each():
    """Replays of two graphs between the program's own eager work, every replay against the eager step."""
    import torch
    steps, eager = [Step(3), Step(4)], [Step(3), Step(4)]
    graphs = []
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for s in steps:
            s.inputs(30)
            s.run()
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                s.run()
            graphs.append(g)
        torch.cuda.synchronize()
        for rep in range(4):
            for s, e, g in zip(steps, eager, graphs):
                s.inputs(40 + rep)
                e.inputs(40 + rep)
                e.run()
                torch.cuda.synchronize()
                g.replay()
                torch.cuda.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(s.results(), e.results())), rep
        _check(steps[0], *steps[0].inputs(43))
    del graphs


def test_captured_long_table_gradient_and_list():
    """The forms for long batches and long lists, captured: three launches more, the list's table written before."""
    import torch
    n, v, e = 30000, 3000, 24
    s = C.dense_embed_shape(v, e, C.F32, C.BF16)
    torch.manual_seed(5)
    dY = torch.randn((n, e), device="cuda").bfloat16()
    ids = torch.zeros(n, dtype=torch.int64, device="cuda")
    dT = torch.empty((v, e), device="cuda")
    many = [torch.empty(17, device="cuda") for _ in range(200)] + [dT]
    outs = [torch.empty_like(x) for x in many]
    plan = C.GradPlan(many, outs)
    ws = torch.empty(C.comera_dense_embed_workspace_bytes(s, n), dtype=torch.uint8, device="cuda")
    norm = torch.zeros(1, device="cuda")

    def step():
        C.comera_dense_embed_backward(s, ids, n, dY, 1.0, 3, dT, ws)
        C.comera_grad_clip(plan.handle, 1.0, 1.0, norm, None, ws)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step()
        for rep in range(3):
            ids.copy_((torch.rand(n, device="cuda") ** 3 * v).long())
            for x in many[:-1]:
                x.normal_()
            step()
            torch.cuda.synchronize()
            want = [x.clone() for x in outs] + [norm.clone(), dT.clone()]
            for x in outs:
                x.zero_()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs + [norm, dT], want)), rep
    del g
