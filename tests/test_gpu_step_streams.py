"""A training step on another stream, and a captured one, against results that
are kept apart: every buffer that the step writes is filled with NaN before
the run that is checked, so nothing of the first run can stand in for it."""
import pytest

from paper_2405_14377_amd import comera as C
from tests.test_gpu_step_together import Step

pytestmark = pytest.mark.gpu


def _results(step):
    return [x.clone() for x in [step.out, step.norm, step.grads["T"], step.dX] + step.clipped]


def _forget(step):
    for x in [step.X, step.H, step.Xn, step.out, step.A, step.dA, step.F, step.dF, step.dH, step.dXn, step.dX,
              step.norm, *step.grads.values(), *step.dG[0], *step.dG[1], *step.clipped]:
        x.fill_(float("nan"))
    step.ws.fill_(0xFF)


def test_step_on_another_stream():
    """Every output of the step, that of the second norm among them, is the other stream's own."""
    import torch
    step = Step(2)
    step.inputs(21)
    step.run()
    want = _results(step)
    _forget(step)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step.run()
    side.synchronize()
    assert not any(x.isnan().any() for x in want)
    assert all(torch.equal(a, b) for a, b in zip(_results(step), want))


def test_captured_long_table_gradient_and_list():
    """Replays of a long batch's table gradient and a long list's clipping write all that the eager step wrote."""
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
    written = outs + [norm, dT]

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
        for rep in range(4):
            ids.copy_((torch.rand(n, device="cuda") ** 3 * v).long())
            for x in many[:-1]:
                x.normal_()
            step()
            torch.cuda.synchronize()
            want = [x.clone() for x in written]
            assert not any(x.isnan().any() for x in want)
            for x in written:
                x.fill_(float("nan"))
            ws.fill_(0xFF)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(written, want)), rep
    del g
