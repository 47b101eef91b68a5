"""The tuning calls give the same bits whatever their workspace held before: nothing of it is read that the call has not written."""
import pytest
import torch

from paper_2601_21109_b200 import binding as cwl
from test_gpu_factors import factor
from test_gpu_head import operands

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,d,V", [(1, 64, 500), (40, 72, 3001), (100, 2048, 1000), (300, 1032, 5003), (1100, 96, 4000), (5000, 64, 60001)])
@pytest.mark.parametrize("kw", [dict(), dict(want_dx=True), dict(want_dw=True), dict(want_dx=True, want_dw=True)])
@pytest.mark.parametrize("grad", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("backward", [False, True])
def test_head_loss(T, d, V, kw, grad, backward):
    if backward and not kw:
        return
    X, W, y, w = operands(T, T, d, V)
    y[::3] = -1
    if backward:
        kw = dict(kw, want_loss=False, lse=cwl.cwl_head_loss(X, W, y, weight=w).lse, dloss=torch.rand(T, device="cuda"))
    n = cwl.cwl_head_loss_workspace_bytes(T, d, V, kw.get("want_dx", False), kw.get("want_dw", False))
    got = []
    for fill in (0, 255, 1):
        ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
        o = cwl.cwl_head_loss(X, W, y, weight=w, grad_dtype=grad, workspace=ws, **kw)
        got.append([t.clone() for t in (o.loss, o.dX, o.dW) if t is not None])
    assert all(torch.equal(a, b) for other in got[1:] for a, b in zip(got[0], other))
    assert all(bool(torch.isfinite(t).all()) for t in got[0])


@pytest.mark.parametrize("shapes", [[(16, 300), (64, 5000)], [(100, 400), (400, 200), (33, 90)], [(256, 3000)]])
@pytest.mark.parametrize("steps", [1, 2, 5])
def test_factors(shapes, steps):
    got = []
    for fill in (0, 255, 1):
        us = [factor(i, *s) for i, s in enumerate(shapes)]
        p, m = [torch.ones_like(u) for u in us], [torch.ones_like(u) for u in us]
        n = cwl.OrthogonalizeCall(us, [torch.empty_like(u) for u in us], steps=steps).workspace.numel()
        ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
        o = cwl.cwl_orthogonalize(us, steps=steps, workspace=ws)
        ws.fill_(fill)
        cwl.FactorStep(p, None, us, m, steps=steps, workspace=ws)(0.1)
        got.append(list(o) + p + m)
    assert all(torch.equal(a, b) for other in got[1:] for a, b in zip(got[0], other))
    assert all(bool(torch.isfinite(t).all()) for t in got[0])
