"""The tuning step that the projection, the head's loss, the adapter gradients and the factors' update make up together."""
import numpy as np
import pytest
import torch

from paper_2601_21109_b200 import binding as cwl
from paper_2601_21109_b200 import distill_ladder, tune_ladder

pytestmark = pytest.mark.gpu


def gate_of(t, table, T, R):
    tab = table.to_host()
    gate = np.zeros((T, R))
    for c in range(tab["n_chunks"]):
        for r in range(tab["offsets"][c], tab["offsets"][c + 1]):
            j = r - tab["offsets"][c]
            lam = (j + 1) / (t.window + 1) if c > 0 and j < t.window else 1.0
            gate[r, :tab["rank"][c]] += lam * tab["scale"][c]
            if lam < 1:
                gate[r, :tab["rank"][c - 1]] += (1 - lam) * tab["scale"][c - 1]
    return torch.from_numpy(gate).cuda()


@pytest.mark.parametrize("T,dim,V,R", [(200, 128, 1008, 16), (333, 256, 2512, 64)])
def test_gradients_and_update_equal_those_of_the_plain_form(T, dim, V, R):
    """The whole chain against torch's own differentiation of the same step in fp64, and the update against its formula."""
    t = tune_ladder.synthetic(T, dim, V, R=R, lr=0.05, weight_decay=0.1)
    t.gradients()
    gate = gate_of(t, t.table, T, R)
    A, B = t.A.double().requires_grad_(), t.B.double().requires_grad_()
    hidden = t.X.double() @ t.W.double() + (gate * (t.X.double() @ A)) @ B
    # the projection hands its result on in bf16: its values are the rounded ones, their derivative is 1
    hidden = hidden + (t.forward().double() - hidden).detach()
    logq = torch.log_softmax(hidden @ t.head.double(), 1)
    on = t.targets >= 0
    loss = torch.where(on, -logq.gather(1, t.targets.clamp(min=0).long()[:, None])[:, 0], 0.0) * t.weight.double()
    loss.sum().backward()
    assert float((t.loss.double() - loss.detach()).abs().max()) <= 1e-4 * float(t.weight.max())
    # gradients of the head's input are bf16 (2^-9 of a number on the average, and as much again in E), the factors' fp32
    for got, ref in ((t.dA, A.grad), (t.dB, B.grad)):
        assert float((got.double() - ref).norm() / ref.norm()) <= 2.0 ** -8
    before = [p.clone() for p in t.master]
    grads = [g.clone() for g in (t.dA, t.dB)]
    t.update(t.lr, t.momentum, t.weight_decay)
    for p0, p, g, m, low in zip(before, t.master, grads, t.moments, (t.A, t.B)):
        assert torch.equal(m, g)                           # the first step's momentum
        o, = cwl.cwl_orthogonalize([(g.double() + float(np.float32(t.momentum)) * g.double()).float()])
        want = (1 - t.lr * t.weight_decay) * p0.double() - t.lr * max(1.0, p.shape[0] / p.shape[1]) ** 0.5 * o.double()
        assert float((p.double() - want).abs().max()) <= 1e-6 * float(want.abs().max())
        assert torch.equal(low, p.bfloat16())
    assert int(t.status.item()) == 0


def test_a_captured_step_equals_a_launched_one():
    a, b = (tune_ladder.synthetic(300, 256, 2000, R=32) for _ in range(2))
    graph = a.capture()                                    # one step is taken, and one recorded
    b.step()
    for _ in range(3):
        graph.replay()
        b.step()
    torch.cuda.synchronize()
    for x, y in zip(a.master + a.moments + [a.loss], b.master + b.moments + [b.loss]):
        assert torch.equal(x, y)


def test_the_commands_run(capsys, monkeypatch):
    for module, extra in ((tune_ladder, []), (distill_ladder, ["--optimizer", "muon"])):
        monkeypatch.setattr("sys.argv", ["x", "--steps", "4", "--tokens", "256", "--width", "256", "--vocab", "2048", *extra])
        module.main()
        out = capsys.readouterr().out
        assert "before" in out and "after" in out


def test_losses_are_finite_and_weights_move():
    t = tune_ladder.synthetic(512, 256, 4096, R=64)
    start = [p.clone() for p in t.master]
    for _ in range(5):
        t.step()
    assert int(t.status.item()) == 0 and bool(torch.isfinite(t.loss).all())
    assert all(not torch.equal(p, q) for p, q in zip(start, t.master))
