"""The training step that the log-probability, distillation and adapter-gradient calls make up with the projection."""
import numpy as np
import pytest
import torch

from paper_2601_21109_b200.distill_ladder import synthetic

pytestmark = pytest.mark.gpu


def test_gradients_equal_those_of_the_plain_form():
    """The whole chain against torch's own differentiation of the same step in fp64 (projection, gate, softmax, loss)."""
    T, dim, V, R, tau = 200, 128, 512, 16, 2.0
    d = synthetic(T, dim, V, R=R, top_k=8, temperature=tau)
    d.gradients()
    t = d.table.to_host()
    gate = np.zeros((T, R))
    for c in range(t["n_chunks"]):
        for r in range(t["offsets"][c], t["offsets"][c + 1]):
            j = r - t["offsets"][c]
            lam = (j + 1) / (d.window + 1) if c > 0 and j < d.window else 1.0
            gate[r, :t["rank"][c]] += lam * t["scale"][c]
            if lam < 1:
                gate[r, :t["rank"][c - 1]] += (1 - lam) * t["scale"][c - 1]
    gate = torch.from_numpy(gate).cuda()
    A, B = d.A.double().requires_grad_(), d.B.double().requires_grad_()
    y = d.X.double() @ d.W.double() + (gate * (d.X.double() @ A)) @ B
    # the projection hands its logits on in bf16: their values are the rounded ones, their derivative is 1
    y = y + (d.forward().double() - y).detach()
    logq = torch.log_softmax(y / tau, 1)
    ids, lp = d.teacher.top_ids.long(), d.teacher.top_logprobs.double()
    p = lp.exp()
    rest = (1 - p.sum(1)).clamp(min=0)
    q_rest = 1 - logq.gather(1, ids).exp().sum(1)
    loss = tau ** 2 * ((p * (lp - logq.gather(1, ids))).sum(1) + rest * (rest / q_rest).log()) / T
    loss.sum().backward()
    # bf16 gradients of the logits: half a spacing, 2^-8 of a number, in every one of the terms that a gradient sums
    assert float((d.loss.double() - loss.detach()).abs().max()) <= 1e-5 * tau ** 2
    for got, ref in ((d.dA, A.grad), (d.dB, B.grad)):
        assert float((got.double() - ref).norm() / ref.norm()) <= 2.0 ** -8


def test_training_brings_the_prefixes_closer_to_the_full_adapter():
    d = synthetic(512, 256, 2048, R=64, lr=2e-3)
    d.gradients()
    before, agree = float(d.loss.sum()), d.agreement()
    for _ in range(60):
        d.step()
    d.gradients()
    after = float(d.loss.sum())
    assert int(d.status.item()) == 0
    assert after < 0.7 * before and d.agreement() > agree
