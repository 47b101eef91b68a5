"""Marshalled factor calls follow their tensors: new storage, other strides, replaced attributes of the two ladders."""
import pytest
import torch

from paper_2601_21109_b200 import binding as cwl
from paper_2601_21109_b200 import distill_ladder, tune_ladder

pytestmark = pytest.mark.gpu
SHAPES = [(64, 300), (300, 100)]


def padded(t, pad):
    """The same values in another place, rows `pad` elements further apart."""
    out = torch.full((t.shape[0], t.shape[1] + pad), 7.0, dtype=t.dtype, device=t.device)[:, :t.shape[1]]
    return out.copy_(t)


@pytest.mark.parametrize("pad", [0, 3, 8])
def test_orthogonalize_follows_new_storage(pad):
    torch.manual_seed(0)
    us = [torch.randn(*s, device="cuda") for s in SHAPES]
    call = cwl.OrthogonalizeCall(us, [torch.empty_like(u) for u in us])
    outs = call()
    kept = [t.data for t in us + list(outs)]               # what the call was made with stays allocated, and untouched
    before = [t.clone() for t in kept]
    for u in us:
        u.data = padded(torch.randn_like(u), pad)
    for o in outs:
        o.data = padded(torch.zeros_like(o), pad)
    call()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, cwl.cwl_orthogonalize([u.clone() for u in us])))
    assert all(torch.equal(a, b) for a, b in zip(kept, before))


@pytest.mark.parametrize("which", ["master", "low", "grad", "momentum"])
@pytest.mark.parametrize("pad", [0, 5])
def test_step_follows_new_storage(which, pad):
    def make():
        torch.manual_seed(1)
        p, g, m = ([torch.randn(*s, device="cuda") for s in SHAPES] for _ in range(3))
        return dict(master=p, low=[t.bfloat16() for t in p], grad=g, momentum=m)

    def call_of(s):
        return cwl.FactorStep(s["master"], s["low"], s["grad"], s["momentum"])
    a, b = make(), make()
    call = call_of(a)
    call(0.1)
    call_of(b)(0.1)
    kept = [t.data for t in a[which]]
    before = [t.clone() for t in kept]
    for t, same in zip(a[which], b[which]):
        t.data = padded(t.data, pad)
        t.mul_(1.25), same.mul_(1.25)
    call(0.1)
    call_of(b)(0.1)
    torch.cuda.synchronize()
    for name in a:
        assert all(torch.equal(x, y) for x, y in zip(a[name], b[name])), name
    assert all(torch.equal(x, y) for x, y in zip(kept, before))


def test_tensors_that_no_longer_fit_are_refused():
    p, g, m = (torch.randn(64, 300, device="cuda") for _ in range(3))
    call = cwl.FactorStep([p], None, [g], [m])
    call(0.1)
    with torch.no_grad():
        p.resize_(64, 400)
    for _ in range(2):                                     # not only the first time
        with pytest.raises(AssertionError):
            call(0.1)
    u = torch.randn(64, 300, device="cuda")
    call = cwl.OrthogonalizeCall([u], [torch.empty_like(u)])
    call()
    u.data = u.data.cpu()
    with pytest.raises(AssertionError):
        call()


def twins(module, **kw):
    return [module.synthetic(256, 128, 2000, R=16, **kw) for _ in range(2)]


@pytest.mark.parametrize("kind", ["distil", "tune"])
def test_ladders_follow_what_is_replaced(kind):
    a, b = twins(distill_ladder, optimizer="muon") if kind == "distil" else twins(tune_ladder)
    for t in (a, b):
        t.step()
    kept = [a.A, a.B, a.dA, a.dB, *a.master] + [m for m, _ in a.moments] if kind == "distil" else [a.A, a.B, a.dA, a.dB, *a.master, *a.moments]
    a.A, a.B, a.dA, a.dB = (t.clone() for t in (a.A, a.B, a.dA, a.dB))
    a.master = [p.clone() for p in a.master]
    a.moments = [(m.clone(), v) for m, v in a.moments] if kind == "distil" else [m.clone() for m in a.moments]
    before = [t.clone() for t in kept]
    for _ in range(2):
        for t in (a, b):
            t.step()
    torch.cuda.synchronize()
    assert torch.equal(a.A, b.A) and torch.equal(a.B, b.B) and torch.equal(a.loss, b.loss)
    assert all(torch.equal(p, q) for p, q in zip(a.master, b.master))
    assert all(torch.equal(p, q) for p, q in zip(kept, before))
    assert a.update is a.update.of(*a.update.keep)         # nothing is made anew for the same tensors
