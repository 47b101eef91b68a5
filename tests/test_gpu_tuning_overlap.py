"""Tuning calls on matrices that share a buffer: between one another's rows as if they were apart, in one another's place refused."""
import pytest
import torch

from paper_2601_21109_b200 import binding as cwl

pytestmark = pytest.mark.gpu


def beside(*tensors):
    """The tensors as columns of one buffer."""
    return torch.cat(tensors, 1).split([t.shape[1] for t in tensors], 1)


@pytest.mark.parametrize("T,d,V", [(5, 64, 96), (300, 72, 1000)])
def test_head_gradients_beside_their_inputs(T, d, V):
    torch.manual_seed(0)
    X, W = torch.randn(T, d, device="cuda").bfloat16(), torch.randn(d, V, device="cuda").bfloat16()
    y = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32)
    want = cwl.cwl_head_loss(X, W, y, want_dx=True, want_dw=True)
    X2, dX = beside(X, torch.zeros_like(X))
    W2, dW = beside(W, torch.zeros_like(W))
    got = cwl.cwl_head_loss(X2, W2, y, dX=dX, dW=dW)
    assert torch.equal(got.dX, want.dX) and torch.equal(got.dW, want.dW) and torch.equal(X2, X) and torch.equal(W2, W)
    for kw in (dict(dX=X2), dict(dW=W2), dict(dX=X2.as_strided((T, d), X2.stride(), X2.storage_offset() + 1))):
        with pytest.raises(cwl.CwlError):
            cwl.cwl_head_loss(X2, W2, y, **kw)
    assert torch.equal(X2, X) and torch.equal(W2, W)


@pytest.mark.parametrize("rows,cols", [(16, 96), (300, 40), (130, 200)])
def test_factors_beside_and_in_one_anothers_place(rows, cols):
    torch.manual_seed(0)
    g, m, p = (torch.randn(rows, cols, device="cuda") for _ in range(3))
    want, = cwl.cwl_orthogonalize([g])
    u, o = beside(g, torch.zeros_like(g))
    cwl.cwl_orthogonalize([u], [o])
    assert torch.equal(o, want) and torch.equal(u, g)
    with pytest.raises(cwl.CwlError):
        cwl.cwl_orthogonalize([u], [u])
    assert torch.equal(u, g)
    alone = p.clone(), m.clone()
    cwl.FactorStep([alone[0]], None, [g], [alone[1]])(0.1)
    p2, g2, m2 = beside(p, g, m)
    cwl.FactorStep([p2], None, [g2], [m2])(0.1)
    assert torch.equal(p2, alone[0]) and torch.equal(m2, alone[1]) and torch.equal(g2, g)
    low = p2.view(torch.bfloat16)[:, :cols]
    for kw, error in ((dict(masters=[g2]), cwl.CwlError), (dict(momenta=[g2]), cwl.CwlError), (dict(momenta=[p2]), AssertionError),
                      (dict(lows=[low]), AssertionError), (dict(lows=[g2.view(torch.bfloat16)[:, :cols]]), cwl.CwlError)):
        with pytest.raises(error):
            cwl.FactorStep(**{**dict(masters=[p2], lows=None, grads=[g2], momenta=[m2]), **kw})(0.1)
    assert torch.equal(p2, alone[0]) and torch.equal(g2, g)


def test_a_tensor_written_twice_is_refused():
    u, v, o, m = (torch.randn(16, 96, device="cuda") for _ in range(4))
    with pytest.raises(AssertionError):
        cwl.cwl_orthogonalize([u, v], [o, o])
    with pytest.raises(AssertionError):
        cwl.FactorStep([o, o], None, [u, v], [m, torch.empty_like(m)])
    p, q = cwl.cwl_orthogonalize([u, u])                   # reading twice is fine
    assert torch.equal(p, q)
