"""Backward calls of cwl_head_loss (lse given) for each gradient alone and both, against 64 bits.

The tolerances are those of test_gpu_head: what a logit, an exponential, the roundings of dZ and of the result and the fp32 sums
may lose.  Workspaces come full of NaN, so that a number that is read before it is written shows."""
import pytest
import torch

from paper_2601_21109_b200 import binding as cwl
from test_gpu_head import check_gradients, operands, reference

pytestmark = pytest.mark.gpu
WANTED = {"dX": (True, False), "dW": (False, True), "both": (True, True)}


def backward(T, d, V, wanted, grad, share_off=0.0):
    want_dx, want_dw = WANTED[wanted]
    X, W, y, w = operands(T + d, T, d, V)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(V)
    y = torch.where(torch.rand(T, device="cuda", generator=gen) < share_off, -1, y)
    lse = cwl.cwl_head_loss(X, W, y, weight=w).lse
    up = torch.rand(T, device="cuda", generator=gen) - 0.5
    if share_off > 0:
        up[::5] = 0.0
    ws = torch.full((cwl.cwl_head_loss_workspace_bytes(T, d, V, want_dx, want_dw),), 255, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    o = cwl.cwl_head_loss(X, W, y, weight=w, dloss=up, lse=lse, want_loss=False, want_dx=want_dx, want_dw=want_dw, grad_dtype=grad,
                          workspace=ws, status_word=status)
    assert int(status.item()) == 0 and o.loss is None and o.lse is lse
    assert (o.dX is not None) == want_dx and (o.dW is not None) == want_dw
    check_gradients(reference(X, W, y, w, dloss=up, lse=lse), o.dX, o.dW, T, V)
    if want_dx:
        assert not bool(o.dX[(y < 0) | (up == 0)].any())


@pytest.mark.parametrize("T,d,V", [(1, 4096, 3200), (5, 33, 31), (48, 512, 3001), (64, 72, 1000), (65, 200, 1000), (129, 1000, 2049), (300, 1024, 5003),
                                   (1000, 24, 20011)])
@pytest.mark.parametrize("wanted", list(WANTED))
@pytest.mark.parametrize("grad", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("share_off", [0.0, 0.3])
def test_each_gradient(T, d, V, wanted, grad, share_off):
    backward(T, d, V, wanted, grad, share_off)


@pytest.mark.parametrize("T,d,V", [(16384, 64, 20000), (4099, 72, 50001), (48, 64, 600000), (3, 24, 540001)])
@pytest.mark.parametrize("wanted", list(WANTED))
@pytest.mark.parametrize("grad", [torch.bfloat16, torch.float32])
def test_a_vocabulary_in_pieces(T, d, V, wanted, grad):
    """The vocabulary does not fit one piece of the workspace: what the pieces leave adds up."""
    backward(T, d, V, wanted, grad, 0.2)
