"""Few rows over a vocabulary of several pieces: head_few_kernel's logits, references and sums carried from piece to piece, forward and
backward, against 64 bits with the tolerances of test_gpu_head."""
import pytest
import torch

from paper_2601_21109_b200 import binding as cwl
from test_gpu_head import check_gradients, operands, reference, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,d,V", [(1, 64, 540007), (40, 72, 600000), (64, 24, 1100000)])
@pytest.mark.parametrize("grad", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("slope", ["flat", "up", "down"])
def test_loss_and_gradient(T, d, V, grad, slope):
    """`up`: logits grow along the vocabulary, so that every piece outgrows the references of those before; `down`: the first piece's
    reference lies above all that comes."""
    X, W, y, w = operands(T, T, d, V)
    if slope != "flat":
        W.mul_(torch.linspace(0.1, 30.0, V, device="cuda"))
    if slope == "down":
        W.copy_(W.flip(1))
    y[::9] = -1
    if T > 1:
        y[1], y[2] = 0, V - 1
    ws = torch.full((cwl.cwl_head_loss_workspace_bytes(T, d, V, True),), 255, dtype=torch.uint8, device="cuda")
    o = cwl.cwl_head_loss(X, W, y, weight=w, want_dx=True, grad_dtype=grad, workspace=ws)
    r = reference(X, W, y, w)
    within(o.lse, r["lse"], r["tl"], "lse")
    within(o.loss, r["loss"], r["tloss"], "loss")
    check_gradients(r, o.dX, None, T, V)
