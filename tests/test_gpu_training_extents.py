"""As many rows, and as long a row, as an int32 holds: row and element numbers are stepped past 2^31 without wrapping round."""
import pytest
import torch

from paper_2601_21109_b200 import binding as cwl

pytestmark = pytest.mark.gpu
MOST = 2 ** 31 - 1


def parts(n, step=1 << 28):
    return ((a, min(a + step, n)) for a in range(0, n, step))


def test_log_probabilities_of_the_most_rows():
    z = torch.empty(MOST, 1, dtype=torch.bfloat16, device="cuda")
    for a, b in parts(MOST):
        z[a:b].normal_()
    o = cwl.cwl_token_logprobs(z)
    for a, b in parts(MOST):
        assert torch.equal(o.lse[a:b], z[a:b, 0].float()) and not bool(o.entropy[a:b].any())


def test_distillation_of_the_most_rows():
    """One token, of which the teacher is sure: no loss and no gradient; a quarter of the rows is not trained on."""
    z = torch.empty(MOST, 1, dtype=torch.bfloat16, device="cuda")
    z.normal_()
    ids = torch.zeros(MOST, 1, dtype=torch.int32, device="cuda")
    vals = torch.zeros(MOST, 1, device="cuda")
    loss = torch.full((MOST,), 7.0, device="cuda")
    grad = torch.full((MOST, 1), 7.0, dtype=torch.bfloat16, device="cuda")
    cwl.cwl_distill_topk(z, ids, vals, teacher="logprobs", loss=loss, dlogits=grad)
    for a, b in parts(MOST):
        assert not bool(loss[a:b].any()) and not bool(grad[a:b].any())


def test_alternatives_of_the_longest_row():
    """Large logits in a few threads' elements of the last slice, so that the exact selection walks it to its end."""
    V = MOST
    z = torch.zeros(1, V, dtype=torch.bfloat16, device="cuda")
    start = V - (1 << 22)
    v = torch.arange(start, V, device="cuda")
    z[0, start:] = torch.where(v % 2048 < 80, 20.0, 0.0).bfloat16()
    at = torch.cat([V - 1 - 37 * torch.arange(50, device="cuda")])
    z[0, at] = (30.0 + torch.arange(50, device="cuda")).bfloat16()
    o = cwl.cwl_token_logprobs(z, top_k=128)
    rest = start + torch.nonzero((z[0, start:] == 20.0)).flatten()[:78]
    want = torch.cat([at.flip(0), rest]).to(torch.int32)
    assert torch.equal(o.top_ids[0], want)
