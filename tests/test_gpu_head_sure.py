"""Gradients of tokens that the model is sure of, in calls that want dW, against 64 bits.

Where the target's probability is near 1, 1 - q_y has the relative precision of the other tokens' probabilities: a forward call adds
those up, a backward call takes it from z_y - lse as it is given.  So every dZ, the target's among them, is within
r = 2.02 (ez + el) + share of itself: twice a logit's error (d 2^-23 of its terms' magnitudes) and an exponential's (test_gpu_head),
and 2^-8 where dZ is one bf16 number, 2^-16 where it is two or more.  The products add V or T terms in fp32 and round to their type."""
import pytest
import torch

from paper_2601_21109_b200 import binding as cwl
from test_gpu_head import within

pytestmark = pytest.mark.gpu
SHARE = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -16}
OUT = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def compare(o, X, W, dz, r, grad):
    """dX and dW of a call from dZ (64 bits), each entry of which may be off by r of itself (one r a row)."""
    x, wt, u = X.double(), W.double(), 2.0 ** -23
    if o.dX is not None:
        ref = dz @ wt.T
        within(o.dX, ref, (dz.abs() * (r[:, None] + W.shape[1] * u)) @ wt.abs().T + ref.abs() * OUT[grad], "dX")
    if o.dW is not None:
        ref = x.T @ dz
        within(o.dW, ref, x.abs().T @ (dz.abs() * (r[:, None] + len(x) * u)) + ref.abs() * OUT[grad], "dW")


@pytest.mark.parametrize("T", [20, 100, 300, 1500])
@pytest.mark.parametrize("low,high", [(0.0, 50.0), (20.0, 30.0)])
@pytest.mark.parametrize("want_dx", [False, True])
@pytest.mark.parametrize("grad", [torch.bfloat16, torch.float32])
def test_forward(T, low, high, want_dx, grad):
    d, V = 256, 3000
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T)
    W = (torch.randn(d, V, device="cuda", generator=gen) * d ** -0.5).bfloat16()
    y = torch.randint(0, V, (T,), device="cuda", generator=gen, dtype=torch.int32)
    y[::7] = 0
    toward = W[:, y.long()].t().float()
    gap = torch.linspace(low, high, T, device="cuda")[:, None]
    X = (torch.randn(T, d, device="cuda", generator=gen) * 0.5 + gap * toward / (toward ** 2).sum(1, keepdim=True)).bfloat16()
    w = torch.rand(T, device="cuda", generator=gen) + 0.5
    o = cwl.cwl_head_loss(X, W, y, weight=w, want_dx=want_dx, want_dw=True, grad_dtype=grad)
    x, wt, at = X.double(), W.double(), y.long()[:, None]
    z = x @ wt
    dz = (z - torch.logsumexp(z, 1, keepdim=True)).exp().scatter(1, at, 0.0)
    rest = dz.sum(1, keepdim=True)
    assert float(rest.min()) < 1e-8               # 3000 e^-30 = 2.8e-10, times e to a difference of logits of deviation 0.7
    dz = dz.scatter(1, at, -rest) * w.double()[:, None]
    ez = d * 2.0 ** -23 * (x.abs() @ wt.abs()).amax(1)
    el = (2 * z.abs().amax(1) + 4) * 2.0 ** -22 + 1024 * 2.0 ** -24
    compare(o, X, W, dz, 2.02 * (ez + el) + SHARE[grad], grad)
    # the loss, too: of a sure token it is what the others add up to, and as exact relative to itself; of others, where it is
    # w ln 2 or more, two logits and a sum are off by w (2 ez + el) < 3 (ez + el) w ln 2
    loss = -torch.log1p(-rest[:, 0]) * w.double()
    within(o.loss, loss, (3 * (ez + el) + 2.0 ** -22) * loss, "loss")


@pytest.mark.parametrize("T", [20, 100, 300])
@pytest.mark.parametrize("wanted", [(True, False), (False, True), (True, True)])
@pytest.mark.parametrize("grad", [torch.bfloat16, torch.float32])
def test_backward_of_exact_logits(T, wanted, grad):
    """Logits that are small multiples of a half, summed without error: what is left of the target is expm1 of an exact difference,
    0 where lse rounds to its logit."""
    d, V = 16, 600
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T)
    W = (torch.randint(-4, 5, (d, V), device="cuda", generator=gen) / 4.0).bfloat16()
    y = torch.randint(0, V, (T,), device="cuda", generator=gen, dtype=torch.int32)
    X = (8 * W[:, y.long()].T).contiguous()
    z, at = X.double() @ W.double(), y.long()[:, None]
    lse = torch.logsumexp(z, 1).float()
    up = torch.rand(T, device="cuda", generator=gen) + 0.5
    o = cwl.cwl_head_loss(X, W, y, dloss=up, lse=lse, want_loss=False, want_dx=wanted[0], want_dw=wanted[1], grad_dtype=grad)
    dz = z - lse.double()[:, None]
    dz = dz.exp().scatter(1, at, dz.gather(1, at).expm1()) * up.double()[:, None]
    assert float(dz.gather(1, at).abs().min()) < 1e-6
    r = (2 * z.abs().amax(1) + 4) * 2.0 ** -22 + SHARE[grad]
    compare(o, X, W, dz, r, grad)
