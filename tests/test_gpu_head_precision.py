"""What cwl_head_loss keeps of gradients that are small or asked for in 32 bits, against 64 bits."""
import pytest
import torch

from paper_2601_21109_b200 import binding as cwl

pytestmark = pytest.mark.gpu


def exact(X, W, y, w, lse=None):
    """dX and dW in 64 bits; 1 - q_y is what the others add up to."""
    x, wt, at = X.double(), W.double(), y.long()[:, None]
    z = x @ wt
    norm = torch.logsumexp(z, 1) if lse is None else lse.double()
    dz = (z - norm[:, None]).exp().scatter(1, at, 0.0)
    if lse is None:
        dz.scatter_(1, at, -dz.sum(1, keepdim=True))
    else:
        dz.scatter_(1, at, (z.gather(1, at) - norm[:, None]).expm1())
    dz = dz * w.double()[:, None]
    return dz @ wt.T, x.T @ dz, z


@pytest.mark.parametrize("T,V", [(20, 3000), (100, 3000), (300, 3000), (1500, 3000), (1500, 100001)])
@pytest.mark.parametrize("grad", [torch.bfloat16, torch.float32])
def test_rows_of_sure_tokens(T, V, grad):
    """Targets up to 140 above the others: every row's gradient that fp32 can hold has the relative precision of the rest.  Row by
    row: E's rounding and dX's (2^-9 each at most in a norm, taken whole), and twice what a logit of up to 200 loses in 16
    truncated steps (2^-23 of it each: 2^-11.3)."""
    d = 256
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T)
    buf = torch.zeros(d, (V + 7) // 8 * 8, dtype=torch.bfloat16, device="cuda")
    W = buf[:, :V].copy_(torch.randn(d, V, device="cuda", generator=gen) * d ** -0.5)
    y = torch.randint(0, V, (T,), device="cuda", generator=gen, dtype=torch.int32)
    y[::7] = 0                                          # the column that rows take their reference from
    gap = torch.linspace(0, 140, T, device="cuda")[torch.randperm(T, device="cuda", generator=gen)]
    toward = W[:, y.long()].t().float()
    X = (torch.randn(T, d, device="cuda", generator=gen) + gap[:, None] * toward / (toward ** 2).sum(1, keepdim=True)).bfloat16()
    w = torch.rand(T, device="cuda", generator=gen) + 0.5
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    o = cwl.cwl_head_loss(X, W, y, weight=w, want_dx=True, grad_dtype=grad, status_word=status)
    assert int(status.item()) == 0
    ref, _, z = exact(X, W, y, w)
    assert float(z.abs().max()) < 200
    size = ref.norm(dim=1)
    held = size > 1e-33
    assert int(held.sum()) > T // 2 and bool((size[held] < 1e-28).any())
    off = (o.dX.double() - ref).norm(dim=1)
    assert float((off[held] / size[held]).max()) <= 2.0 ** -7 + 2.0 ** -10
    assert float(off.max() / size.max()) <= 2.0 ** -7 and bool(torch.isfinite(o.loss).all())
    others = torch.logsumexp(z.scatter(1, y.long()[:, None], -torch.inf), 1)
    loss = w.double() * torch.nn.functional.softplus(others - z.gather(1, y.long()[:, None])[:, 0])
    assert float((o.loss.double() - loss).abs().max()) <= 1.5 * 200 * (2.0 ** -19 + 2.0 ** -22)


@pytest.mark.parametrize("T,want_dw", [(20, True), (300, True), (700, True), (300, False), (700, False)])
@pytest.mark.parametrize("backward", [False, True])
def test_gradients_of_32_bits_of_a_wide_head(T, want_dw, backward):
    """fp32 gradients do not carry what a tensor core's sum of 8192 products loses.  Logits leave it after 64 steps, each of which drops
    2^-24 on average of a sum that is half of the last one on average: 2^-19 of a logit, which a probability loses; the
    two numbers that stand for a probability leave 2^-17 of it."""
    d, V = 8192, 3000
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T)
    W = (torch.randn(d, V, device="cuda", generator=gen) * (3.0 * d ** -0.5)).bfloat16()
    y = torch.randint(0, V, (T,), device="cuda", generator=gen, dtype=torch.int32)
    X = torch.randn(T, d, device="cuda", generator=gen).bfloat16()
    w = torch.full((T,), 1.0 / T, device="cuda")
    z = X.double() @ W.double()
    kw = dict(lse=torch.logsumexp(z, 1).float(), want_loss=False) if backward else {}
    o = cwl.cwl_head_loss(X, W, y, weight=w, want_dx=True, want_dw=want_dw, grad_dtype=torch.float32, **kw)
    dx, dw, z = exact(X, W, y, w, kw.get("lse"))
    bound = 2.0 ** -19 * float(z.abs().max()) + 2.0 ** -17
    assert bound < 4e-5
    assert float((o.dX.double() - dx).norm() / dx.norm()) <= bound
    if want_dw:
        assert float((o.dW.double() - dw).norm() / dw.norm()) <= bound


@pytest.mark.parametrize("T", [3, 100, 400])
@pytest.mark.parametrize("want_dx", [False, True])
def test_loss_of_sure_tokens(T, want_dx):
    """The loss of a token whose target stands out is as exact as its logits are apart, not as they are large: the differences of exact
    logits (small multiples of powers of two, 16 products) are exact, and what the others add up to has 2^-22 of itself per
    exponential and 2^-24 per sum of at most 1024."""
    d, V = 16, 600
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T)
    W = (torch.randint(-4, 5, (d, V), device="cuda", generator=gen) / 4.0).bfloat16()
    X = (torch.randint(-8, 9, (T, d), device="cuda", generator=gen) / 4.0).bfloat16()
    z = X.double() @ W.double()
    y = z.argmax(1).int()
    o = cwl.cwl_head_loss(X, W, y, want_dx=want_dx)
    apart = z - z.gather(1, y.long()[:, None])
    ref = torch.log1p(apart.exp().scatter(1, y.long()[:, None], 0.0).sum(1))
    assert float((o.loss.double() - ref).abs().max()) <= (2 * float(apart.abs().max()) + 4) * 2.0 ** -22 + 1024 * 2.0 ** -24
