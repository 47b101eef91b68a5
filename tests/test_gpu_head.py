"""cwl_head_loss against its definition in 64 bits and against differences.

Tolerances, entry by entry, from the arithmetic.  A logit is an fp32 sum of d products (2^-23 d of the sum of their magnitudes,
however they cancel): ez.  An exponential's argument is rounded at the size of the logits and the function itself is good to
2^-22; at most 1024 of them are added up one after the other: el.  So lse is within ez + el, a probability within twice that of
itself, dZ is rounded to bf16 (2^-8 of a number), and the products with W and X sum V or T terms in fp32 (2^-23 of their
magnitudes each) and are rounded to their own type (2^-8 or 2^-24)."""
import pytest
import torch

from paper_2601_21109_b200 import binding as cwl

pytestmark = pytest.mark.gpu


def operands(seed, T, d, V, pad=0, spread=3.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def m(r, c, std):
        buf = torch.full((r, (c + pad + 7) // 8 * 8), 9.0, dtype=torch.bfloat16, device="cuda")
        buf[:, :c].copy_(torch.randn(r, c, device="cuda", generator=gen) * std)
        return buf[:, :c]
    X, W = m(T, d, 1.0), m(d, V, spread * d ** -0.5)
    y = torch.randint(0, V, (T,), device="cuda", generator=gen, dtype=torch.int32)
    w = torch.rand(T, device="cuda", generator=gen) + 0.5
    return X, W, y, w


def reference(X, W, y, w, dloss=None, lse=None):
    """Everything in 64 bits, with the tolerances of loss, lse and dZ."""
    V, d = W.shape[1], W.shape[0]
    x, wt = X.double(), W.double()
    on = (y >= 0) & (y < V) & (w != 0)
    if dloss is not None:
        on &= dloss != 0
    x = torch.where(on[:, None], x, 0.0)
    z = x @ wt
    ez = (d * 2.0 ** -23 * (x.abs() @ wt.abs())).amax(1)
    el = (2 * z.abs().amax(1) + 4) * 2.0 ** -22 + 1024 * 2.0 ** -24
    own = torch.logsumexp(z, 1)
    norm = own if lse is None else lse.double()
    zy = z.gather(1, y.clamp(0, V - 1).long()[:, None])[:, 0]
    up = torch.where(on, w.double() * (1 if dloss is None else dloss.double()), 0.0)
    q = (z - norm[:, None]).exp()
    at = y.clamp(0, V - 1).long()[:, None]
    if lse is None:                                     # 1 - q_y is what the others add up to (64 bits do not hold 1 - 1e-17)
        dz = q.scatter(1, at, 0.0)
        dz.scatter_(1, at, -dz.sum(1, keepdim=True))
    else:
        dz = q.scatter_add(1, at, torch.full((len(y), 1), -1.0, dtype=torch.float64, device=z.device))
    dz = dz * up[:, None]
    tz = q * (up.abs() * 2.02 * (ez + el))[:, None] + dz.abs() * 2.0 ** -8
    loss = torch.where(on, w.double() * (own - zy), 0.0)
    tl = torch.where(on, ez + el + own.abs() * 2.0 ** -23, 0.0)
    return dict(on=on, x=x, W=wt, lse=torch.where(on, own, 0.0), tl=tl, loss=loss, tloss=w.double().abs() * (2 * tl) + loss.abs() * 2.0 ** -22,
                dz=dz, tz=tz)


def within(got, ref, tol, what):
    over = (got.double() - ref).abs() - tol * 1.01 - 1e-30
    assert bool(torch.isfinite(got).all()), f"{what}: not finite"
    assert float(over.max()) <= 0, f"{what}: over tolerance by {float(over.max()):.3e}"


def check_gradients(r, dX, dW, T, V):
    u = 2.0 ** -23
    if dX is not None:
        out = 2.0 ** -8 if dX.dtype == torch.bfloat16 else 2.0 ** -24
        ref = r["dz"] @ r["W"].T
        within(dX, ref, (r["tz"] + V * u * r["dz"].abs()) @ r["W"].abs().T + ref.abs() * out, "dX")
        if float(ref.norm()) > 0:       # what 2^-8 of every dZ, of either sign, comes to in a norm, and the rounding of dX
            assert float((dX.double() - ref).norm() / ref.norm()) <= 2.0 ** -8 + out
    if dW is not None:
        out = 2.0 ** -8 if dW.dtype == torch.bfloat16 else 2.0 ** -24
        ref = r["x"].T @ r["dz"]
        within(dW, ref, r["x"].abs().T @ (r["tz"] + T * u * r["dz"].abs()) + ref.abs() * out, "dW")


def check(X, W, y, w, **kw):
    T, V = X.shape[0], W.shape[1]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    o = cwl.cwl_head_loss(X, W, y, weight=w, status_word=status, **kw)
    assert int(status.item()) == 0
    r = reference(X, W, y, torch.ones_like(y, dtype=torch.float32) if w is None else w)
    within(o.lse, r["lse"], r["tl"], "lse")
    within(o.loss, r["loss"], r["tloss"], "loss")
    check_gradients(r, o.dX, o.dW, T, V)
    return o


SIZES = [(1, 64, 500), (1, 4096, 32000), (2, 16, 8), (7, 8, 1), (3, 1, 17), (5, 33, 31), (48, 512, 3001), (127, 200, 1000), (128, 64, 512), (129, 1000, 2049),
         (255, 136, 777), (256, 256, 256), (257, 72, 4097), (300, 1024, 5003), (777, 2048, 1234), (1000, 24, 20011), (1536, 640, 8192)]


@pytest.mark.parametrize("T,d,V", SIZES)
def test_loss_alone(T, d, V):
    check(*operands(T + d, T, d, V))


@pytest.mark.parametrize("T,d,V", SIZES)
def test_loss_and_gradients(T, d, V):
    X, W, y, w = operands(T + d, T, d, V, pad=3)
    check(X, W, y, w, want_dx=True, want_dw=True)
    check(X, W, y, w, want_dx=True, grad_dtype=torch.float32)
    check(X, W, y, None, want_dw=True, grad_dtype=torch.float32)


@pytest.mark.parametrize("T,d,V", SIZES)
def test_backward_call(T, d, V):
    X, W, y, w = operands(T + d, T, d, V)
    f = cwl.cwl_head_loss(X, W, y, weight=w)
    g = torch.rand(T, device="cuda") - 0.5
    g[::5] = 0.0
    o = cwl.cwl_head_loss(X, W, y, weight=w, dloss=g, lse=f.lse, want_loss=False, want_dx=True, want_dw=True, grad_dtype=torch.float32)
    assert o.loss is None and o.lse is f.lse
    check_gradients(reference(X, W, y, w, dloss=g, lse=f.lse), o.dX, o.dW, T, V)


@pytest.mark.parametrize("T,d,V", [(9, 64, 700), (300, 136, 2049), (600, 512, 1000)])
@pytest.mark.parametrize("share", [0.0, 0.02, 0.5, 1.0])
def test_rows_that_do_not_count(T, d, V, share):
    """Rows without a target or of weight 0 have zeros everywhere, whatever their activations hold."""
    X, W, y, w = operands(T, T, d, V)
    off = torch.rand(T, device="cuda") < share
    half = torch.rand(T, device="cuda") < 0.5
    y = torch.where(off & half, -1, y)
    w = torch.where(off & ~half, 0.0, w)
    X[off] = float("nan")
    o = check(X, W, y, w, want_dx=True, want_dw=True)
    for t in (o.loss, o.lse, o.dX):
        assert not bool(t[off].any())
    check(X, W, y, w, want_dx=True, want_dw=True, grad_dtype=torch.float32)


def test_a_vocabulary_in_pieces():
    X, W, y, w = operands(1, 16384, 64, 20000)
    y[::7] = -1
    check(X, W, y, w, want_dx=True, want_dw=True)
    check(X, W, y, w, want_dx=True, grad_dtype=torch.float32)


@pytest.mark.parametrize("grad", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d,V,spread", [(60, 64, 3000, 60.0), (700, 136, 4504, 40.0), (16384, 16, 20000, 100.0)])
def test_logits_far_apart(T, d, V, spread, grad):
    """Logits hundreds above the row's reference, more so from piece to piece: columns that outgrow it take another one."""
    X, W, y, w = operands(7, T, d, V)
    W.copy_(W * torch.linspace(0.1, spread / 3.0, V, device="cuda"))
    check(X, W, y, w, want_dx=True, grad_dtype=grad)
    check(X, W.flip(1).contiguous(), y, w, want_dx=True, grad_dtype=grad)
    W[:, 0] = 0                                                     # the reference itself far above all others
    W[0, 0] = 100.0
    X[:, 0] = X[:, 0].abs() + 1
    check(X, W, y, w, want_dx=True, grad_dtype=grad)


@pytest.mark.parametrize("T,d,V", [(20, 64, 3000), (300, 256, 5000)])
def test_gradients_of_tokens_that_the_model_is_sure_of(T, d, V):
    """Where the target's probability is near 1 what is left of dX is small, and its error is relative to that: in one call
    1 - q_y is a sum of the others, not a difference."""
    X, W, y, w = operands(11, T, d, V)
    col = W[:, y.long()].T.float()
    X.copy_(X * 0.2 + 1.6 * col / col.norm(dim=1, keepdim=True) * torch.linspace(2, 9, T, device="cuda")[:, None])
    r = reference(X, W, y, w)
    rest = 1 - torch.exp(-r["loss"] / w.double())
    assert float(rest.min()) < 1e-3
    ez = d * 2.0 ** -23 * (X.double().abs() @ W.double().abs()).amax(1)     # of a logit: a relative error of a probability
    for grad in (torch.bfloat16, torch.float32):
        o = cwl.cwl_head_loss(X, W, y, weight=w, want_dx=True, grad_dtype=grad)
        ref = r["dz"] @ r["W"].T
        size = (r["dz"].abs() @ r["W"].abs().T)
        # every term of the sum: its rounding, twice the logits' errors, the fp32 sums; nothing of the size of W_y alone
        share = 2.0 ** -8 if grad == torch.bfloat16 else 2.0 ** -16
        tol = size * (share + V * 2.0 ** -23 + 4 * ez[:, None] + 2.0 ** -19) + ref.abs() * (2.0 ** -8 if grad == torch.bfloat16 else 2.0 ** -24)
        within(o.dX, ref, tol, "dX")


@pytest.mark.parametrize("T", [1, 2, 40, 500])
def test_fp32_gradients_of_few_rows_carry_fp32(T):
    """One row's dZ rounded to 16 bits would show in a whole column of dW: three numbers keep it to 2^-24."""
    X, W, y, w = operands(T, T, 320, 2000)
    o = cwl.cwl_head_loss(X, W, y, weight=w, want_dx=True, want_dw=True, grad_dtype=torch.float32)
    r = reference(X, W, y, w)
    for got, ref in ((o.dX, r["dz"] @ r["W"].T), (o.dW, r["x"].T @ r["dz"])):
        assert float((got.double() - ref).norm() / ref.norm()) <= 4e-6
