"""Calls of the head's loss and of the factors that the size tests do not make: outputs and workspaces with guards around them,
targets out of range, activations that are not finite, offsets past 2^31, graphs, streams, differences, waits that run out."""
import pytest
import torch

from paper_2601_21109_b200 import binding as cwl
from test_gpu_head import check, operands, reference, within

pytestmark = pytest.mark.gpu
CWL_ERR_INVALID_ARG, CWL_ERR_TIMEOUT = 1, 7
SHAPES = [(5, 64, 700), (64, 128, 3000), (65, 72, 1000), (300, 512, 2049), (1100, 96, 4000)]


def guarded(rows, cols, pitch, offset, dtype):
    buf = torch.full((rows * pitch + offset + 64,), 5.0, dtype=dtype, device="cuda")
    return buf, buf[offset:offset + rows * pitch].view(rows, pitch)[:, :cols]


def untouched(buf, view, rows, cols, pitch, offset):
    inside = torch.zeros(buf.shape, dtype=torch.bool, device="cuda")
    inside[offset:offset + rows * pitch].view(rows, pitch)[:, :cols] = True
    return bool((buf[~inside] == 5.0).all())


@pytest.mark.parametrize("T,d,V", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pad,offset", [(0, 0), (1, 1), (3, 2), (8, 8)])
def test_nothing_outside_outputs_and_workspace(T, d, V, dtype, pad, offset):
    X, W, y, w = operands(T, T, d, V)
    y[1::4] = -1
    bx, dX = guarded(T, d, d + pad, offset, dtype)
    bw, dW = guarded(d, V, V + pad, offset, dtype)
    need = cwl.cwl_head_loss_workspace_bytes(T, d, V, True, True)
    ws = torch.full((need + 4096,), 171, dtype=torch.uint8, device="cuda")
    check(X, W, y, w, dX=dX, dW=dW, workspace=ws[:need])
    assert untouched(bx, dX, T, d, d + pad, offset) and untouched(bw, dW, d, V, V + pad, offset)
    assert bool((ws[need:] == 171).all())
    need = cwl.cwl_head_loss_workspace_bytes(T, d, V, True)
    ws.fill_(171)
    check(X, W, y, w, dX=dX, workspace=ws[:need])
    assert untouched(bx, dX, T, d, d + pad, offset) and bool((ws[need:] == 171).all())


@pytest.mark.parametrize("T,d,V", SHAPES)
def test_targets_out_of_range(T, d, V):
    X, W, y, w = operands(T, T, d, V)
    y[0], y[T // 2] = V, 2 ** 31 - 1
    y[1] = -2 ** 31
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    o = cwl.cwl_head_loss(X, W, y, weight=w, want_dx=True, want_dw=True, status_word=status)
    assert int(status.item()) == 1 << CWL_ERR_INVALID_ARG
    bad = torch.zeros(T, dtype=torch.bool, device="cuda")
    bad[0] = bad[T // 2] = True
    assert bool(torch.isnan(o.loss[bad]).all()) and bool(torch.isnan(o.lse[bad]).all()) and not bool(o.dX[bad].any())
    assert not bool(o.loss[1].any()) and not bool(o.dX[1].any())
    y2 = torch.where(bad, -1, y)
    p = cwl.cwl_head_loss(X, W, y2, weight=w, want_dx=True, want_dw=True)
    assert torch.equal(o.loss[~bad], p.loss[~bad]) and torch.equal(o.dX, p.dX) and torch.equal(o.dW, p.dW)


def test_no_rows():
    X, W, y, w = operands(1, 4, 64, 100)
    o = cwl.cwl_head_loss(X[:0], W, y[:0], weight=w[:0], want_dx=True, want_dw=True)
    assert o.loss.shape == (0,) and o.dX.shape == (0, 64) and not bool(o.dW.any())
    o = cwl.cwl_head_loss(X[:0], W, y[:0])                    # tensors of no rows have no address
    assert o.loss.shape == (0,) and o.dX is None
    for T in (1, 70, 600):
        X, W, y, w = operands(T, T, 64, 1000)
        for yy, ww in ((torch.full_like(y, -1), w), (y, torch.zeros_like(w))):
            for grad in (torch.bfloat16, torch.float32):
                o = cwl.cwl_head_loss(X, W, yy, weight=ww, want_dx=True, want_dw=True, grad_dtype=grad)
                assert not any(bool(t.any()) for t in (o.loss, o.lse, o.dX, o.dW))
                assert not bool(cwl.cwl_head_loss(X, W, yy, weight=ww, want_dx=True, grad_dtype=grad).dX.any())


@pytest.mark.parametrize("T,d,V", SHAPES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_activations_that_are_not_finite_stay_in_their_row(T, d, V, bad):
    X, W, y, w = operands(T, T, d, V)
    good = cwl.cwl_head_loss(X, W, y, weight=w, want_dx=True)
    X[2, d // 2] = bad
    o = cwl.cwl_head_loss(X, W, y, weight=w, want_dx=True)
    alone = cwl.cwl_head_loss(X, W, y, weight=w)
    others = torch.arange(T, device="cuda") != 2
    for a in (o, alone):
        assert bool(torch.isnan(a.loss[2])) and bool(torch.isnan(a.lse[2]))
    assert bool(torch.isnan(o.dX[2]).all())
    assert torch.equal(o.loss[others], good.loss[others]) and torch.equal(o.dX[others], good.dX[others])


@pytest.mark.parametrize("T", [3, 40, 200])
def test_rows_do_not_depend_on_their_company(T):
    """The same tokens among others, packed or not: the same sums in the same order wherever the schedule is the same."""
    X, W, y, w = operands(T, T, 128, 2000)
    a = cwl.cwl_head_loss(X, W, y, weight=w, want_dx=True, grad_dtype=torch.float32)
    y2 = y.clone()
    y2[::3] = -1
    b = cwl.cwl_head_loss(X, W, y2, weight=w, want_dx=True, grad_dtype=torch.float32)
    on = y2 >= 0
    assert torch.equal(a.loss[on], b.loss[on]) and torch.equal(a.lse[on], b.lse[on])
    assert float((a.dX[on] - b.dX[on]).norm() / a.dX[on].norm()) < 1e-6


def test_gradient_against_differences():
    T, d, V = 30, 64, 500
    X, W, y, w = operands(2, T, d, V, spread=1.0)
    X.copy_((X * 16).round() / 16)                       # multiples of 2^-4 below 16: steps of 2^-5 are exact
    X.clamp_(-3.5, 3.5)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    D = torch.randint(-1, 2, X.shape, device="cuda", generator=gen).to(torch.bfloat16)
    h = 2.0 ** -5
    f = [cwl.cwl_head_loss((X + s * h * D).contiguous(), W, y, weight=w).loss.double() for s in (1, -1)]
    assert bool(((X + h * D).double() == X.double() + h * D.double()).all())
    o = cwl.cwl_head_loss(X, W, y, weight=w, want_dx=True, grad_dtype=torch.float32)
    got = (o.dX.double() * D.double()).sum(1)
    want = (f[0] - f[1]) / (2 * h)
    reach = (D.double() @ W.double()).abs().amax(1)
    r = reference(X, W, y, w)
    # the third derivative along D is at most (2 reach)^3; a loss is good to tloss; dX to 2^-16 of what it sums
    tol = w.double() * (2 * reach) ** 3 * h ** 2 / 6 + 2 * r["tloss"] / (2 * h) + 2.0 ** -16 * (r["dz"].abs() @ r["W"].abs().T).sum(1)
    assert bool(((got - want).abs() <= tol).all())


@pytest.mark.parametrize("T,d,V", SHAPES)
@pytest.mark.parametrize("kw", [dict(), dict(want_dx=True), dict(want_dx=True, want_dw=True), dict(want_dx=True, grad_dtype=torch.float32)])
def test_the_same_bits_in_a_graph_and_on_another_stream(T, d, V, kw):
    X, W, y, w = operands(T, T, d, V)
    y[::5] = -1
    want = [t for t in cwl.cwl_head_loss(X, W, y, weight=w, **kw) if t is not None]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:                                    # two calls at once, each with a workspace of its own
        with torch.cuda.stream(s):
            got.append([t for t in cwl.cwl_head_loss(X, W, y, weight=w, **kw) if t is not None])
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = [t for t in cwl.cwl_head_loss(X, W, y, weight=w, **kw) if t is not None]
    for _ in range(2):
        for t in out:
            t.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    y.copy_(torch.where(y < 0, 3, -1))                   # other rows count now: the graph goes by what it finds
    graph.replay()
    torch.cuda.synchronize()
    fresh = [t for t in cwl.cwl_head_loss(X, W, y, weight=w, **kw) if t is not None]
    assert all(torch.equal(a, b) for a, b in zip(out, fresh))


def test_offsets_past_two_to_the_31():
    """A head of 2.4e9 numbers under few and many rows, activations of 2.2e9 under a small vocabulary, a wide factor."""
    d, V = 8192, 300000
    W = torch.empty(d, V, dtype=torch.bfloat16, device="cuda")
    for r in range(0, d, 512):
        W[r:r + 512].normal_(0, 3 * d ** -0.5)
    for T in (3, 300):
        X = torch.randn(T, d, device="cuda").bfloat16()
        y = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32)
        y[0] = V - 1
        o = cwl.cwl_head_loss(X, W, y, want_dx=True)
        z = torch.cat([X[:3].double() @ W[:, c:c + 50000].double() for c in range(0, V, 50000)], 1)
        lse = torch.logsumexp(z, 1)
        loss = lse - z.gather(1, y[:3].long()[:, None])[:, 0]
        assert float((o.loss[:3].double() - loss).abs().max()) <= 1e-3
        q = (z - lse[:, None]).exp()
        q.scatter_add_(1, y[:3].long()[:, None], torch.full((3, 1), -1.0, dtype=torch.float64, device="cuda"))
        dX = sum(q[:, c:c + 50000] @ W[:, c:c + 50000].double().T for c in range(0, V, 50000))
        assert float((o.dX[:3].double() - dX).norm() / dX.norm()) <= 2.0 ** -8
    del W, z, q
    T, d, V = 540000, 4096, 64
    X = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    for r in range(0, T, 54000):
        X[r:r + 54000].normal_()
    W = (torch.randn(d, V, device="cuda") * d ** -0.5).bfloat16()
    y = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32)
    y[::2] = -1
    o = cwl.cwl_head_loss(X, W, y, want_dx=True)
    rows = torch.cat([torch.arange(0, 64), torch.arange(T - 64, T)]).cuda()
    r = reference(X[rows], W, y[rows], torch.ones(128, device="cuda"))
    within(o.loss[rows], r["loss"], r["tloss"], "loss")
    ref = r["dz"] @ r["W"].T
    assert float((o.dX[rows].double() - ref).norm() / ref.norm()) <= 2.0 ** -8


def timed(call):
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    with cwl.test_hooks():
        cwl.cwl_debug_training_set(wait_limit_ns=20_000_000, withhold=True)      # 20 ms
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        call(status)
        end.record()
        torch.cuda.synchronize()                                                 # returns: nothing hangs
        assert int(status.item()) == 1 << CWL_ERR_TIMEOUT
        assert start.elapsed_time(end) < 3000.0                                  # some wait limits


@pytest.mark.parametrize("T,d,V", [(40, 256, 3000), (200, 2048, 3000), (700, 256, 6000)])
@pytest.mark.parametrize("kw", [dict(), dict(want_dx=True), dict(want_dw=True)])
def test_products_that_wait_for_a_block_that_never_comes(T, d, V, kw):
    X, W, y, w = operands(T, T, d, V)
    want = [t for t in cwl.cwl_head_loss(X, W, y, weight=w, **kw) if t is not None]
    timed(lambda status: cwl.cwl_head_loss(X, W, y, weight=w, status_word=status, **kw))
    got = [t for t in cwl.cwl_head_loss(X, W, y, weight=w, **kw) if t is not None]
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def refused(call, tensors, name, host):
    with pytest.raises(AssertionError):
        call(**{**tensors, name: host})


def test_tensors_elsewhere_are_refused():
    T, d, V = 8, 64, 96
    X, W, y, w = operands(1, T, d, V)
    f = lambda *s: torch.rand(*s, device="cuda")   # noqa: E731
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(cwl.cwl_head_loss_workspace_bytes(T, d, V, True, True), dtype=torch.uint8, device="cuda")
    good = dict(X=X, W=W, targets=y, weight=w, loss=f(T), lse=f(T), dX=f(T, d), dW=f(d, V), workspace=ws, status_word=status)
    cwl.cwl_head_loss(**good)
    for name in good:
        refused(cwl.cwl_head_loss, good, name, good[name].cpu())
    refused(cwl.cwl_head_loss, good, "targets", y.long())
    refused(cwl.cwl_head_loss, good, "W", W.float())
    refused(cwl.cwl_head_loss, good, "dW", f(d, V).bfloat16())
    refused(cwl.cwl_head_loss, good, "dloss", f(T))
    back = dict(X=X, W=W, targets=y, lse=f(T), dloss=f(T), want_loss=False, want_dx=True)
    cwl.cwl_head_loss(**back)
    refused(cwl.cwl_head_loss, back, "dloss", f(T).cpu())
    refused(cwl.cwl_head_loss, back, "lse", None)
    u, o = f(8, 40), f(8, 40)
    for a, b in ((u.cpu(), o), (u, o.cpu()), (u, f(40, 8)), (u[0], o[0])):
        with pytest.raises(AssertionError):
            cwl.OrthogonalizeCall([a], [b])
    with pytest.raises(AssertionError):
        cwl.OrthogonalizeCall([u], [o], workspace=torch.empty(1 << 20, dtype=torch.uint8))
    with pytest.raises(cwl.CwlError):
        cwl.OrthogonalizeCall([u], [o], workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))()
    with pytest.raises(cwl.CwlError):
        cwl.cwl_orthogonalize([f(300, 400)])
    for bad in (dict(masters=[u.bfloat16()]), dict(lows=[u]), dict(momenta=[f(8, 41)]), dict(grads=[u.cpu()]), dict(scales=[1.0, 2.0])):
        kw = dict(masters=[u], lows=None, grads=[f(8, 40)], momenta=[f(8, 40)], **{})
        kw.update(bad)
        with pytest.raises(AssertionError):
            cwl.FactorStep(**kw)


def test_factors_past_two_to_the_31_and_in_guarded_workspace():
    rows, cols, pitch = 40, 300, 60_000_000                 # rows 240 MB apart: the last one starts past 2^31 elements
    buf = torch.zeros(39 * pitch + cols, device="cuda")
    u = buf.as_strided((rows, cols), (pitch, 1))
    u.copy_(torch.randn(rows, cols, device="cuda"))
    dense = u.contiguous()
    assert torch.equal(cwl.cwl_orthogonalize([u])[0], cwl.cwl_orthogonalize([dense])[0])
    del buf, u
    us = [torch.randn(r, c, device="cuda") for r, c in ((64, 500), (3, 900), (200, 300), (700, 150))]
    call = cwl.OrthogonalizeCall(us, [torch.empty_like(x) for x in us])
    need = call.workspace.numel()
    ws = torch.full((need + 4096,), 171, dtype=torch.uint8, device="cuda")
    want = [o.clone() for o in call()]
    got = cwl.OrthogonalizeCall(us, [torch.empty_like(x) for x in us], workspace=ws[:need])()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and bool((ws[need:] == 171).all())


def test_two_updates_at_once():
    sets = []
    for seed in range(2):
        torch.manual_seed(seed)
        shapes = [(64, 700), (700, 64), (130, 300)]
        p, g, m = ([torch.randn(*s, device="cuda") for s in shapes] for _ in range(3))
        sets.append((p, g, m))
    alone = []
    for p, g, m in sets:
        q, n = [t.clone() for t in p], [t.clone() for t in m]
        cwl.FactorStep(q, None, g, n)(0.1)
        alone.append(q + n)
    torch.cuda.synchronize()
    calls = [cwl.FactorStep(p, None, g, m) for p, g, m in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    for c, s in zip(calls, streams):
        c(0.1, stream=s)
    torch.cuda.synchronize()
    for (p, g, m), want in zip(sets, alone):
        assert all(torch.equal(a, b) for a, b in zip(p + m, want))
