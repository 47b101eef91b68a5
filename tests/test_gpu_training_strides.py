"""Matrices of one row or one column, whose strides in that dimension may be anything, answer like contiguous ones."""
import pytest
import torch

from paper_2601_21109_b200 import binding as cwl

pytestmark = pytest.mark.gpu


def one_row(t, stride):
    """The single row of `t` in storage of its own, with a row stride that says nothing."""
    return t.clone().as_strided(t.shape, (stride, 1))


def column(t):
    """A [n, 1] matrix whose column stride says nothing."""
    return t.reshape(1, -1).clone().t()


def test_one_row():
    V, K = 501, 7
    z = torch.randn(1, V, device="cuda")
    want = cwl.cwl_token_logprobs(z, top_k=K)
    for stride in (0, 1, 3, V, 4096):
        got = cwl.cwl_token_logprobs(one_row(z, stride), top_k=K)
        assert torch.equal(got.top_ids, want.top_ids) and torch.equal(got.lse, want.lse)
    loss, grad = cwl.cwl_distill_topk(z, want.top_ids, want.top_logprobs, teacher="logprobs", temperature=1.5)
    for a, b, c in ((0, 1, 2), (V, K, 40), (1000, 40, K), (1, 0, 0)):
        x = one_row(z, a)
        out = one_row(z, c)
        for kw in ({}, {"dlogits": out}, {"dlogits": x}):
            l, g = cwl.cwl_distill_topk(x, one_row(want.top_ids, b), one_row(want.top_logprobs, c), teacher="logprobs", temperature=1.5, **kw)
            assert torch.equal(l, loss) and torch.equal(g, grad)


def test_one_column():
    T = 33
    z = torch.randn(T, 1, device="cuda")
    got = cwl.cwl_token_logprobs(column(z), top_k=1)
    assert torch.equal(got.lse, z[:, 0]) and bool((got.top_logprobs == 0).all()) and bool((got.top_ids == 0).all())
    V = 700
    wide = torch.randn(T, V, device="cuda")
    ids, vals = torch.randint(0, V, (T, 1), dtype=torch.int32, device="cuda"), torch.full((T, 1), -0.5, device="cuda")
    want = cwl.cwl_distill_topk(wide, ids, vals, teacher="logprobs")
    for i, v in ((column(ids), vals), (ids, column(vals)), (column(ids), column(vals)), (ids[:, :1], vals)):
        got = cwl.cwl_distill_topk(wide, i, v, teacher="logprobs")
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_gradients_of_one_token():
    d, R = 64, 16
    m = lambda *s: torch.rand(*s, device="cuda").bfloat16()   # noqa: E731
    X, dY, A, B = m(1, d), m(1, d), m(d, R), m(R, d)
    tab = cwl.DeviceChunkTable.from_host([0, 1], [R], [1.0], [1])
    want = cwl.cwl_apply_grads(X, dY, A, B, tab, 0)
    for a, b in ((0, 1), (65, 64), (d, 77), (1000, 3)):
        got = cwl.cwl_apply_grads(one_row(X, a), one_row(dY, b), A, B, tab, 0)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_strided_columns_are_refused():
    z = torch.randn(4, 64, device="cuda")
    ids, vals = torch.zeros(4, 3, dtype=torch.int32, device="cuda"), torch.zeros(4, 3, device="cuda")
    with pytest.raises(AssertionError):
        cwl.cwl_token_logprobs(z[:, ::2])
    with pytest.raises(AssertionError):
        cwl.cwl_distill_topk(z[:, ::2], ids, vals)
    with pytest.raises(AssertionError):
        cwl.cwl_distill_topk(z, ids.t().contiguous().t(), vals)
    with pytest.raises(AssertionError):
        cwl.cwl_distill_topk(z, ids, torch.zeros(4, 5, device="cuda")[:, :3])
