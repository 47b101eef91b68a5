"""Refusals and sizes of the head-loss, orthogonalisation and factor-step calls that need no device: every one is reported
before anything touches CUDA."""
import ctypes
import math

import pytest

from paper_2601_21109_b200 import binding as cwl


@pytest.fixture(scope="module")
def L():
    from paper_2601_21109_b200 import build
    build.build()
    return cwl.lib()


P = 4096     # an address that is aligned and never read: the calls below end before any launch


def head(L, X=P, ldx=64, W=P, ldw=96, T=8, d=64, V=96, targets=P, weight=None, dloss=None, loss=P, lse=P, dX=None, lddx=64, dW=None,
         lddw=96, dtype=1, ws=P, n=1 << 40):
    return L.cwl_head_loss(X, ldx, W, ldw, T, d, V, targets, weight, dloss, loss, lse, dX, lddx, dW, lddw, dtype, ws, n, None, None)


def test_head_loss_refusals(L):
    assert head(L, T=0) == 0 and head(L, T=0, dX=P) == 0 and head(L, T=0, X=None, targets=None, loss=None, lse=None) == 0
    assert head(L, T=-1) == 1 and head(L, d=0) == 1 and head(L, V=0) == 1 and head(L, dtype=2) == 1 and head(L, dtype=7) == 1
    assert head(L, T=(1 << 24) + 1) == 3 and head(L, V=(1 << 24) + 1) == 3 and head(L, d=(1 << 20) + 1) == 3
    assert head(L, X=None) == 1 and head(L, W=None) == 1 and head(L, targets=None) == 1
    assert head(L, loss=None) == 1                                    # nothing wanted
    assert head(L, loss=None, lse=None, dX=P) == 1                    # a backward call without lse
    assert head(L, dloss=P) == 1 and head(L, dloss=P, dX=P) == 1      # an upstream gradient in a forward call
    for name in ("X", "W"):
        assert head(L, **{name: P + 8}) == 2
    assert head(L, ldx=56) == 2 and head(L, ldx=68) == 2 and head(L, ldw=88) == 2 and head(L, ldw=100) == 2
    assert head(L, dX=P + 1) == 2 and head(L, dX=P + 2, dtype=0) == 2 and head(L, dW=P + 2, dtype=0) == 2
    assert head(L, dX=P, lddx=63) == 2 and head(L, dW=P, lddw=95) == 2
    assert head(L, ws=None) == 5 and head(L, ws=P + 16) == 5 and head(L, n=1000) == 5
    assert head(L, dX=P, n=cwl.cwl_head_loss_workspace_bytes(8, 64, 96)) == 5


def test_head_loss_workspace(L):
    w = cwl.cwl_head_loss_workspace_bytes
    assert w(0, 64, 96) == 0 and w(8, 0, 96) == 0 and w(8, 64, 0, True) == 0 and w((1 << 24) + 1, 64, 96) == 0
    assert 0 < w(8, 64, 96) <= w(8, 64, 96, True) and w(8, 64, 96) <= w(8, 64, 96, False, True)
    # pieces: twice the vocabulary does not take twice the room, and no logits are kept
    full = 16384 * 128000 * 2
    assert w(16384, 4096, 128000, True) < 0.6 * full
    assert w(16384, 4096, 128000, True) < 1.1 * w(16384, 4096, 64000, True)


def factor(rows=64, cols=96, grad=P, ldg=96, m=P, ldm=96, out=P, ldo=96, low=None, ldl=96, scale=1.0):
    return cwl.CFactor(rows, cols, grad, ldg, m, ldm, out, ldo, low, ldl, scale)


def iteration(steps=5, a=3.4, b=-4.7, c=2.0, eps=1e-7):
    return cwl.CNewtonSchulz(steps, a, b, c, eps)


def ortho(L, f=None, n=1, tin=0, tout=0, it=None, ws=P, size=1 << 40):
    arr = (cwl.CFactor * 1)(f if f is not None else factor())
    it = it if it is not None else iteration()
    return L.cwl_orthogonalize(arr, n, tin, tout, ctypes.byref(it), ws, size, None)


def step(L, f=None, n=1, tin=0, it=None, lr=0.1, beta=0.9, decay=0.0, ws=P, size=1 << 40):
    arr = (cwl.CFactor * 1)(f if f is not None else factor())
    it = it if it is not None else iteration()
    return L.cwl_factor_step(arr, n, tin, ctypes.byref(it), lr, beta, decay, 1, ws, size, None)


@pytest.mark.parametrize("call", [ortho, step])
def test_factor_refusals(L, call):
    assert call(L, n=0) == 0 and call(L, n=-1) == 1 and call(L, tin=3) == 1 and call(L, tin=-1) == 1
    for bad in (iteration(steps=0), iteration(steps=17), iteration(a=math.nan), iteration(b=math.inf), iteration(c=-math.inf), iteration(eps=-1.0),
                iteration(eps=math.nan)):
        assert call(L, it=bad) == 1
    assert call(L, factor(rows=0)) == 1 and call(L, factor(cols=-1)) == 1
    assert call(L, factor(rows=257, cols=300, ldg=300, ldm=300, ldo=300)) == 3
    assert call(L, factor(rows=4, cols=(1 << 22) + 1, ldg=1 << 23, ldm=1 << 23, ldo=1 << 23)) == 3
    assert call(L, factor(grad=None)) == 1 and call(L, factor(out=None)) == 1
    assert call(L, factor(grad=P + 2)) == 2 and call(L, factor(out=P + 2)) == 2
    assert call(L, factor(ldg=95)) == 2 and call(L, factor(ldo=95)) == 2 and call(L, factor(ldg=1 << 31)) == 2
    assert call(L, ws=None) == 5 and call(L, ws=P + 16) == 5 and call(L, size=100) == 5
    assert L.cwl_orthogonalize(None, 1, 0, 0, ctypes.byref(iteration()), P, 1 << 40, None) == 1
    assert L.cwl_orthogonalize((cwl.CFactor * 1)(factor()), 1, 0, 0, None, P, 1 << 40, None) == 1


def test_orthogonalize_and_step_refusals(L):
    assert ortho(L, tout=2) == 1
    assert step(L, factor(m=None)) == 1 and step(L, factor(m=P + 2)) == 2 and step(L, factor(ldm=95)) == 2
    assert step(L, factor(low=P + 1)) == 2 and step(L, factor(low=P, ldl=95)) == 2
    assert step(L, factor(scale=math.nan)) == 1
    for v in (math.nan, math.inf):
        assert step(L, lr=v) == 1 and step(L, decay=v) == 1 and step(L, beta=v) == 1
    assert step(L, beta=1.0) == 1 and step(L, beta=-0.1) == 1


def test_factor_workspace(L):
    w = lambda *shapes: int(L.cwl_orthogonalize_workspace_bytes((cwl.CFactor * len(shapes))(*[cwl.CFactor(r, c) for r, c in shapes]), len(shapes)))   # noqa: E731
    assert L.cwl_orthogonalize_workspace_bytes(None, 3) == 0 and w((0, 5)) == 0 and w((300, 300)) == 0
    assert 0 < w((16, 100)) <= w((64, 4096)) < w((256, 4096))
    assert ctypes.sizeof(cwl.CFactor) == 80 and ctypes.sizeof(cwl.CNewtonSchulz) == 40


def test_struct_offsets_match_the_header(L):
    assert cwl.CFactor.grad.offset == 8 and cwl.CFactor.momentum.offset == 24 and cwl.CFactor.out.offset == 40
    assert cwl.CFactor.low.offset == 56 and cwl.CFactor.scale.offset == 72 and cwl.CNewtonSchulz.a.offset == 8
