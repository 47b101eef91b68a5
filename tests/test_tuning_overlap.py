"""Outputs of the head-loss, orthogonalisation and factor-step calls that overlap what the call still reads are refused before
anything touches CUDA; matrices that only lie between one another's rows are not taken for overlapping."""
import ctypes
import itertools

import pytest

from paper_2601_21109_b200 import binding as cwl


@pytest.fixture(scope="module")
def L():
    from paper_2601_21109_b200 import build
    build.build()
    return cwl.lib()


# addresses that are aligned and never read: calls whose tensors do not overlap are not made here
BASE, FAR = 1 << 40, 1 << 30
WS = 1 << 45
REFUSED = 1


def head(L, X, W, dX, dW, T=8, d=64, V=96, ldx=64, ldw=96, lddx=64, lddw=96, dtype=1):
    return L.cwl_head_loss(X, ldx, W, ldw, T, d, V, BASE + 9 * FAR, None, None, BASE + 10 * FAR, None, dX, lddx, dW, lddw, dtype, WS, 1 << 44, None, None)


def test_head_loss(L):
    X, W, out = BASE, BASE + FAR, BASE + 2 * FAR
    x_bytes, w_bytes = 8 * 64 * 2, 64 * 96 * 2
    assert head(L, X, W, X, None) == REFUSED and head(L, X, W, W, None) == REFUSED
    assert head(L, X, W, None, W) == REFUSED and head(L, X, W, None, X) == REFUSED
    assert head(L, X, W, out, out) == REFUSED
    for off in (-w_bytes + 2, -2, 2, w_bytes - 2):                       # partly
        assert head(L, X, W, None, W + off) == REFUSED
    for off in (-x_bytes + 2, x_bytes - 2):
        assert head(L, X, W, X + off, None) == REFUSED
    assert head(L, X, W, X + 2 * 64, None, ldx=128, lddx=100) == REFUSED   # rows of other distances that meet


def factors(*items):
    return (cwl.CFactor * len(items))(*items)


ITERATION = cwl.CNewtonSchulz(5, 3.4, -4.7, 2.0, 1e-7)


def ortho(L, f, tin=0, tout=0):
    return L.cwl_orthogonalize(factors(f), 1, tin, tout, ctypes.byref(ITERATION), WS, 1 << 44, None)


def step(L, f, tin=0):
    return L.cwl_factor_step(factors(f), 1, tin, ctypes.byref(ITERATION), 0.1, 0.9, 0.0, 1, WS, 1 << 44, None)


@pytest.mark.parametrize("rows,cols", [(1, 1), (16, 96), (96, 16), (200, 300)])
def test_orthogonalize(L, rows, cols):
    n = rows * cols
    for tin, tout, off in ((0, 0, 0), (1, 1, 0), (0, 1, 0), (1, 0, 0), (0, 0, 4 * (n - 1)), (0, 0, -4 * (n - 1)), (1, 0, 2 * (n - 1) // 4 * 4)):
        assert ortho(L, cwl.CFactor(rows, cols, BASE, cols, None, 0, BASE + off, cols), tin, tout) == REFUSED


def test_step(L):
    rows, cols = 70, 96
    places = [BASE + i * FAR for i in range(4)]
    for a, b in itertools.combinations(range(4), 2):
        at = list(places)
        at[b] = at[a] + 64
        g, m, p, low = at
        for tin in (0, 1, 2):
            assert step(L, cwl.CFactor(rows, cols, g, cols, m, cols, p, cols, low, cols, 1.0), tin) == REFUSED
    g, m, p, _ = places
    assert step(L, cwl.CFactor(rows, cols, g, cols, m, cols, g, cols, None, 0, 1.0)) == REFUSED


def spans(a, b):
    """Do two lists of (first byte, last byte + 1) meet?"""
    return any(s < f and t < e for s, e in a for t, f in b)


def test_exact(L):
    """The test of two matrices against every byte of them, over small shapes, distances and offsets."""
    with cwl.test_hooks() as hooks:
        f = hooks.cwl_debug_overlap
    f.restype = ctypes.c_int32
    f.argtypes = [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64] * 2
    seen = set()
    for ra, wa, pa, rb, wb, pb in itertools.product((1, 2, 4), (1, 3, 4), (4, 7), (1, 3), (1, 2, 5), (5, 7, 11)):
        for off in range(-30, 31):
            a = [(1000 + i * pa, 1000 + i * pa + wa) for i in range(ra)]
            b = [(1000 + off + i * pb, 1000 + off + i * pb + wb) for i in range(rb)]
            want = spans(a, b)
            assert bool(f(1000, ra, wa, pa, 1000 + off, rb, wb, pb)) == want
            assert bool(f(1000 + off, rb, wb, pb, 1000, ra, wa, pa)) == want
            seen.add(want)
    assert seen == {False, True}
    assert not f(1000, 0, 4, 4, 1000, 3, 4, 4)
