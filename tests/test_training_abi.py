"""Refusals and sizes of the log-probability, distillation and adapter-gradient calls that need no device: every one is
reported before anything touches CUDA."""
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


def logprobs(L, logits=P, dtype=0, ld=32, T=4, V=32, targets=None, temp=1.0, k=0, logprob=None, ids=None, top=None):
    return L.cwl_token_logprobs(logits, dtype, ld, T, V, targets, temp, k, logprob, P, P, ids, top, None, None)


def test_token_logprobs_refusals(L):
    assert logprobs(L, T=0) == 0
    assert logprobs(L, T=-1) == 1 and logprobs(L, V=0) == 1 and logprobs(L, k=-1) == 1 and logprobs(L, dtype=3) == 1
    for t in (0.0, -1.0, math.inf, math.nan):
        assert logprobs(L, temp=t) == 1
    assert logprobs(L, k=33, ids=P, top=P) == 1                       # more than there are tokens
    assert logprobs(L, V=4096, ld=4096, k=129, ids=P, top=P) == 3     # more than CWL_MAX_TOP_K
    assert logprobs(L, logits=None) == 1 and logprobs(L, k=2) == 1    # nowhere to put the alternatives
    assert logprobs(L, targets=P) == 1 and logprobs(L, logprob=P) == 1
    assert logprobs(L, ld=31) == 2 and logprobs(L, logits=P + 2) == 2 and logprobs(L, logits=P + 1, dtype=1) == 2


def distill(L, logits=P, dtype=0, ld=32, T=4, V=32, ids=P, vals=P, ldt=8, K=8, mode=0, temp=1.0, loss=P, dlogits=2 * P, ldd=32):
    return L.cwl_distill_topk(logits, dtype, ld, T, V, ids, vals, ldt, K, mode, temp, None, None, loss, dlogits, ldd, None, None)


def test_distill_topk_refusals(L):
    assert distill(L, T=0) == 0
    assert distill(L, T=-1) == 1 and distill(L, V=0) == 1 and distill(L, K=0) == 1 and distill(L, dtype=-1) == 1
    assert distill(L, mode=2) == 1 and distill(L, temp=0.0) == 1 and distill(L, temp=math.nan) == 1
    assert distill(L, K=129, ldt=129) == 3
    widest = 8 * 208 * 1024 // 4
    assert distill(L, V=widest + 1, ld=widest + 1, ldd=widest + 1) == 3
    assert distill(L, logits=None) == 1 and distill(L, ids=None) == 1 and distill(L, vals=None) == 1
    assert distill(L, loss=None, dlogits=None) == 1
    assert distill(L, ld=31) == 2 and distill(L, ldt=7) == 2 and distill(L, ldd=31) == 2
    assert distill(L, logits=P + 1, dtype=2) == 2 and distill(L, dlogits=P + 2) == 2
    assert distill(L, dlogits=P, ldd=40) == 2                         # in place, but with another stride


def grads(L, X=P, ldx=64, dY=P, lddy=64, A=P, lda=16, B=P, ldb=64, T=8, d_in=64, d_out=64, R=16, window=0, mode=0, dA=P, ldda=16,
          dB=P, lddb=64, dtype=1, ws=P, n=1 << 20, table=None):
    t = table if table is not None else cwl.CChunkTable(P, P, P, P, P, P, 1)
    return L.cwl_apply_grads(X, ldx, dY, lddy, A, lda, B, ldb, T, d_in, d_out, R, t, window, mode, dA, ldda, dB, lddb, dtype, ws, n,
                             None, None)


def test_apply_grads_refusals(L):
    assert grads(L, T=-1) == 1 and grads(L, d_in=0) == 1 and grads(L, R=0) == 1 and grads(L, window=-1) == 1
    assert grads(L, mode=2) == 1 and grads(L, dtype=2) == 1 and grads(L, dA=None) == 1 and grads(L, dB=None) == 1
    assert grads(L, d_in=72, ldx=72) == 3 and grads(L, d_out=40) == 3 and grads(L, R=8) == 3 and grads(L, R=272, lda=272, ldda=272) == 3
    assert grads(L, X=None) == 1 and grads(L, dY=None) == 1 and grads(L, A=None) == 1 and grads(L, B=None) == 1
    assert grads(L, table=cwl.CChunkTable(None, P, P, P, P, P, 1)) == 1
    for name in ("X", "dY", "A", "B", "dA", "dB"):
        assert grads(L, **{name: P + 8}) == 2, name
    for name in ("ldx", "lddy", "lda", "ldb", "ldda", "lddb"):
        base = {"lda": 16, "ldda": 16}.get(name, 64)
        assert grads(L, **{name: base - 8}) == 2 and grads(L, **{name: base + 4}) == 2, name
    assert grads(L, ws=None) == 5 and grads(L, ws=P + 16) == 5 and grads(L, n=64) == 5


def test_apply_grads_workspace(L):
    """H' and G, each two bf16 halves of [T, R] in rows of 2 R (R <= 128) or of R rounded up to 64, plus R."""
    w = cwl.cwl_apply_grads_workspace_bytes
    assert w(2048, 4096, 4096, 64) == 2 * 2048 * 128 * 2
    assert w(100, 64, 64, 144) == 2 * ((100 * (192 + 144) * 2 + 255) // 256 * 256)
    assert w(0, 64, 64, 16) == 0 and w(1, 16, 16, 16) == 512


def test_hooks_of_the_training_calls_exist_in_the_test_build_only(L):
    from paper_2601_21109_b200 import build
    assert not hasattr(ctypes.CDLL(build.LIB), "cwl_debug_training_set")
    assert hasattr(ctypes.CDLL(build.LIB_HOOKS), "cwl_debug_training_set")
