"""The failure path of the distillation and gradient kernels without a device fault: with the test hook (test build of the
library only) one copy that they wait for is never made; the waits run out after a short limit, the kernels report
CWL_ERR_TIMEOUT in the status word and return, and the next ordinary call on the same context is correct."""
import pytest
import torch

from paper_2601_21109_b200 import binding as cwl

pytestmark = pytest.mark.gpu
CWL_ERR_TIMEOUT = 7


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
        assert start.elapsed_time(end) < 2000.0                                  # a few wait limits, not seconds


@pytest.mark.parametrize("T,V,dtype", [(400, 24000, torch.bfloat16), (300, 32000, torch.float32)])   # one block a row; pairs of blocks
def test_distillation_that_waits_for_a_slice_that_never_comes(T, V, dtype):
    z = torch.randn(T, V, device="cuda").to(dtype)
    o = cwl.cwl_token_logprobs(z + 0.1, top_k=8)
    want = cwl.cwl_distill_topk(z, o.top_ids, o.top_logprobs, teacher="logprobs")
    timed(lambda status: cwl.cwl_distill_topk(z, o.top_ids, o.top_logprobs, teacher="logprobs", status_word=status))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = cwl.cwl_distill_topk(z, o.top_ids, o.top_logprobs, teacher="logprobs", status_word=status)
    assert int(status.item()) == 0 and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("T,d_in,d_out,R", [(256, 1024, 1024, 16), (2048, 512, 512, 64), (2048, 512, 512, 256)])
def test_gradients_that_wait_for_a_block_that_never_comes(T, d_in, d_out, R):
    X, dY, A, B = (torch.randn(r, c, device="cuda").bfloat16() for r, c in ((T, d_in), (T, d_out), (d_in, R), (R, d_out)))
    tab = cwl.DeviceChunkTable.from_host([0, T], [R], [1.0], [1])
    want = cwl.cwl_apply_grads(X, dY, A, B, tab, 0)
    timed(lambda status: cwl.cwl_apply_grads(X, dY, A, B, tab, 0, status_word=status))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = cwl.cwl_apply_grads(X, dY, A, B, tab, 0, status_word=status)
    assert int(status.item()) == 0 and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
