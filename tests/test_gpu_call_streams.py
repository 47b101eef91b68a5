"""Calls given a stream of their own: what they allocate belongs to that stream, so that nothing else gets it while they run."""
import pytest
import torch

from paper_2601_21109_b200 import binding as cwl

pytestmark = pytest.mark.gpu


class Recorder:
    """The library, with the addresses that its calls are given noted."""

    def __init__(self, real):
        self.real, self.addresses = real, []

    def __getattr__(self, name):
        call = getattr(self.real, name)

        def noted(*args):
            self.addresses += [a for a in args if isinstance(a, int) and a > 1 << 32]
            return call(*args)
        return noted


def normal(*shape):
    return (torch.randn(*shape, device="cuda") * 0.1).bfloat16()


def calls():
    T, d, V, R = 96, 128, 1024, 16
    X, W, A, B, dY = normal(T, d), normal(d, V), normal(d, R), normal(R, V), normal(T, V)
    y = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32)
    table = cwl.DeviceChunkTable.from_host([0, 40, T], [R, R // 2], [1.0, 1.0], [1, 0])
    score, cu = torch.rand(T, device="cuda"), torch.tensor([0, T], device="cuda", dtype=torch.int32)
    policy = cwl.make_policy([4, 8, 16], [1.0, 1.0, 1.0], [0.3, 0.6], 4, 16, 2)
    logits = torch.randn(T, V, device="cuda")
    ids, zeros = y[:, None].contiguous(), torch.zeros(T, 1, device="cuda")
    us = [torch.randn(s, device="cuda") for s in ((16, 96), (100, 130))]
    keep = locals()
    return keep, {
        "head loss": lambda s: cwl.cwl_head_loss(X, W, y, want_dx=True, want_dw=True, stream=s),
        "orthogonalize": lambda s: cwl.cwl_orthogonalize(us, stream=s),
        "apply": lambda s: cwl.cwl_apply(X, W, A, B, table, 2, stream=s),
        "apply grouped": lambda s: cwl.cwl_apply_grouped(X, [W, W], [A, A], [B, B], table, 2, stream=s),
        "apply grads": lambda s: cwl.cwl_apply_grads(X, dY, A, B, table, 2, stream=s),
        "partition": lambda s: cwl.cwl_partition(score, cu, policy, stream=s),
        "batch align": lambda s: cwl.cwl_batch_align(score, cu, policy, 1, stream=s),
        "score": lambda s: cwl.cwl_score_tokens(logits, stream=s),
        "logprobs": lambda s: cwl.cwl_token_logprobs(logits, y, 4, stream=s),
        "distill": lambda s: cwl.cwl_distill_topk(logits, ids, zeros, stream=s),
        "ladder": lambda s: cwl.cwl_ladder_build(A, B, stream=s),
    }


def segments(stream):
    return [(s["address"], s["address"] + s["total_size"]) for s in torch.cuda.memory_snapshot() if s["stream"] == stream]


def values(out):
    if torch.is_tensor(out):
        return [out]
    if isinstance(out, dict):
        out = list(out.values())
    elif hasattr(out, "__dict__") and not isinstance(out, tuple):
        out = list(vars(out).values())
    return [t for x in out for t in values(x)] if isinstance(out, (list, tuple)) else []


@pytest.mark.parametrize("name", list(calls()[1]) if torch.cuda.is_available() else ["no device"])
def test_what_a_call_allocates_belongs_to_its_stream(name, monkeypatch):
    keep, made = calls()
    want = [t.clone() for t in values(made[name](None))]
    torch.cuda.synchronize()
    given = [(t.data_ptr(), t.data_ptr() + t.untyped_storage().nbytes()) for x in keep.values() for t in values(x)]
    recorder = Recorder(cwl.lib())
    monkeypatch.setattr(cwl, "lib", lambda: recorder)
    stream = torch.cuda.Stream()
    out = made[name](stream)
    here = segments(stream.cuda_stream)
    own = [a for a in recorder.addresses if a != stream.cuda_stream and not any(b <= a < e for b, e in given)]
    own += [t.data_ptr() for t in values(out) if t.numel()]
    assert own and all(any(b <= a < e for b, e in here) for a in own)
    torch.cuda.synchronize()
    got = values(out)
    assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_kept_call_that_is_dropped_keeps_its_workspace_until_it_has_run():
    us = [torch.randn(64, 4096, device="cuda")]
    call = cwl.OrthogonalizeCall(us, [torch.empty_like(us[0])])
    at, n = call.workspace.data_ptr(), call.workspace.numel()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        torch.cuda._sleep(200_000_000)                     # a tenth of a second
    call(stream=stream)
    del call
    others = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(3)]
    assert not stream.query()
    assert all(t.data_ptr() + n <= at or t.data_ptr() >= at + n for t in others)
    torch.cuda.synchronize()
