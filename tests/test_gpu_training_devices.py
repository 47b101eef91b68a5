"""Tensors that are not on the device are refused before anything is launched, in every place of the three calls."""
import pytest
import torch

from paper_2601_21109_b200 import binding as cwl

pytestmark = pytest.mark.gpu


def refused(call, tensors, name, host):
    with pytest.raises(AssertionError):
        call(**{**tensors, name: host})


def test_log_probabilities():
    z, t = torch.randn(4, 64, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    good = dict(logits=z, targets=t, top_k=2, out=cwl.TokenLogprobs(4, 2), status_word=torch.zeros(1, dtype=torch.int32, device="cuda"))
    cwl.cwl_token_logprobs(**good)
    for name in ("logits", "targets", "status_word"):
        refused(cwl.cwl_token_logprobs, good, name, good[name].cpu())
    refused(cwl.cwl_token_logprobs, good, "out", cwl.TokenLogprobs(4, 2, device="cpu"))
    refused(cwl.cwl_token_logprobs, good, "status_word", torch.zeros(1, device="cuda"))


def test_distillation():
    T, V, K = 4, 64, 3
    f = lambda *s: torch.rand(*s, device="cuda")   # noqa: E731
    good = dict(logits=f(T, V), teacher_ids=torch.zeros(T, K, dtype=torch.int32, device="cuda"), teacher_values=f(T, K), weight=f(T),
                dloss=f(T), loss=f(T), dlogits=f(T, V), status_word=torch.zeros(1, dtype=torch.int32, device="cuda"))
    cwl.cwl_distill_topk(**good)
    for name in good:
        refused(cwl.cwl_distill_topk, good, name, good[name].cpu())
    refused(cwl.cwl_distill_topk, good, "status_word", torch.zeros(1, dtype=torch.int64, device="cuda"))


def test_adapter_gradients():
    T, d, R = 32, 64, 16
    m = lambda *s: torch.rand(*s, device="cuda").bfloat16()   # noqa: E731
    table = lambda where: cwl.DeviceChunkTable.from_host([0, T], [R], [1.0], [1], device=where)   # noqa: E731
    ws = torch.empty(cwl.cwl_apply_grads_workspace_bytes(T, d, d, R), dtype=torch.uint8, device="cuda")
    good = dict(X=m(T, d), dY=m(T, d), A=m(d, R), B=m(R, d), table=table("cuda"), window=0, dA=m(d, R), dB=m(R, d), workspace=ws,
                status_word=torch.zeros(1, dtype=torch.int32, device="cuda"))
    cwl.cwl_apply_grads(**good)
    for name in ("X", "dY", "A", "B", "dA", "dB", "workspace", "status_word"):
        refused(cwl.cwl_apply_grads, good, name, good[name].cpu())
    refused(cwl.cwl_apply_grads, good, "table", table("cpu"))
    for part in ("offsets", "rank", "scale", "flags", "n_chunks"):
        mixed = table("cuda")
        setattr(mixed, part, getattr(mixed, part).cpu())
        refused(cwl.cwl_apply_grads, good, "table", mixed)
    refused(cwl.cwl_apply_grads, good, "workspace", ws.repeat(2)[::2])
    refused(cwl.cwl_apply_grads, good, "workspace", ws.view(torch.int32))
