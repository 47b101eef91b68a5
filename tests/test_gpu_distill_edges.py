"""cwl_distill_topk where the student leaves next to nothing, or nothing, outside the teacher's entries: against the
definition in 64 bits, in logarithms.

Tolerances (u = 2^-24) are those of the sums: S within eps = u (4 + 3 log2 V + V/256 + 40) relative.  ln q_rest is ln S_out
- ln S_row and an exact distance of two maxima, so the rest's share of the loss is within p_rest 2 eps and what p_rest
itself is off, 20 u, times its logarithm.  An outside gradient is p_rest 2^t / S_out: relative 2 eps + u (30 + 3 |t|), t its
distance from the largest logit outside in powers of two, and 20 u / p_rest from p_rest."""
import numpy as np
import pytest
import torch

from paper_2601_21109_b200 import binding as cwl

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -24}
# one small block a row; a pipelined block a row; pairs and eights of blocks a row; (without gradients) the stream of many rows
FORMS = [(40, 1003), (300, 12007), (3, 32003), (165, 60007), (745, 12007)]


def definition(zt, ids, vals, mode, tau):
    """loss [T], gradient [T, V] for weight 1, the masses outside, and their logarithm for the student; fp64"""
    z, i, u = zt.double() / tau, ids.long(), vals.double()
    logq = torch.log_softmax(z, 1)
    p = torch.softmax(u / tau, 1) if mode == "logits" else u.exp()
    lp = torch.log_softmax(u / tau, 1) if mode == "logits" else u
    rest = (1.0 - p.sum(1)).clamp(min=0.0) if mode == "logprobs" else torch.zeros_like(p[:, 0])
    held = torch.zeros(z.shape, dtype=torch.bool, device=z.device).scatter_(1, i, True)
    out = logq.masked_fill(held, float("-inf"))
    lq_rest = torch.logsumexp(out, 1)
    loss = tau * tau * (torch.where(p > 0, p * (lp - logq.gather(1, i)), 0.0).sum(1)
                        + torch.where(rest > 0, rest * (rest.log() - lq_rest), 0.0))
    grad = logq.exp() * (p.sum(1) + rest)[:, None]
    share = torch.where(held, 0.0, (out - lq_rest[:, None]).exp())
    grad = tau * (grad.scatter_add(1, i, -p) - share * rest[:, None])
    return loss, grad, rest, lq_rest, share


def eps_of(V):
    return U * (4 + 3 * np.log2(V + 1) + V / 256 + 40)


@pytest.mark.parametrize("mode", ["logits", "logprobs"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("gap,tau", [(60.0, 1.0), (87.0, 1.0), (88.5, 1.0), (104.0, 1.0), (130.0, 2.0), (700.0, 1.0), (10000.0, 1.0), (12.0, 0.1)])
def test_outside_mass_far_below_the_entries(gap, tau, dtype, mode):
    outside_below(gap, tau, dtype, mode)


@pytest.mark.parametrize("mode", ["logits", "logprobs"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("gap", [15.0, 24.0, 31.0, 34.0, 37.0, 45.0])
def test_outside_mass_where_it_stops_showing_beside_the_entries(gap, dtype, mode):
    """2^-40 of the row is 27.7 nats below it; the mass of thousands of tokens reaches it with the tokens further down.  Nearer, an
    element's exponent counts from the row's maximum."""
    outside_below(gap, 1.0, dtype, mode, from_row_maximum=True)


def outside_below(gap, tau, dtype, mode, from_row_maximum=False):
    K = 8
    tau = float(np.float32(tau))
    for T, V in FORMS:
        gen = torch.Generator(device="cuda")
        gen.manual_seed(V + int(gap))
        z = torch.randn(T, V, device="cuda", generator=gen) * tau - gap
        ids = torch.rand(T, V, device="cuda", generator=gen).topk(K, dim=1).indices.to(torch.int32)
        z.scatter_(1, ids.long(), torch.rand(T, K, device="cuda", generator=gen) * 3 * tau)
        zt = z.to(DT[dtype])
        vals = torch.randn(T, K, device="cuda", generator=gen)
        if mode == "logprobs":
            vals = torch.log_softmax(vals, 1) + np.log(0.8)            # a fifth of the teacher's mass is outside
        loss, grad = cwl.cwl_distill_topk(zt, ids, vals, teacher=mode, temperature=tau)
        alone, _ = cwl.cwl_distill_topk(zt, ids, vals, teacher=mode, temperature=tau, want_grad=False)
        rl, rg, rest, lq_rest, share = definition(zt, ids, vals, mode, tau)
        eps = eps_of(V)
        mag = 12.0 + vals.double().abs().amax(1)                       # of the entries' logarithms
        tol = tau * tau * (2 * eps + 12 * U * mag + torch.where(rest > 0, 20 * U * (1 + (rest.log() - lq_rest).abs()), 0.0)) + 4 * U * rl.abs()
        for got in (loss, alone):
            assert bool(torch.isfinite(got).all())
            assert float(((got.double() - rl).abs() - tol).max()) <= 0
        held = share == 0
        top = zt.double().masked_fill(torch.zeros_like(held).scatter_(1, ids.long(), True), float("-inf")).amax(1, keepdim=True)
        if from_row_maximum:
            top = zt.double().amax(1, keepdim=True)
        far = ((zt.double() - top).abs() / tau * 1.4427).clamp(max=200.0)
        tol = rg.abs() * (2 * eps + U * (30 + 3 * far) + torch.where(rest > 0, 20 * U / rest, 0.0)[:, None])
        tol += rg.abs() * HALF_ULP[dtype] * 1.01 + TINY[dtype] * 1.01
        tol.scatter_add_(1, ids.long(), tau * (U * (14 + 4 * (vals.double().abs() + np.log(K + 1))) + 6 * eps))
        assert bool(torch.isfinite(grad).all())
        assert float(((grad.double() - rg).abs() - tol).max()) <= 0


def test_one_outcome_outside_at_the_edge_of_fp32():
    """Eight entries at 0 and one logit at -87 or below: with a teacher that leaves nothing to it its gradient is q itself."""
    ids = torch.arange(8, dtype=torch.int32, device="cuda")[None]
    for at in (-80.0, -87.0, -88.0, -95.0, -103.0, -200.0):
        z = torch.zeros(1, 9, device="cuda")
        z[0, 8] = at
        loss, grad = cwl.cwl_distill_topk(z, ids, torch.zeros(1, 8, device="cuda"), teacher="logits")
        assert abs(float(loss)) <= 1e-6 and float(grad[0, :8].abs().max()) <= 1e-6
        assert abs(float(grad[0, 8]) - np.exp(at) / 8) <= 1e-5 * np.exp(at) / 8 + 2.0 ** -126


RECORDS = [(64, 100, 100, None), (200, 128, 128, None), (64, 40, 40, None), (300, 12007, 64, 64), (300, 12007, 100, 20), (3, 32003, 128, 128),
           (165, 60007, 64, 33), (760, 12007, 64, 50), (800, 8200, 128, 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mask", [float("-inf"), -1.0e4, "lowest"])
@pytest.mark.parametrize("T,V,K,allowed", RECORDS)
def test_a_record_of_every_allowed_token_has_no_rest(T, V, K, allowed, mask, dtype):
    """The entries hold every token that the row allows: what 1 - sum p shows of a rest is the rounding of the record, and the
    student, which equals its teacher, has no loss.  Tolerance: the log-probabilities of the record and of the student are each
    within eps_S + 6 u (|ln p| + ln K), weighted by p."""
    for tau in (1.0, 0.7, 2.0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(T + V)
        z = torch.randn(T, V, device="cuda", generator=gen) * torch.rand(T, 1, device="cuda", generator=gen) * 3
        if allowed is not None:
            keep = torch.rand(T, V, device="cuda", generator=gen).topk(allowed, dim=1).indices
            held = torch.zeros(T, V, dtype=torch.bool, device="cuda").scatter_(1, keep, True)
            z.masked_fill_(~held, torch.finfo(DT[dtype]).min if mask == "lowest" else mask)
        zt = z.to(DT[dtype])
        o = cwl.cwl_token_logprobs(zt, top_k=K, temperature=tau)
        loss, grad = cwl.cwl_distill_topk(zt, o.top_ids, o.top_logprobs, teacher="logprobs", temperature=tau)
        alone, _ = cwl.cwl_distill_topk(zt, o.top_ids, o.top_logprobs, teacher="logprobs", temperature=tau, want_grad=False)
        tol = tau * tau * (2 * eps_of(V) + 12 * U * (1 + 2 * np.log(K)))
        for got in (loss, alone):
            assert bool(torch.isfinite(got).all()) and float(got.abs().max()) <= tol
        assert bool(torch.isfinite(grad).all()) and float(grad.abs().max()) <= tol / tau + HALF_ULP[dtype] * tol / tau


def test_a_rest_that_the_record_can_tell_from_none_is_kept():
    """A teacher that leaves 1e-5 outside, to a student that allows nothing there: the divergence is infinite."""
    for T, V in FORMS:
        z = torch.full((T, V), float("-inf"), device="cuda")
        z[:, :4] = torch.randn(T, 4, device="cuda")
        ids = torch.arange(4, dtype=torch.int32, device="cuda").repeat(T, 1)
        vals = torch.log_softmax(z[:, :4], 1) + np.log1p(-1e-5)
        loss, grad = cwl.cwl_distill_topk(z, ids, vals, teacher="logprobs")
        alone, _ = cwl.cwl_distill_topk(z, ids, vals, teacher="logprobs", want_grad=False)
        assert bool(torch.isinf(loss).all()) and bool(torch.isinf(alone).all()) and bool((grad[:, 4:] == 0).all())


def test_repeated_ids_give_the_same_bits_every_time():
    """Many entries name the same few tokens, from different warps: which of them counts the token must not depend on timing."""
    for T, V in ((745, 12007), (2000, 8200), (300, 12007), (40, 1003)):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(V)
        z = torch.randn(T, V, device="cuda", generator=gen)
        ids = torch.randint(0, V, (T, 40), device="cuda", generator=gen, dtype=torch.int32).repeat(1, 4)[:, :128].contiguous()
        ids = ids.gather(1, torch.rand(T, 128, device="cuda", generator=gen).argsort(1))
        z.scatter_(1, ids.long(), torch.rand(T, 128, device="cuda", generator=gen) * 6)
        vals = torch.randn(T, 128, device="cuda", generator=gen)
        first, _ = cwl.cwl_distill_topk(z, ids, vals, want_grad=False)
        for _ in range(60):
            again, _ = cwl.cwl_distill_topk(z, ids, vals, want_grad=False)
            assert torch.equal(first, again)


@pytest.mark.parametrize("temperature", [1.2e-38, 1e-39, 1e-42])
@pytest.mark.parametrize("mode", ["logits", "logprobs"])
def test_the_smallest_temperatures(mode, temperature):
    """Student and teacher put all mass on the same token: nothing to learn; gradients scale with the temperature."""
    for T, V in FORMS:
        z = torch.randn(T, V, device="cuda")
        z[:, 9] = 8.0
        ids = torch.tensor([[9, 4, 6]], dtype=torch.int32, device="cuda").repeat(T, 1)
        vals = torch.tensor([[8.0, 1.0, 0.0]] if mode == "logits" else [[0.0, -1e30, -2e30]], device="cuda").repeat(T, 1)
        loss, grad = cwl.cwl_distill_topk(z, ids, vals, teacher=mode, temperature=temperature)
        alone, _ = cwl.cwl_distill_topk(z, ids, vals, teacher=mode, temperature=temperature, want_grad=False)
        assert bool((loss == 0).all()) and bool((alone == 0).all()) and bool((grad == 0).all())


def test_rows_without_entries_teach_nothing_whatever_they_hold():
    """Teacher logits, every entry padding: loss and gradient are 0, of a row with NaN or +inf logits or none allowed too."""
    for T, V in FORMS:
        z = torch.randn(T, V, device="cuda")
        z[0, 5], z[1, 7], z[2] = float("nan"), float("inf"), float("-inf")
        ids = torch.full((T, 6), -1, dtype=torch.int32, device="cuda")
        vals = torch.full((T, 6), float("nan"), device="cuda")
        if T > 5:
            ids[5:, 2] = 11
            vals[5:, 2] = 1.0
        for dlogits in (None, z.clone()):
            loss, grad = cwl.cwl_distill_topk(z, ids, vals, dlogits=dlogits)
            alone, _ = cwl.cwl_distill_topk(z, ids, vals, want_grad=False)
            n = min(T, 5)
            assert bool((loss[:n] == 0).all()) and bool((alone[:n] == 0).all()) and bool((grad[:n] == 0).all())
            assert bool(torch.isfinite(loss).all()) and bool((loss[n:] > 0).all()) and torch.allclose(loss, alone, rtol=1e-5, atol=0)
