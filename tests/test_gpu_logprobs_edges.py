"""cwl_token_logprobs at the ends of its range: near-certain tokens, the smallest temperatures, numbers next to zero."""
import numpy as np
import pytest
import torch

from paper_2601_21109_b200 import binding as cwl

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V", [(2000, 32000), (3000, 4099), (40, 32000), (1, 50021)])
def test_no_log_probability_is_positive(dtype, T, V):
    """m is the row's maximum and the largest term of S is 1 itself, so S >= 1 and no log-probability exceeds 0; a near-certain
    token's is ln S of an S of 1 and little more: what it loses are the terms' roundings beside the 1 (as many as a thread has,
    each half a spacing at most) and 2 u of its own."""
    for tau in (1.0, 0.6):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(T + V)
        z = torch.randn(T, V, device="cuda", generator=gen) * 0.7
        at = torch.randint(0, V, (T, 1), device="cuda", generator=gen)
        z.scatter_(1, at, 12.0 + 14.0 * torch.rand(T, 1, device="cuda", generator=gen))
        zt = z.to(DT[dtype])
        t = zt.float().argmax(1).to(torch.int32)
        o = cwl.cwl_token_logprobs(zt, t, top_k=3, temperature=tau)
        assert float(o.logprob.max()) <= 0 and float(o.top_logprobs.max()) <= 0
        d = (zt.double() - zt.double().amax(1, keepdim=True)) / float(np.float32(tau))
        ref = -torch.log(torch.exp(d).sum(1))
        # the row's small terms as a whole are off by their own relative error (dist up to 40 powers of two)
        tol = (V / 256 + 40) * U + ref.abs() * U * (8 + 3 * 60)
        assert float(((o.logprob.double() - ref).abs() - tol).max()) <= 0


@pytest.mark.parametrize("temperature", [1.2e-38, 1e-39, 1e-42, 1.5e-45, 3.0e38])
@pytest.mark.parametrize("T,V", [(3, 20011), (400, 20011), (5, 200)])
def test_the_smallest_and_largest_temperatures(temperature, T, V):
    """All mass on the largest logits, dealt evenly to those that are equal; or on every allowed token alike."""
    z = torch.randn(T, V, device="cuda")
    z[:, 3], z[:, 150], z[:, 7] = 9.0, 9.0, float("-inf")
    t = torch.tensor([3, 150, 8] * T, dtype=torch.int32, device="cuda")[:T]
    o = cwl.cwl_token_logprobs(z, t, top_k=3, temperature=temperature)
    if temperature < 1:
        want = torch.where(t == 8, float("-inf"), -float(np.log(2.0)))
        assert torch.allclose(o.entropy, torch.full_like(o.entropy, float(np.log(2.0))), rtol=1e-6)
        assert bool((o.top_ids[:, :2] == torch.tensor([3, 150], dtype=torch.int32, device="cuda")).all())
        assert bool((o.top_logprobs[:, 2] < -1e30).all())
        at = t != 8
        assert torch.allclose(o.logprob[at], want[at].float(), rtol=1e-6) and bool((o.logprob[~at] < -1e30).all())
    else:
        assert torch.allclose(o.logprob, torch.full_like(o.logprob, -float(np.log(V - 1))), rtol=1e-5)
        assert torch.allclose(o.entropy, torch.full_like(o.entropy, float(np.log(V - 1))), rtol=1e-5)


def test_zeros_above_a_row_of_the_smallest_negative_number():
    """More zeros than are wanted, all in a few threads' elements, in a row otherwise full of -2^-149: the zeros come first, the
    lowest indices of them."""
    for T in (3, 400):
        V, K = 8192, 64
        z = torch.full((T, V), -(2.0 ** -149), device="cuda")
        zeros = torch.cat([torch.arange(c * 512, c * 512 + 20) for c in range(16)])        # five vectors of each batch
        z[:, zeros.cuda()] = 0.0
        o = cwl.cwl_token_logprobs(z, top_k=K)
        assert bool((o.top_ids == zeros[:K].to(torch.int32).cuda()).all())
