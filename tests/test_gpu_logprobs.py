"""cwl_token_logprobs against its definition in 64 bits.

Tolerances, from the arithmetic (u = 2^-24): a term 2^t carries 4 u from the exponential and 3 u |t| from its exponent, and
the |t| weighted by the terms themselves is at most log2 V; a sum of n terms in 256 cells carries at most n/256 + 40
roundings.  So S is within eps_S = u (4 + 3 log2 V + V/256 + 40) relative, ln S within eps_S + u |ln S|, and each output
adds the roundings of its own few operations."""
import numpy as np
import pytest
import torch

from paper_2601_21109_b200 import binding as cwl

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def on_device(z, dtype, pad=0, offset=0):
    """[T, V] on the device as a view whose rows start `offset` elements into rows of V + pad (+ offset)."""
    T, V = z.shape
    buf = torch.full((T, V + pad + offset), 7.0, dtype=DT[dtype], device="cuda")
    view = buf[:, offset:offset + V]
    view.copy_(torch.from_numpy(z).cuda())
    return view


def reference(zt, targets, top_k, tau):
    z = zt.double().cpu().numpy()
    T, V = z.shape
    with np.errstate(all="ignore"):
        bad = ~(z.max(1) < np.inf) | (z.max(1) == -np.inf)
        m = np.where(bad, 0.0, z.max(1))
        d = (z - m[:, None]) / tau
        e = np.exp(d)
        s = e.sum(1)
        lse = np.where(bad, np.nan, m / tau + np.log(s))
        ent = np.where(bad, np.nan, np.log(s) - np.where(e > 0, d * e, 0.0).sum(1) / s)
        ids = np.argsort(-z, axis=1, kind="stable")[:, :top_k].astype(np.int64)
        top = np.take_along_axis(d, ids, 1) - np.log(s)[:, None]
    ids[bad], top[bad] = -1, np.nan
    lp = None
    if targets is not None:
        t = np.clip(targets, 0, V - 1)
        with np.errstate(all="ignore"):
            lp = d[np.arange(T), t] - np.log(s)
        lp[bad] = np.nan
        lp[targets < 0] = 0.0
        lp[targets >= V] = np.nan
    return dict(lse=lse, entropy=ent, logprob=lp, top_ids=ids, top_logprobs=top, m=m, V=V)


def close(got, ref, tol, what):
    got = got.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(ref)), what
    inf = np.isinf(ref)
    assert np.array_equal(got[inf], ref[inf]), what
    fine = np.isfinite(ref)
    over = np.abs(got[fine] - ref[fine]) - np.broadcast_to(tol, ref.shape)[fine]
    assert over.size == 0 or over.max() <= 0, f"{what}: over tolerance by {over.max():.3e}"


def check(zt, targets=None, top_k=0, tau=1.0, **kw):
    tt = None if targets is None else torch.from_numpy(targets.astype(np.int32)).cuda()
    o = cwl.cwl_token_logprobs(zt, tt, top_k=top_k, temperature=tau, **kw)
    tau32 = float(np.float32(tau))
    r = reference(zt, targets, top_k, tau32)
    V = r["V"]
    eps = U * (4 + 3 * np.log2(V + 1) + V / 256 + 40)
    with np.errstate(all="ignore"):
        mag = np.abs(np.nan_to_num(r["lse"])) + np.abs(r["m"]) / tau32
        close(o.lse, r["lse"], eps + 4 * U * mag, "lse")
        close(o.entropy, r["entropy"], 2 * eps * (1 + np.log(V + 1)) + 4 * U, "entropy")
        if targets is not None:
            close(o.logprob, r["logprob"], eps + 6 * U * (np.abs(np.nan_to_num(r["logprob"], posinf=0, neginf=0)) + np.log(V + 1)), "logprob")
        if top_k:
            assert np.array_equal(o.top_ids.cpu().numpy(), r["top_ids"]), "top_ids"
            close(o.top_logprobs, r["top_logprobs"],
                  eps + 6 * U * (np.abs(np.nan_to_num(r["top_logprobs"], posinf=0, neginf=0)) + np.log(V + 1)), "top_logprobs")
    return o


def rows(seed, T, V):
    rng = np.random.default_rng(seed)
    return (rng.standard_normal((T, V)) / rng.uniform(0.3, 3.0, size=(T, 1))).astype(np.float32)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,top_k,tau,pad", [
    (1, 32000, 20, 1.0, 0), (3, 1, 1, 1.0, 0), (5, 2, 2, 0.7, 1), (7, 127, 127, 1.0, 0), (37, 1000, 128, 1.3, 5),
    (64, 32003, 20, 0.7, 0), (9, 50021, 64, 2.0, 3), (300, 4099, 8, 1.0, 0), (333, 2048, 1, 1.0, 8), (2, 131072, 128, 1.0, 0),
    (150, 8192, 0, 1.0, 0)])
def test_sizes_and_types(dtype, T, V, top_k, tau, pad):
    z = rows(T * 1000 + V, T, V)
    targets = np.random.default_rng(V).integers(0, V, T)
    targets[::5] = -1
    check(on_device(z, dtype, pad), targets, top_k, tau)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("offset", [1, 2, 3, 5, 7])
def test_rows_that_start_anywhere(dtype, offset):
    check(on_device(rows(offset, 11, 3001), dtype, pad=2, offset=offset), np.arange(11), 16)
    check(on_device(rows(offset, 1, 9001), dtype, pad=2, offset=offset), np.arange(1), 16)     # one row, several CTAs


@pytest.mark.parametrize("T", [6, 400])           # rows shared by a cluster, and one CTA a row
def test_special_rows(T):
    V = 20011
    z = rows(3, T, V)
    z[0, 5] = np.nan
    z[1, V - 1] = np.inf
    z[2, :] = -np.inf
    z[3, 1:] = -np.inf                            # one token allowed
    z[4, :] = np.finfo(np.float32).min            # the type's lowest value everywhere: uniform
    z[5, 10:] = np.finfo(np.float32).min          # ... as a mask
    check(on_device(z, "f32"), np.zeros(T, np.int64), 12)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T", [4, 200])
def test_ties_go_to_the_lowest_index(dtype, T):
    V = 30011
    z = np.zeros((T, V), np.float32)
    z[0] = 3.25                                   # all equal
    z[1, ::2] = -0.0                              # zeros of both signs are equal
    z[2] = np.tile(np.array([1.0, 2.0, 2.0], np.float32), V // 3 + 1)[:V]
    z[3] = np.random.default_rng(0).integers(0, 40, V)
    o = check(on_device(z, dtype), np.arange(T), 100)
    assert o.top_ids[0].tolist() == list(range(100))


@pytest.mark.parametrize("allowed", [1, 3, 19, 20, 21, 500])
def test_rows_with_few_allowed_tokens(allowed):
    V, K = 32000, 20
    for T in (2, 180):
        rng = np.random.default_rng(allowed)
        z = np.full((T, V), -np.inf, np.float32)
        for t in range(T):
            z[t, rng.choice(V, allowed, replace=False)] = rng.standard_normal(allowed)
        check(on_device(z, "f32"), z.argmax(1), K)
        check(on_device(z, "bf16"), z.argmax(1), K)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("mask", [-np.inf, "lowest", -1.0e4, 0.0])
@pytest.mark.parametrize("V,top_k", [(32000, 20), (13363, 128), (900, 64), (70001, 128)])
def test_rows_full_of_one_value(dtype, mask, V, top_k):
    """Most logits hold one value (a mask, a floor), which a good part of the listed ones then is, lowest index first."""
    lowest = {"f32": np.finfo(np.float32).min, "f16": -65504.0, "bf16": -3.3895313892515355e38}[dtype]
    fill = lowest if mask == "lowest" else mask
    for T, allowed in ((3, 5), (3, 100), (160, 40), (640, 250)):
        rng = np.random.default_rng(allowed)
        z = np.full((T, V), fill, np.float32)
        for t in range(T):
            z[t, rng.choice(V, allowed, replace=False)] = rng.standard_normal(allowed) + (t % 2) * 2
        check(on_device(z, dtype), None, top_k)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V", [(1, 3909), (4, 29879), (21, 13363), (30, 57744), (500, 6000), (700, 12345), (9, 1024)])
def test_many_alternatives_of_short_slices(dtype, T, V):
    check(on_device(rows(T + V, T, V), dtype), None, 128)
    check(on_device(np.round(rows(T + V, T, V) * 3), dtype), None, 100)          # few different values


@pytest.mark.parametrize("dtype,stride", [("f32", 1024), ("bf16", 2048), ("f16", 2048)])
def test_large_logits_gathered_in_few_cells(dtype, stride):
    """Elements `stride` apart belong to the same thread: everything large sits in five threads' elements, so that the
    bound from the threads' maxima is far too low and thousands of logits lie above it."""
    T, V, K = 160, 160000, 20
    rng = np.random.default_rng(5)
    z = (rng.standard_normal((T, V)) * 0.1).astype(np.float32)
    v = np.arange(V)
    vec = 4 if dtype == "f32" else 8
    z[:, (v % stride) < 10 * vec] += 20.0 + rng.standard_normal((T, int(((v % stride) < 10 * vec).sum()))).astype(np.float32)
    check(on_device(z, dtype), None, K)
    # and with many of them equal
    z[:, (v % stride) < 10 * vec] = 20.0
    check(on_device(z, dtype), None, K)


def test_sorted_rows():
    V = 40000
    z = np.stack([np.linspace(-5, 5, V), np.linspace(5, -5, V)]).astype(np.float32)
    check(on_device(z, "f32"), np.array([0, V - 1]), 128)
    check(on_device(np.repeat(z, 100, 0), "f32"), None, 128)


@pytest.mark.parametrize("dtype,V", [("bf16", 9001), ("f32", 5003), ("f16", 16384)])
@pytest.mark.parametrize("top_k", [1, 64, 128])
def test_a_row_answers_the_same_among_many(dtype, V, top_k):
    """Rows of every kind, thousands at once, against calls on parts of them: a row's answer does not depend on the others."""
    T = 7200
    gen = torch.Generator(device="cuda")
    gen.manual_seed(V + top_k)
    z = torch.randn(T, V, device="cuda", generator=gen) / (0.3 + 2.7 * torch.rand(T, 1, device="cuda", generator=gen))
    z[0::16] = torch.randint(0, 40, (T // 16, V), device="cuda", generator=gen).float()          # ties
    z[1::16] = 2.5
    few = torch.rand(T // 16, V, device="cuda", generator=gen) < 10.0 / V                        # fewer allowed than listed
    z[2::16] = torch.where(few, z[2::16], float("-inf"))
    z[2::16, 7] = 1.0
    v = torch.arange(V, device="cuda")
    z[3::16] += 30.0 * ((v % 512) < 8)                                                           # large logits in few cells
    z[4::16] -= 30.0 * v / V
    z[5::16] = z[5::16].sort(dim=1).values
    z[6::160, 11], z[22::160, V - 1] = float("nan"), float("inf")
    z[38::160] = float("-inf")
    z[54::160] = -60000.0
    z = z.to(DT[dtype])
    t = torch.randint(-1, V, (T,), dtype=torch.int32, device="cuda", generator=gen)
    o = cwl.cwl_token_logprobs(z, t, top_k=top_k, temperature=0.8)
    for a in range(0, T, 2400):
        b = slice(a, a + 2400)
        w = cwl.cwl_token_logprobs(z[b], t[b].contiguous(), top_k=top_k, temperature=0.8)
        assert torch.equal(o.top_ids[b], w.top_ids)
        for x, y in ((o.lse[b], w.lse), (o.logprob[b], w.logprob), (o.top_logprobs[b], w.top_logprobs), (o.entropy[b], w.entropy)):
            assert torch.equal(torch.nan_to_num(x, nan=7.0), torch.nan_to_num(y, nan=7.0))


def test_bad_targets_are_flagged_and_good_ones_are_not():
    z = on_device(rows(1, 6, 300), "f32")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    check(z, np.array([0, 299, -1, -7, 5, 5]), 3, status_word=status)
    assert int(status.item()) == 0
    check(z, np.array([0, 300, -1, 2 ** 31 - 1, 5, 5]), 3, status_word=status)
    assert int(status.item()) == 1 << 1


def test_writes_only_its_outputs_and_answers_the_same_again():
    T, V, K = 70, 5003, 9
    z = on_device(rows(8, T, V), "bf16", pad=4)
    keep = z.clone()
    o = cwl.TokenLogprobs(T, K)
    base = o.lse._base if o.lse._base is not None else o.lse
    base.fill_(float("nan"))
    t = torch.arange(T, dtype=torch.int32, device="cuda")
    cwl.cwl_token_logprobs(z, t, top_k=K, out=o)
    first = [x.clone() for x in (o.lse, o.entropy, o.logprob, o.top_ids, o.top_logprobs)]
    assert not any(bool(torch.isnan(x.float()).any()) for x in first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        base.fill_(float("nan"))
        cwl.cwl_token_logprobs(z, t, top_k=K, out=o)
    side.synchronize()
    for a, b in zip(first, (o.lse, o.entropy, o.logprob, o.top_ids, o.top_logprobs)):
        assert torch.equal(a, b)
    assert torch.equal(z, keep)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cwl.cwl_token_logprobs(z, t, top_k=K, out=o)
    base.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(first, (o.lse, o.entropy, o.logprob, o.top_ids, o.top_logprobs)):
        assert torch.equal(a, b)


def test_agrees_with_the_complexity_score():
    V = 32000
    z = on_device(rows(12, 40, V), "f32")
    ent = cwl.cwl_token_logprobs(z).entropy
    score = cwl.cwl_score_tokens(z)
    assert float((ent / np.log(V) - score).abs().max()) <= 2e-5


def test_rows_past_two_to_the_31_elements():
    """The last row begins past 2^31 elements: offsets are 64-bit."""
    V = 16
    T = (1 << 31) // 1024 + 3
    buf = torch.empty(T * 1024, dtype=torch.bfloat16, device="cuda")
    z = buf.view(T, 1024)[:, :V]
    z.copy_(torch.randn(T, V, device="cuda"))
    o = cwl.cwl_token_logprobs(z, top_k=2)
    last = z[-4:].contiguous()
    w = cwl.cwl_token_logprobs(last, top_k=2)
    assert torch.equal(o.top_ids[-4:], w.top_ids) and torch.equal(o.lse[-4:], w.lse)


def test_refusals():
    z = torch.zeros(4, 16, device="cuda")
    for kw, status in ((dict(top_k=17), 1), (dict(top_k=-1), None), (dict(temperature=0.0), 1), (dict(temperature=-1.0), 1),
                       (dict(temperature=float("inf")), 1), (dict(temperature=float("nan")), 1)):
        with pytest.raises((cwl.CwlError, RuntimeError)) as e:
            cwl.cwl_token_logprobs(z, **kw)
        assert status is None or e.value.status == status
    with pytest.raises(cwl.CwlError) as e:
        cwl.cwl_token_logprobs(torch.zeros(2, 400, device="cuda"), top_k=129)
    assert e.value.status == 3
    with pytest.raises(AssertionError):
        cwl.cwl_token_logprobs(z.double())
    assert cwl.cwl_token_logprobs(torch.zeros(0, 16, device="cuda"), top_k=2).top_ids.shape == (0, 2)
    L = cwl.lib()
    assert L.cwl_token_logprobs(z.data_ptr(), 0, 15, 4, 16, None, 1.0, 0, None, None, None, None, None, None, None) == 2
    assert L.cwl_token_logprobs(z.data_ptr() + 2, 0, 16, 3, 16, None, 1.0, 0, None, None, None, None, None, None, None) == 2
    assert L.cwl_token_logprobs(z.data_ptr(), 5, 16, 4, 16, None, 1.0, 0, None, None, None, None, None, None, None) == 1
    assert L.cwl_token_logprobs(z.data_ptr(), 0, 16, 4, 16, z.data_ptr(), 1.0, 0, None, None, None, None, None, None, None) == 1
    assert L.cwl_token_logprobs(z.data_ptr(), 0, 16, 4, 16, None, 1.0, 2, None, None, None, None, None, None, None) == 1
