"""cwl_distill_topk against its definition in 64 bits, and its gradient against differences of that definition.

Tolerances, from the arithmetic (u = 2^-24).  As for the log-probabilities, S is within eps_S = u (4 + 3 log2 V + V/256 +
40) relative and an exponential within 4 u + 3 u |t|, |t| the distance of its logit from the maximum in powers of two (a
term of weight below 2^-24 of the row moves nothing, so |t| <= 24 counts for sums).  A gradient entry outside the
teacher's is a product of four such factors: relative error 2 eps_S + u (20 + 3 |t|) of q_v times the gradient's scale
(with p_rest / q_rest up to `amplify`).  An entry of the teacher adds the rounding of p_j (10 u, plus 3 u |u_j|).  The loss
is a sum of p_j ln(p_j / q_j) whose logarithms are within 2 eps_S + u * 6 (|ln p| + |ln q|)."""
import numpy as np
import pytest
import torch

from paper_2601_21109_b200 import binding as cwl

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}     # of a number rounded to 24, 8 and 11 significant bits
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -24}      # spacing of the type's smallest numbers (ftz for fp32)


def definition(z, ids, vals, mode, tau, w, dloss):
    """fp64 loss [T] and gradient [T, V] of the definition; z fp64 numpy, ids < 0 padding."""
    T, V = z.shape
    loss, grad = np.zeros(T), np.zeros((T, V))
    info = []
    for t in range(T):
        if w[t] == 0:
            info.append((0.0, 1.0))
            continue
        keep = ids[t] >= 0
        i, u = ids[t][keep], vals[t][keep]
        m = z[t].max()
        if not m < np.inf or m == -np.inf:
            loss[t], grad[t] = np.nan, np.nan
            info.append((0.0, 1.0))
            continue
        with np.errstate(all="ignore"):
            d = (z[t] - m) / tau
            lq = d - np.log(np.exp(d).sum())
            q = np.exp(lq)
            if mode == "logits":
                if len(u) == 0:
                    info.append((0.0, 1.0))
                    continue
                p = np.exp((u - u.max()) / tau)
                lp = (u - u.max()) / tau - np.log(p.sum())
                p = p / p.sum()
                rest = 0.0
            else:
                p, lp = np.exp(u), u
                rest = max(0.0, 1.0 - p.sum())
            inside = np.zeros(V, bool)
            inside[i] = True
            q_rest = q[~inside].sum()
            kl = np.where(p > 0, p * (lp - lq[i]), 0.0).sum()
            if rest > 0:
                kl += rest * (np.log(rest) - np.log(q_rest))
            g = q * (p.sum() + rest)
            np.subtract.at(g, i, p)
            if rest > 0 and q_rest > 0:
                g[~inside] -= rest * q[~inside] / q_rest
        loss[t] = w[t] * tau * tau * kl
        grad[t] = g * w[t] * tau * dloss[t]
        info.append((rest, q_rest))
    return loss, grad, info


def teacher_of(z, K, mode, tau, seed, short=True):
    rng = np.random.default_rng(seed)
    T, V = z.shape
    with np.errstate(all="ignore"):
        y = np.where(np.isfinite(z), z, -30.0) + 0.7 * rng.standard_normal(z.shape)
        if mode == "logprobs":
            y = y / tau
            m = y.max(1, keepdims=True)
            y = y - m - np.log(np.exp(y - m).sum(1, keepdims=True))
    ids = np.argsort(-y, axis=1, kind="stable")[:, :K].astype(np.int32)
    vals = np.take_along_axis(y, ids, 1).astype(np.float32)
    if short:
        for t in range(0, T, 3):
            ids[t, K - K // 3:] = -1
            vals[t, K - K // 3:] = np.nan                      # what padding holds is not read
    return ids, vals


def device(z, dtype, pad=0, offset=0):
    T, V = z.shape
    buf = torch.full((T, V + pad + offset), 3.0, dtype=DT[dtype], device="cuda")
    v = buf[:, offset:offset + V]
    v.copy_(torch.from_numpy(z).cuda())
    return v


def check(zt, ids, vals, mode, tau=1.0, w=None, dloss=None, dtype="f32", dlogits=None, status=None, grad_too=True):
    T, V = zt.shape
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()   # noqa: E731
    z64 = zt.double().cpu().numpy()
    loss, grad = cwl.cwl_distill_topk(zt, dev(ids), dev(vals), teacher=mode, temperature=tau, weight=dev(w), dloss=dev(dloss),
                                      dlogits=dlogits, status_word=status, want_grad=grad_too)
    tau64 = float(np.float32(tau))
    w64 = np.ones(T) if w is None else w.astype(np.float64)
    d64 = np.ones(T) if dloss is None else dloss.astype(np.float64)
    ids_ok = np.where(ids >= V, -1, ids)
    rl, rg, info = definition(z64, ids_ok, vals.astype(np.float64), mode, tau64, w64, d64)
    gl, gg = loss.double().cpu().numpy(), grad.double().cpu().numpy() if grad_too else rg
    eps = U * (4 + 3 * np.log2(V + 1) + V / 256 + 40)
    assert np.array_equal(np.isnan(gl), np.isnan(rl)) and np.array_equal(np.isinf(gl), np.isinf(rl))
    assert np.array_equal(np.isnan(gg), np.isnan(rg))
    for t in range(T):
        if np.isnan(rl[t]) or w64[t] == 0:
            continue
        scale = abs(w64[t] * tau64 * d64[t])
        rest, q_rest = info[t]
        with np.errstate(all="ignore"):
            m = z64[t].max()
            dist = np.minimum(np.abs(z64[t] - m) / tau64 * 1.4427, 200.0)
            q = np.exp((z64[t] - m) / tau64)
            q = q / q.sum()
        amplify = 1.0 + (rest / q_rest if q_rest > 0 else 0.0)
        # p_rest = 1 - sum p carries the roundings of the p's, relative to 1
        rest_err = (20 * U / q_rest if (rest > 0 and q_rest > 0) else 0.0)
        tol = scale * (q * (amplify * (3 * eps + U * (30 + 3 * dist)) + rest_err))
        i = ids_ok[t][ids_ok[t] >= 0]
        u_mag = np.abs(vals[t][ids_ok[t] >= 0].astype(np.float64))
        np.add.at(tol, i, scale * U * (14 + 4 * (u_mag + np.log(len(i) + 1))) * 1.0)
        tol = tol + np.abs(rg[t]) * HALF_ULP[dtype] * 1.01 + TINY[dtype] * 1.01
        over = np.abs(gg[t] - rg[t]) - tol
        assert over.max() <= 0, f"row {t}: gradient over tolerance by {over.max():.3e} at {over.argmax()}"
        if np.isfinite(rl[t]):
            with np.errstate(all="ignore"):
                lq = np.maximum(np.log(q[i]) if len(i) else np.zeros(1), -200.0)
                mag = np.abs(lq).max() + (u_mag.max() if len(i) else 0.0) + (abs(np.log(q_rest)) if q_rest > 0 else 0.0) + 1.0
            tol_l = abs(w64[t]) * tau64 ** 2 * (2 * eps + 12 * U * mag + (20 * U * (1 + abs(np.log(rest / q_rest)))
                                                                         if rest > 0 and q_rest > 0 else 0.0)) + abs(rl[t]) * 4 * U
            assert abs(gl[t] - rl[t]) <= tol_l, f"row {t}: loss {gl[t]} against {rl[t]}, tolerance {tol_l:.2e}"
    return loss, grad


def rows(seed, T, V):
    rng = np.random.default_rng(seed)
    z = (rng.standard_normal((T, V)) / rng.uniform(0.4, 3.0, size=(T, 1))).astype(np.float32)
    for t in range(T):
        z[t, rng.integers(0, V, 5)] += 6.0
    return z


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("mode", ["logits", "logprobs"])
@pytest.mark.parametrize("T,V,K,tau,pad", [
    (1, 32000, 64, 1.0, 0), (7, 32003, 8, 2.0, 5), (5, 1, 1, 1.0, 0), (4, 2, 1, 1.0, 3), (9, 130, 128, 1.5, 0),
    (40, 1003, 20, 0.7, 0), (330, 517, 16, 1.0, 1), (170, 4099, 100, 2.0, 0), (3, 131072, 128, 1.0, 0), (2, 9001, 1, 1.0, 0)])
def test_sizes_and_types(dtype, mode, T, V, K, tau, pad):
    zt = device(rows(T + V, T, V), dtype, pad)
    ids, vals = teacher_of(zt.double().cpu().numpy(), K, mode, tau, V)
    rng = np.random.default_rng(T)
    w = rng.uniform(0.5, 2.0, T).astype(np.float32)
    w[1::4] = 0.0
    check(zt, ids, vals, mode, tau, w, rng.uniform(-1.5, 1.5, T).astype(np.float32), dtype)


@pytest.mark.parametrize("T,V,dtype", [(592, 20003, "bf16"), (600, 11000, "f32"), (591, 20003, "bf16"), (640, 22528, "f16"), (592, 22529, "bf16")])
def test_rows_on_both_sides_of_the_small_blocks(T, V, dtype):
    zt = device(rows(V, T, V), dtype, 1)
    ids, vals = teacher_of(zt.double().cpu().numpy(), 33, "logprobs", 1.0, V)
    w = np.ones(T, np.float32)
    w[::7] = 0.0
    check(zt, ids, vals, "logprobs", 1.0, w, None, dtype)


@pytest.mark.parametrize("T,V,dtype", [(310, 53240, "bf16"), (310, 53257, "f16"), (301, 26619, "f32"), (160, 150001, "bf16"), (165, 100003, "f32")])
def test_rows_in_the_longest_slices(T, V, dtype):
    zt = device(rows(V, T, V), dtype, 1)
    ids, vals = teacher_of(zt.double().cpu().numpy(), 33, "logprobs", 1.0, V)
    w = np.ones(T, np.float32)
    w[::7] = 0.0
    check(zt, ids, vals, "logprobs", 1.0, w, None, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("offset,out_offset", [(1, 1), (3, 0), (0, 5), (6, 7)])
def test_rows_that_start_anywhere(dtype, offset, out_offset):
    for T in (2, 180):                                     # several CTAs a row, and one
        zt = device(rows(offset, T, 20011 if T == 2 else 2003), dtype, pad=3, offset=offset)
        V = zt.shape[1]
        ids, vals = teacher_of(zt.double().cpu().numpy(), 12, "logprobs", 1.0, 1)
        guard = torch.full((T + 1, V + 16), float("nan"), dtype=DT[dtype], device="cuda")
        check(zt, ids, vals, "logprobs", dtype=dtype, dlogits=guard[:T, out_offset:out_offset + V])
        assert bool(torch.isnan(guard[T]).all()) and bool(torch.isnan(guard[:, :out_offset]).all())
        assert bool(torch.isnan(guard[:, out_offset + V:]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("mode", ["logits", "logprobs"])
@pytest.mark.parametrize("T,V,K,tau,pad", [(740, 16411, 128, 1.0, 0), (760, 9001, 20, 2.0, 3), (800, 8200, 1, 0.7, 1), (741, 50021, 64, 1.0, 0)])
def test_the_loss_alone_of_many_rows(dtype, mode, T, V, K, tau, pad):
    zt = device(rows(T + V, T, V), dtype, pad)
    ids, vals = teacher_of(zt.double().cpu().numpy(), K, mode, tau, V)
    w = np.random.default_rng(T).uniform(0.5, 2.0, T).astype(np.float32)
    w[1::4] = 0.0
    check(zt, ids, vals, mode, tau, w, None, dtype, grad_too=False)


def test_the_loss_alone_of_special_rows():
    T, V, K = 745, 12007, 10
    z = rows(4, T, V)
    ids, vals = teacher_of(z.astype(np.float64), K, "logprobs", 1.0, 9, short=False)
    z[0, 100], z[1, 200], z[2, :] = np.nan, np.inf, -np.inf
    z[3, ~np.isin(np.arange(V), ids[3])] = -np.inf
    z[4, ids[4, 0]] = -np.inf
    ids[5] = -1
    z[6, :] = np.finfo(np.float32).min
    z[7, ~np.isin(np.arange(V), ids[7])] = np.finfo(np.float32).min
    z[8, :] += 50000.0                                     # far from 0: the exact form of the exponent
    ids[9, 1:] = ids[9, 0]
    z[10, ids[10, 2]] = np.nan
    zt = device(z, "f32")
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()   # noqa: E731
    for mode in ("logits", "logprobs"):
        alone, _ = cwl.cwl_distill_topk(zt, dev(ids), dev(vals), teacher=mode, want_grad=False)
        both, _ = cwl.cwl_distill_topk(zt, dev(ids), dev(vals), teacher=mode)
        rl, _, _ = definition(zt.double().cpu().numpy(), ids, vals.astype(np.float64), mode, 1.0, np.ones(T), np.ones(T))
        for got in (alone, both):
            g = got.double().cpu().numpy()
            assert np.array_equal(np.isnan(g), np.isnan(rl)) and np.array_equal(np.isinf(g), np.isinf(rl))
            fine = np.isfinite(rl)
            assert np.allclose(g[fine], rl[fine], rtol=2e-4, atol=2e-4)


def test_wide_rows_take_a_cluster():
    for V, dtype in ((160000, "f32"), (300000, "f32"), (250007, "bf16")):
        zt = device(rows(V, 2, V), dtype)
        ids, vals = teacher_of(zt.double().cpu().numpy(), 64, "logprobs", 1.0, 3)
        check(zt, ids, vals, "logprobs", dtype=dtype)


@pytest.mark.parametrize("mode", ["logits", "logprobs"])
@pytest.mark.parametrize("T", [8, 300])
def test_special_rows(mode, T):
    V, K = 12007, 10
    z = rows(4, T, V)
    ids, vals = teacher_of(z.astype(np.float64), K, mode, 1.0, 9, short=False)
    z[0, 100] = np.nan
    z[1, 200] = np.inf
    z[2, :] = -np.inf
    keep = ids[3].copy()
    z[3, ~np.isin(np.arange(V), keep)] = -np.inf           # the student allows the teacher's entries only: no mass outside
    z[4, ids[4, 0]] = -np.inf                              # it forbids one that the teacher wants: infinite loss
    ids[5] = -1                                            # no entries
    z[6, :] = np.finfo(np.float32).min                     # the type's lowest value everywhere
    z[7, ~np.isin(np.arange(V), ids[7])] = np.finfo(np.float32).min
    w = np.ones(T, np.float32)
    zt = device(z, "f32")
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()   # noqa: E731
    loss, grad = cwl.cwl_distill_topk(zt, dev(ids), dev(vals), teacher=mode, weight=dev(w))
    rl, rg, _ = definition(z.astype(np.float64), ids, vals.astype(np.float64), mode, 1.0, w.astype(np.float64), np.ones(T))
    gl, gg = loss.double().cpu().numpy(), grad.double().cpu().numpy()
    assert np.array_equal(np.isnan(gl), np.isnan(rl)) and np.array_equal(np.isinf(gl), np.isinf(rl)), (gl[:8], rl[:8])
    assert np.array_equal(np.isnan(gg), np.isnan(rg))
    assert gl[5] == 0.0 or mode == "logprobs"
    fine = np.isfinite(rl)
    assert np.allclose(gl[fine], rl[fine], rtol=2e-4, atol=2e-4)
    fine = np.isfinite(rg)
    assert np.allclose(gg[fine], rg[fine], rtol=0, atol=4e-5)


def test_masked_rows_are_not_read():
    """Rows of weight 0 may hold anything: their loss and gradient are exactly 0."""
    T, V = 50, 3001
    z = rows(2, T, V)
    ids, vals = teacher_of(z.astype(np.float64), 8, "logprobs", 1.0, 2)
    w = np.ones(T, np.float32)
    w[:20] = 0.0
    z[:20] = np.nan
    zt = device(z, "f32")
    loss, grad = check(zt, ids, vals, "logprobs", w=w)
    assert bool((loss[:20] == 0).all()) and bool((grad[:20] == 0).all())


def test_repeated_and_out_of_range_ids():
    T, V, K = 5, 700, 12
    z = rows(6, T, V)
    ids, vals = teacher_of(z.astype(np.float64), K, "logits", 1.0, 6, short=False)
    ids[0, 5] = ids[0, 2]
    ids[1, :] = ids[1, 0]
    zt = device(z, "f32")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    check(zt, ids, vals, "logits", status=status)
    assert int(status.item()) == 0
    ids[2, 3] = V
    ids[3, 0] = 2 ** 31 - 1
    ids[4, 1] = -5
    check(zt, ids, vals, "logits", status=status)
    assert int(status.item()) == 1 << 1


def test_gradient_against_differences_of_the_definition():
    T, V, K, tau = 3, 60, 6, 1.7
    z = rows(11, T, V).astype(np.float64)
    for mode in ("logits", "logprobs"):
        ids, vals = teacher_of(z, K, mode, tau, 11)
        w = np.array([0.5, 1.0, 2.0], np.float32)
        dl = np.array([1.0, -2.0, 0.7], np.float32)
        _, grad = check(device(z.astype(np.float32), "f32"), ids, vals, mode, tau, w, dl)
        z32 = z.astype(np.float32).astype(np.float64)
        h = 1e-5
        num = np.zeros((T, V))
        for v in range(V):
            up, dn = z32.copy(), z32.copy()
            up[:, v] += h
            dn[:, v] -= h
            args = (ids, vals.astype(np.float64), mode, tau, w.astype(np.float64), np.ones(T))
            num[:, v] = (definition(up, *args)[0] - definition(dn, *args)[0]) / (2 * h) * dl
        # central differences: h^2 times a third derivative of order w tau^-1, and rounding of order 1e-16 / h
        assert np.abs(grad.double().cpu().numpy() - num).max() <= 1e-6


def test_forward_then_backward_equals_one_call_and_in_place():
    T, V, K = 90, 8003, 20
    for dtype in ("f32", "bf16"):
        zt = device(rows(5, T, V), dtype, pad=5)
        ids, vals = (torch.from_numpy(a).cuda() for a in teacher_of(zt.double().cpu().numpy(), K, "logprobs", 1.0, 5))
        dl = torch.rand(T, device="cuda")
        both = cwl.cwl_distill_topk(zt, ids, vals, teacher="logprobs", dloss=dl)
        loss, none = cwl.cwl_distill_topk(zt, ids, vals, teacher="logprobs", want_grad=False)
        assert none is None and torch.equal(loss, both[0])
        none, grad = cwl.cwl_distill_topk(zt, ids, vals, teacher="logprobs", dloss=dl, want_loss=False)
        assert none is None and torch.equal(grad, both[1])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            cwl.cwl_distill_topk(zt, ids, vals, teacher="logprobs", dloss=dl, dlogits=zt)
        side.synchronize()
        assert torch.equal(zt, both[1])


def test_teacher_rows_with_a_pitch_and_a_captured_step():
    T, V, K = 33, 3001, 7
    z = rows(15, T, V)
    zt = device(z, "bf16")
    ids, vals = teacher_of(zt.double().cpu().numpy(), K, "logprobs", 1.0, 5)
    wide_i = torch.full((T, K + 4), -3, dtype=torch.int32, device="cuda")
    wide_v = torch.full((T, K + 4), float("nan"), device="cuda")
    wide_i[:, :K].copy_(torch.from_numpy(ids))
    wide_v[:, :K].copy_(torch.from_numpy(vals))
    a = cwl.cwl_distill_topk(zt, wide_i[:, :K], wide_v[:, :K], teacher="logprobs")
    b = cwl.cwl_distill_topk(zt, wide_i[:, :K].contiguous(), wide_v[:, :K].contiguous(), teacher="logprobs")
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    loss, grad = torch.zeros(T, device="cuda"), torch.zeros_like(a[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cwl.cwl_distill_topk(zt, wide_i[:, :K], wide_v[:, :K], teacher="logprobs", loss=loss, dlogits=grad)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(loss, a[0]) and torch.equal(grad, a[1])


def test_a_student_that_equals_its_teacher_has_no_loss_and_no_gradient():
    T, V, K = 20, 9001, 50
    zt = device(rows(21, T, V), "f32")
    for tau in (1.0, 2.0):
        o = cwl.cwl_token_logprobs(zt, top_k=K, temperature=tau)
        loss, grad = cwl.cwl_distill_topk(zt, o.top_ids, o.top_logprobs, teacher="logprobs", temperature=tau)
        # the log-probabilities are rounded to fp32: relative error of a p about 2^-24 |ln p| + eps_S
        assert float(loss.abs().max()) <= 2e-5 and float(grad.abs().max()) <= 2e-5


def test_refusals():
    z = torch.zeros(4, 16, device="cuda")
    ids = torch.zeros(4, 3, dtype=torch.int32, device="cuda")
    vals = torch.zeros(4, 3, device="cuda")
    for kw, status in ((dict(temperature=0.0), 1), (dict(temperature=float("nan")), 1)):
        with pytest.raises(cwl.CwlError) as e:
            cwl.cwl_distill_topk(z, ids, vals, **kw)
        assert e.value.status == status
    with pytest.raises(cwl.CwlError) as e:
        cwl.cwl_distill_topk(torch.zeros(1, 200, device="cuda"), torch.zeros(1, 129, dtype=torch.int32, device="cuda"),
                             torch.zeros(1, 129, device="cuda"))
    assert e.value.status == 3
    with pytest.raises(cwl.CwlError) as e:
        cwl.cwl_distill_topk(torch.zeros(1, 430000, device="cuda"), ids[:1], vals[:1])
    assert e.value.status == 3
    with pytest.raises(cwl.CwlError) as e:
        cwl.cwl_distill_topk(z, ids, vals, want_loss=False, want_grad=False)
    assert e.value.status == 1
    with pytest.raises(KeyError):
        cwl.cwl_distill_topk(z, ids, vals, teacher="else")
    with pytest.raises(AssertionError):
        cwl.cwl_distill_topk(z, ids.long(), vals)
    with pytest.raises(AssertionError):
        cwl.cwl_distill_topk(z, ids, vals, weight=torch.ones(3, device="cuda"))
    p, L = z.data_ptr(), cwl.lib()
    args = lambda ld=16, ldt=3, ldd=16, k=3, mode=0, dt=0: (p, dt, ld, 4, 16, ids.data_ptr(), vals.data_ptr(), ldt, k, mode, 1.0,   # noqa: E731
                                                            None, None, None, p, ldd, None, None)
    assert L.cwl_distill_topk(*args(ld=15)) == 2 and L.cwl_distill_topk(*args(ldt=2)) == 2
    assert L.cwl_distill_topk(*args(ldd=15)) == 2 and L.cwl_distill_topk(*args(ldd=17)) == 2    # in place with another stride
    assert L.cwl_distill_topk(*args(k=0)) == 1 and L.cwl_distill_topk(*args(mode=2)) == 1 and L.cwl_distill_topk(*args(dt=3)) == 1
    loss, grad = cwl.cwl_distill_topk(torch.zeros(0, 16, device="cuda"), ids[:0], vals[:0])
    assert loss.shape == (0,) and grad.shape == (0, 16)
