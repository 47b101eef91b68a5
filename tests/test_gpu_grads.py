"""cwl_apply_grads against its definition in 64 bits and against differences of the projection.

Tolerances, entry by entry, from the arithmetic: H' and G are rounded to bf16 (half a spacing, 2^-8 relative) after an fp32
sum of d products (2^-23 d of the sum of their magnitudes, however the products cancel); the fold sums T products of them
in fp32 (2^-23 T of the magnitudes); the result is rounded to its own type (2^-8 or 2^-24 relative)."""
import numpy as np
import pytest
import torch

from gpu_util import dev_table
from paper_2601_21109_b200 import binding as cwl

pytestmark = pytest.mark.gpu


def table(seed, T, R, chunk, first=0, last=None, seqs=1):
    """Chunks of about `chunk` rows covering [first, last), ranks from 0 to R, `seqs` sequences."""
    rng = np.random.default_rng(seed)
    last = T if last is None else last
    cuts, t = [first], first
    while last - t > chunk:
        t += int(rng.integers(max(1, chunk // 2), chunk + 1))
        cuts.append(t)
    n = len(cuts)
    flags = np.zeros(n, np.int32)
    flags[0] = 1
    for s in range(1, seqs):
        flags[s * n // seqs] = 1
    return dict(offsets=np.array(cuts + [last], np.int32), rank=rng.choice([0, max(1, R // 4), R // 2, R], n).astype(np.int32),
                scale=rng.uniform(0.25, 4.0, n).astype(np.float32), flags=flags, rung=np.zeros(n, np.int32), n_chunks=n)


def gate_of(tab, T, R, window, centred=False):
    g = np.zeros((T, R))
    off, rank, scale, flags, C = tab["offsets"], tab["rank"], tab["scale"].astype(np.float64), tab["flags"], tab["n_chunks"]
    before = window // 2
    after = window - before
    for c in range(C):
        for t in range(off[c], off[c + 1]):
            j, length = t - off[c], off[c + 1] - off[c]
            lam, cin, cout = 1.0, c, c
            if centred:
                if c > 0 and not flags[c] & 1 and j < after:
                    lam, cout = (before + j + 1) / (window + 1), c - 1
                elif c + 1 < C and not flags[c + 1] & 1 and length - j <= before:
                    lam, cin = (before - (length - j) + 1) / (window + 1), c + 1
            elif c > 0 and not flags[c] & 1 and j < window:
                lam, cout = (j + 1) / (window + 1), c - 1
            g[t, :rank[cin]] += lam * scale[cin]
            if lam < 1:
                g[t, :rank[cout]] += (1 - lam) * scale[cout]
    return g


def operands(seed, T, d_in, d_out, R, pad=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def m(r, c, std):
        buf = torch.full((r, c + pad), 9.0, dtype=torch.bfloat16, device="cuda")
        buf[:, :c].copy_(torch.randn(r, c, device="cuda", generator=gen) * std)
        return buf[:, :c]
    return m(T, d_in, 1.0), m(T, d_out, 0.5), m(d_in, R, d_in ** -0.5), m(R, d_out, R ** -0.5)


def check(X, dY, A, B, tab, window, centred=False, **kw):
    T, d_in = X.shape
    d_out, R = dY.shape[1], A.shape[1]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dA, dB = cwl.cwl_apply_grads(X, dY, A, B, dev_table(tab), window, centred=centred, status_word=status, **kw)
    assert int(status.item()) == 0
    g = torch.from_numpy(gate_of(tab, T, R, window, centred)).cuda()
    x, dy, a, b = (t.double() for t in (X, dY, A, B))
    H, G = g * (x @ a), g * (dy @ b.T)
    u = 2.0 ** -23
    errH = H.abs() * 2.0 ** -8 + g * d_in * u * (x.abs() @ a.abs())
    errG = G.abs() * 2.0 ** -8 + g * d_out * u * (dy.abs() @ b.abs().T)
    out = 2.0 ** -8 if dA.dtype == torch.bfloat16 else 2.0 ** -24
    for got, ref, tol, what in ((dA, x.T @ G, x.abs().T @ (errG + T * u * G.abs()), "dA"),
                                (dB, H.T @ dy, (errH + T * u * H.abs()).T @ dy.abs(), "dB")):
        over = (got.double() - ref).abs() - (tol * 1.01 + ref.abs() * out + 1e-30)
        assert bool(torch.isfinite(got).all()) and float(over.max()) <= 0, f"{what}: over tolerance by {float(over.max()):.3e}"
    return dA, dB


@pytest.mark.parametrize("T,d_in,d_out,R,chunk,window", [
    (256, 1024, 1024, 16, 32, 4), (1, 64, 64, 16, 32, 4), (2, 16, 16, 16, 8, 0), (37, 144, 80, 32, 8, 8), (129, 336, 1040, 48, 40, 8),
    (300, 512, 320, 64, 50, 8), (1000, 4096, 256, 64, 96, 8), (513, 272, 4112, 128, 64, 3), (700, 1024, 2064, 256, 100, 8),
    (65, 640, 640, 240, 30, 5), (2048, 4096, 4096, 64, 96, 8), (5000, 256, 512, 144, 200, 8)])
def test_sizes(T, d_in, d_out, R, chunk, window):
    X, dY, A, B = operands(T + R, T, d_in, d_out, R)
    tab = table(T, T, R, chunk, seqs=3 if T > 100 else 1)
    check(X, dY, A, B, tab, window)
    check(X, dY, A, B, tab, window, grad_dtype=torch.float32)


@pytest.mark.parametrize("T,d_in,d_out,R,chunk,window", [
    (8256, 3600, 4112, 48, 300, 8), (2050, 12304, 13328, 16, 100, 4), (8200, 4096, 3856, 128, 200, 8), (4133, 10128, 4240, 80, 64, 8),
    (16384, 2064, 2048, 32, 500, 6)])
def test_many_rows(T, d_in, d_out, R, chunk, window):
    X, dY, A, B = operands(T + R, T, d_in, d_out, R)
    tab = table(T, T, R, chunk, seqs=3)
    check(X, dY, A, B, tab, window)
    check(X, dY, A, B, tab, window, grad_dtype=torch.float32)


@pytest.mark.parametrize("T,d_in,d_out,R", [(300, 512, 320, 64), (777, 256, 1040, 144), (129, 1024, 640, 16), (2000, 272, 512, 256)])
def test_fp32_gradients_carry_more_than_bf16(T, d_in, d_out, R):
    """H' and G are kept as two bf16 numbers: what they lose is 2^-17 of a number (half of the low one's spacing), so an fp32
    gradient is within 2^-16 of the magnitudes that it sums, beside the fp32 sums themselves."""
    X, dY, A, B = operands(T, T, d_in, d_out, R)
    tab = table(T, T, R, 40)
    dA, dB = cwl.cwl_apply_grads(X, dY, A, B, dev_table(tab), 4, grad_dtype=torch.float32)
    g = torch.from_numpy(gate_of(tab, T, R, 4)).cuda()
    x, dy, a, b = (t.double() for t in (X, dY, A, B))
    H, G = g * (x @ a), g * (dy @ b.T)
    u = 2.0 ** -23
    for got, ref, tol in ((dA, x.T @ G, x.abs().T @ (G.abs() * (2.0 ** -16 + T * u) + g * d_out * u * (dy.abs() @ b.abs().T))),
                          (dB, H.T @ dy, (H.abs() * (2.0 ** -16 + T * u) + g * d_in * u * (x.abs() @ a.abs())).T @ dy.abs())):
        assert float(((got.double() - ref).abs() - tol - ref.abs() * 2.0 ** -23).max()) <= 0


@pytest.mark.parametrize("window", [0, 1, 7, 8])
def test_centred_windows(window):
    X, dY, A, B = operands(3, 400, 256, 320, 64)
    check(X, dY, A, B, table(3, 400, 64, 30, seqs=2), window, centred=True)


def test_matrices_with_a_pitch_and_guards():
    T, d_in, d_out, R = 333, 272, 208, 48
    X, dY, A, B = operands(9, T, d_in, d_out, R, pad=24)
    for dt in (torch.bfloat16, torch.float32):
        ga = torch.full((d_in + 3, R + 8), float("nan"), dtype=dt, device="cuda")
        gb = torch.full((R + 3, d_out + 8), float("nan"), dtype=dt, device="cuda")
        check(X, dY, A, B, table(9, T, R, 40), 4, dA=ga[:d_in, :R], dB=gb[:R, :d_out])
        assert bool(torch.isnan(ga[d_in:]).all()) and bool(torch.isnan(ga[:, R:]).all())
        assert bool(torch.isnan(gb[R:]).all()) and bool(torch.isnan(gb[:, d_out:]).all())


def test_rows_outside_every_chunk_and_empty_tables():
    T, d, R = 500, 256, 32
    X, dY, A, B = operands(4, T, d, d, R)
    check(X, dY, A, B, table(4, T, R, 40, first=70, last=333), 4)
    empty = dict(offsets=np.zeros(1, np.int32), rank=np.zeros(0, np.int32), scale=np.zeros(0, np.float32), flags=np.zeros(0, np.int32),
                 rung=np.zeros(0, np.int32), n_chunks=0)
    dA, dB = cwl.cwl_apply_grads(X, dY, A, B, dev_table(empty), 4)
    assert not bool(dA.any()) and not bool(dB.any())
    none = torch.full((d, R), 5.0, dtype=torch.bfloat16, device="cuda")
    dA, dB = cwl.cwl_apply_grads(X[:0], dY[:0], A, B, dev_table(empty), 4, dA=none)
    assert not bool(dA.any()) and not bool(dB.any())


def test_against_differences_of_the_projection():
    """The projection is linear in A and in B, so a central difference of <Y, dY> in 64 bits is the derivative itself."""
    T, d_in, d_out, R, window = 60, 48, 64, 16, 4
    X, dY, A, B = operands(6, T, d_in, d_out, R)
    tab = table(6, T, R, 12)
    dA, dB = check(X, dY, A, B, tab, window, grad_dtype=torch.float32)
    g = torch.from_numpy(gate_of(tab, T, R, window)).cuda()
    x, dy, a, b = (t.double() for t in (X, dY, A, B))

    def value(aa, bb):
        return float((((g * (x @ aa)) @ bb) * dy).sum())
    scale_a, scale_b = float(dA.abs().max()), float(dB.abs().max())
    rng = np.random.default_rng(0)
    for _ in range(20):
        i, j, k, n = (int(rng.integers(0, m)) for m in (d_in, R, R, d_out))
        e = torch.zeros_like(a)
        e[i, j] = 0.5
        assert abs(value(a + e, b) - value(a - e, b) - float(dA[i, j])) <= 2.0 ** -7 * scale_a
        e = torch.zeros_like(b)
        e[k, n] = 0.5
        assert abs(value(a, b + e) - value(a, b - e) - float(dB[k, n])) <= 2.0 ** -7 * scale_b


def test_gradient_of_the_input_is_the_projection_on_transposed_factors():
    T, d_in, d_out, R = 300, 256, 512, 32
    X, dY, A, B = operands(12, T, d_in, d_out, R)
    W = (torch.randn(d_in, d_out, device="cuda") * d_in ** -0.5).bfloat16()
    tab = table(12, T, R, 40)
    dX = cwl.cwl_apply(dY.contiguous(), W.t().contiguous(), B.t().contiguous(), A.t().contiguous(), dev_table(tab), 4)
    g = torch.from_numpy(gate_of(tab, T, R, 4)).cuda()
    ref = dY.double() @ W.double().T + (g * (dY.double() @ B.double().T)) @ A.double().T
    assert float((dX.double() - ref).norm() / ref.norm()) <= 1e-2


def test_same_bits_again_on_another_stream_and_in_a_graph():
    T, d_in, d_out, R = 900, 1024, 768, 64
    X, dY, A, B = operands(5, T, d_in, d_out, R)
    tab = dev_table(table(5, T, R, 70))
    ws = torch.empty(cwl.cwl_apply_grads_workspace_bytes(T, d_in, d_out, R), dtype=torch.uint8, device="cuda")
    ws.fill_(255)
    dA, dB = cwl.cwl_apply_grads(X, dY, A, B, tab, 8, workspace=ws)
    ws.random_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        eA, eB = cwl.cwl_apply_grads(X, dY, A, B, tab, 8, workspace=ws)
    side.synchronize()
    assert torch.equal(dA, eA) and torch.equal(dB, eB)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cwl.cwl_apply_grads(X, dY, A, B, tab, 8, dA=eA, dB=eB, workspace=ws)
    eA.zero_(), eB.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(dA, eA) and torch.equal(dB, eB)


def test_refusals():
    X, dY, A, B = operands(1, 32, 64, 64, 16)
    tab = dev_table(table(1, 32, 16, 8))

    def status(**kw):
        with pytest.raises(cwl.CwlError) as e:
            cwl.cwl_apply_grads(kw.pop("X", X), kw.pop("dY", dY), kw.pop("A", A), kw.pop("B", B), kw.pop("tab", tab), kw.pop("window", 4), **kw)
        return e.value.status
    assert status(window=-1) == 1
    assert status(workspace=torch.empty(64, dtype=torch.uint8, device="cuda")) == 5
    assert status(grad_dtype=torch.float16) == 1
    assert status(X=torch.zeros(32, 72, dtype=torch.bfloat16, device="cuda"), A=torch.zeros(72, 16, dtype=torch.bfloat16, device="cuda")) == 3
    assert status(A=torch.zeros(64, 8, dtype=torch.bfloat16, device="cuda"), B=torch.zeros(8, 64, dtype=torch.bfloat16, device="cuda")) == 3
    assert status(A=torch.zeros(64, 272, dtype=torch.bfloat16, device="cuda"), B=torch.zeros(272, 64, dtype=torch.bfloat16, device="cuda")) == 3
    wide = torch.zeros(32, 65, dtype=torch.bfloat16, device="cuda")
    assert status(X=wide[:, :64]) == 2 and status(X=wide.view(-1)[1:1 + 32 * 64].view(32, 64)) == 2
    with pytest.raises(AssertionError):
        cwl.cwl_apply_grads(X, dY[:16], A, B, tab, 4)
    with pytest.raises(AssertionError):
        cwl.cwl_apply_grads(X.float(), dY, A, B, tab, 4)
