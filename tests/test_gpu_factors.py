"""cwl_orthogonalize and cwl_factor_step against their definitions in 64 bits.

Tolerances, entry by entry: the R x R polynomial Q is computed in 64 bits and rounded to fp32 (2^-24 of a number), its product
with U sums R terms in fp32 (2^-24 of the magnitudes summed, each), and the result is rounded to its own type; 2^-40 of the
magnitudes stands for the 64-bit part.  The momentum is one fused multiply-add (2^-24)."""
import pytest
import torch

from paper_2601_21109_b200 import binding as cwl

pytestmark = pytest.mark.gpu
ABC = cwl.NS_COEFFICIENTS


def factor(seed, rows, cols, dtype=torch.float32, spread=2.5, pad=0, offset=0):
    """A matrix of falling spectrum in a buffer of its own pitch, from an element on that may be unaligned."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    R = min(rows, cols)
    u = (torch.randn(rows, R, device="cuda", generator=gen) * torch.logspace(0, -spread, R, device="cuda")) @ \
        torch.randn(R, cols, device="cuda", generator=gen)
    buf = torch.full((rows * (cols + pad) + offset,), 7.0, dtype=dtype, device="cuda")
    out = buf[offset:].view(rows, cols + pad)[:, :cols]
    out.copy_(u)
    return out


def polynomial(u, steps, abc=ABC, eps=1e-7):
    """(Q, U with its short side first) in 64 bits, O = Q U."""
    x = u.double()
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    size = x.norm()
    unit = 0.0 if float(size) == 0 else 1.0 / (size + eps)
    g = (x @ x.T) * unit ** 2
    eye = torch.eye(len(g), dtype=torch.float64, device="cuda")
    q = eye.clone()
    for _ in range(steps):
        p = abc[0] * eye + abc[1] * g + abc[2] * g @ g
        q, g = p @ q, p @ g @ p
    return q * unit, x, tall


def reference(u, steps, abc=ABC, eps=1e-7):
    q, x, tall = polynomial(u, steps, abc, eps)
    o, tol = q @ x, ((len(q) + 2) * 2.0 ** -24 + 2.0 ** -40) * (q.abs() @ x.abs())
    return (o.T, tol.T) if tall else (o, tol)


def within(got, ref, tol, what=""):
    over = (got.double() - ref).abs() - tol * 1.01 - 1e-35
    assert bool(torch.isfinite(got).all()), f"{what}: not finite"
    assert float(over.max()) <= 0, f"{what}: over tolerance by {float(over.max()):.3e}"


HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SHAPES = [(1, 1), (1, 7), (9, 1), (2, 3), (16, 1024), (1024, 16), (8, 300), (33, 5001), (5001, 33), (64, 64), (64, 4096), (4096, 64), (63, 65),
          (65, 63), (65, 65), (65, 1000), (1000, 129), (128, 2048), (256, 256), (256, 3000), (11008, 256), (200, 4097)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype,out", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float32)])
def test_sizes_and_types(rows, cols, dtype, out):
    u = factor(rows + cols, rows, cols, dtype)
    o, = cwl.cwl_orthogonalize([u], out_dtype=out)
    ref, tol = reference(u, 5)
    within(o, ref, tol + ref.abs() * HALF[out])


@pytest.mark.parametrize("pad,offset", [(1, 0), (0, 1), (3, 2), (4, 4), (8, 0)])
@pytest.mark.parametrize("rows,cols", [(31, 210), (210, 31), (100, 300), (300, 100)])
def test_strides_and_offsets(rows, cols, pad, offset):
    for dtype in HALF:
        u = factor(5, rows, cols, dtype, pad=pad, offset=offset)
        out = torch.bfloat16 if dtype == torch.bfloat16 else torch.float32
        buf = torch.full((rows * (cols + pad) + offset,), 3.0, dtype=out, device="cuda")
        o = buf[offset:].view(rows, cols + pad)[:, :cols]
        cwl.cwl_orthogonalize([u], [o])
        ref, tol = reference(u, 5)
        within(o, ref, tol + ref.abs() * HALF[out])
        if pad:
            assert bool((buf[offset:].view(rows, cols + pad)[:, cols:] == 3.0).all())
        assert bool((buf[:offset] == 3.0).all())


@pytest.mark.parametrize("steps,abc,eps", [(1, ABC, 1e-7), (2, ABC, 0.0), (3, (1.5, -0.5, 0.0), 1e-7), (10, (3.0, -16 / 5, 6 / 5), 1e-3), (16, (1.875, -1.25, 0.375), 0.0)])
@pytest.mark.parametrize("rows,cols", [(40, 500), (500, 150)])
def test_steps_and_coefficients(steps, abc, eps, rows, cols):
    u = factor(3, rows, cols, spread=1.0)
    o, = cwl.cwl_orthogonalize([u], steps=steps, coefficients=abc, eps=eps)
    ref, tol = reference(u, steps, abc, eps)
    within(o, ref, tol + ref.abs() * 2.0 ** -24)


def test_singular_values_follow_the_scalar_iteration():
    """The classical cubic iteration towards the polar factor: singular vectors stay, singular values go through
    s -> 1.5 s - 0.5 s^3 one by one (those below 1.5^-16 have not arrived after 16 steps), which does not use the products at all."""
    for rows, cols in ((48, 700), (900, 100)):
        u = factor(4, rows, cols, spread=0.5)
        o, = cwl.cwl_orthogonalize([u], steps=16, coefficients=(1.5, -0.5, 0.0), eps=0.0)
        left, s, right = torch.linalg.svd(u.double(), full_matrices=False)
        s = s / s.norm()
        for _ in range(16):
            s = 1.5 * s - 0.5 * s ** 3
        assert float(s.max()) > 0.999
        assert float((o.double() - (left * s) @ right).norm()) <= 1e-5 * min(rows, cols) ** 0.5


@pytest.mark.parametrize("rows,cols", [(24, 333), (333, 24), (100, 400), (400, 100)])
def test_small_large_empty_and_deficient(rows, cols):
    u = factor(6, rows, cols, spread=1.0)
    for scale in (1e-30, 1e-18, 1e18, 1e36):
        x = u * scale
        o, = cwl.cwl_orthogonalize([x], eps=0.0)
        ref, tol = reference(x, 5, eps=0.0)
        within(o, ref, tol + ref.abs() * 2.0 ** -24, f"scale {scale}")
    for eps in (0.0, 1e-7):
        o, = cwl.cwl_orthogonalize([torch.zeros_like(u)], eps=eps)
        assert not bool(o.any())
    d = u.clone()
    d[::3] = 0
    d[:, 1::2] = d[:, :1]
    o, = cwl.cwl_orthogonalize([d])
    ref, tol = reference(d, 5)
    within(o, ref, tol + ref.abs() * 2.0 ** -24, "deficient")
    if rows < cols:
        assert not bool(o[::3].any())
    for bad in (float("nan"), float("inf")):
        d = u.clone()
        d[rows // 2, cols // 2] = bad
        good = u.clone()
        o, p = cwl.cwl_orthogonalize([d, good])
        assert bool(torch.isnan(o).all()) and bool(torch.isfinite(p).all())


def test_many_factors_in_a_call():
    """More than a launch's descriptors hold, of mixed sizes; every one as if it were alone, up to the order of 64-bit sums."""
    shapes = [(16 + 8 * (i % 9), 64 + 40 * (i % 13)) if i % 2 else (64 + 24 * (i % 17), 1 + i % 80) for i in range(600)]
    us = [factor(i, r, c) for i, (r, c) in enumerate(shapes)]
    os_ = cwl.cwl_orthogonalize(us)
    for i in range(0, 600, 7):
        ref, tol = reference(us[i], 5)
        within(os_[i], ref, tol + ref.abs() * 2.0 ** -24, str(shapes[i]))
    assert cwl.cwl_orthogonalize([]) == []


def step_operands(seed, rows, cols, dtype):
    g = factor(seed, rows, cols, dtype)
    m = factor(seed + 1, rows, cols) * 8
    p = torch.randn(rows, cols, device="cuda")
    return g, m, p, p.bfloat16()


def check_step(g, m, p, low, lr, beta, decay, nesterov, scale, run, steps=5):
    m0, p0 = m.clone(), p.clone()
    run()
    b = float(torch.tensor(beta, dtype=torch.float32))
    ref_m = b * m0.double() + g.double()
    within(m, ref_m, ref_m.abs() * 2.0 ** -24, "momentum")
    u = (g.double() + b * m.double()).float() if nesterov else m
    # a rounding of u that falls the other way (a tie after the rounding to 64 bits) moves O by less than what is allowed for Q
    ref, tol = reference(u, steps)
    keep = 1.0 - lr * decay
    ref_p = keep * p0.double() - lr * scale * ref
    tol_p = 1.01 * lr * scale * (tol + ref.abs() * 2.0 ** -23) + (p0.abs().double() + ref_p.abs()) * 2.0 ** -23
    within(p, ref_p, tol_p, "master")
    if low is not None:
        assert torch.equal(low, p.bfloat16())


@pytest.mark.parametrize("rows,cols", [(1, 1), (16, 1024), (1024, 16), (33, 501), (64, 4096), (4096, 64), (65, 640), (900, 200), (256, 2000)])
@pytest.mark.parametrize("dtype", list(HALF))
@pytest.mark.parametrize("nesterov", [True, False])
def test_step(rows, cols, dtype, nesterov):
    g, m, p, low = step_operands(rows, rows, cols, dtype)
    scale = max(1.0, rows / cols) ** 0.5
    call = cwl.FactorStep([p], [low], [g], [m])
    for _ in range(2):                                     # the second one on the first one's results
        check_step(g, m, p, low, 0.02, 0.95, 0.1, nesterov, scale, lambda: call(0.02, 0.95, 0.1, nesterov))


@pytest.mark.parametrize("rows,cols", [(31, 210), (210, 31), (100, 300), (300, 100)])
def test_step_with_strides(rows, cols):
    def view(dtype, offset):
        return torch.full((rows * (cols + 5) + offset,), 2.0, dtype=dtype, device="cuda")[offset:].view(rows, cols + 5)[:, :cols]
    g0, m0, p0, _ = step_operands(1, rows, cols, torch.float32)
    g, m, p, low = view(torch.bfloat16, 3), view(torch.float32, 1), view(torch.float32, 2), view(torch.bfloat16, 1)
    g.copy_(g0), m.copy_(m0), p.copy_(p0)
    call = cwl.FactorStep([p], [low], [g], [m], scales=[0.5])
    check_step(g, m, p, low, 0.05, 0.9, 0.0, True, 0.5, lambda: call(0.05, 0.9))
    for t in (g, m, p, low):
        assert bool((t.as_strided((rows, 5), (cols + 5, 1), t.storage_offset() + cols)[:-1] == 2.0).all())


def test_steps_of_many_factors_and_no_copies():
    shapes = [(64, 300), (300, 64), (100, 200), (7, 50)] * 120
    ops = [step_operands(i, r, c, torch.bfloat16) for i, (r, c) in enumerate(shapes)]
    gs, ms, ps, _ = map(list, zip(*ops))
    before = [(m.clone(), p.clone()) for m, p in zip(ms, ps)]
    cwl.FactorStep(ps, None, gs, ms)(0.1, 0.8, 0.0, False)
    for i in range(0, len(shapes), 11):
        m, p = before[i]
        g2, m2, p2 = gs[i], m.clone(), p.clone()
        check_step(g2, m2, p2, None, 0.1, 0.8, 0.0, False, max(1.0, p.shape[0] / p.shape[1]) ** 0.5,
                   lambda: cwl.FactorStep([p2], None, [g2], [m2])(0.1, 0.8, 0.0, False))
        assert torch.equal(ms[i], m2)
        ref, tol = reference(m2, 5)
        within(ps[i], p2.double(), 2.2 * 0.1 * max(1.0, p.shape[0] / p.shape[1]) ** 0.5 * tol + p2.abs().double() * 2.0 ** -22, "in company")


@pytest.mark.parametrize("rows,cols", [(64, 4096), (300, 100)])
def test_the_same_bits_again_on_another_stream_and_in_a_graph(rows, cols):
    u = factor(9, rows, cols)
    o = torch.empty_like(u)
    call = cwl.OrthogonalizeCall([u], [o])
    call()
    want = o.clone()
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    o.zero_()
    torch.cuda.synchronize()
    call(stream=other)
    other.synchronize()
    assert torch.equal(o, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want)
    u.copy_(factor(10, rows, cols))                        # new values in the same place
    graph.replay()
    torch.cuda.synchronize()
    ref, tol = reference(u, 5)
    within(o, ref, tol + ref.abs() * 2.0 ** -24)
