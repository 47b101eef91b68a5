"""Factors at the ends of fp32's range: O does not depend on how small or large they are, denormals and many steps included.

The reference and its tolerance (64 bits; Q and the product in fp32) are those of test_gpu_factors."""
import pytest
import torch

from paper_2601_21109_b200 import binding as cwl
from test_gpu_factors import ABC, factor, reference, within

pytestmark = pytest.mark.gpu
SCALES = [1e-42, 1e-39, 1e-37, 1e-33, 1e-12, 1e-9, 1e9, 1e12, 1e33, 1e37]
SHAPES = [(1, 5), (24, 333), (333, 24), (64, 64), (100, 400), (400, 100)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("steps,abc", [(5, ABC), (16, ABC), (1, ABC), (16, (1.5, -0.5, 0.0))])
def test_orthogonalize(rows, cols, scale, steps, abc):
    x = factor(6, rows, cols, spread=1.0) * scale
    assert bool(torch.isfinite(x).all()) and bool(x.any())
    o, plain = cwl.cwl_orthogonalize([x, factor(7, rows, cols)], steps=steps, coefficients=abc, eps=0.0)
    ref, tol = reference(x, steps, abc, 0.0)
    within(o, ref, tol + ref.abs() * 2.0 ** -24, f"scale {scale}")
    ref, tol = reference(factor(7, rows, cols), steps, abc, 0.0)
    within(plain, ref, tol + ref.abs() * 2.0 ** -24, "its neighbour")


@pytest.mark.parametrize("dtype,scale", [(torch.bfloat16, 1e-37), (torch.bfloat16, 1e37), (torch.float16, 1e-6), (torch.float16, 1e3)])
@pytest.mark.parametrize("rows,cols", [(24, 333), (333, 24), (100, 400), (401, 100), (399, 101)])
def test_short_types(dtype, scale, rows, cols):
    x = factor(6, rows, cols, dtype=torch.float32, spread=1.0).mul(scale).to(dtype)
    o, = cwl.cwl_orthogonalize([x], eps=0.0)
    ref, tol = reference(x, 5, eps=0.0)
    within(o, ref, tol + ref.abs() * 2.0 ** -24)


@pytest.mark.parametrize("rows,cols", [(24, 333), (333, 24), (100, 401), (400, 100)])
@pytest.mark.parametrize("scale", [1e-38, 1e-35, 1e36])
@pytest.mark.parametrize("nesterov", [True, False])
def test_step(rows, cols, scale, nesterov):
    """The master moves by the same O; the momentum keeps the gradient's own scale."""
    g, m, p = factor(1, rows, cols, spread=1.0) * scale, factor(2, rows, cols, spread=1.0) * scale, torch.randn(rows, cols, device="cuda")
    m0, p0 = m.clone(), p.clone()
    cwl.FactorStep([p], None, [g], [m], eps=0.0, scales=[0.5])(0.125, 0.5, 0.0, nesterov)
    assert torch.equal(m, torch.addcmul(g, torch.full_like(m0, 0.5), m0))           # a half is exact but for denormals' last bit
    u = g + 0.5 * m if nesterov else m
    ref, tol = reference(u, 5, eps=0.0)
    want = p0.double() - 0.0625 * ref
    within(p, want, 0.0625 * 1.01 * (tol + ref.abs() * 2.0 ** -23) + (p0.abs().double() + want.abs()) * 2.0 ** -23, "master")
