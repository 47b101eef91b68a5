"""cwl_apply_grads held to what its arithmetic loses as a whole, at every tile width: the norm of the error.

H' and G are pairs of bf16 numbers: 2^-16 of a number at most, of either sign.  The products' sums are kept in fp32, one addition
per 16 terms, of which each loses 2^-24 of the sum on average whichever way it rounds: (T + d) / 16 of them through both products.
A gradient rounded to bf16 adds half a spacing over sqrt 3, 2^-8 / sqrt 3.  (A pair's low half that went missing would show as
2^-9 / sqrt 3 = 1.1e-3, a block of 64 rows as sqrt(64 / T).)"""
import math

import pytest
import torch

from gpu_util import dev_table
from paper_2601_21109_b200 import binding as cwl
from test_gpu_grads import gate_of, operands, table

pytestmark = pytest.mark.gpu


def wide_tiles(T, d_in, d_out, R):
    """The library's rule for 256 columns of X / dY a block in the second product, as its comment states it."""
    if not 64 < R <= 128:
        return False
    tiles, blocks, split = -(-d_in // 256) - (-d_out // 256), -(-T // 64), 1
    while split < 8 and tiles * split * 2 <= 148 and (blocks // (split * 2) >= 4):
        split *= 2
    return tiles * split >= 96 and blocks // split >= 16


@pytest.mark.parametrize("T,d_in,d_out,R,wide", [
    (4133, 10128, 4240, 80, True), (8200, 4096, 3856, 128, True), (2100, 6416, 6400, 96, True), (4096, 4096, 11008, 112, True),
    (1500, 14096, 11008, 80, True), (4133, 1040, 1024, 80, False), (4100, 4096, 4096, 64, False), (3000, 2064, 4096, 16, False),
    (5000, 4112, 2048, 144, False), (2500, 1024, 3600, 256, False)])
def test_norm_of_the_error(T, d_in, d_out, R, wide):
    assert wide_tiles(T, d_in, d_out, R) == wide
    X, dY, A, B = operands(T + R, T, d_in, d_out, R)
    tab = table(T, T, R, 96, seqs=3)
    g = torch.from_numpy(gate_of(tab, T, R, 8)).cuda()
    x, dy, a, b = (t.double() for t in (X, dY, A, B))
    rA, rB = x.T @ (g * (dy @ b.T)), (g * (x @ a)).T @ dy
    for dtype, rounding in ((torch.float32, 0.0), (torch.bfloat16, 2.0 ** -8 / math.sqrt(3))):
        dA, dB = cwl.cwl_apply_grads(X, dY, A, B, dev_table(tab), 8, grad_dtype=dtype)
        for got, ref, d in ((dA, rA, d_out), (dB, rB, d_in)):
            assert float((got.double() - ref).norm() / ref.norm()) <= 2.0 ** -16 + (T + d) / 16 * 2.0 ** -24 + rounding
            # column by column of R too: a rung's factors by themselves
            by_rank = (got.double() - ref).norm(dim=0) / ref.norm(dim=0).clamp(min=1e-30) if ref.shape[1] == R else \
                (got.double() - ref).norm(dim=1) / ref.norm(dim=1).clamp(min=1e-30)
            assert float(by_rank.max()) <= 2 * (2.0 ** -16 + (T + d) / 16 * 2.0 ** -24) + rounding
