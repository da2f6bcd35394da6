"""Coefficients that take singular values and polynomials far from 1, on the GPU against the 64-bit reference.

The limit is that of the ordinary coefficients (see test_gpu_orthogonalize.py): the reference run again with random errors of the split
products' size.  It is relative to what goes into a product, so it holds wherever the operands' scales fit what they hold: singular
values of the iterates up to 2^7 and values of the polynomials up to 2^18, which is what these cases stay within on these matrices."""
import numpy as np
import pytest
import torch

import matrix_reference as R
from test_gpu_orthogonalize import B, allowed, matrices, ws_for  # noqa: F401 (B is a fixture)

pytestmark = pytest.mark.gpu

# one workgroup a matrix, single steps, pairs of steps (520 x 4160 and its transpose)
SHAPES = [(40, 60), (300, 300), (200, 333), (520, 2080), (2080, 520), (520, 4160), (4160, 520)]
COEFFS = {
    "polynomials whose product is 400": ((20.0, 0.0, 0.0),) * 2,
    "polynomials whose product is 400 at zero": ((20.0, -30.0, 12.0), (20.0, -0.1, 0.0)),
    "growing iterates": ((10.0, 0.0, 0.0),) * 3,
    "growing iterates with all terms": ((30.0, -20.0, 4.0), (3.0, 0.01, 1e-6), (2.0, -1e-4, 1e-9)),
    "large polynomials of small iterates": ((1e-4, 0.0, 0.0), (1e5, -3e12, 2e20), (1.5, -0.5, 0.0)),
    "shrinking iterates": ((1e-3, 0.0, 0.0),) * 4,
    "only the last term": ((0.0, 0.0, 1e3), (1.5, -0.5, 0.0)),
    # polynomials that a singular value of 1 would take to 1e5 or 1e6, and those of these matrices, 0.06 .. 0.27, do not
    "spread 1": ((4.3, 0.0, 3.65), (5.02, -8.38, 8.65), (9.57, -14.08, 3.88)),
    "spread 2": ((2.6175, 1.3031, 8.6122), (-3.9471, 2.0601, 2.0932), (1.5754, -4.4213, 17.619)),
    "spread 3": ((5.1162, -18.353, 0.1407), (3.0831, -17.024, 7.2357), (8.4672, -20.598, 10.514)),
    "spread 4": ((3.2826, 6.3356, -2.6979), (9.4196, 1.318, 4.8708), (3.5985, -8.075, 0.1589)),
    "zero": ((0.0, 0.0, 0.0),) * 2,
}


@pytest.mark.parametrize("which", list(COEFFS))
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_the_range_follows_the_coefficients(B, rows, cols, which):  # noqa: F811
    co = tuple(tuple(float(np.float32(v)) for v in c) for c in COEFFS[which])
    x = matrices(1, rows, cols, "plain", rows + cols)
    out = torch.full_like(x, 5.0).cuda()
    B.qesgd_orthogonalize(x.cuda(), rows, cols, 1, co, 0.0, out, ws_for(B, rows, cols, 1))
    got, x64 = out.double().cpu().numpy()[0], x.double().numpy()[0]
    want = R.newton_schulz(x64, co, 0.0)
    off, limit = np.linalg.norm(got - want), allowed(x64, want, co, 2.0 ** -24, 0.0)
    print(which, rows, cols, "size %.2g off %.2g allowed %.2g" % (np.linalg.norm(want), off, limit))
    assert off <= limit


def test_a_scale_that_no_coefficient_moves(B):  # noqa: F811
    """Powers of two in the coefficients: p(2^k X) scaled back is the same polynomial, so the results are the same bits."""
    for rows, cols in SHAPES:
        x = matrices(1, rows, cols, "plain", 3).cuda()
        ws = ws_for(B, rows, cols, 1)
        want, got = torch.empty_like(x), torch.empty_like(x)
        a, b, c = 3.0, -3.5, 1.25
        B.qesgd_orthogonalize(x, rows, cols, 1, ((1.0, 0.0, 0.0), (a, b, c), (a, b, c)), 0.0, want, ws)
        for k in (-9, -3, 7):
            s = 2.0 ** k
            B.qesgd_orthogonalize(x, rows, cols, 1, ((s, 0.0, 0.0), (a / s, b / s ** 3, c / s ** 5), (a, b, c)), 0.0, got, ws)
            assert torch.equal(got, want), (rows, cols, k)
