"""Matrices whose rows, columns or elements differ by orders of magnitude, on the GPU against 64 bits: the whole result, every row and
every column.

How far a result may be off follows from how the kernels hold numbers.  An operand's number is moved by at most 2^-22 of itself (two fp16
numbers of 11 bits), or by 2^-36 in scaled units (half of fp16's smallest number, over 2048); the scale puts the largest singular value
that the coefficients allow between 2^14 and 2^15, so that is 2^-50 of this bound.  A product leaves out lo lo, 2^-22 of each term, and adds up in
fp32.  The partial sums of that can be as large as the sum S of the terms' magnitudes, however small the result: a s + b s^3 + c s^5 is 3.4 - 4.8 + 2.0
at s = 1, and a goes into the sum at once where the others come in over the whole contraction.  n / 16 additions, each off by at most 2^-24 S, come to
(n / 16 / 3)^(1/2) 2^-24 S where they are independent: 2^-22 S for n = 768.  The 64-bit reference is run again with random errors of that size, number by number, in
the products that the kernels make (two steps at once: G P, P G P, P' P), and a result may be off by eight times what they do, row by row.
Where a row is one large number among small ones, its error in one such run is one random number, which may be small by chance: the size
is the root of the mean square over eight runs, which is below a quarter of its expectation once in 7500 (chi-square, 8 degrees of freedom)."""
import pytest
import torch

import matrix_reference as R
from test_gpu_orthogonalize import B, ws_for  # noqa: F401 (B is a fixture)

pytestmark = pytest.mark.gpu
A, B_, C = R.USUAL[0]
MOST_X, MOST_G, MOST_P = 1.2023, 1.4455, 3.4446                # of the usual coefficients: singular values stay below, P(0) = a

# one workgroup a matrix (and at the end of that), single steps, pairs of steps, either orientation
SHAPES = [(64, 64), (48, 341), (341, 48), (97, 97), (300, 300), (512, 1024), (1024, 512), (520, 4160), (4160, 520)]


def badly_scaled(rows, cols, kind, ratio):
    g = torch.Generator(device="cuda").manual_seed(rows + 3 * cols)
    x = torch.randn(rows, cols, generator=g, device="cuda")
    small = x * ratio
    if kind == "element":
        small[3, 5] = 32.0
    elif kind == "row":
        small[3] = x[3]
    elif kind == "column":
        small[:, 5] = x[:, 5]
    elif kind == "graded rows":
        small = x * ratio ** torch.linspace(0, 1, rows, device="cuda")[:, None]
    elif kind == "block":
        small[:rows // 2, :cols // 2] = x[:rows // 2, :cols // 2]
    return small


def newton_schulz(x, steps, moved=None, pairs=False):
    """moved: the number of a run with errors, None for none."""
    g = torch.Generator(device="cuda").manual_seed(moved or 0)
    X = x / x.norm()
    X = X.T.contiguous() if X.shape[0] > X.shape[1] else X

    def noise(like):
        return torch.randn(like.shape, generator=g, device="cuda", dtype=torch.float64)

    def times(a, b, most_a, most_b):
        if moved is not None:
            a, b = a + 2.0 ** -50 * most_a * noise(a), b + 2.0 ** -50 * most_b * noise(b)
        c = a @ b
        if moved is not None:
            c = c + 2.0 ** -22 * (noise(c) * ((a * a) @ (b * b)).sqrt() + noise(c) * (a.abs() @ b.abs()))
        return c

    def polynomial(G):
        P = B_ * G + C * times(G, G, MOST_G, MOST_G)
        P.diagonal().add_(A)
        return P

    alone = 2 * ((steps // 2 + 1) // 2) if pairs and steps % 2 else steps
    i = 0
    while i < steps:
        pair = pairs and i != alone
        P, most = polynomial(G := times(X, X.T.contiguous(), MOST_X, MOST_X)), MOST_P
        if pair:
            G = times(times(G, P, MOST_G, MOST_P), P, MOST_G, MOST_P)
            P, most = times(polynomial(G), P, MOST_P, MOST_P), MOST_P ** 2
        X = times(P, X, most, MOST_X)
        i += 2 if pair else 1
    return X.T if x.shape[0] > x.shape[1] else X


def moved_by(x, steps, want, pairs=False):
    """Mean square of what the errors do to each number, over eight runs."""
    return sum((newton_schulz(x, steps, run, pairs) - want).square() for run in range(8)) / 8


@pytest.mark.parametrize("steps", [5, 10])
@pytest.mark.parametrize("ratio", [1e-2, 1e-4, 1e-6, 1e-8, 1e-10])
@pytest.mark.parametrize("kind", ["element", "row", "column", "graded rows", "block"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_every_row_and_column(B, rows, cols, kind, ratio, steps):  # noqa: F811
    x = badly_scaled(rows, cols, kind, ratio)
    out = torch.full_like(x, 5.0)
    B.qesgd_orthogonalize(x, rows, cols, 1, R.USUAL[:1] * steps, 0.0, out, ws_for(B, rows, cols, 1))
    want = newton_schulz(x.double(), steps)
    moved = moved_by(x.double(), steps, want, pairs=max(rows, cols) == 4160)
    off = out.double() - want
    for what, dim in (("whole", (0, 1)), ("rows", 1), ("columns", 0)):
        size = want.norm(dim=dim)
        limit = 8 * (moved.sum(dim=dim).sqrt() + 2.0 ** -22 * size)
        worst = off.norm(dim=dim) / limit
        print("%s: off %.1e, at most %.2g of what is allowed" % (what, float((off.norm(dim=dim) / size).max()), float(worst.max())))
        assert bool((worst <= 1).all()), what


def test_momentum_and_batches(B):  # noqa: F811
    """The update on three matrices, one of them badly scaled: its small rows come out as from that matrix alone."""
    for rows, cols in ((64, 64), (300, 517)):
        g = torch.stack([badly_scaled(rows, cols, "row", r) for r in (1.0, 1e-6, 1e-3)])
        m, step = torch.zeros_like(g), torch.empty_like(g)
        B.qesgd_orthogonal_update(g, rows, cols, 3, m, 0.5, True, R.USUAL, 0.0, 1.0, step, None, None, None, None, ws_for(B, rows, cols, 3))
        for i in range(3):
            want = newton_schulz(g[i].double(), 5)             # g + mu m = 1.5 g: the same matrix after its norm
            limit = 8 * (moved_by(g[i].double(), 5, want).sum(dim=1).sqrt() + 2.0 ** -22 * want.norm(dim=1))
            assert bool(((step[i].double() - want).norm(dim=1) <= limit).all()), i
