"""Captured graphs, NaN, zeros and extreme magnitudes on the kernels that only larger shapes reach: the 4-bit product with its contraction in
pieces, and the orthogonalisation as separate launches (single steps, pairs of steps, pieces)."""
import numpy as np
import pytest
import torch

import matrix_reference as R
from test_gpu_mx4 import B, host, matrix, product_limit  # noqa: F401 (B is a fixture)
from test_gpu_orthogonalize import EPS, HALF_STEP, allowed, matrices, ws_for

pytestmark = pytest.mark.gpu
PIECES = [(300, 40, 8200), (512, 1000, 25_088), (1, 1000, 25_088)]


def quantised(B, x, seed=0, mode=None):  # noqa: F811
    r, c = x.shape
    p = B.alloc_mx4(B.qesgd_mx4_layout_query(r, c))
    B.qesgd_mx4_quantize_pack(x, c, 0, r, c, 1, B.MX4_NEAREST if mode is None else mode, seed, 0, p, 0)
    return p


@pytest.mark.parametrize("M,N,K", PIECES)
def test_a_product_in_pieces_from_graphs_that_share_its_workspace(B, M, N, K):  # noqa: F811
    need = B.qesgd_mx4_product_workspace_bytes(M, N, K)
    assert need > 0
    x, w = matrix(M, K, torch.bfloat16, 1).cuda(), matrix(N, K, torch.bfloat16, 2).cuda()
    px, pw, ws = quantised(B, x), quantised(B, w), B.alloc_workspace(need + 256).fill_(0xFF)
    y, y2 = (torch.zeros(M, N, device="cuda", dtype=torch.bfloat16) for _ in range(2))

    def work(a, to):
        B.qesgd_mx4_product(a, pw, M, N, K, to, N, workspace=ws[:need])

    other = quantised(B, x.flip(1).contiguous())
    work(px, y)
    work(other, y2)
    torch.cuda.synchronize()
    want, want2 = y.clone(), y2.clone()
    code, scale = R.quantize(host(x))
    a = R.values(code, scale, K)
    code, scale = R.quantize(host(w))
    b = R.values(code, scale, K)
    assert (np.abs(host(want) - a @ b.T) <= product_limit(a, b, a @ b.T, torch.bfloat16)).all()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for g, args in zip(graphs, ((px, y), (other, y2))):
        with torch.cuda.graph(g):
            work(*args)
    for i in range(6):
        y.zero_()
        y2.zero_()
        ws[:need].fill_(0xFF)                                   # NaN: nothing of an earlier call is read
        graphs[i & 1].replay()
        graphs[1 - (i & 1)].replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(y2, want2), i
        assert bool((ws[need:] == 0xFF).all())
        assert np.isfinite(torch.randn(1 << 16, device="cuda").sum().item())


@pytest.mark.parametrize("M,N,K", PIECES)
def test_nan_stays_in_its_row_of_a_product_in_pieces(B, M, N, K):  # noqa: F811
    need = B.qesgd_mx4_product_workspace_bytes(M, N, K)
    assert need > 0
    for at in (3, K // 2, K - 1):                               # in the first, a middle and the last piece
        x, w = matrix(M, K, torch.float32, 1, False), matrix(N, K, torch.float32, 2, False)
        x[M // 2, at] = float("nan")
        w[5, K - 1 - at] = float("inf")
        c = torch.empty(M, N, device="cuda")
        B.qesgd_mx4_product(quantised(B, x.cuda()), quantised(B, w.cuda()), M, N, K, c, N, workspace=B.alloc_workspace(need))
        want = torch.zeros(M, N, dtype=torch.bool)
        want[M // 2] = True
        want[:, 5] = True
        assert torch.equal(torch.isnan(c).cpu(), want), at


GENERAL = [(300, 200), (200, 900), (97, 97), (520, 4160), (1040, 130)]


@pytest.mark.parametrize("dtype,size", [("f32", 1e-42), ("f32", 1e-30), ("f32", 1e30), ("bf16", 1e-38), ("bf16", 1e-30), ("bf16", 1e30), ("f16", 2e-7), ("f16", 1e4)])
@pytest.mark.parametrize("rows,cols", GENERAL)
def test_magnitudes_whose_squares_leave_the_type(B, rows, cols, dtype, size):  # noqa: F811
    """The norm is taken in 64 bits.  eps = 0, so that it does not swallow the smallest."""
    assert ws_for(B, rows, cols, 1) is not None
    t = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    x = (matrices(1, rows, cols, "plain", 3).double() * size).to(t)
    assert bool(torch.isfinite(x).all()) and bool(x.any())
    out = torch.empty_like(x).cuda()
    B.qesgd_orthogonalize(x.cuda(), rows, cols, 1, R.USUAL, 0.0, out, ws_for(B, rows, cols, 1))
    x64 = x[0].double().numpy()
    want = R.newton_schulz(x64, R.USUAL, 0.0)
    # fp16: half of its smallest number for every one that is below its normal range
    limit = allowed(x64, want, R.USUAL, HALF_STEP[dtype], 0.0) + ((rows * cols) ** 0.5 * 2.0 ** -25 if dtype == "f16" else 0.0)
    assert np.linalg.norm(out[0].double().cpu().numpy() - want) <= limit


@pytest.mark.parametrize("momentum", [False, True])
@pytest.mark.parametrize("size", [1e-42, 1e-30, 1e30])
@pytest.mark.parametrize("rows,cols", GENERAL[:2])
def test_updates_of_such_magnitudes(B, rows, cols, size, momentum):  # noqa: F811
    x = (matrices(1, rows, cols, "plain", 3).double() * size).float()
    m = torch.zeros_like(x).cuda() if momentum else None
    step = torch.empty_like(x).cuda()
    B.qesgd_orthogonal_update(x.cuda(), rows, cols, 1, m, 0.5, True, R.USUAL, 0.0, 1.0, step, None, None, None, None, ws_for(B, rows, cols, 1))
    x64 = ((x + np.float32(0.5) * x) if momentum else x)[0].double().numpy()
    want = R.newton_schulz(x64, R.USUAL, 0.0)
    assert np.linalg.norm(step[0].double().cpu().numpy() - want) <= allowed(x64, want, R.USUAL, 2.0 ** -24, 0.0)
    assert m is None or torch.equal(m.cpu(), x)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols", GENERAL)
def test_zeros_give_zeros_and_nan_stays_in_its_matrix(B, rows, cols, dtype):  # noqa: F811
    x = matrices(3, rows, cols, "plain", 1).to(dtype)
    x[0] = 0.0
    x[1, rows // 2, cols - 1] = float("nan")
    for eps in (0.0, EPS):
        out = torch.full((3, rows, cols), 9.0, device="cuda", dtype=dtype)
        B.qesgd_orthogonalize(x.cuda(), rows, cols, 3, R.USUAL, eps, out, ws_for(B, rows, cols, 3))
        assert (out[0] == 0).all()
        assert torch.isnan(out[1]).all()
        again = x.clone()
        again[1] = 1.0                                          # the others' results have nothing to do with it
        clean = torch.empty_like(out)
        B.qesgd_orthogonalize(again.cuda(), rows, cols, 3, R.USUAL, eps, clean, ws_for(B, rows, cols, 3))
        assert torch.equal(clean[2], out[2]) and torch.equal(clean[0], out[0])


@pytest.mark.parametrize("n,rows,cols", [(1, 33, 480), (4, 40, 450), (1, 90, 417), (2, 300, 290), (1, 257, 161)])
def test_short_pieces_and_contractions(B, n, rows, cols):  # noqa: F811
    """X X^T over 15, 14, 10 and 6 steps of 32, in pieces of three where it is cut up, and products of m x m matrices over 2 to 10."""
    assert ws_for(B, rows, cols, n) is not None
    x = matrices(n, rows, cols, "decay", rows)
    out = torch.full((n, rows, cols), 9.0, device="cuda")
    B.qesgd_orthogonalize(x.cuda(), rows, cols, n, R.USUAL, EPS, out, ws_for(B, rows, cols, n))
    for i in range(n):
        x64 = x[i].double().numpy()
        want = R.newton_schulz(x64)
        assert np.linalg.norm(out[i].double().cpu().numpy() - want) <= allowed(x64, want, R.USUAL, 2.0 ** -24), i
