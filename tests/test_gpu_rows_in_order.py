"""Rows that lie in the groups' order already (order None): row r is row r of x, whatever `per` says of the pairs that an order would hold."""
import numpy as np
import pytest
import torch

from expert_reference import TYPES
from test_gpu_grouped import ints, packed_noise, tokens

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_1901_03040_amd import binding
    assert torch.cuda.is_available()
    binding.lib()
    return binding


@pytest.mark.parametrize("per", [2, 3, 7, 1 << 20])
@pytest.mark.parametrize("mode", [0, 1], ids=["nearest", "stochastic"])
@pytest.mark.parametrize("T", [150, 40], ids=["all rows", "rows beyond x"])
def test_packing(B, T, mode, per):
    n, cols, E = 150, 200, 4
    x, offsets = tokens(T, cols, torch.bfloat16, 1).cuda(), ints([0, 30, 31, 100, n])
    lay, lay_t = B.qesgd_mx4_layout_query(n, cols), B.qesgd_mx4_layout_query(cols, B.qesgd_mx4_grouped_columns(n, E))
    for rows, columns in ((True, False), (False, True), (True, True)):
        out = []
        for number in (1, per):
            p, pt = (B.alloc_mx4(v).fill_(0xA5) for v in (lay, lay_t))
            B.qesgd_mx4_quantize_groups(x, cols, T, None, number, offsets, E, n, cols, mode, 5, 6, p if rows else None, packed_t=pt if columns else None)
            out.append((p, pt))
        assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1]), (rows, columns)


@pytest.mark.parametrize("per", [2, 3, 7, 1 << 20])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_single_rows(B, dtype, per):
    n, N, K = 12, 100, 300
    x = tokens(n, K, TYPES[dtype], 2).cuda()
    for E, offsets in ((1, None), (3, ints([0, 5, 5, n]))):
        w = packed_noise(B, N, K, E, 3)[0].cuda()
        ws = B.alloc_workspace(B.qesgd_mx4_vector_product_workspace_bytes(n, N, K, E))
        out = []
        for number in (1, per):
            y = torch.zeros(n, N, dtype=TYPES[dtype], device="cuda")
            B.qesgd_mx4_vector_product(x, K, n, None, number, w, w.stride(0), offsets, E, n, N, K, y, N, workspace=ws)
            out.append(y)
        assert out[0].any() and torch.equal(*out)


def test_an_order_is_still_divided(B):
    """The same rows by an order of pairs, three to a token, and without one."""
    T, k, cols, E = 30, 3, 130, 2
    x, offsets = tokens(T, cols, torch.float32, 4).cuda(), ints([0, 40, T * k])
    order = np.random.default_rng(1).permutation(T * k)
    picked = x[torch.from_numpy(order // k).cuda()]
    lay, out = B.qesgd_mx4_layout_query(T * k, cols), []
    for src, rows, by in ((x, T, ints(order)), (picked, T * k, None)):
        p = B.alloc_mx4(lay).zero_()
        B.qesgd_mx4_quantize_groups(src, cols, rows, by, k, offsets, E, T * k, cols, B.MX4_NEAREST, 0, 0, p)
        out.append(p)
    assert torch.equal(*out)
