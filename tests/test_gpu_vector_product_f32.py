"""Products of single rows of 16 bits with results in fp32: nothing of the sums is rounded away, in one launch and in pieces."""
import numpy as np
import pytest
import torch

import expert_reference as X
from expert_reference import ONE, host
from test_gpu_grouped import ints, packed_noise
from test_gpu_vector_product import rows

pytestmark = pytest.mark.gpu
HALVES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def B():
    from paper_1901_03040_amd import binding
    assert torch.cuda.is_available()
    binding.lib()
    return binding


@pytest.mark.parametrize("t", HALVES, ids=["bf16", "f16"])
@pytest.mark.parametrize("n,N,K,E", [(1, 1, 1, 1), (1, 130, 384, 1), (1, 1000, 2049, 1), (6, 40, 1000, 1), (16, 512, 512, 1), (40, 30, 128, 1), (33, 141, 513, 5), (100, 64, 2049, 9),
                                     (16, 4100, 5000, 1), (33, 5000, 9000, 1), (7, 100, 70_000, 3)])
def test_against_64_bits(B, n, N, K, E, t):
    rng = np.random.default_rng(n + N)
    pw, w = packed_noise(B, N, K, E, n + N + K)
    x, pw = rows(n, K, t, N), pw.cuda()
    offsets = [0, n] if E == 1 else X.group_sizes(rng, E, n, "ragged")
    ws = B.alloc_workspace(B.qesgd_mx4_vector_product_workspace_bytes(n, N, K, E))
    y = torch.full((n * (N + 3) + 1,), 3.0, device="cuda")
    B.qesgd_mx4_vector_product(x.cuda(), K, n, None, 1, pw, pw.stride(0), None if E == 1 else ints(offsets), E, n, N, K, y[1:], N + 3, workspace=ws)
    narrow = torch.full((n, N + 3), 3.0, dtype=t, device="cuda")
    B.qesgd_mx4_vector_product(x.cuda(), K, n, None, 1, pw, pw.stride(0), None if E == 1 else ints(offsets), E, n, N, K, narrow, N + 3, workspace=ws)
    got = torch.as_strided(y, (n, N + 3), (N + 3, 1), 1)
    assert torch.equal(got.to(t), narrow)                       # the results of 16 bits are these, rounded
    got = host(got)
    assert y[0] == 3.0 and (got[:, N:] == 3.0).all() and (got[:offsets[0]] == 3.0).all() and (got[offsets[-1]:] == 3.0).all()
    x64 = host(x)
    for e in range(E):
        s = slice(offsets[e], offsets[e + 1])
        # at most two exact products of each element and as many additions in any order, the parts' sums added
        limit = (2 * K + 2) * ONE * (np.abs(x64[s]) @ np.abs(w[e]).T)
        assert (np.abs(got[s, :N] - x64[s] @ w[e].T) <= limit).all(), e


def test_types_that_are_refused(B):
    pw = packed_noise(B, 16, 32, 1, 1)[0].cuda()
    for x, y in ((torch.float32, torch.bfloat16), (torch.bfloat16, torch.float16), (torch.float16, torch.bfloat16), (torch.bfloat16, torch.float64), (torch.int16, torch.float32)):
        a, c = torch.zeros(2, 32, dtype=x, device="cuda"), torch.zeros(2, 16, dtype=y, device="cuda")
        with pytest.raises(B.QesgdError):
            B.qesgd_mx4_vector_product(a, 32, 2, None, 1, pw, 0, None, 1, 2, 16, 32, c, 16)
