"""Products of single rows whose contraction is cut into pieces (two launches and a workspace): captured, on two streams, and beside the program's own calls."""
import pytest
import torch

from test_gpu_grouped import ints, packed_noise

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_1901_03040_amd import binding
    assert torch.cuda.is_available()
    binding.lib()
    return binding


SIZES = [(16, 4100, 5000, 1), (33, 5000, 9000, 1), (7, 100, 70_000, 3)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,N,K,E", SIZES)
def test_in_graphs_and_on_two_streams(B, n, N, K, E, dtype):
    """Each job has a workspace of its own; every replay gives what a call alone gives, also where its workspace held something else before."""
    need = B.qesgd_mx4_vector_product_workspace_bytes(n, N, K, E)
    assert need > 0
    w = packed_noise(B, N, K, E, 2)[0].cuda()
    x = torch.randn(n, K, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    offsets = None if E == 1 else ints([0, 2, 2, n])

    def job():
        y, ws = torch.zeros(n, N, dtype=dtype, device="cuda"), B.alloc_workspace(need)

        def run():
            B.qesgd_mx4_vector_product(x, K, n, None, 1, w, w.stride(0), offsets, E, n, N, K, y, N, workspace=ws)
        return y, ws, run

    jobs = [job() for _ in range(2)]
    jobs[0][2]()
    torch.cuda.synchronize()
    want = jobs[0][0].clone()
    assert want.any()
    streams, graphs = [torch.cuda.Stream() for _ in jobs], []
    for (_, _, run), s in zip(jobs, streams):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            run()
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            run()
        graphs.append(g)
    for turn in range(4):
        for y, ws, _ in jobs:
            y.zero_()
            ws.fill_(0xFF)                                      # NaN
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                for _ in range(3):
                    g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(y, want) for y, _, _ in jobs), turn
        # the pieces' sums were there: rows of 16 bits of the first size fit one launch's memory whole
        assert all(bool((ws != 0xFF).any()) for _, ws, _ in jobs) or (K == 5000 and dtype != torch.float32), turn
        jobs[turn % 2][2]()                                     # the program's own call between the replays
        assert torch.equal(jobs[turn % 2][0], want), turn
