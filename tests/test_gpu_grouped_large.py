"""Grouped products that are large enough for workgroups with several tiles one after the other, and for streaming stores, against 64 bits."""
import numpy as np
import pytest
import torch

import expert_reference as X
from expert_reference import ONE, TYPES
from test_gpu_grouped import ints, packed_noise

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_1901_03040_amd import binding
    assert torch.cuda.is_available()
    binding.lib()
    return binding


def within(got, a, b, dtype):
    """got = a b^T: n exact products added in fp32 in any order, one rounding.  a [M, n] and b [N, n] in 64 bits on the GPU."""
    want, size = a @ b.T, a.abs() @ b.abs().T
    limit = a.shape[1] * ONE * size + X.HALF_STEP[dtype] * want.abs() * (1 + 2.0 ** -10) + X.LEAST[dtype]
    off = (got.double() - want).abs() - limit
    return bool((off <= 0).all())


def on_gpu(v):
    return torch.from_numpy(v).cuda()


# steps of the contraction: one half, one, two with a half, an odd number, many
@pytest.mark.parametrize("kind", ["ragged", "even", "one", "none"])
@pytest.mark.parametrize("n,N,K,E", [(10_000, 4100, 100, 5), (9000, 4100, 250, 3), (10_000, 4096, 300, 70), (12_000, 3900, 700, 2), (17_000, 2060, 1100, 4)])
def test_product(B, n, N, K, E, kind):
    dtype = list(TYPES.values())[(n + K) % 3]
    offsets = X.group_sizes(np.random.default_rng(K), E, n, kind)
    pa, a = packed_noise(B, n, K, 1, n + K)
    pb, b = packed_noise(B, N, K, E, N + 2 * K)
    pa, pb, a = pa[0].cuda(), pb.cuda(), on_gpu(a[0])
    ws = B.alloc_workspace(B.qesgd_mx4_grouped_product_workspace_bytes(n, N, K, E))
    out = []
    for _ in range(2):
        c = torch.full((n, N), 3.0, dtype=dtype, device="cuda")
        B.qesgd_mx4_grouped_product(pa, pb, pb.stride(0), ints(offsets), E, n, N, K, c, N, workspace=ws)
        out.append(c)
    assert torch.equal(*out)
    assert (c[offsets[-1]:] == 3.0).all() and (c[:offsets[0]] == 3.0).all()
    for e in range(E):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        assert within(c[lo:hi], a[lo:hi], on_gpu(b[e]), dtype), e


@pytest.mark.parametrize("kind", ["ragged", "even", "one", "none"])
@pytest.mark.parametrize("n,N,K,E", [(1500, 3000, 2000, 7), (700, 2500, 2310, 9), (300, 1030, 1000, 40), (9000, 4096, 2300, 4)])
def test_gradient(B, n, N, K, E, kind):
    dtype = list(TYPES.values())[(n + N) % 3]
    offsets = X.group_sizes(np.random.default_rng(K), E, n, kind)
    columns = X.group_columns(n, E)
    pa, a = packed_noise(B, N, columns, 1, n + K)
    pb, b = packed_noise(B, K, columns, 1, N + 2 * K)
    pa, pb, a, b = pa[0].cuda(), pb[0].cuda(), on_gpu(a[0]), on_gpu(b[0])
    ws = B.alloc_workspace(B.qesgd_mx4_grouped_gradient_workspace_bytes(n, N, K, E))
    out = []
    for _ in range(2):
        d = torch.full((E, N, K), 3.0, dtype=dtype, device="cuda")
        B.qesgd_mx4_grouped_gradient(pa, pb, ints(offsets), E, n, N, K, d, workspace=ws)
        out.append(d)
    assert torch.equal(*out)
    at = 0
    for e in range(E):
        wide = int(offsets[e + 1] - offsets[e] + 127) // 128 * 128
        assert within(d[e], a[:, at:at + wide], b[:, at:at + wide], dtype), e
        at += wide


@pytest.mark.parametrize("dtype", list(TYPES))
def test_streamed_results(B, dtype):
    """Results of 192 MiB and more, in whole lines and with rows that are none."""
    t = TYPES[dtype]
    size = torch.empty((), dtype=t).element_size()
    E, K = 3, 128
    for N in (8192, 8200):
        n = (200 << 20) // (N * size) + 77
        offsets = X.group_sizes(np.random.default_rng(N), E, n, "ragged")
        pa, a = packed_noise(B, n, K, 1, n)
        pb, b = packed_noise(B, N, K, E, N)
        c = torch.full((n, N), 3.0, dtype=t, device="cuda")
        B.qesgd_mx4_grouped_product(pa[0].cuda(), pb.cuda(), pb.shape[1], ints(offsets), E, n, N, K, c, N)
        a = on_gpu(a[0])
        assert (c[offsets[-1]:] == 3.0).all()
        for e in range(E):
            lo, hi = int(offsets[e]), int(offsets[e + 1])
            assert within(c[lo:hi], a[lo:hi], on_gpu(b[e]), t), (N, e)
        del c
    # gradients: enough experts for as much
    N, K, n = 1024, 1024, 500
    E = (200 << 20) // (N * K * size) + 1
    offsets, columns = X.group_sizes(np.random.default_rng(1), E, n, "ragged"), X.group_columns(n, E)
    pa, a = packed_noise(B, N, columns, 1, 5)
    pb, b = packed_noise(B, K, columns, 1, 6)
    d = torch.full((E, N, K), 3.0, dtype=t, device="cuda")
    B.qesgd_mx4_grouped_gradient(pa[0].cuda(), pb[0].cuda(), ints(offsets), E, n, N, K, d)
    a, b, at = on_gpu(a[0]), on_gpu(b[0]), 0
    for e in range(E):
        wide = int(offsets[e + 1] - offsets[e] + 127) // 128 * 128
        assert within(d[e], a[:, at:at + wide], b[:, at:at + wide], t), e
        at += wide


@pytest.mark.parametrize("dtype", list(TYPES))
def test_weighted_sum_of_many_rows(B, dtype):
    """Calls that stream: rows of more than the memory-side cache, tokens of 128 MiB and more; and rows that are no whole lines."""
    t = TYPES[dtype]
    size = torch.empty((), dtype=t).element_size()
    for N, k in ((4096, 2), (4100, 2), (512, 1)):
        T = (300 << 20) // (N * size * k) + 5
        n = T * k
        g = torch.Generator(device="cuda").manual_seed(N)
        rows, dy = torch.randn(n, N, generator=g, device="cuda").to(t), torch.randn(T, N, generator=g, device="cuda").to(t)
        gates = torch.rand(T, k, generator=g, device="cuda")
        slots = torch.randperm(n, generator=g, device="cuda").int()
        slots[::13] = -1
        out, drows, dgates = torch.empty_like(dy), torch.full_like(rows, 9.0), torch.empty_like(gates)
        B.qesgd_combine(rows, N, n, slots, gates, T, k, N, out, N)
        B.qesgd_combine_backward(dy, N, rows, N, n, slots, gates, T, k, N, drows, N, dgates)
        s, half, least = slots.reshape(T, k).long(), X.HALF_STEP[t], X.LEAST[t]
        touched = torch.zeros(n, dtype=torch.bool, device="cuda")
        for t0 in range(0, T, 8192):
            p = slice(t0, min(T, t0 + 8192))
            want = torch.zeros(s[p].shape[0], N, dtype=torch.float64, device="cuda")
            mag = torch.zeros_like(want)
            for j in range(k):
                there = s[p, j] >= 0
                r = rows[s[p, j].clamp(min=0)].double() * there[:, None]
                w, d = gates[p, j:j + 1].double(), dy[p].double()
                want += w * r
                mag += (w * r).abs()
                dot, dmag = (r * d).sum(1), (r * d).abs().sum(1)
                assert ((dgates[p, j].double() - dot).abs() <= (N + 1) * ONE * dmag).all()
                at = s[p, j][there]
                v = (w * d)[there]
                assert ((drows[at].double() - v).abs() <= (half + ONE) * v.abs() * (1 + 2.0 ** -10) + least).all()
                touched[at] = True
            assert ((out[p].double() - want).abs() <= (k + 1) * ONE * mag + half * want.abs() * (1 + 2.0 ** -10) + least).all()
        assert (drows[~touched] == 9.0).all()


@pytest.mark.parametrize("kind", ["ragged", "even", "one", "none"])
@pytest.mark.parametrize("n,N,K,E", [(64, 512, 8192, 8), (5, 33, 9000, 2), (300, 64, 4100, 4), (1, 4096, 4096, 1), (90, 131, 12_345, 3), (40, 60, 2900, 30)])
def test_long_contractions_in_pieces(B, n, N, K, E, kind):
    need = B.qesgd_mx4_grouped_product_workspace_bytes(n, N, K, E)
    assert need > 0 and need % (4 * n * N) == 0
    dtype = list(TYPES.values())[(n + K) % 3]
    offsets = X.group_sizes(np.random.default_rng(K), E, n, kind)
    pa, a = packed_noise(B, n, K, 1, n + K)
    pb, b = packed_noise(B, N, K, E, N + 2 * K)
    pa, pb, a, ldc = pa[0].cuda(), pb.cuda(), on_gpu(a[0]), N + 3
    ws = torch.full((need + 256,), 0x7F, dtype=torch.uint8, device="cuda")
    out = []
    for _ in range(2):
        c = torch.full((n, ldc), 3.0, dtype=dtype, device="cuda")
        B.qesgd_mx4_grouped_product(pa, pb, pb.stride(0), ints(offsets), E, n, N, K, c, ldc, workspace=ws[:need])
        out.append(c)
    assert torch.equal(*out) and (ws[need:] == 0x7F).all()
    assert (c[offsets[-1]:] == 3.0).all() and (c[:offsets[0]] == 3.0).all() and (c[:, N:] == 3.0).all()
    for e in range(E):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        assert within(c[lo:hi, :N], a[lo:hi], on_gpu(b[e]), dtype), e
    with pytest.raises(B.QesgdError):
        B.qesgd_mx4_grouped_product(pa, pb, pb.stride(0), ints(offsets), E, n, N, K, c, ldc, workspace=ws[:need - 1])


@pytest.mark.parametrize("kind", ["ragged", "even", "one", "none"])
@pytest.mark.parametrize("n,N,K,E", [(20_000, 64, 64, 1), (30_000, 100, 41, 2), (60_000, 256, 131, 3), (16_384, 33, 64, 4)])
def test_gradients_of_long_groups_in_pieces(B, n, N, K, E, kind):
    need = B.qesgd_mx4_grouped_gradient_workspace_bytes(n, N, K, E)
    assert need > 0 and need % (4 * E * N * K) == 0
    dtype = list(TYPES.values())[(n + K) % 3]
    offsets = X.group_sizes(np.random.default_rng(K), E, n, kind)
    columns = X.group_columns(n, E)
    pa, a = packed_noise(B, N, columns, 1, n + K)
    pb, b = packed_noise(B, K, columns, 1, N + 2 * K)
    pa, pb, a, b = pa[0].cuda(), pb[0].cuda(), on_gpu(a[0]), on_gpu(b[0])
    ws = torch.full((need + 256,), 0x7F, dtype=torch.uint8, device="cuda")
    out = []
    for _ in range(2):
        d = torch.full((E * N * K + 64,), 3.0, dtype=dtype, device="cuda")
        B.qesgd_mx4_grouped_gradient(pa, pb, ints(offsets), E, n, N, K, d, workspace=ws[:need])
        out.append(d)
    assert torch.equal(*out) and (d[E * N * K:] == 3.0).all() and (ws[need:] == 0x7F).all()
    at, got = 0, d[:E * N * K].view(E, N, K)
    for e in range(E):
        wide = int(offsets[e + 1] - offsets[e] + 127) // 128 * 128
        assert within(got[e], a[:, at:at + wide], b[:, at:at + wide], dtype), e
        at += wide


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("n,N,K,E", [(3000, 555, 1088, 13), (400, 2300, 1408, 4), (9000, 4100, 960, 3)])
def test_gradients_in_whole_lines(B, n, N, K, E, dtype):
    """Results of 12 MB and more whose rows are whole lines, in 64 to 256 rows and columns a tile, the last ones short."""
    t, offsets, columns = TYPES[dtype], X.group_sizes(np.random.default_rng(K), E, n, "ragged"), X.group_columns(n, E)
    pa, a = packed_noise(B, N, columns, 1, n + K)
    pb, b = packed_noise(B, K, columns, 1, N + 2 * K)
    a, b = on_gpu(a[0]), on_gpu(b[0])
    ws = B.alloc_workspace(B.qesgd_mx4_grouped_gradient_workspace_bytes(n, N, K, E))
    d = torch.full((E * N * K + 640,), 3.0, dtype=t, device="cuda")
    B.qesgd_mx4_grouped_gradient(pa[0].cuda(), pb[0].cuda(), ints(offsets), E, n, N, K, d[:E * N * K], workspace=ws)
    assert (d[E * N * K:] == 3.0).all()
    d, at = d[:E * N * K].view(E, N, K), 0
    for e in range(E):
        wide = int(offsets[e + 1] - offsets[e] + 127) // 128 * 128
        assert within(d[e], a[:, at:at + wide], b[:, at:at + wide], t), e
        at += wide


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("N", [63, 65, 126, 130, 253, 254, 255, 1021, 1022, 1025])
def test_rows_that_do_not_end_with_four_columns(B, N, dtype):
    """Every rest of four, rows that begin at any element, and what lies between them left as it was; tiles of 64, 128 and 256."""
    t = TYPES[dtype]
    for n, K, E in ((150, 200, 3), (1500, 700, 4), (9000, 300, 5)):
        offsets = X.group_sizes(np.random.default_rng(N), E, n, "ragged")
        pa, a = packed_noise(B, n, K, 1, n + K)
        pb, b = packed_noise(B, N, K, E, N + 2 * K)
        pb, a = pb.cuda(), on_gpu(a[0])
        ldc = N + 3
        c = torch.full((n * ldc + 7,), 3.0, dtype=t, device="cuda")
        ws = B.alloc_workspace(B.qesgd_mx4_grouped_product_workspace_bytes(n, N, K, E))
        B.qesgd_mx4_grouped_product(pa[0].cuda(), pb, pb.stride(0), ints(offsets), E, n, N, K, c[1:], ldc, workspace=ws)
        rows = torch.as_strided(c, (n, ldc), (ldc, 1), 1)
        assert c[0] == 3.0 and (rows[:, N:] == 3.0).all() and (c[n * ldc + 1:] == 3.0).all()
        assert (rows[offsets[-1]:] == 3.0).all() and (rows[:offsets[0]] == 3.0).all()
        for e in range(E):
            lo, hi = int(offsets[e]), int(offsets[e + 1])
            assert within(rows[lo:hi, :N], a[lo:hi], on_gpu(b[e]), t), (n, e)


def test_pieces_in_graphs_and_on_two_streams(B):
    """Calls of two launches, each with a workspace of its own, captured and run side by side: every replay gives what a call alone gives."""
    E, n, N, K = 2, 64, 300, 9000
    o, far = ints([0, 30, n]), ints([0, 7000, 16_384])
    a, w = packed_noise(B, n, K, 1, 1)[0][0].cuda(), packed_noise(B, N, K, E, 2)[0].cuda()
    columns = X.group_columns(16_384, E)
    ga, gb = packed_noise(B, 64, columns, 1, 3)[0][0].cuda(), packed_noise(B, 41, columns, 1, 4)[0][0].cuda()
    x = torch.randn(n, K, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()

    def job():
        out = [torch.zeros(n, N, device="cuda"), torch.zeros(E, 64, 41, device="cuda"), torch.zeros(n, N, dtype=torch.bfloat16, device="cuda")]
        sizes = [B.qesgd_mx4_grouped_product_workspace_bytes(n, N, K, E), B.qesgd_mx4_grouped_gradient_workspace_bytes(16_384, 64, 41, E),
                 B.qesgd_mx4_vector_product_workspace_bytes(n, N, K, E)]
        ws = [B.alloc_workspace(s) for s in sizes]

        def run():
            B.qesgd_mx4_grouped_product(a, w, w.stride(0), o, E, n, N, K, out[0], N, workspace=ws[0])
            B.qesgd_mx4_grouped_gradient(ga, gb, far, E, 16_384, 64, 41, out[1], workspace=ws[1])
            B.qesgd_mx4_vector_product(x, K, n, None, 1, w, w.stride(0), o, E, n, N, K, out[2], N, workspace=ws[2])
        return out, run, sizes

    jobs = [job() for _ in range(2)]
    assert jobs[0][2][0] > 0 and jobs[0][2][1] > 0
    jobs[0][1]()
    torch.cuda.synchronize()
    want = [t.clone() for t in jobs[0][0]]
    assert all(t.any() for t in want)
    streams, graphs = [torch.cuda.Stream() for _ in jobs], []
    for (out, run, _), s in zip(jobs, streams):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            run()
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            run()
        graphs.append(g)
    for turn in range(5):
        for out, _, _ in jobs:
            for t in out:
                t.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                for _ in range(3):
                    g.replay()
        torch.cuda.synchronize()
        for out, _, _ in jobs:
            assert all(torch.equal(t, v) for t, v in zip(out, want)), turn
        jobs[turn % 2][1]()                                    # the program's own calls between the replays
        assert all(torch.equal(t, v) for t, v in zip(jobs[turn % 2][0], want)), turn
