"""Products of single rows with packed 4-bit matrices on the GPU against the 64-bit reference."""
import numpy as np
import pytest
import torch

import expert_reference as X
from expert_reference import ONE, TYPES, host
from test_gpu_grouped import ints, packed_noise

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_1901_03040_amd import binding
    assert torch.cuda.is_available()
    binding.lib()
    return binding


def rows(T, K, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(T, K, generator=g) * torch.exp2(torch.randint(-6, 3, (T, 1), generator=g).float())).to(dtype)


def limit(x, w, want, dtype):
    """At most three exact products of each element and as many additions in fp32 in any order, the parts' sums added: (3 K + 2) 2^-24 of the sum of
    the products' magnitudes (the parts of an element have its sign, so their magnitudes add up to its own); then one rounding."""
    return (3 * x.shape[1] + 2) * ONE * (np.abs(x) @ np.abs(w).T) + X.rounded(want, dtype)


ONE_MATRIX = [(1, 1, 1), (1, 16, 32), (1, 130, 384), (1, 1000, 2049), (2, 33, 129), (5, 65, 640), (6, 40, 1000), (8, 257, 130), (9, 48, 8200), (16, 512, 512),
              (17, 100, 257), (40, 30, 128), (1, 20, 30_000), (16, 64, 5000), (3, 4100, 96)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("n,N,K", ONE_MATRIX)
def test_one_matrix(B, n, N, K, dtype):
    t = TYPES[dtype]
    pw, w = packed_noise(B, N, K, 1, n + N + K)
    ld, ldy = K + 3, N + 5
    base = torch.full((n * ld + 9,), float("nan"), dtype=t)    # what lies between the rows is not read
    x = rows(n, K, t, N)
    torch.as_strided(base, (n, K), (ld, 1), 1).copy_(x)
    base, out = base.cuda(), []
    for _ in range(2):
        y = torch.full((n, ldy), 3.0, dtype=t, device="cuda")
        B.qesgd_mx4_vector_product(base[1:], ld, n, None, 1, pw.cuda(), 0, None, 1, n, N, K, y, ldy,
                                   workspace=B.alloc_workspace(B.qesgd_mx4_vector_product_workspace_bytes(n, N, K, 1)))
        out.append(y)
    assert torch.equal(*out)
    got = host(out[0])
    want = host(x) @ w[0].T
    off = np.abs(got[:, :N] - want) - limit(host(x), w[0], want, t)
    assert (got[:, N:] == 3.0).all()
    assert (off <= 0).all(), np.argwhere(off > 0)[:4]


EXPERTS = [(1, 2, 3, 20, 40), (4, 2, 8, 130, 300), (12, 4, 64, 141, 513), (16, 8, 9, 64, 2049), (50, 1, 3, 33, 1000), (7, 3, 200, 48, 96), (30, 2, 2, 515, 4100)]


@pytest.mark.parametrize("kind", ["ragged", "even", "one", "none"])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T,k,E,N,K", EXPERTS)
def test_rows_of_experts(B, T, k, E, N, K, dtype, kind):
    t, n = TYPES[dtype], T * k
    rng = np.random.default_rng(T + K)
    offsets, order = X.group_sizes(rng, E, n, kind), rng.permutation(n)
    if n > 10:
        order[::7] = -1
        order[3] = T * k + 9
    pw, w = packed_noise(B, N, K, E, N)
    slab = torch.zeros(E, pw.shape[1] + 256, dtype=torch.uint8)
    slab[:, :pw.shape[1]] = pw
    x = rows(T, K, t, 5)
    y = torch.full((n, N), 3.0, dtype=t, device="cuda")
    slab = slab.cuda()
    B.qesgd_mx4_vector_product(x.cuda(), K, T, ints(order), k, slab, slab.stride(0), ints(offsets), E, n, N, K, y, N,
                               workspace=B.alloc_workspace(B.qesgd_mx4_vector_product_workspace_bytes(n, N, K, E)))
    got = host(y)
    source = np.where(order < 0, T, np.minimum(order // k, T))
    picked = np.concatenate((host(x), np.zeros((1, K))))[source]
    assert (got[offsets[-1]:] == 3.0).all() and (got[:offsets[0]] == 3.0).all()
    for e in range(E):
        lo, hi = offsets[e], offsets[e + 1]
        want = picked[lo:hi] @ w[e].T
        off = np.abs(got[lo:hi] - want) - limit(picked[lo:hi], w[e], want, t)
        assert (off <= 0).all(), (e, np.argwhere(off > 0)[:4])


def test_every_code_and_scale(B):
    """One row picks out each element in turn: all 16 codes with all 256 scales.  255 marks a NaN; 253 and 254 are not the format's (its largest
    exponent is 125): their largest elements, 4 * 2^126 and more, are beyond fp32's and bf16's range, infinities, and zero times an infinity is NaN."""
    N, K = 256, 32
    lay = B.qesgd_mx4_layout_query(N, K)
    p = torch.zeros(lay.bytes, dtype=torch.uint8)
    codes = p.numpy()[:N * lay.row_codes].reshape(N, -1)
    codes[:, :8] = [0x10, 0x32, 0x54, 0x76, 0x98, 0xBA, 0xDC, 0xFE]
    p.numpy()[lay.scales_off:lay.scales_off + N * lay.row_scales].reshape(N, -1)[:, 0] = np.arange(256)
    grid = np.array([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6])
    want = grid[None, :] * np.ldexp(1.0, np.arange(256) - 127)[:, None]
    for t in TYPES.values():
        x = torch.eye(16, K).to(t).cuda()
        y = torch.empty(16, N, dtype=t, device="cuda")
        B.qesgd_mx4_vector_product(x, K, 16, None, 1, p.cuda(), 0, None, 1, 16, N, K, y, N)
        got = host(y).T
        assert np.isnan(got[255]).all()
        with np.errstate(over="ignore"):
            ref = torch.from_numpy(want[:253]).to(torch.float32).to(t).double().numpy()
        # below the least normal number of bf16 an element counts as itself or as zero
        small = np.abs(want[:253]) < 2.0 ** -126
        assert np.array_equal(got[:253][~small], ref[~small])
        assert ((got[:253][small] == ref[small]) | (got[:253][small] == 0)).all()


@pytest.mark.parametrize("dtype", list(TYPES))
def test_infinities_and_nan_stay_in_their_row(B, dtype):
    t, K, N = TYPES[dtype], 200, 40
    pw, w = packed_noise(B, N, K, 1, 3)
    x = rows(6, K, t, 1)
    x[1, 150], x[3, 2], x[4, 199] = float("nan"), float("inf"), -float("inf")
    x[5] = torch.finfo(t).max
    y = torch.empty(6, N, dtype=torch.float32 if t == torch.float32 else t, device="cuda")
    B.qesgd_mx4_vector_product(x.cuda(), K, 6, None, 1, pw.cuda(), 0, None, 1, 6, N, K, y, N)
    got = host(y)
    clean = host(x)
    with np.errstate(invalid="ignore"):
        want = np.stack([(clean[i] * w[0]).sum(1) for i in range(6)])     # 0 times infinity is NaN
    assert np.isnan(got[1]).all()
    assert np.array_equal(np.isnan(got[3:5]), np.isnan(want[3:5])) and np.array_equal(np.isposinf(got[3:5]), np.isposinf(want[3:5]))
    for i in (0, 2):
        assert (np.abs(got[i] - want[i]) <= limit(clean[i:i + 1], w[0], want[i:i + 1], t)[0]).all()


def test_small_and_large_numbers_of_f32(B):
    """Three parts hold a number of fp32 whole, whatever its size, down to where the last one's exponent ends."""
    K, N = 128, 16
    lay = B.qesgd_mx4_layout_query(N, K)
    p = torch.zeros(lay.bytes, dtype=torch.uint8)
    p[:N * lay.row_codes] = 0x22                                # ones
    p[lay.scales_off:lay.scales_off + N * lay.row_scales] = 127
    g = torch.Generator().manual_seed(1)
    x = torch.zeros(13, K)
    for i in range(13):
        x[i, i] = (1 + torch.rand(1, generator=g)).float() * 2.0 ** (-102 + 17 * i)
    y = torch.empty(13, N, device="cuda")
    B.qesgd_mx4_vector_product(x.cuda(), K, 13, None, 1, p.cuda(), 0, None, 1, 13, N, K, y, N)
    want = x.sum(1)
    # the parts' sums are added in fp32, the smaller ones first: two roundings
    assert (torch.abs(y[:, 0].cpu().double() - want.double()) <= 2 * ONE * want.double()).all()


def test_graph_and_side_stream(B):
    T, k, E, N, K = 4, 2, 16, 300, 700
    n = T * k
    rng = np.random.default_rng(1)
    offsets, order = ints(X.group_sizes(rng, E, n, "ragged")), ints(rng.permutation(n))
    pw, _ = packed_noise(B, N, K, E, 9)
    w, x = pw.cuda(), rows(T, K, torch.bfloat16, 2).cuda()
    y = torch.zeros(n, N, dtype=torch.bfloat16, device="cuda")
    ws = B.alloc_workspace(B.qesgd_mx4_vector_product_workspace_bytes(n, N, K, E))

    def work():
        B.qesgd_mx4_vector_product(x, K, T, order, k, w, w.stride(0), offsets, E, n, N, K, y, N, workspace=ws)

    work()
    torch.cuda.synchronize()
    want = y.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        work()
    side.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for i in range(3):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), i
        assert np.isfinite(torch.randn(1 << 16, device="cuda").sum().item())


LONG = [(16, 1000, 8192, 1), (16, 4096, 4096, 1), (40, 70, 9000, 1), (16, 33, 6001, 3), (64, 512, 5000, 2),
        (16, 4100, 5000, 1), (2, 30, 50_001, 1), (33, 5000, 9000, 1), (4, 20, 40_000, 2), (7, 100, 70_000, 3), (64, 4096, 4096, 1)]
PIECES = LONG[5:]


@pytest.mark.parametrize("n,N,K,E", PIECES)
def test_long_rows_need_room_for_their_pieces(B, n, N, K, E):
    need = B.qesgd_mx4_vector_product_workspace_bytes(n, N, K, E)
    assert need >= 2 * 4 * n * N and need % (4 * n * N) == 0


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("n,N,K,E", LONG)
def test_long_rows_in_pieces(B, n, N, K, E, dtype):
    """Several workgroups to a row: the same sums in another order, rows of no group left, a workspace that held NaN, every run the same."""
    t, need = TYPES[dtype], B.qesgd_mx4_vector_product_workspace_bytes(n, N, K, E)
    pw, w = packed_noise(B, N, K, E, n + N)
    offsets = [0, n] if E == 1 else [2] + [2 + (n - 3) * (e + 1) // E for e in range(E)]
    x, pw = rows(n, K, t, 8), pw.cuda()
    ws, out = torch.full((max(need // 4, 1),), float("nan"), device="cuda").view(torch.uint8), []
    for _ in range(2):
        y = torch.full((n, N + 3), 3.0, dtype=t, device="cuda")
        B.qesgd_mx4_vector_product(x.cuda(), K, n, None, 1, pw, pw.stride(0), None if E == 1 else ints(offsets), E, n, N, K, y, N + 3, workspace=ws)
        out.append(y)
        ws.view(torch.float32).fill_(float("nan"))
    assert torch.equal(*out)
    got = host(out[0])
    assert (got[:, N:] == 3.0).all() and (got[:offsets[0]] == 3.0).all() and (got[offsets[-1]:] == 3.0).all()
    for e in range(E):
        lo, hi = offsets[e], offsets[e + 1]
        want = host(x[lo:hi]) @ w[e].T
        off = np.abs(got[lo:hi, :N] - want) - limit(host(x[lo:hi]), w[e], want, t)
        assert (off <= 0).all(), (e, np.argwhere(off > 0)[:4])
    kept = out[0].clone()
    for short in (None, ws[:need - 16]) if need else ():
        with pytest.raises(B.QesgdError):
            B.qesgd_mx4_vector_product(x.cuda(), K, n, None, 1, pw, pw.stride(0), None if E == 1 else ints(offsets), E, n, N, K, out[0], N + 3, workspace=short)
    assert torch.equal(out[0], kept)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_few_rows_of_many_experts(B, dtype):
    """As many experts as make the kernel take its rows in larger tiles, the reference on the GPU in 64 bits, an expert at a time."""
    t, E, n, N, K = TYPES[dtype], 300, 600, 270, 2100
    rng = np.random.default_rng(4)
    sizes = rng.multinomial(n - 5, rng.dirichlet(np.full(E, 2.0)))
    offsets, order = np.concatenate(([3], 3 + np.cumsum(sizes))), rng.permutation(n)
    lay = B.qesgd_mx4_layout_query(N, K)
    g = torch.Generator(device="cuda").manual_seed(2)
    slab = torch.randint(0, 256, (E, lay.bytes), dtype=torch.uint8, device="cuda", generator=g)
    codes, scales = slab[:, :N * lay.row_codes].view(E, N, -1), slab[:, lay.scales_off:lay.scales_off + N * lay.row_scales].view(E, N, -1)
    scales.copy_(120 + scales % 14)
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device="cuda")
    x = rows(n // 2, K, t, 5).cuda()
    y = torch.full((n, N), 3.0, dtype=t, device="cuda")
    B.qesgd_mx4_vector_product(x, K, n // 2, ints(order), 2, slab, slab.stride(0), ints(offsets), E, n, N, K, y, N,
                               workspace=B.alloc_workspace(B.qesgd_mx4_vector_product_workspace_bytes(n, N, K, E)))
    got, picked = host(y), host(x)[order // 2]
    assert (got[:3] == 3.0).all() and (got[offsets[-1]:] == 3.0).all()
    for e in range(E):
        lo, hi = offsets[e], offsets[e + 1]
        if lo == hi:
            continue
        c = codes[e].long()
        w = grid[torch.stack((c & 15, c >> 4), -1).view(N, -1)] * torch.exp2(scales[e].double() - 127).repeat_interleave(32, 1)
        w = w[:, :K].cpu().numpy()
        want = picked[lo:hi] @ w.T
        off = np.abs(got[lo:hi] - want) - limit(picked[lo:hi], w, want, t)
        assert (off <= 0).all(), (e, np.argwhere(off > 0)[:4])
