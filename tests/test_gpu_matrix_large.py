"""The operators for matrix parameters at sizes where they change kernels, tiles or the number of pieces, and where offsets pass 32 bits.
The 64-bit forms are evaluated on the GPU."""
import numpy as np
import pytest
import torch

import matrix_reference as R

pytestmark = pytest.mark.gpu
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


@pytest.fixture(scope="module")
def B():
    from paper_1901_03040_amd import binding
    assert torch.cuda.is_available()
    binding.lib()
    return binding


def packed_noise(B, rows, cols, seed):
    """Any bytes are a packed matrix, but for the zeros behind its columns.  Scales 2^-3 .. 2^3."""
    lay = B.qesgd_mx4_layout_query(rows, cols)
    g = torch.Generator(device="cuda").manual_seed(seed)
    p = torch.randint(0, 256, (lay.bytes,), generator=g, dtype=torch.uint8, device="cuda")
    codes = p[:rows * lay.row_codes].view(rows, -1)
    codes[:, (cols + 1) // 2:] = 0
    if cols % 2:
        codes[:, cols // 2] &= 15
    p[lay.scales_off:] = torch.randint(124, 131, (lay.bytes - lay.scales_off,), generator=g, dtype=torch.uint8, device="cuda")
    return lay, p


def unpacked(lay, p, first=0, rows=None, dtype=torch.float64):
    rows = lay.rows if rows is None else rows
    codes = p[first * lay.row_codes:(first + rows) * lay.row_codes].view(rows, -1)
    scales = p[lay.scales_off + first * lay.row_scales:lay.scales_off + (first + rows) * lay.row_scales].view(rows, -1)
    table = torch.tensor(np.concatenate((R.MAGNITUDES, -R.MAGNITUDES)), dtype=dtype, device="cuda")
    q = torch.stack((table[(codes & 15).int()], table[(codes >> 4).int()]), 2).view(rows, -1, 32)
    return (q * torch.exp2(scales.to(dtype) - 127)[:, :, None]).view(rows, -1)[:, :lay.cols]


def check_product(a, b, c, K):
    """As in the tests of small products: K 2^-24 of the sum of magnitudes for fp32 sums in any order, half a step of the output."""
    want = a @ b.T
    limit = K * 2.0 ** -24 * (a.abs() @ b.abs().T) + HALF_STEP[c.dtype] * want.abs() * (1 + 2.0 ** -10) + (2.0 ** -25 if c.dtype == torch.float16 else 0)
    off = (c.double() - want).abs() - limit
    assert bool((off <= 0).all()), torch.nonzero(off > 0)[:4]


# few rows at the ends of that kernel's range (16 rows, 16 steps of 256, 8192 columns) and just beyond; long contractions in pieces;
# tiles of 64, 128 and 256, whole and cut off, with a half step at the end and without
PRODUCTS = [(16, 8192, 4096), (17, 8192, 4096), (16, 8193, 4096), (16, 515, 4097), (1, 8192, 3968), (3, 31, 33),
            (1, 1000, 25088), (16, 999, 25000), (512, 1000, 25088), (5, 300, 100_001), (200, 200, 1 << 17), (257, 129, 1 << 20),
            (1024, 2048, 1024), (1000, 2111, 1100), (1024, 4096, 4096), (1500, 4001, 4000), (4096, 4096, 512), (2049, 5001, 833), (3000, 5000, 700),
            (1, 20_000, 64), (20_000, 3, 200)]


@pytest.mark.parametrize("M,N,K,dtype", [(*c, t) for c in PRODUCTS for t in HALF_STEP if t == torch.float32 or c[2] <= 30_000])
def test_product(B, M, N, K, dtype):
    la, pa = packed_noise(B, M, K, M + K)
    lb, pb = packed_noise(B, N, K, N + 2 * K)
    if dtype == torch.float16:                                  # sums stay in range
        pa[la.scales_off:] = 120
    ldc = N + 3
    c = torch.full((M, ldc), 3.0, dtype=dtype, device="cuda")
    need = B.qesgd_mx4_product_workspace_bytes(M, N, K)
    ws = None if need == 0 else B.alloc_workspace(need + 256).fill_(0xFF)
    B.qesgd_mx4_product(pa, pb, M, N, K, c, ldc, workspace=None if ws is None else ws[:need])
    assert bool((c[:, N:] == 3.0).all()) and (ws is None or bool((ws[need:] == 0xFF).all()))
    check_product(unpacked(la, pa), unpacked(lb, pb), c[:, :N], K)
    again = torch.empty_like(c)
    B.qesgd_mx4_product(pa, pb, M, N, K, again, ldc, workspace=ws)
    assert torch.equal(again[:, :N], c[:, :N])


def test_product_operand_beyond_32_bits(B):
    M, N, K = 1 << 20, 40, 1 << 13                              # 4 GiB of codes
    la, pa = packed_noise(B, M, K, 1)
    lb, pb = packed_noise(B, N, K, 2)
    assert M * la.row_codes >= 1 << 32
    c = torch.empty(M, N, device="cuda")
    B.qesgd_mx4_product(pa, pb, M, N, K, c, N, workspace=B.alloc_workspace(B.qesgd_mx4_product_workspace_bytes(M, N, K)))
    b = unpacked(lb, pb)
    for first in (0, M // 2 - 100, M - 200):
        check_product(unpacked(la, pa, first, 200), b, c[first:first + 200], K)
    # the same operand on the other side
    c = torch.empty(N, M, device="cuda")
    B.qesgd_mx4_product(pb, pa, N, M, K, c, M, workspace=B.alloc_workspace(B.qesgd_mx4_product_workspace_bytes(N, M, K)))
    for first in (0, M // 2 - 100, M - 200):
        check_product(b, unpacked(la, pa, first, 200), c[:, first:first + 200], K)


def test_product_result_beyond_32_bits(B):
    M, N, K = 70_000, 66_000, 64                                # 4.6e9 numbers
    la, pa = packed_noise(B, M, K, 1)
    lb, pb = packed_noise(B, N, K, 2)
    c = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    B.qesgd_mx4_product(pa, pb, M, N, K, c, N, workspace=B.alloc_workspace(B.qesgd_mx4_product_workspace_bytes(M, N, K)))
    for r, s in ((0, 0), (M - 300, N - 300), (65_075, 100), (35_000, 65_900)):
        check_product(unpacked(la, pa, r, 100), unpacked(lb, pb, s, 100), c[r:r + 100, s:s + 100], K)


def test_codes_of_matrices_beyond_32_bits(B):
    """Both forms of 4.4e9 numbers: the tails equal those of the tail alone (nearest), and the stochastic ones what the reference makes of
    their coordinates' numbers."""
    rows, cols = (1 << 25) + 128, 128
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn(rows, cols, generator=g, device="cuda", dtype=torch.bfloat16)
    tail = 256                                                  # rows, a multiple of 128
    lay, lay_t = B.qesgd_mx4_layout_query(rows, cols), B.qesgd_mx4_layout_query(cols, rows)
    p, t = B.alloc_mx4(lay), B.alloc_mx4(lay_t)
    xt = x[-tail:].double().cpu().numpy()
    for mode in (B.MX4_NEAREST, B.MX4_STOCHASTIC):
        stochastic = mode == B.MX4_STOCHASTIC
        for rows_alone in (True, False):
            p.fill_(0xA5)
            B.qesgd_mx4_quantize_pack(x, cols, 0, rows, cols, 1, mode, 7, 1, p, 0, packed_t=None if rows_alone else t, worker=2)
            r = variates_from((rows - tail) * 128, tail * 128, 7, 1, 2).reshape(tail, 128) if stochastic else None
            code, scale = quantize_with(xt, r)
            got = p[(rows - tail) * lay.row_codes:rows * lay.row_codes].view(tail, -1).cpu().numpy()
            assert np.array_equal(got, R.pack(code))
            got = p[lay.scales_off + (rows - tail) * 4:lay.scales_off + rows * 4].view(tail, -1).cpu().numpy()
            assert np.array_equal(got, scale)
        wide = lay_t.row_codes * 2
        r = np.stack([variates_from(c * wide + rows - tail, tail, 7, 1, 2) for c in range(cols)]) if stochastic else None
        code, scale = quantize_with(xt.T, r)
        at = (rows - tail) // 2
        assert np.array_equal(t[:cols * lay_t.row_codes].view(cols, -1)[:, at:at + tail // 2].cpu().numpy(), R.pack(code))
        at = (rows - tail) // 32
        got = t[lay_t.scales_off:lay_t.scales_off + cols * lay_t.row_scales].view(cols, -1)[:, at:at + tail // 32].cpu().numpy()
        assert np.array_equal(got, scale)
    # back to numbers: the last of 4.4e9
    z = torch.empty(rows * cols, device="cuda")
    B.qesgd_mx4_quantize_pack(x, cols, 0, rows, cols, 1, B.MX4_NEAREST, 0, 0, p, 0)
    B.qesgd_mx4_unpack_aggregate_update(p, 0, 1, rows, cols, None, z, None, None)
    want = R.values(*quantize_with(xt, None), cols).astype(np.float32)
    assert np.array_equal(z[-tail * cols:].view(tail, cols).cpu().numpy(), want)


def variates_from(first, count, seed, rnd, worker):
    """The variates of coordinates first .. first + count - 1, first a multiple of 8."""
    g = np.arange(first // 8, (first + count) // 8, dtype=np.uint64)
    zero = np.zeros_like(g)
    w = np.stack(R.philox(g & np.uint64(0xFFFFFFFF), g >> np.uint64(32), zero + np.uint64(worker), zero + np.uint64(rnd), seed), 1)
    return np.stack((w & np.uint64(0xFFFF), w >> np.uint64(16)), 2).reshape(-1).astype(np.int64)


def quantize_with(x, variates):
    """R.quantize with the variates given (columns a multiple of 128), or to nearest without."""
    kept, R.variates = R.variates, lambda *_: variates
    try:
        return R.quantize(x, variates is not None)
    finally:
        R.variates = kept


def newton_schulz(x, coeffs, eps=1e-7, noise=0.0):
    g = torch.Generator(device="cuda").manual_seed(0)
    X = x / (x.norm() + eps)
    X = X.T.contiguous() if X.shape[0] > X.shape[1] else X

    def times(a, b):
        c = a @ b
        if noise:
            c += noise * torch.randn(c.shape, generator=g, device="cuda", dtype=torch.float64) * a.norm(dim=1)[:, None] * b.norm(dim=0)[None, :]
        return c

    for a, b, c in coeffs:
        G = times(X, X.T.contiguous())
        P = b * G + c * times(G, G)
        P.diagonal().add_(a)
        X = times(P, X)
    return X.T if x.shape[0] > x.shape[1] else X


# single steps and pairs (the longer side at least twice the shorter), tiles of 64, 128 and 256, the contraction in pieces and whole, both
# orientations, cut-off tiles, batches, every number of steps modulo the pairs
ORTHOGONAL = [(1, 520, 2080, 5), (1, 2080, 520, 5), (1, 520, 2080, 1), (1, 520, 2080, 2), (1, 520, 2080, 3), (1, 520, 2080, 4), (1, 520, 2080, 6),
              (1, 1030, 1999, 5), (1, 2048, 2048, 5), (1, 3001, 2011, 4), (1, 1000, 9001, 5), (1, 9001, 1000, 2), (1, 2100, 7777, 5),
              (1, 4100, 4100, 2), (1, 4096, 9000, 3), (6, 700, 900, 3), (12, 1024, 1024, 2), (40, 100, 300, 5), (3, 130, 50_001, 5),
              (1, 2048, 8192, 3), (1, 5632, 11_264, 2), (1, 1, 100_000, 5), (1, 70_000, 2, 5), (1000, 20, 1100, 5), (300, 97, 97, 3), (70, 96, 170, 5), (3, 96, 160, 5), (3, 161, 96, 5), (2, 32, 512, 5), (2, 33, 512, 5), (2, 513, 32, 5)]


@pytest.mark.parametrize("n,rows,cols,steps", ORTHOGONAL)
def test_orthogonalize(B, n, rows, cols, steps):
    """What a result may be off by: as in the tests of small matrices, from the reference with random errors of the split products' size."""
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    rank = max(1, min(rows, cols) // 8)
    x = torch.randn(n, rows, cols, generator=g, device="cuda")
    for i in range(0, n, 2):                                    # every other one with strong directions
        strong = torch.randn(rows, rank, generator=g, device="cuda") / (1 + torch.arange(rank, device="cuda"))
        x[i] = 0.05 * x[i] + strong @ torch.randn(rank, cols, generator=g, device="cuda")
    co = R.USUAL[:1] * steps
    need = B.qesgd_orthogonalize_workspace_bytes(rows, cols, n)
    ws = B.alloc_workspace(need + 256).fill_(0xFF) if need else None
    out = torch.full((n * rows * cols + 64,), 5.0, device="cuda")
    B.qesgd_orthogonalize(x, rows, cols, n, co, 1e-7, out, None if ws is None else ws[:need])
    assert bool((out[n * rows * cols:] == 5.0).all()) and (ws is None or bool((ws[need:] == 0xFF).all()))
    got = out[:n * rows * cols].view(n, rows, cols)
    for i in sorted({0, 1 % n, n // 2, n - 1}):
        x64 = x[i].double()
        want = newton_schulz(x64, co)
        moved = newton_schulz(x64, co, noise=2.0 ** -22 / max(rows, cols) ** 0.5) if min(rows, cols) > 1 else want
        size = float(want.norm())
        limit = 8 * (float((moved - want).norm()) + 2.0 ** -22 * size) + 2.0 ** -24 * size
        off = float((got[i].double() - want).norm())
        print("%d: off %.2g of %.2g allowed" % (i, off / size, limit / size))
        assert off <= limit, i
    B.qesgd_orthogonalize(x, rows, cols, n, co, 1e-7, x, ws)    # in place, and the same bits again
    assert torch.equal(x, got)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols", [(300, 500), (1024, 8192), (8200, 1030), (2048, 8192), (8100, 2040)])
def test_orthogonalize_types(B, rows, cols, dtype):
    """Half a step of the type more, and for fp16 half of its smallest subnormal for every number."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = (torch.randn(rows, cols, generator=g, device="cuda") * 1e-2).to(dtype)
    co, out = R.USUAL[:2], torch.empty_like(x)
    B.qesgd_orthogonalize(x, rows, cols, 1, co, 1e-7, out, B.alloc_workspace(B.qesgd_orthogonalize_workspace_bytes(rows, cols, 1)))
    want = newton_schulz(x.double(), co)
    moved = newton_schulz(x.double(), co, noise=2.0 ** -22 / max(rows, cols) ** 0.5)
    limit = 8 * float((moved - want).norm()) + (8 * 2.0 ** -22 + HALF_STEP[dtype]) * float(want.norm())
    limit += (rows * cols) ** 0.5 * 2.0 ** -25 if dtype == torch.float16 else 0.0
    assert float((out.double() - want).norm()) <= limit


@pytest.mark.parametrize("n,rows,cols", [(1, 4096, 300_000), (60_000, 300, 260)])
def test_orthogonalize_beyond_32_bits(B, n, rows, cols):
    """Numbers whose byte offsets, in the matrices and in the workspace, pass 2^32: one long matrix, and many."""
    co = R.USUAL[:1]
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(n, rows, cols, generator=g, device="cuda")
    assert x.numel() * 4 > 1 << 32
    out = torch.empty_like(x)
    B.qesgd_orthogonalize(x, rows, cols, n, co, 1e-7, out, B.alloc_workspace(B.qesgd_orthogonalize_workspace_bytes(rows, cols, n)))
    for i in sorted({0, n - 1}):
        # off by a product's error in G and P each, and the split of X: 2^-22 of every row's norm, five times over
        step = 1 << 16
        G = sum(x[i, :, c:c + step].double() @ x[i, :, c:c + step].double().T.contiguous() for c in range(0, cols, step))
        norm = float(G.trace()) ** 0.5 + 1e-7
        G /= norm ** 2
        a, b, c = co[0]
        P = b * G + c * (G @ G)
        P.diagonal().add_(a)
        want = P @ (x[i, :, -2000:].double() / norm)
        assert float((out[i, :, -2000:].double() - want).norm()) <= 5 * 2.0 ** -22 * float(want.norm()) * max(1.0, a / float(torch.linalg.eigvalsh(P).abs().min()))


def test_two_calls_at_once(B):
    """On two streams, each with a workspace of its own: the same bits as one after the other."""
    rows, cols = 520, 2080
    M, N, K = 512, 1000, 25_088
    assert B.qesgd_mx4_product_workspace_bytes(M, N, K) > 0
    x = torch.randn(2, 1, rows, cols, generator=torch.Generator(device="cuda").manual_seed(0), device="cuda")
    out, alone = torch.empty_like(x), torch.empty_like(x)
    pa, pb = [packed_noise(B, M, K, i)[1] for i in range(2)], [packed_noise(B, N, K, 5 + i)[1] for i in range(2)]
    c, c_alone = (torch.empty(2, M, N, device="cuda") for _ in range(2))
    wx = [B.alloc_workspace(B.qesgd_orthogonalize_workspace_bytes(rows, cols, 1)) for _ in range(2)]
    wp = [B.alloc_workspace(B.qesgd_mx4_product_workspace_bytes(M, N, K)) for _ in range(2)]

    def work(i, to, product):
        for _ in range(5):
            B.qesgd_orthogonalize(x[i], rows, cols, 1, R.USUAL, 1e-7, to[i], wx[i])
            B.qesgd_mx4_product(pa[i], pb[i], M, N, K, product[i], N, workspace=wp[i])

    for i in range(2):
        work(i, alone, c_alone)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i, stream in enumerate(streams):
        with torch.cuda.stream(stream):
            work(i, out, c)
    torch.cuda.synchronize()
    assert torch.equal(out, alone) and torch.equal(c, c_alone)


def test_views_are_refused(B):
    x, out = torch.randn(64, 64, device="cuda"), torch.empty(64, 64, device="cuda")
    row = torch.randn(64, device="cuda").expand(64, 64)
    calls = [lambda v: B.qesgd_orthogonalize(v, 64, 64, 1, R.USUAL, 1e-7, out, None), lambda v: B.qesgd_orthogonalize(x, 64, 64, 1, R.USUAL, 1e-7, v, None)]
    for at in range(5):
        def update(v, at=at):
            t = [x, None, out, None, None, None, None]
            t[at] = v
            if at >= 4:
                t[3], t[4], t[5] = (torch.empty(64, 64, device="cuda") if i != at else v for i in (3, 4, 5))
            g, m, step, z, w, u, zsum = t
            B.qesgd_orthogonal_update(g, 64, 64, 1, m, 0.9, True, R.USUAL, 1e-7, 1.0, step, z, w, u, zsum, None)
        calls.append(update)
    for call in calls:
        for v in (x.t(), row, torch.randn(64, 128, device="cuda")[:, :64]):
            with pytest.raises(B.QesgdError) as e:
                call(v)
            assert e.value.code == B.ERR_STRIDE


def test_hyperparameters_of_other_types(B):
    x = torch.randn(40, 60, device="cuda")
    a, b = torch.empty_like(x), torch.empty_like(x)
    B.qesgd_orthogonal_update(x, 40, 60, 1, None, 0.5, True, R.USUAL, 1e-7, -0.25, a, None, None, None, None, None)
    B.qesgd_orthogonal_update(x, 40, 60, 1, None, np.float32(0.5), True, np.array(R.USUAL), np.float64(1e-7), torch.tensor(-0.25), b, None, None,
                              None, None, None)
    assert torch.equal(a, b)


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("rows,cols", [(40, 50), (1, 9), (300, 200), (200, 900), (1, 3000)])
def test_what_is_not_finite_takes_its_whole_matrix(B, rows, cols, bad):
    x = torch.randn(3, rows, cols, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    ws = B.alloc_workspace(B.qesgd_orthogonalize_workspace_bytes(rows, cols, 3))
    want, out = torch.empty_like(x), torch.empty_like(x)
    B.qesgd_orthogonalize(x, rows, cols, 3, R.USUAL, 1e-7, want, ws)
    x[1, rows // 2, cols // 3] = bad
    B.qesgd_orthogonalize(x, rows, cols, 3, R.USUAL, 1e-7, out, ws)
    assert bool(torch.isnan(out[1]).all())
    assert torch.equal(out[0], want[0]) and torch.equal(out[2], want[2])
