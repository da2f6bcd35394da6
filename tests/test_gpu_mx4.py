"""4-bit microscaled codes on the GPU against the 64-bit reference: every byte of codes and scales, the mean and update bit for bit,
products within their rounding."""
import numpy as np
import pytest
import torch

import matrix_reference as R

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


@pytest.fixture(scope="module")
def B():
    from paper_1901_03040_amd import binding
    assert torch.cuda.is_available()
    binding.lib()
    return binding


def matrix(rows, cols, dtype, seed, special=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp2(torch.randint(-9, 4, (rows, 1), generator=g).float())
    x *= torch.rand(rows, cols, generator=g) > 0.05
    if special and rows * cols > 64:
        flat = x.view(-1)
        flat[::37] = torch.tensor([-0.0, 0.25, 0.75, 1.5, 6.0, 7.0, -5.0, 2.5, 3.5, 1e-5])[torch.arange(len(flat[::37])) % 10]
    return x.to(dtype)


def host(x):
    return x.detach().double().cpu().numpy()


def check_packed(B, packed, rows, cols, code, scale, what):
    lay = B.qesgd_mx4_layout_query(rows, cols)
    got = packed.cpu().numpy()
    codes = got[:rows * lay.row_codes].reshape(rows, -1)
    scales = got[lay.scales_off:lay.scales_off + rows * lay.row_scales].reshape(rows, -1)
    bad = np.argwhere(scales != scale)
    assert not len(bad), (what, "scale bytes", bad[:4])
    bad = np.argwhere(codes != R.pack(code))
    assert not len(bad), (what, "codes", bad[:4])
    assert (got[rows * lay.row_codes:lay.scales_off] == 0xA5).all() and (got[lay.scales_off + rows * lay.row_scales:] == 0xA5).all(), what


SHAPES = [(1, 1), (1, 31), (1, 32), (1, 129), (3, 5), (2, 128), (7, 384), (33, 127), (64, 256), (130, 300), (1, 5000), (1, 4096),
          (257, 1001), (600, 7)]


@pytest.mark.parametrize("mode", ["nearest", "stochastic"])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantize_every_byte(B, rows, cols, dtype, mode):
    x = matrix(rows, cols, TYPES[dtype], rows * 1000 + cols).cuda()
    m = B.MX4_STOCHASTIC if mode == "stochastic" else B.MX4_NEAREST
    seed, rnd, worker = 0x123456789ABCDEF, 9, 5
    lay, lay_t = B.qesgd_mx4_layout_query(rows, cols), B.qesgd_mx4_layout_query(cols, rows)
    want = R.quantize(host(x), mode == "stochastic", seed, rnd, worker)
    want_t = R.quantize(host(x).T, mode == "stochastic", seed, rnd, worker)
    for which in ("rows", "columns", "both"):
        p, t = B.alloc_mx4(lay).fill_(0xA5), B.alloc_mx4(lay_t).fill_(0xA5)
        B.qesgd_mx4_quantize_pack(x, cols, 0, rows, cols, 1, m, seed, rnd, None if which == "columns" else p, 0,
                                  packed_t=None if which == "rows" else t, worker=worker)
        if which != "columns":
            check_packed(B, p, rows, cols, *want, which)
        if which != "rows":
            check_packed(B, t, cols, rows, *want_t, which)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("offset,extra", [(0, 3), (1, 0), (3, 5), (8, 64)])
def test_quantize_workers_strides_and_offsets(B, dtype, offset, extra):
    """Three workers, rows that are longer than the matrix and start at any element."""
    rows, cols, K = 37, 203, 3
    ld = cols + extra
    stride = rows * ld + 11
    whole = matrix(1, offset + K * stride, TYPES[dtype], 7).cuda().view(-1)
    x = whole[offset:]
    lay, lay_t = B.qesgd_mx4_layout_query(rows, cols), B.qesgd_mx4_layout_query(cols, rows)
    p, t = B.alloc_mx4(lay, K).fill_(0xA5), B.alloc_mx4(lay_t, K).fill_(0xA5)
    B.qesgd_mx4_quantize_pack(x, ld, stride, rows, cols, K, B.MX4_STOCHASTIC, 11, 2, p, p.stride(0), packed_t=t,
                              packed_t_stride=t.stride(0), worker=4)
    q = B.alloc_mx4(lay, K).fill_(0xA5)
    B.qesgd_mx4_quantize_pack(x, ld, stride, rows, cols, K, B.MX4_STOCHASTIC, 11, 2, q, q.stride(0), worker=4)
    assert torch.equal(p, q)
    for k in range(K):
        xk = host(torch.as_strided(x, (rows, cols), (ld, 1), offset + k * stride))
        check_packed(B, p[k], rows, cols, *R.quantize(xk, True, 11, 2, 4 + k), k)
        check_packed(B, t[k], cols, rows, *R.quantize(xk.T, True, 11, 2, 4 + k), k)


@pytest.mark.parametrize("mode", ["nearest", "stochastic"])
def test_quantize_ends_of_the_range(B, mode):
    """Subnormals, the largest numbers, zeros of either sign, infinities and NaN, each in blocks of its own."""
    big = float(np.finfo(np.float32).max)
    rows = [[1e-45, -1e-45, 3e-45], [1.1754944e-38, 5e-39], [2.0 ** -125, 2.0 ** -126, -2.0 ** -127], [big, -big, big / 2, big / 3],
            [1.5 * 2.0 ** 127, 2.0 ** 127, 2.0 ** 126], [float(np.nextafter(np.float32(1.5 * 2.0 ** 127), np.float32(0)))],
            [0.0, -0.0], [float("inf"), 1.0], [float("-inf"), -1.0], [float("nan"), 2.0], [6.0], [float(np.nextafter(np.float32(6), np.float32(7)))]]
    x = torch.zeros(len(rows), 96)
    for i, r in enumerate(rows):
        x[i, 33:33 + len(r)] = torch.tensor(r, dtype=torch.float32)
        x[i, 70] = 1.0                                         # the next block is not touched by its neighbour
    seed = 3
    want = R.quantize(host(x), mode == "stochastic", seed, 0, 0)
    want_t = R.quantize(host(x).T, mode == "stochastic", seed, 0, 0)
    lay, lay_t = B.qesgd_mx4_layout_query(*x.shape), B.qesgd_mx4_layout_query(*x.T.shape)
    p, t = B.alloc_mx4(lay).fill_(0xA5), B.alloc_mx4(lay_t).fill_(0xA5)
    B.qesgd_mx4_quantize_pack(x.cuda(), 96, 0, x.shape[0], 96, 1, B.MX4_STOCHASTIC if mode == "stochastic" else B.MX4_NEAREST, seed, 0, p, 0, packed_t=t)
    check_packed(B, p, *x.shape, *want, "rows")
    check_packed(B, t, *x.T.shape, *want_t, "columns")


def packed_noise(B, rows, cols, K, seed, spread=20):
    """Any bytes are a packed matrix."""
    lay = B.qesgd_mx4_layout_query(rows, cols)
    g = torch.Generator().manual_seed(seed)
    p = torch.randint(0, 256, (K, lay.bytes), generator=g, dtype=torch.uint8)
    p[:, lay.scales_off:] = torch.randint(127 - spread, 127 + spread, (K, lay.bytes - lay.scales_off), generator=g, dtype=torch.uint8)
    return lay, p


def unpacked(lay, row):
    b = row.numpy()
    codes = b[:lay.rows * lay.row_codes].reshape(lay.rows, -1)
    code = np.stack((codes & 15, codes >> 4), 2).reshape(lay.rows, -1)
    return R.values(code, b[lay.scales_off:lay.scales_off + lay.rows * lay.row_scales].reshape(lay.rows, -1), lay.cols)


@pytest.mark.parametrize("K", [1, 2, 3, 5, 8, 16, 64])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 130), (5, 7), (3, 128), (40, 384), (33, 1001), (1, 70_001)])
def test_mean_and_update_bit_for_bit(B, rows, cols, K):
    lay, p = packed_noise(B, rows, cols, K, rows + cols + K)
    g = torch.Generator().manual_seed(K)
    d = rows * cols
    w, zs = torch.randn(d, generator=g), torch.randn(d, generator=g)
    acc = np.zeros(d, np.float32)
    for k in range(K):
        acc = acc + unpacked(lay, p[k]).astype(np.float32).reshape(-1)
    z = acc / np.float32(K)
    room = 64
    out = {n: torch.full((d + room,), 7.0, device="cuda") for n in ("z", "u", "zs")}
    out["zs"][:d] = zs.cuda()
    pc, wc = p.cuda(), w.cuda()
    B.qesgd_mx4_unpack_aggregate_update(pc, pc.stride(0), K, rows, cols, wc, out["z"], out["u"], out["zs"])
    for n, want in (("z", z), ("u", w.numpy() + z), ("zs", zs.numpy() + z)):
        assert np.array_equal(out[n][:d].cpu().numpy(), want), n
        assert (out[n][d:] == 7.0).all(), n
    only = torch.full((d + room,), 7.0, device="cuda")
    B.qesgd_mx4_unpack_aggregate_update(pc, pc.stride(0), K, rows, cols, None, only, None, None)
    assert torch.equal(only, out["z"])
    B.qesgd_mx4_unpack_aggregate_update(pc, pc.stride(0), K, rows, cols, wc, None, wc, None)       # in place
    assert torch.equal(wc, out["u"][:d])
    only[:d] = zs.cuda()
    B.qesgd_mx4_unpack_aggregate_update(pc, pc.stride(0), K, rows, cols, None, None, None, only)
    assert torch.equal(only, out["zs"])


def test_decoding_every_byte_and_scale(B):
    lay = B.qesgd_mx4_layout_query(256, 512)
    p = torch.empty(1, lay.bytes, dtype=torch.uint8)
    p[0, :256 * 256] = torch.arange(256, dtype=torch.uint8).repeat(256)
    p[0, lay.scales_off:lay.scales_off + 256 * 16] = torch.arange(256, dtype=torch.uint8).repeat_interleave(16)
    z = torch.empty(256 * 512, device="cuda")
    B.qesgd_mx4_unpack_aggregate_update(p.cuda(), lay.bytes, 1, 256, 512, None, z, None, None)
    with np.errstate(over="ignore"):
        want = unpacked(lay, p[0]).astype(np.float32)
    assert np.array_equal(z.cpu().numpy().reshape(256, 512), want, equal_nan=True)


PRODUCTS = [(1, 1, 1), (1, 16, 32), (1, 1000, 128), (1, 515, 4000), (2, 33, 129), (16, 64, 256), (17, 130, 384), (37, 1000, 2049),
            (100, 64, 640), (128, 128, 128), (129, 257, 1000), (255, 511, 320), (300, 40, 8200), (520, 777, 511)]


def product_limit(a, b, want, dtype):
    """Element products are exact; a sum of n terms in fp32 in any order is off by at most n 2^-24 of the sum of magnitudes (n 2^-24 for
    n - 1 additions, first order); rounding to the output type by half a step."""
    return a.shape[1] * 2.0 ** -24 * (np.abs(a) @ np.abs(b).T) + HALF_STEP[dtype] * np.abs(want) * (1 + 2.0 ** -10) + (2.0 ** -25 if dtype == torch.float16 else 0)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_product(B, M, N, K, dtype):
    t = TYPES[dtype]
    la, pa = packed_noise(B, M, K, 1, M + K, 3)
    lb, pb = packed_noise(B, N, K, 1, N + 2 * K, 3)
    # what is behind the last column counts for nothing only because the format has zeros there
    for lay, p in ((la, pa), (lb, pb)):
        b = p[0].numpy()
        codes = b[:lay.rows * lay.row_codes].reshape(lay.rows, -1)
        codes[:, (K + 1) // 2:] = 0
        if K % 2:
            codes[:, K // 2] &= 15
    a, b = unpacked(la, pa[0]), unpacked(lb, pb[0])
    want = a @ b.T
    ldc = N + 5
    c = torch.full((M, ldc), 3.0, dtype=t, device="cuda")
    ws = B.alloc_workspace(B.qesgd_mx4_product_workspace_bytes(M, N, K))
    B.qesgd_mx4_product(pa.cuda(), pb.cuda(), M, N, K, c, ldc, workspace=ws)
    got = host(c)
    assert (got[:, N:] == 3.0).all()
    off = np.abs(got[:, :N] - want) - product_limit(a, b, want, t)
    assert (off <= 0).all(), np.argwhere(off > 0)[:4]
    again = torch.full((M, ldc), 3.0, dtype=t, device="cuda")
    B.qesgd_mx4_product(pa.cuda(), pb.cuda(), M, N, K, again, ldc, workspace=ws)
    assert torch.equal(again, c)                               # no order of additions that comes and goes


@pytest.mark.parametrize("M,N", [(3, 40), (150, 140)])
def test_product_nan_stays_in_its_row(B, M, N):
    K = 300
    x, w = matrix(M, K, torch.float32, 1, False), matrix(N, K, torch.float32, 2, False)
    x[M - 2, 250] = float("nan")
    w[5, 17] = float("inf")
    px, pw = B.alloc_mx4(B.qesgd_mx4_layout_query(M, K)), B.alloc_mx4(B.qesgd_mx4_layout_query(N, K))
    B.qesgd_mx4_quantize_pack(x.cuda(), K, 0, M, K, 1, B.MX4_NEAREST, 0, 0, px, 0)
    B.qesgd_mx4_quantize_pack(w.cuda(), K, 0, N, K, 1, B.MX4_NEAREST, 0, 0, pw, 0)
    c = torch.empty(M, N, device="cuda")
    B.qesgd_mx4_product(px, pw, M, N, K, c, N, workspace=B.alloc_workspace(B.qesgd_mx4_product_workspace_bytes(M, N, K)))
    nan = torch.isnan(c).cpu()
    want = torch.zeros(M, N, dtype=torch.bool)
    want[M - 2] = True
    want[:, 5] = True
    assert torch.equal(nan, want)


@pytest.mark.parametrize("M,N,K", [(64, 96, 160), (130, 70, 200)])
def test_a_layers_gradients_against_the_formula_and_differences(B, M, N, K):
    """y = Q(x) Q(w)^T, dx = Q(dy) Q(w), dw = Q(dy)^T Q(x), all from one read of each operand.  The operands are such that their 4-bit
    forms along either side are exact, so the gradients are those of y: they are checked against differences too."""
    g = torch.Generator().manual_seed(M)
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])

    def exact(r, c):
        x = grid[torch.randint(0, 8, (r, c), generator=g)] * (torch.randint(0, 2, (r, c), generator=g) * 2.0 - 1)
        x[:, ::16] = 6.0                                       # every block along either side has the same scale
        x[::16, :] = 4.0
        return x

    x, w, dy = exact(M, K), exact(N, K), exact(M, N)
    packed = {}
    for n, v in (("x", x), ("w", w), ("dy", dy)):
        r, c = v.shape
        packed[n] = B.alloc_mx4(B.qesgd_mx4_layout_query(r, c)), B.alloc_mx4(B.qesgd_mx4_layout_query(c, r))
        B.qesgd_mx4_quantize_pack(v.cuda(), c, 0, r, c, 1, B.MX4_NEAREST, 0, 0, packed[n][0], 0, packed_t=packed[n][1])

    def product(a, b, m, n, k):
        c = torch.empty(m, n, device="cuda")
        B.qesgd_mx4_product(a, b, m, n, k, c, n, workspace=B.alloc_workspace(B.qesgd_mx4_product_workspace_bytes(m, n, k)))
        return c.double().cpu()

    y = product(packed["x"][0], packed["w"][0], M, N, K)
    dx = product(packed["dy"][0], packed["w"][1], M, K, N)
    dw = product(packed["dy"][1], packed["x"][1], N, K, M)
    # sums of at most 200 multiples of 1/4 up to 36: exact in fp32
    assert torch.equal(y, x.double() @ w.double().T)
    assert torch.equal(dx, dy.double() @ w.double())
    assert torch.equal(dw, dy.double().T @ x.double())
    loss = lambda a, b: ((a.double() @ b.double().T) * dy.double()).sum()      # noqa: E731, linear in either operand: a difference is exact
    for i, j in [(0, 0), (M - 1, K - 1), (M // 2, 3)]:
        step = torch.zeros(M, K)
        step[i, j] = 1.0
        assert abs(float(loss(x + step, w) - loss(x, w) - dx[i, j])) <= 1e-9
    for i, j in [(0, 0), (N - 1, K - 1), (N // 2, 3)]:
        step = torch.zeros(N, K)
        step[i, j] = 1.0
        assert abs(float(loss(x, w + step) - loss(x, w) - dw[i, j])) <= 1e-9


def test_side_stream_and_graph(B):
    """A captured and replayed round on packed operands equals the eager one, replay after replay, and two graphs that share a workspace
    do not disturb each other when they run one after the other."""
    M, N, K = 48, 200, 1100
    x, w = matrix(M, K, torch.bfloat16, 1).cuda(), matrix(N, K, torch.bfloat16, 2).cuda()
    px, pw = B.alloc_mx4(B.qesgd_mx4_layout_query(M, K)), B.alloc_mx4(B.qesgd_mx4_layout_query(N, K))
    ws = B.alloc_workspace(max(B.qesgd_mx4_product_workspace_bytes(M, N, K), 256))
    y = torch.zeros(M, N, device="cuda", dtype=torch.bfloat16)

    def work():
        B.qesgd_mx4_quantize_pack(x, K, 0, M, K, 1, B.MX4_STOCHASTIC, 1, 2, px, 0)
        B.qesgd_mx4_quantize_pack(w, K, 0, N, K, 1, B.MX4_NEAREST, 1, 2, pw, 0)
        B.qesgd_mx4_product(px, pw, M, N, K, y, N, workspace=ws)

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
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for g in graphs:
        with torch.cuda.graph(g):
            work()
    for i in range(4):
        y.zero_()
        px.zero_()
        graphs[i & 1].replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), i
        assert np.isfinite(torch.randn(1 << 16, device="cuda").sum().item())
