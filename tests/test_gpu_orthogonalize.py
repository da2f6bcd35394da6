"""The orthogonalised update on the GPU against the 64-bit reference.

How far a result may be off is taken from the reference itself: the kernels' products hold each operand as two fp16 numbers (off by
at most 2^-23 of the number, and 2^-24 of the largest lost) and sum in fp32, so every product is moved by about 2^-22 of the norms of the row and column
that went into it.  The reference is run again with random errors of that size in every product (noise), and a result may be
off by eight times what that does to it, plus half a step of the output's type."""
import numpy as np
import pytest
import torch

import matrix_reference as R

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
EPS = 1e-7


@pytest.fixture(scope="module")
def B():
    from paper_1901_03040_amd import binding
    assert torch.cuda.is_available()
    binding.lib()
    return binding


def matrices(n, rows, cols, kind, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, rows, cols, generator=g)
    if kind == "decay":                                        # singular values that fall off, and a few strong directions
        r = max(1, min(rows, cols) // 8)
        x = 0.05 * x + (torch.randn(n, rows, r, generator=g) / (1 + torch.arange(r))) @ torch.randn(n, r, cols, generator=g)
    if kind == "rank1":
        x = torch.randn(n, rows, 1, generator=g) @ torch.randn(n, 1, cols, generator=g)
    return x


def allowed(x, want, coeffs, half_step, eps=EPS):
    """Norm of what a result may be off by."""
    rng = np.random.default_rng(0)
    moved = R.newton_schulz(x, coeffs, eps, noise=2.0 ** -22 / np.sqrt(max(x.shape)), rng=rng) if min(x.shape) > 1 else want
    return 8 * (np.linalg.norm(moved - want) + 2.0 ** -22 * np.linalg.norm(want)) + half_step * np.linalg.norm(want)


def ws_for(B, rows, cols, n):
    need = B.qesgd_orthogonalize_workspace_bytes(rows, cols, n)
    return B.alloc_workspace(need).fill_(0xFF) if need else None       # NaN everywhere: nothing may be read before it is written


SHAPES = [(1, 1), (1, 7), (9, 1), (2, 2), (5, 3), (16, 16), (31, 33), (32, 32), (33, 31), (64, 64), (64, 576), (65, 130), (100, 100), (127, 129),
          (129, 127), (128, 512), (300, 64), (500, 40), (200, 333), (257, 256), (384, 640), (1000, 520),
          (96, 96), (48, 341), (17, 900), (16, 1024), (64, 256), (64, 257), (96, 170), (97, 97), (1024, 90), (130, 2100), (600, 1800)]


@pytest.mark.parametrize("kind", ["plain", "decay", "rank1"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_against_64_bits(B, rows, cols, kind):
    x = matrices(1, rows, cols, kind, rows + 7 * cols) * 1e-3
    out = torch.full_like(x, 5.0).cuda()
    B.qesgd_orthogonalize(x.cuda(), rows, cols, 1, R.USUAL, EPS, out, ws_for(B, rows, cols, 1))
    got, x64 = out.double().cpu().numpy()[0], x.double().numpy()[0]
    want = R.newton_schulz(x64)
    off, limit = np.linalg.norm(got - want), allowed(x64, want, R.USUAL, HALF_STEP["f32"])
    print(rows, cols, kind, "off %.2g of %.2g allowed" % (off / np.linalg.norm(want), limit / np.linalg.norm(want)))
    assert off <= limit


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("n,rows,cols", [(3, 40, 72), (2, 150, 90), (5, 64, 64), (2, 129, 300)])
def test_batches_types_and_in_place(B, n, rows, cols, dtype):
    x = (matrices(n, rows, cols, "decay", n) * torch.tensor([1.0, 1e-3, 30.0, 1e-2, 5.0])[:n, None, None]).to(TYPES[dtype])
    dev = x.cuda()
    out = torch.empty_like(dev)
    ws = ws_for(B, rows, cols, n)
    B.qesgd_orthogonalize(dev, rows, cols, n, R.USUAL, EPS, out, ws)
    B.qesgd_orthogonalize(dev, rows, cols, n, R.USUAL, EPS, dev, ws)
    assert torch.equal(dev, out)
    for i in range(n):
        x64 = x[i].double().numpy()
        want = R.newton_schulz(x64)
        off = np.linalg.norm(out[i].double().cpu().numpy() - want)
        assert off <= allowed(x64, want, R.USUAL, HALF_STEP[dtype]), i


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 9])
def test_other_coefficients_and_numbers_of_steps(B, steps):
    classical = ((15 / 8, -10 / 8, 3 / 8),) * steps
    mixed = tuple((1.5 + 0.1 * i, -0.5 - 0.05 * i, 0.02 * i) for i in range(steps))
    x = matrices(1, 70, 180, "plain", steps)
    for co in (classical, mixed):
        out = torch.empty(1, 70, 180, device="cuda")
        B.qesgd_orthogonalize(x.cuda(), 70, 180, 1, co, 0.0, out, ws_for(B, 70, 180, 1))
        co32 = tuple(tuple(float(np.float32(v)) for v in c) for c in co)
        want = R.newton_schulz(x[0].double().numpy(), co32, 0.0)
        assert np.linalg.norm(out[0].double().cpu().numpy() - want) <= allowed(x[0].double().numpy(), want, co32, 2.0 ** -24, 0.0)


@pytest.mark.parametrize("size", [1e-42, 1e-30, 1e30])
def test_magnitudes_whose_squares_leave_fp32(B, size):
    """The norm is taken in 64 bits.  eps = 0, so that it does not swallow the smallest."""
    x = (matrices(1, 48, 80, "plain", 3).double() * size).float()
    out = torch.empty_like(x).cuda()
    B.qesgd_orthogonalize(x.cuda(), 48, 80, 1, R.USUAL, 0.0, out, ws_for(B, 48, 80, 1))
    want = R.newton_schulz(x[0].double().numpy(), R.USUAL, 0.0)
    assert np.linalg.norm(out[0].double().cpu().numpy() - want) <= allowed(x[0].double().numpy(), want, R.USUAL, 2.0 ** -24, 0.0)


def test_zeros_give_zeros_and_nan_stays_in_its_matrix(B):
    x = matrices(3, 40, 50, "plain", 1)
    x[0] = 0.0
    x[1, 3, 4] = float("nan")
    for eps in (0.0, EPS):
        out = torch.full((3, 40, 50), 9.0, device="cuda")
        B.qesgd_orthogonalize(x.cuda(), 40, 50, 3, R.USUAL, eps, out, ws_for(B, 40, 50, 3))
        assert (out[0] == 0).all()
        assert torch.isnan(out[1]).all()
        alone = torch.empty(1, 40, 50, device="cuda")
        B.qesgd_orthogonalize(x[2:].cuda().contiguous(), 40, 50, 1, R.USUAL, eps, alone, ws_for(B, 40, 50, 1))
        assert torch.equal(alone[0], out[2])


@pytest.mark.parametrize("momentum", [False, True])
@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("n,rows,cols", [(1, 30, 50), (2, 90, 60), (3, 64, 64), (1, 300, 517)])
def test_update(B, n, rows, cols, nesterov, momentum):
    """Three rounds: momentum bit for bit in fp32, the rest from the reference on the same momentum."""
    shape, mu, alpha = (n, rows, cols), 0.9, -0.05
    g = torch.Generator().manual_seed(rows)
    w, z, zs = (torch.randn(shape, generator=g) for _ in range(3))
    m = torch.randn(shape, generator=g) if momentum else None
    dev = {k: v.cuda() for k, v in (("w", w), ("z", z), ("zs", zs))}
    dm = m.cuda() if momentum else None
    step, u = torch.empty(shape, device="cuda"), torch.empty(shape, device="cuda")
    ws = ws_for(B, rows, cols, n)
    z64, zs64 = z.double().numpy(), zs.double().numpy()
    slack = 0.0
    for r in range(3):
        grad = matrices(n, rows, cols, "decay", r)
        B.qesgd_orthogonal_update(grad.cuda(), rows, cols, n, dm, mu, nesterov, R.USUAL, EPS, alpha, step, dev["z"], dev["w"], u, dev["zs"], ws)
        x = grad.numpy()
        if momentum:
            m = torch.from_numpy(np.float32(mu) * m.numpy() + x)
            assert torch.equal(dm.cpu(), m)
            x = x + np.float32(mu) * m.numpy() if nesterov else m.numpy()
        want = np.stack([R.newton_schulz(v.astype(np.float64)) for v in x]) * float(np.float32(alpha))
        limit = sum(allowed(v.astype(np.float64), want[i] / float(np.float32(alpha)), R.USUAL, 2.0 ** -24) for i, v in enumerate(x)) * abs(alpha)
        assert np.linalg.norm(step.double().cpu().numpy() - want) <= limit
        # z, u and zsum from the kernel's own step: fp32 sums, bit for bit
        s32 = step.cpu().numpy()
        z = z.numpy() + s32 if r == 0 else z + s32
        zs = zs.numpy() + z if r == 0 else zs + z
        assert np.array_equal(dev["z"].cpu().numpy(), z)
        assert np.array_equal(u.cpu().numpy(), w.numpy() + z)
        assert np.array_equal(dev["zs"].cpu().numpy(), zs)


def test_update_optional_outputs(B):
    shape = (1, 50, 70)
    g, z0 = matrices(*shape, "plain", 1).cuda(), torch.randn(shape).cuda()
    ws = ws_for(B, 50, 70, 1)
    step, z, u, w, zs = (torch.zeros(shape, device="cuda") for _ in range(5))
    z.copy_(z0)
    B.qesgd_orthogonal_update(g, 50, 70, 1, None, 0.0, False, R.USUAL, EPS, 2.0, step, z, w, u, zs, ws)
    only = torch.zeros(shape, device="cuda")
    B.qesgd_orthogonal_update(g, 50, 70, 1, None, 0.0, False, R.USUAL, EPS, 2.0, only, None, None, None, None, ws)
    assert torch.equal(only, step)
    only.copy_(z0)
    B.qesgd_orthogonal_update(g, 50, 70, 1, None, 0.0, False, R.USUAL, EPS, 2.0, None, only, None, None, None, ws)
    assert torch.equal(only, z)
    only.copy_(z0)
    B.qesgd_orthogonal_update(g, 50, 70, 1, None, 0.0, False, R.USUAL, EPS, 2.0, None, only, w, w, None, ws)       # in place
    assert torch.equal(w, u)


@pytest.mark.parametrize("n,rows,cols", [(2, 64, 64), (1, 200, 333), (1, 700, 130)])
def test_the_same_bits_again_on_another_stream_and_from_graphs(B, n, rows, cols):
    """Two captured graphs share the workspace, the program works between the replays."""
    x = matrices(n, rows, cols, "decay", 4).cuda()
    ws = ws_for(B, rows, cols, n)
    out, m = torch.zeros_like(x), torch.zeros_like(x)

    def work():
        B.qesgd_orthogonal_update(x, rows, cols, n, m, 0.5, True, R.USUAL, EPS, 1.0, out, None, None, None, None, ws)

    work()
    torch.cuda.synchronize()
    want = [out.clone()]
    for _ in range(4):
        work()
        torch.cuda.synchronize()
        want.append(out.clone())
    m.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    side.synchronize()
    assert torch.equal(out, want[0])
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for gr in graphs:
        with torch.cuda.graph(gr):
            work()
    m.zero_()
    for i in range(5):
        out.zero_()
        graphs[i & 1].replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i]), i
        assert np.isfinite(torch.randn(1 << 16, device="cuda").sum().item())
