"""Results of 16 bits whose experts' rows stay in fp32 between the product and the weighted sum: one rounding, against 64 bits."""
import numpy as np
import pytest
import torch

import expert_reference as X
from expert_reference import ONE, host
from test_gpu_route import COMBINE, slots_for

pytestmark = pytest.mark.gpu
HALVES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def B():
    from paper_1901_03040_amd import binding
    assert torch.cuda.is_available()
    binding.lib()
    return binding


@pytest.mark.parametrize("t", HALVES, ids=["bf16", "f16"])
@pytest.mark.parametrize("T,k,N", COMBINE + [(40, 2, 4), (40, 2, 5), (40, 2, 12), (7, 12, 300)])
def test_combine_and_its_gradients(B, T, k, N, t):
    R = T * k + 3
    g = torch.Generator().manual_seed(T + N)
    # rows that are longer than N and begin at any element, what lies between them NaN
    rows = torch.full((R * (N + 3) + 5,), float("nan"))
    r32 = torch.randn(R, N, generator=g)
    torch.as_strided(rows, (R, N), (N + 3, 1), 1).copy_(r32)
    rows, r64 = rows.cuda()[1:], r32.double().numpy()
    dy = torch.randn(T * (N + 1) + 5, generator=g).to(t).cuda()[3:]
    d64 = host(torch.as_strided(dy, (T, N), (N + 1, 1)))
    gates = torch.rand(T, k, generator=g).cuda()
    slots = slots_for(T, k, R, N)
    s = torch.from_numpy(slots).cuda()
    for weights in (gates, None):
        out = torch.full((T, N + 2), 9.0, dtype=t, device="cuda")
        B.qesgd_combine(rows, N + 3, R, s, weights, T, k, N, out, N + 2)
        want, mag = X.combine(r64, slots, None if weights is None else host(weights), T, k)
        assert (out[:, N:] == 9.0).all()
        # k products and sums in fp32, one rounding to t
        assert (np.abs(host(out)[:, :N] - want) <= (k + 1) * ONE * mag + X.rounded(want, t)).all()
    drows = torch.full((R, N + 2), 9.0, dtype=t, device="cuda")
    dgates = torch.full((T * k + 4,), 9.0, device="cuda")
    B.qesgd_combine_backward(dy, N + 1, rows, N + 3, R, s, gates, T, k, N, drows, N + 2, dgates)
    wg, size = np.zeros(T * k), np.zeros(T * k)
    for i, slot in enumerate(slots):
        if slot >= 0:
            wg[i], size[i] = d64[i // k] @ r64[slot], np.abs(d64[i // k]) @ np.abs(r64[slot])
    assert (dgates[T * k:] == 9.0).all()
    assert (np.abs(host(dgates)[:T * k] - wg) <= (N + 1) * ONE * size).all()
    # the rows' gradients have nothing of the rows
    alone = torch.full_like(drows, 9.0)
    B.qesgd_combine_backward(dy, N + 1, None, 0, R, s, gates, T, k, N, alone, N + 2, None)
    assert torch.equal(alone, drows)
    one = torch.empty_like(dgates)
    B.qesgd_combine_backward(dy, N + 1, rows, N + 3, R, s, None, T, k, N, None, 0, one)
    assert torch.equal(one[:T * k], dgates[:T * k])


@pytest.mark.parametrize("t", HALVES, ids=["bf16", "f16"])
def test_sums_of_large_calls(B, t):
    """Results written past the caches, and rows read so: 600 MB of rows, the reference on the GPU a part at a time."""
    T, k, N = 24_000, 2, 3136
    g = torch.Generator(device="cuda").manual_seed(1)
    rows, dy = torch.randn(T * k, N, device="cuda", generator=g), torch.randn(T, N, device="cuda", generator=g).to(t)
    gates = torch.rand(T, k, device="cuda", generator=g)
    slots = torch.randperm(T * k, device="cuda", generator=g).int()
    out, drows, dgates = torch.empty(T, N, dtype=t, device="cuda"), torch.empty(T * k, N, dtype=t, device="cuda"), torch.empty(T, k, device="cuda")
    B.qesgd_combine(rows, N, T * k, slots, gates, T, k, N, out, N)
    B.qesgd_combine_backward(dy, N, rows, N, T * k, slots, gates, T, k, N, drows, N, dgates)
    half, least = X.HALF_STEP[t] * (1 + 2.0 ** -10), X.LEAST[t]
    for lo in range(0, T, 4000):
        at = slots.view(T, k)[lo:lo + 4000].long()
        picked, d, w = rows[at].double(), dy[lo:lo + 4000].double()[:, None], gates[lo:lo + 4000].double()[:, :, None]
        terms = picked * w
        want = terms.sum(1)
        assert bool(((out[lo:lo + 4000].double() - want).abs() <= (k + 1) * ONE * terms.abs().sum(1) + half * want.abs() + least).all()), lo
        want = w * d
        assert bool(((drows[at].double() - want).abs() <= (ONE + half) * want.abs() + least).all()), lo
        terms = picked * d
        assert bool(((dgates[lo:lo + 4000].double() - terms.sum(2)).abs() <= (N + 1) * ONE * terms.abs().sum(2)).all()), lo


def test_what_is_refused(B):
    T, k, N, R = 4, 2, 16, 8
    i32 = dict(dtype=torch.int32, device="cuda")
    rows, half = torch.zeros(R, N, device="cuda"), torch.zeros(R, N, dtype=torch.bfloat16, device="cuda")
    slots, gates, dg = torch.arange(R, **i32), torch.ones(T, k, device="cuda"), torch.zeros(T, k, device="cuda")
    # rows of 16 bits beside another type, and the gradients in the place of rows of another type
    for out in (torch.zeros(T, N, device="cuda"), torch.zeros(T, N, dtype=torch.float16, device="cuda")):
        with pytest.raises(B.QesgdError):
            B.qesgd_combine(half, N, R, slots, gates, T, k, N, out, N)
        with pytest.raises(B.QesgdError):
            B.qesgd_combine_backward(out, N, half, N, R, slots, gates, T, k, N, None, 0, dg)
    dy = torch.zeros(T, N, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(B.QesgdError) as e:
        B.qesgd_combine_backward(dy, N, rows, N, R, slots, gates, T, k, N, rows.reshape(-1).view(torch.bfloat16), N, dg)
    assert e.value.code == B.ERR_DTYPE
    with pytest.raises(ValueError):                             # half as many rows as the call reads
        B.qesgd_combine(rows[:4], N, R, slots, gates, T, k, N, dy, N)


def test_from_a_graph(B):
    T, k, N = 50, 3, 200
    R = T * k
    rows, dy = torch.randn(R, N, device="cuda"), torch.randn(T, N, device="cuda").to(torch.bfloat16)
    slots, gates = torch.from_numpy(slots_for(T, k, R, 3)).cuda(), torch.rand(T, k, device="cuda")
    out, drows, dg = torch.zeros_like(dy), torch.zeros(R, N, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, k, device="cuda")

    def work():
        B.qesgd_combine(rows, N, R, slots, gates, T, k, N, out, N)
        B.qesgd_combine_backward(dy, N, rows, N, R, slots, gates, T, k, N, drows, N, dg)

    work()
    torch.cuda.synchronize()
    want = [v.clone() for v in (out, drows, dg)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for i in range(4):
        for v in (out, drows, dg):
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(v, w) for v, w in zip((out, drows, dg), want)), i
        assert np.isfinite(torch.randn(1 << 16, device="cuda").sum().item())
