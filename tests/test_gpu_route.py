"""The router and the weighted sum of the experts' rows on the GPU against the 64-bit reference: choices, places and order exactly, gates,
sums and gradients within their roundings."""
import numpy as np
import pytest
import torch

import expert_reference as X
from expert_reference import HALF_STEP, ONE, TYPES, host

pytestmark = pytest.mark.gpu
GUARD = -77


@pytest.fixture(scope="module")
def B():
    from paper_1901_03040_amd import binding
    assert torch.cuda.is_available()
    binding.lib()
    return binding


def logits(T, E, dtype, seed, closed=0.0, ties=False):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, E, generator=g) * 2
    if ties:
        x = torch.round(x)                                     # few values: ties in every row
    if closed:
        u = torch.rand(T, 1, generator=g)
        x[(u < closed) | ((u < 2 * closed) & (torch.rand(T, E, generator=g) < 0.7))] = -float("inf")
    return x.to(dtype)


def run_route(B, x, k, all_, ld=None):
    T, E = x.shape
    pairs = T * k
    out = dict(experts=torch.full((pairs + 8,), GUARD, dtype=torch.int32), gates=torch.full((pairs + 8,), float(GUARD)),
               offsets=torch.full((E + 9,), GUARD, dtype=torch.int32), order=torch.full((pairs + 8,), GUARD, dtype=torch.int32),
               slots=torch.full((pairs + 8,), GUARD, dtype=torch.int32))
    out = {n: t.cuda() for n, t in out.items()}
    ws = B.alloc_workspace(B.qesgd_route_workspace_bytes(T, E, k))
    B.qesgd_route(x, ld or x.stride(0), T, E, k, B.GATE_ALL if all_ else B.GATE_CHOSEN, *(out[n] for n in ("experts", "gates", "offsets", "order", "slots")),
                  workspace=ws)
    for n, count in (("experts", pairs), ("gates", pairs), ("offsets", E + 1), ("order", pairs), ("slots", pairs)):
        assert (out[n][count:] == GUARD).all(), n
        out[n] = out[n][:count]
    return out


def check_route(x, k, all_, out):
    T, E = x.shape
    l = host(x)
    experts, gates, offsets, order, slots = X.route(l, k, all_)
    assert np.array_equal(out["experts"].cpu().numpy().reshape(T, k), experts)
    assert np.array_equal(out["offsets"].cpu().numpy(), offsets)
    got = out["order"].cpu().numpy()
    assert np.array_equal(got[:len(order)], order) and (got[len(order):] == GUARD).all()
    assert np.array_equal(out["slots"].cpu().numpy(), slots)
    # a gate's error is its row's softmax error at most: over the chosen there are fewer terms
    limit = gates * X.softmax_error(l).max(1, keepdims=True) + 2.0 ** -140
    off = np.abs(host(out["gates"]).reshape(T, k) - gates)
    assert (off <= limit).all(), (off - limit).max()


SHAPES = [(1, 1, 1), (1, 8, 8), (1, 64, 2), (3, 5, 2), (2, 16, 16), (7, 9, 1), (63, 33, 4), (65, 64, 2), (129, 65, 3), (500, 17, 16), (300, 130, 8),
          (257, 257, 6), (40, 600, 5), (20, 1024, 16), (4100, 4, 2), (20_011, 12, 3), (9000, 1000, 2),
          (701, 160, 16), (135, 192, 8), (501, 224, 7), (301, 300, 5), (300, 330, 4), (401, 384, 6), (333, 512, 16), (201, 640, 9), (400, 768, 3), (299, 1024, 12)]


@pytest.mark.parametrize("all_", [True, False], ids=["all", "chosen"])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T,E,k", SHAPES)
def test_route(B, T, E, k, dtype, all_):
    x = logits(T, E, TYPES[dtype], T + E, ties=T % 2 == 1).cuda()
    check_route(x, k, all_, run_route(B, x, k, all_))


@pytest.mark.parametrize("all_", [True, False], ids=["all", "chosen"])
@pytest.mark.parametrize("T,E,k", [(1, 8, 3), (70, 8, 8), (200, 64, 4), (1000, 257, 6), (5000, 33, 2), (300, 200, 16), (211, 512, 9), (150, 1024, 5)])
def test_closed_experts_and_padded_tokens(B, T, E, k, all_):
    x = logits(T, E, torch.float32, 3, closed=0.3).cuda()
    check_route(x, k, all_, run_route(B, x, k, all_))
    x.fill_(-float("inf"))
    out = run_route(B, x, k, all_)
    assert (out["experts"] == -1).all() and (out["slots"] == -1).all() and not out["gates"].any() and not out["offsets"].any()
    assert (out["order"] == GUARD).all()


def test_lowest_values_zeros_of_both_signs_nan_and_infinity(B):
    low = torch.finfo(torch.float32).min
    inf, nan = float("inf"), float("nan")
    x = torch.tensor([[low, low, low, low], [low, 0.0, -0.0, low], [-0.0, 0.0, -1.0, -2.0], [1e-45, -1e-45, 0.0, -inf], [88.0, -88.0, 300.0, -300.0],
                      [1.0, nan, 2.0, 3.0], [nan, nan, -inf, 0.0], [inf, 1.0, 2.0, 0.0], [-inf, -inf, 5.0, -inf]]).cuda()
    for all_ in (True, False):
        out = run_route(B, x, 3, all_)
        e, g = out["experts"].cpu().numpy().reshape(-1, 3), host(out["gates"]).reshape(-1, 3)
        check_route(x[:5], 3, all_, run_route(B, x[:5], 3, all_))
        assert e[:5].tolist() == [[0, 1, 2], [1, 2, 0], [0, 1, 2], [0, 2, 1], [2, 0, 1]]
        assert e[5:].tolist() == [[1, 3, 2], [0, 1, 3], [0, 2, 1], [2, -1, -1]]     # a NaN counts as the largest
        assert np.isnan(g[5:8]).all() and g[8].tolist() == [1.0, 0.0, 0.0]


@pytest.mark.parametrize("dtype", list(TYPES))
def test_strides_and_offsets(B, dtype):
    whole = logits(50, 40, TYPES[dtype], 1).cuda()
    view = whole[:, 3:26]
    out = run_route(B, view, 4, True)
    check_route(view.contiguous(), 4, True, out)
    # one row: its stride is nothing to the call
    check_route(view[:1].contiguous(), 4, True, run_route(B, view[:1], 4, True, ld=0))


@pytest.mark.parametrize("all_", [True, False], ids=["all", "chosen"])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T,E,k", SHAPES)
def test_route_backward(B, T, E, k, dtype, all_):
    t = TYPES[dtype]
    x = logits(T, E, t, T * 3 + E, closed=0.1).cuda()
    out = run_route(B, x, k, all_)
    dg = torch.randn(T, k, generator=torch.Generator().manual_seed(T))
    ld = E + 3
    dl = torch.full((T, ld), 5.0, dtype=t, device="cuda")
    B.qesgd_route_backward(x if all_ else None, E, T, E, k, B.GATE_ALL if all_ else B.GATE_CHOSEN, out["experts"], out["gates"], dg.cuda(), dl, ld)
    assert (dl[:, E:] == 5.0).all()
    l, experts, gates = host(x), out["experts"].cpu().numpy().reshape(T, k), host(out["gates"]).reshape(T, k)
    want, mag = X.route_backward(l, experts, gates, dg.double().numpy(), all_)
    # k products and sums twice, the probability's own error where it is worked out anew, one rounding of the result
    limit = mag * ((2 * k + 6) * ONE + (X.softmax_error(l) if all_ else 0.0)) + X.rounded(want, t) + 2.0 ** -140
    off = np.abs(host(dl)[:, :E] - want)
    assert (off <= limit).all(), (off - limit).max()
    assert (host(dl)[:, :E][l == -np.inf] == 0).all()


def test_route_backward_against_differences(B):
    """The whole router, logits to gates, as a function of one logit after the other.  Differences in 64 bits of the formula the kernel's gates are
    checked against above."""
    T, E, k, h = 6, 11, 3, 1e-5
    x = logits(T, E, torch.float32, 5).cuda()
    dg = torch.randn(T, k, generator=torch.Generator().manual_seed(9))
    for all_ in (True, False):
        out = run_route(B, x, k, all_)
        dl = torch.empty_like(x)
        B.qesgd_route_backward(x, E, T, E, k, B.GATE_ALL if all_ else B.GATE_CHOSEN, out["experts"], out["gates"], dg.cuda(), dl, E)
        l = host(x)
        for e in range(E):
            up, down = l.copy(), l.copy()
            up[:, e] += h
            down[:, e] -= h
            diff = ((X.route(up, k, all_)[1] - X.route(down, k, all_)[1]) * dg.double().numpy()).sum(1) / (2 * h)
            # third derivatives of a softmax are at most 1: h^2 / 6 times the sum of |dgates|, and fp32's roundings
            limit = (h * h + 40 * ONE) * np.abs(dg.double().numpy()).sum(1) + 1e-10
            assert (np.abs(host(dl)[:, e] - diff) <= limit).all()


def test_the_same_expert_twice_and_choices_out_of_range(B):
    """A caller's own choices: contributions to one expert add up, numbers that are none are left out."""
    x = logits(4, 6, torch.float32, 2).cuda()
    experts = torch.tensor([[1, 1], [5, -1], [6, 0], [-7, 1 << 30]], dtype=torch.int32)
    gates, dg = torch.rand(4, 2), torch.randn(4, 2)
    for all_ in (True, False):
        dl = torch.empty_like(x)
        B.qesgd_route_backward(x, 6, 4, 6, 2, B.GATE_ALL if all_ else B.GATE_CHOSEN, experts.cuda(), gates.cuda(), dg.cuda(), dl, 6)
        want, mag = X.route_backward(host(x), experts.numpy(), gates.double().numpy(), dg.double().numpy(), all_)
        assert (np.abs(host(dl) - want) <= mag * 40 * ONE + np.abs(want) * ONE).all()


# ---- the weighted sum ---------------------------------------------------------

COMBINE = [(1, 1, 1), (1, 2, 3), (5, 3, 7), (33, 2, 64), (17, 4, 129), (100, 1, 1000), (3, 16, 515), (9, 5, 2050), (2, 8, 4097), (300, 2, 40)]


def slots_for(T, k, R, seed, missing=0.2):
    rng = np.random.default_rng(seed)
    s = rng.permutation(R)[:T * k].astype(np.int32)
    s[rng.random(T * k) < missing] = -1
    return s


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T,k,N", COMBINE)
def test_combine_and_its_gradients(B, T, k, N, dtype):
    t, R = TYPES[dtype], T * k + 3
    g = torch.Generator().manual_seed(T + N)
    # rows that are longer than N and begin at any element
    rows = torch.randn(R * (N + 3) + 5, generator=g).to(t).cuda()[1:]
    dy = torch.randn(T * (N + 1) + 5, generator=g).to(t).cuda()[3:]
    gates = torch.rand(T, k, generator=g).cuda()
    slots = slots_for(T, k, R, N)
    s = torch.from_numpy(slots).cuda()
    r64 = host(torch.as_strided(rows, (R, N), (N + 3, 1)))
    d64 = host(torch.as_strided(dy, (T, N), (N + 1, 1)))
    for weights in (gates, None):
        out = torch.full((T, N + 2), 9.0, dtype=t, device="cuda")
        B.qesgd_combine(rows, N + 3, R, s, weights, T, k, N, out, N + 2)
        want, mag = X.combine(r64, slots, None if weights is None else host(weights), T, k)
        assert (out[:, N:] == 9.0).all()
        assert (np.abs(host(out)[:, :N] - want) <= (k + 1) * ONE * mag + X.rounded(want, t)).all()
    drows = torch.full((R, N + 2), 9.0, dtype=t, device="cuda")
    dgates = torch.full((T * k + 4,), 9.0, device="cuda")
    B.qesgd_combine_backward(dy, N + 1, rows, N + 3, R, s, gates, T, k, N, drows, N + 2, dgates)
    want = np.full((R, N), 9.0)
    wg, size = np.zeros(T * k), np.zeros(T * k)
    for i, slot in enumerate(slots):
        if slot >= 0:
            want[slot] = host(gates).reshape(-1)[i] * d64[i // k]
            wg[i], size[i] = d64[i // k] @ r64[slot], np.abs(d64[i // k]) @ np.abs(r64[slot])
    assert (drows[:, N:] == 9.0).all() and (dgates[T * k:] == 9.0).all()
    assert (np.abs(host(drows)[:, :N] - want) <= ONE * np.abs(want) + X.rounded(want, t)).all()
    # a sum of N products in any order
    assert (np.abs(host(dgates)[:T * k] - wg) <= (N + 1) * ONE * size).all()
    one = torch.empty_like(dgates)
    B.qesgd_combine_backward(dy, N + 1, rows, N + 3, R, s, None, T, k, N, None, 0, one)
    assert torch.equal(one[:T * k], dgates[:T * k])
    alone = torch.full_like(drows, 9.0)
    B.qesgd_combine_backward(dy, N + 1, None, 0, R, s, gates, T, k, N, alone, N + 2, None)
    assert torch.equal(alone, drows)


def test_combine_without_slots_and_in_place(B):
    T, k, N = 12, 3, 77
    g = torch.Generator().manual_seed(1)
    rows, gates, dy = torch.randn(T * k, N, generator=g).cuda(), torch.rand(T, k, generator=g).cuda(), torch.randn(T, N, generator=g).cuda()
    slots = torch.arange(T * k, dtype=torch.int32).cuda()
    a, b = torch.empty(T, N, device="cuda"), torch.empty(T, N, device="cuda")
    B.qesgd_combine(rows, N, T * k, slots, gates, T, k, N, a, N)
    B.qesgd_combine(rows, N, T * k, None, gates, T, k, N, b, N)
    assert torch.equal(a, b)
    dg, dg2, d = torch.empty(T, k, device="cuda"), torch.empty(T, k, device="cuda"), torch.empty_like(rows)
    B.qesgd_combine_backward(dy, N, rows, N, T * k, slots, gates, T, k, N, d, N, dg)
    B.qesgd_combine_backward(dy, N, rows, N, T * k, None, gates, T, k, N, rows, N, dg2)      # the gradients take the rows' place
    assert torch.equal(rows, d) and torch.equal(dg, dg2)


def test_combine_leaves_out_slots_beyond_the_rows(B):
    T, k, N, R = 5, 2, 40, 7
    rows, gates, dy = torch.randn(R, N).cuda(), torch.rand(T, k).cuda(), torch.randn(T, N).cuda()
    slots = np.array([0, 7, 6, -1, 1 << 30, -(1 << 31), 3, 2, 5, 8], np.int32)
    s = torch.from_numpy(slots).cuda()
    out, room = torch.empty(T, N, device="cuda"), torch.full((R + 4, N), 9.0, device="cuda")
    B.qesgd_combine(rows, N, R, s, gates, T, k, N, out, N)
    want, mag = X.combine(host(rows), slots, host(gates), T, k)
    assert (np.abs(host(out) - want) <= 4 * ONE * mag + ONE * np.abs(want)).all()
    dg = torch.full((T, k), 9.0, device="cuda")
    B.qesgd_combine_backward(dy, N, rows, N, R, s, gates, T, k, N, room[2:], N, dg)
    named = [x for x in slots if 0 <= x < R]
    assert (room[[0, 1, R + 2, R + 3]] == 9.0).all() and (room[2:][[r for r in range(R) if r not in named]] == 9.0).all()
    assert (dg.reshape(-1)[[i for i, x in enumerate(slots) if not 0 <= x < R]] == 0).all()


def test_nan_in_a_row_without_a_token(B):
    """Rows that no pair names are not read: a NaN there stays there."""
    rows = torch.full((4, 8), float("nan")).cuda()
    rows[2] = 1.0
    out = torch.empty(2, 8, device="cuda")
    B.qesgd_combine(rows, 8, 4, torch.tensor([2, -1, -1, -1], dtype=torch.int32).cuda(), torch.tensor([[0.5, 0.0], [0.0, 0.0]]).cuda(), 2, 2, 8, out, 8)
    assert (out[0] == 0.5).all() and (out[1] == 0.0).all()


def test_router_on_a_side_stream_from_a_graph_and_again(B):
    T, E, k = 3000, 40, 3
    x = logits(T, E, torch.bfloat16, 8, closed=0.1).cuda()
    dg = torch.randn(T, k, device="cuda")
    want = run_route(B, x, k, True)
    ws = B.alloc_workspace(B.qesgd_route_workspace_bytes(T, E, k))
    out = {n: torch.zeros_like(v) for n, v in want.items()}
    dl = torch.empty_like(x)

    def work():
        B.qesgd_route(x, E, T, E, k, B.GATE_ALL, *(out[n] for n in ("experts", "gates", "offsets", "order", "slots")), workspace=ws)
        B.qesgd_route_backward(x, E, T, E, k, B.GATE_ALL, out["experts"], out["gates"], dg, dl, E)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    side.synchronize()
    first = dl.clone()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for graph in graphs:
        with torch.cuda.graph(graph):
            work()
    for i in range(4):
        for v in out.values():
            v.fill_(GUARD)
        dl.zero_()
        graphs[i & 1].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[n], want[n]) for n in out) and torch.equal(dl, first), i
