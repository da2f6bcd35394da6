"""The operators for layers of experts together, as the epoch loop runs them: router, rows to their experts and back, gradients, round."""
import numpy as np
import pytest
import torch

import expert_reference as X
import matrix_reference as R
from expert_reference import HALF_STEP, ONE, host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    from paper_1901_03040_amd import epoch_loop
    assert torch.cuda.is_available()
    return epoch_loop


def make(L, E, out, inn, K=2, seed=1234567, **options):
    w = torch.randn(E, out, inn, generator=torch.Generator().manual_seed(E + out)) / inn ** 0.5
    return L.QesgdExpertLoop(w.cuda(), K, seed, **options)


def inputs(T, E, inn, dtype, seed, closed=True):
    g = torch.Generator().manual_seed(seed)
    x, logits = torch.randn(T, inn, generator=g).to(dtype), torch.randn(T, E, generator=g) * 2
    if closed and T > 3:
        logits[1] = -float("inf")                              # padding
        logits[2, 1:] = -float("inf")
    return x.cuda(), logits.cuda()


def close(got, want, mag, dtype, terms):
    assert (np.abs(host(got) - want) <= terms * ONE * mag + X.rounded(want, dtype) * 1.001).all()


@pytest.mark.parametrize("kind", [0, 1], ids=["all", "chosen"])
@pytest.mark.parametrize("E,out,inn,T,k,dtype", [(4, 40, 72, 50, 2, torch.float32), (5, 130, 64, 33, 3, torch.bfloat16), (70, 24, 40, 90, 1, torch.float32),
                                                 (3, 33, 257, 1, 2, torch.float16)])
def test_layer_and_round(L, E, out, inn, T, k, dtype, kind):
    K, seed = 2, 1234567
    loop = make(L, E, out, inn, K, seed, choices=k, gate_kind=kind)
    z, zsum, m = np.zeros((E, out, inn), np.float32), np.zeros((E, out, inn), np.float32), np.zeros((E, out, inn), np.float32)
    for rnd in range(2):
        u = host(loop.u)
        qu, qut = np.stack([X.q(v) for v in u]), np.stack([X.q(v.T) for v in u])
        grads = torch.empty(K, E, out, inn, device="cuda")
        for worker in range(K):
            x, logits = inputs(T, E, inn, dtype, 10 * rnd + worker)
            dy = (torch.randn(T, out, generator=torch.Generator().manual_seed(worker)) * 1e-2).to(dtype).cuda()
            y, saved = loop.forward(x, logits)
            dx, dlogits, dw = loop.backward(dy, saved, worker=worker)
            grads[worker] = dw
            assert y.dtype == dtype and dx.dtype == dtype and dlogits.dtype == logits.dtype and dw.dtype == torch.float32
            assert torch.equal(y, loop.forward(x, logits, gradients=False)[0])
            # each step from what the steps before it gave, so that one rounding is counted at a time
            _, got_rows, _, got_experts, got_gates, got_offsets, got_slots, _, _ = saved
            l = host(logits)
            experts, gates, offsets, order, slots = X.route(l, k, kind == 0)
            assert np.array_equal(host(got_experts).reshape(T, k), experts) and np.array_equal(host(got_offsets), offsets)
            assert np.array_equal(host(got_slots).reshape(-1), slots)
            assert (np.abs(host(got_gates) - gates) <= gates * X.softmax_error(l).max(1, keepdims=True) + 2.0 ** -140).all()
            n, gates = len(order), host(got_gates)
            x64, rows = host(x), host(got_rows)
            a = X.q(x64[order // k])
            for e in range(E):
                s = slice(offsets[e], offsets[e + 1])
                close(got_rows[s], a[s] @ qu[e].T, np.abs(a[s]) @ np.abs(qu[e]).T, dtype, inn)
            want, mag = X.combine(rows, slots, gates, T, k)
            close(y, want, mag, dtype, k + 1)
            # backward: the rows' gradients as they are stored, then rounded without bias
            d64, flat = host(dy), gates.reshape(-1)
            drows = torch.from_numpy((flat[order, None].astype(np.float32) * d64[order // k].astype(np.float32))).to(dtype).double().numpy()
            b = X.q(np.concatenate((drows, np.zeros((T * k - n, out)))), True, seed, loop.round_id, K + worker)[:n]
            dxrows, size = np.zeros((T * k, inn)), np.zeros((T * k, inn))
            columns = X.group_columns(T * k, E)
            turned, begin, _ = X.padded(drows, offsets, columns)
            turned_x, _, _ = X.padded(x64[order // k], offsets, columns)
            bt, at = X.q(turned, True, seed, loop.round_id, K + worker), X.q(turned_x)
            for e in range(E):
                s, c = slice(offsets[e], offsets[e + 1]), slice(begin[e], begin[e] + offsets[e + 1] - offsets[e])
                dxrows[s], size[s] = b[s] @ qut[e].T, np.abs(b[s]) @ np.abs(qut[e]).T
                close(dw[e], bt[:, c] @ at[:, c].T, np.abs(bt[:, c]) @ np.abs(at[:, c]).T, torch.float32, T)
            want, mag = X.combine(dxrows, slots, None, T, k)
            # the rows of dx are stored in dtype before they are added
            spare = X.combine(X.rounded(dxrows, dtype) + out * ONE * size, slots, None, T, k)[0]
            assert (np.abs(host(dx) - want) <= spare + (k + 1) * ONE * (mag + spare) + X.rounded(np.abs(want) + spare, dtype)).all()
            dgates, dmag = np.zeros(T * k), np.zeros(T * k)
            dgates[order] = (d64[order // k] * rows[:n]).sum(1)
            dmag[order] = (out + 1) * ONE * np.abs(d64[order // k] * rows[:n]).sum(1)
            want, mag = X.route_backward(l, experts, gates, dgates.reshape(T, k), kind == 0)
            spare = X.route_backward(l, experts, np.abs(gates), dmag.reshape(T, k), kind == 0)[1]
            assert (np.abs(host(dlogits) - want) <= spare + mag * ((2 * k + 6) * ONE + X.softmax_error(l)) + ONE * np.abs(want) + 1e-30).all()
        acc = np.zeros((E * out, inn), np.float32)
        for worker in range(K):
            acc = acc + X.q(host(grads[worker]).reshape(E * out, inn), True, seed, loop.round_id, worker).astype(np.float32)
        mean = (acc / np.float32(K)).reshape(E, out, inn)
        before = loop.z.cpu().numpy().copy()
        loop.orthogonal_round(grads, 0.02, last=rnd == 1)
        assert np.array_equal(loop.mean.cpu().numpy(), mean)
        m = np.float32(0.95) * m + mean
        assert np.array_equal(loop.momentum.cpu().numpy(), m)
        look = (mean + np.float32(0.95) * m).astype(np.float64)
        z = loop.z.cpu().numpy()
        for e in range(E):
            want = -0.02 * R.newton_schulz(look[e])
            moved = R.newton_schulz(look[e], noise=2.0 ** -22 / np.sqrt(max(out, inn)), rng=np.random.default_rng(0)) * -0.02
            limit = 8 * (np.linalg.norm(moved - want) + 2.0 ** -22 * np.linalg.norm(want)) + 2.0 ** -23 * (np.linalg.norm(z[e]) + np.linalg.norm(before[e]))
            assert np.linalg.norm(z[e].astype(np.float64) - before[e] - want) <= limit
        assert np.array_equal(loop.u.cpu().numpy(), loop.w.cpu().numpy() + z)
        zsum = zsum + z if rnd == 0 else zsum
        assert np.array_equal(loop.zsum.cpu().numpy(), zsum)
    w32 = loop.w.cpu().numpy()
    loop.end_epoch()
    assert np.array_equal(loop.w.cpu().numpy(), w32 + zsum / np.float32(2))


def test_next_tokens(L):
    """A few tokens' rows as they are: against 64 bits with the packed parameters, and a token without experts gives zeros."""
    E, out, inn, T, k = 6, 70, 130, 9, 2
    loop = make(L, E, out, inn, choices=k)
    x, logits = inputs(T, E, inn, torch.float32, 3)
    y = loop.next_tokens(x, logits)
    experts, gates, *_ = X.route(host(logits), k, False)
    x64 = host(x)
    want, mag = np.zeros((T, out)), np.zeros((T, out))
    for t in range(T):
        for j in range(k):
            if experts[t, j] >= 0:
                w = X.q(host(loop.u[experts[t, j]]))
                want[t] += gates[t, j] * (w @ x64[t])
                mag[t] += gates[t, j] * (np.abs(w) @ np.abs(x64[t]))
    assert (np.abs(host(y) - want) <= (3 * inn + E + 130) * ONE * mag).all()
    assert not y[1].any()
    one = L.QesgdMatrixLoop(loop.u[0].clone(), 1, 5)
    w = X.q(host(one.u))
    for rows in (x[:1], x[::2], x.t().contiguous().t()):
        got = one.next_tokens(rows)
        assert (np.abs(host(got) - host(rows) @ w.T) <= (3 * inn + 3) * ONE * (np.abs(host(rows)) @ np.abs(w).T)).all()


def test_views_and_broadcast_gradients(L):
    E, out, inn, T = 4, 48, 80, 20
    loop = make(L, E, out, inn)
    x, logits = inputs(T, E, inn, torch.float32, 1)
    wide = torch.zeros(T, 200, device="cuda")
    wide[:, 7:87] = x
    wl = torch.zeros(T, 9, device="cuda")
    wl[:, 2:6] = logits
    y, saved = loop.forward(x, logits)
    for a, b in ((wide[:, 7:87], wl[:, 2:6]), (x.t().contiguous().t(), logits.t().contiguous().t())):
        got, kept = loop.forward(a, b)
        assert torch.equal(got, y)
    for dy in (torch.full((), 0.37, device="cuda").expand(T, out), torch.randn(out, device="cuda").expand(T, out)):
        for got, want in zip(loop.backward(dy, saved), loop.backward(dy.contiguous(), saved)):
            assert torch.equal(got, want)


def test_parameters_that_are_gone(L):
    loop = make(L, 3, 32, 64)
    x, logits = inputs(8, 3, 64, torch.float32, 1)
    _, saved = loop.forward(x, logits)
    loop.begin_epoch()
    with pytest.raises(AssertionError):
        loop.backward(torch.zeros(8, 32, device="cuda"), saved)


def test_a_layer_and_a_round_from_a_graph(L):
    """Captured once and replayed with other tokens each time: every replay equals the eager calls, whatever the groups' sizes."""
    K, E, out, inn, T = 2, 5, 96, 160, 50

    def start():
        loop = make(L, E, out, inn, K, 11)
        x, logits = inputs(T, E, inn, torch.float32, 3)
        dy = torch.randn(T, out, generator=torch.Generator().manual_seed(4)).cuda()
        return loop, x, logits, dy, torch.empty(K, E, out, inn, device="cuda")

    def step(loop, x, logits, dy, grads):
        loop.round_id = 0                                       # part of the captured calls
        y, saved = loop.forward(x, logits)
        for k in range(K):
            dx, dlogits, dw = loop.backward(dy, saved, worker=k)
            grads[k].copy_(dw)
        loop.orthogonal_round(grads, 0.1)
        return y, dx, dlogits

    def turn(state, i):
        x, logits = inputs(T, E, inn, torch.float32, 20 + i)
        state[1].copy_(x)
        state[2].copy_(logits)

    eager, want = start(), []
    for i in range(4):
        turn(eager, i)
        out_ = step(*eager)
        want.append([t.clone() for t in (*out_, eager[0].u, eager[0].zsum, eager[0].momentum)])
    state = start()
    step(*state)
    fresh = start()[0]
    for name in ("u", "z", "zsum", "momentum", "packed_u", "packed_ut"):
        getattr(state[0], name).copy_(getattr(fresh, name))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out_ = step(*state)
    for i in range(4):
        turn(state, i)
        graph.replay()
        torch.cuda.synchronize()
        for got, ref in zip((*out_, state[0].u, state[0].zsum, state[0].momentum), want[i]):
            assert torch.equal(got, ref), i
        assert np.isfinite(torch.randn(1 << 16, device="cuda").sum().item())
