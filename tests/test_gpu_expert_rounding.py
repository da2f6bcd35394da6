"""A layer of experts with 16-bit activations: results of one rounding, from 64 bits and not from what a kernel stored between; and the loop's rows in
the activations' type, for whoever asks for them."""
import numpy as np
import pytest
import torch

import expert_reference as X
from expert_reference import ONE, host
from test_gpu_expert_loop import inputs, make

pytestmark = pytest.mark.gpu
HALVES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def L():
    from paper_1901_03040_amd import epoch_loop
    assert torch.cuda.is_available()
    return epoch_loop


def layer(loop, x, gates, experts, quantised=True):
    """sum_j gates_j Q(x) Q(u_e)^T in 64 bits, and the sum of the magnitudes."""
    a = X.q(host(x)) if quantised else host(x)
    w = np.stack([X.q(v) for v in host(loop.u)])
    want, mag = np.zeros((len(a), loop.out)), np.zeros((len(a), loop.out))
    for t, row in enumerate(experts):
        for j, e in enumerate(row):
            if e >= 0:
                want[t] += gates[t, j] * (w[e] @ a[t])
                mag[t] += gates[t, j] * (np.abs(w[e]) @ np.abs(a[t]))
    return want, mag


@pytest.mark.parametrize("t", HALVES, ids=["bf16", "f16"])
@pytest.mark.parametrize("E,out,inn,T,k", [(5, 130, 64, 33, 3), (3, 33, 257, 1, 2), (4, 300, 500, 700, 2)])
def test_forward_and_next_tokens_are_rounded_once(L, E, out, inn, T, k, t):
    loop = make(L, E, out, inn, choices=k)
    x, logits = inputs(T, E, inn, t, 3)
    y, saved = loop.forward(x, logits)
    gates, experts = host(saved[4]).reshape(T, k), saved[3].cpu().numpy().reshape(T, k)
    assert y.dtype == t
    want, mag = layer(loop, x, gates, experts)
    # a product's inn terms, k products with gates and their sums in fp32; one rounding
    assert (np.abs(host(y) - want) <= (inn + k + 1) * ONE * mag + X.rounded(want, t)).all()
    y = loop.next_tokens(x, logits)
    want, mag = layer(loop, x, gates, experts, quantised=False)
    assert y.dtype == t and (np.abs(host(y) - want) <= (2 * inn + 2 + k + 1) * ONE * mag + X.rounded(want, t)).all()


@pytest.mark.parametrize("t", HALVES, ids=["bf16", "f16"])
@pytest.mark.parametrize("wide", [True, False], ids=["rows of fp32", "rows of 16 bits"])
def test_gradient_of_the_tokens(L, t, wide):
    """dx from the rows' gradients as they are packed: k rows of fp32 added and rounded once, or rounded, added and rounded again."""
    E, out, inn, T, k, seed = 4, 96, 200, 60, 3, 1234567
    loop = make(L, E, out, inn, 2, seed, choices=k, rows_f32=wide)
    x, logits = inputs(T, E, inn, t, 3)
    dy = (torch.randn(T, out, generator=torch.Generator().manual_seed(1)) * 1e-2).to(t).cuda()
    y, saved = loop.forward(x, logits)
    rows, gates, slots = saved[1], host(saved[4]).reshape(T, k), saved[6].cpu().numpy().reshape(-1)
    assert rows.dtype == (torch.float32 if wide else t)
    dx, dlogits, dw = loop.backward(dy, saved, worker=1)
    assert y.dtype == dx.dtype == t and dw.dtype == torch.float32
    order = np.full((slots >= 0).sum(), -1)
    order[slots[slots >= 0]] = np.flatnonzero(slots >= 0)
    n, d64 = len(order), host(dy)
    drows = torch.from_numpy(gates.reshape(-1)[order, None].astype(np.float32) * d64[order // k].astype(np.float32)).to(t).double().numpy()
    b = X.q(np.concatenate((drows, np.zeros((T * k - n, out)))), True, seed, loop.round_id, loop.K + 1)
    ut, offsets = np.stack([X.q(v.T) for v in host(loop.u)]), saved[5].cpu().numpy()
    dxrows, size = np.zeros((T * k, inn)), np.zeros((T * k, inn))
    for e in range(E):
        s = slice(offsets[e], offsets[e + 1])
        dxrows[s], size[s] = b[s] @ ut[e].T, np.abs(b[s]) @ np.abs(ut[e]).T
    spare = out * ONE * size + (0 if wide else X.rounded(dxrows, t))
    want, mag = X.combine(dxrows, slots, None, T, k)
    spare = X.combine(spare, slots, None, T, k)[0]
    assert (np.abs(host(dx) - want) <= spare + (k + 1) * ONE * (mag + spare) + X.rounded(np.abs(want) + spare, t)).all()
    # and what the sum gives of the rows as they lie there
    want, mag = X.combine(host(rows), slots, gates, T, k)
    assert (np.abs(host(y) - want) <= (k + 1) * ONE * mag + X.rounded(want, t)).all()
    dg, dmag = np.zeros(T * k), np.zeros(T * k)
    dg[order] = (d64[order // k] * host(rows)[:n]).sum(1)
    dmag[order] = (out + 1) * ONE * np.abs(d64[order // k] * host(rows)[:n]).sum(1)
    l, experts = host(logits), saved[3].cpu().numpy().reshape(T, k)
    want, mag = X.route_backward(l, experts, gates, dg.reshape(T, k), False)
    spare = X.route_backward(l, experts, np.abs(gates), dmag.reshape(T, k), False)[1]
    assert (np.abs(host(dlogits) - want) <= spare + mag * (2 * k + 6) * ONE + ONE * np.abs(want) + 1e-30).all()


@pytest.mark.parametrize("wide", [True, False], ids=["rows of fp32", "rows of 16 bits"])
def test_16_bit_activations_from_a_graph(L, wide):
    E, out, inn, T = 5, 96, 160, 50
    loop = make(L, E, out, inn, rows_f32=wide)
    x, logits = inputs(T, E, inn, torch.bfloat16, 3)
    dy = torch.randn(T, out, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).cuda()

    def step():
        y, saved = loop.forward(x, logits)
        return (y, *loop.backward(dy, saved), loop.next_tokens(x[:4], logits[:4]))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(4):
        new = inputs(T, E, inn, torch.bfloat16, 30 + i)
        x.copy_(new[0])
        logits.copy_(new[1])
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, step()):
            assert torch.equal(a, b), i
        assert np.isfinite(torch.randn(1 << 16, device="cuda").sum().item())


def test_a_gradient_of_another_type(L):
    """Beside rows of fp32 any type does; rows of 16 bits take their own."""
    x, logits = inputs(8, 3, 64, torch.bfloat16, 1)
    loop = make(L, 3, 32, 64)
    _, saved = loop.forward(x, logits)
    dy = torch.randn(8, 32, device="cuda").to(torch.bfloat16)
    for t in (torch.bfloat16, torch.float32, torch.float16):
        assert loop.backward(dy.to(t), saved)[0].dtype == t
    loop = make(L, 3, 32, 64, rows_f32=False)
    _, saved = loop.forward(x, logits)
    with pytest.raises(AssertionError):
        loop.backward(dy.float(), saved)
