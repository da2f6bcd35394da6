"""Gradient of the gates where a token's logits hold an infinity or a NaN: its gates are NaN, and so are the formula's gradients of all its open logits."""
import pytest
import torch

from expert_reference import TYPES
from test_gpu_route import run_route

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def B():
    from paper_1901_03040_amd import binding
    assert torch.cuda.is_available()
    binding.lib()
    return binding


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("E", [5, 40, 300, 1000])
def test_gradient(B, E, dtype):
    t, k = TYPES[dtype], 2
    x = torch.randn(7, E, generator=torch.Generator().manual_seed(E)).to(t)
    x[1, 3], x[2, 1], x[3, 0], x[4] = NAN, INF, -INF, -INF
    x[5, 0], x[5, 4], x[6, 1:] = INF, -INF, -INF
    x = x.cuda()
    dg = torch.rand(7, k, generator=torch.Generator().manual_seed(1)).cuda() + 0.5
    closed = x == -INF
    for all_ in (True, False):
        out = run_route(B, x, k, all_)
        dl = torch.full_like(x, 9.0)
        B.qesgd_route_backward(x, E, 7, E, k, B.GATE_ALL if all_ else B.GATE_CHOSEN, out["experts"], out["gates"], dg, dl, E)
        assert (dl[closed] == 0).all()
        assert torch.isfinite(dl[[0, 3, 4, 6]]).all()
        chosen = torch.zeros(7, E, dtype=torch.bool, device="cuda")
        e = out["experts"].view(7, k).long()
        chosen.scatter_(1, e.clamp(min=0), e >= 0)
        for i in (1, 2, 5):
            want = ~closed[i] if all_ else chosen[i]
            assert torch.equal(torch.isnan(dl[i]), want), (i, all_)
            assert (dl[i][~want] == 0).all()
