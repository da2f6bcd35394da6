"""The two kinds of gates where all experts are chosen: the softmax over all logits and that over the chosen ones are one and the same.

Where a lane of the router holds one logit (up to 16 experts) and the logits fall, choice j is expert j and lies in the lane of logit j, so both sums
have the same terms in the same order: the gates are equal in every bit if, and only if, a term of either sum is worked out alike."""
import numpy as np
import pytest
import torch

import expert_reference as X
from expert_reference import TYPES, host
from test_gpu_route import run_route

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_1901_03040_amd import binding
    assert torch.cuda.is_available()
    binding.lib()
    return binding


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("E", [2, 5, 8, 16])
@pytest.mark.parametrize("T", [100, 5000])
def test_gates_of_all_chosen(B, T, E, dtype):
    x = torch.rand(T, E, generator=torch.Generator().manual_seed(E)) * 24
    x = x.to(TYPES[dtype]).sort(dim=1, descending=True)[0].contiguous().cuda()
    a, c = run_route(B, x, E, True), run_route(B, x, E, False)
    for name in ("experts", "offsets", "order", "slots"):
        assert torch.equal(a[name], c[name])
    assert torch.equal(a["gates"], c["gates"]), (a["gates"] != c["gates"]).sum()
    l = host(x)
    _, gates, *_ = X.route(l, E, True)
    assert (np.abs(host(a["gates"]).reshape(T, E) - gates) <= gates * X.softmax_error(l).max(1, keepdims=True)).all()
