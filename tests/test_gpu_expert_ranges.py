"""Layers of experts at the ends of the ranges that the header states: as many tokens as it allows, which are more than one launch numbers threads for."""
import pytest
import torch

from expert_reference import ONE

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_1901_03040_amd import binding
    assert torch.cuda.is_available()
    binding.lib()
    yield binding
    torch.cuda.empty_cache()


def test_choices_of_2_28_tokens(B):
    """Blocks of 64 tokens, 1024 threads each, are 2^32 threads."""
    T, E, part = 1 << 28, 9, 1 << 24
    x = torch.empty(T, E, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    experts, order, slots = (torch.full((T,), -7, dtype=torch.int32, device="cuda") for _ in range(3))
    gates, offsets = torch.zeros(T, device="cuda"), torch.empty(E + 1, dtype=torch.int32, device="cuda")
    B.qesgd_route(x, E, T, E, 1, B.GATE_CHOSEN, experts, gates, offsets, order, slots, workspace=B.alloc_workspace(B.qesgd_route_workspace_bytes(T, E, 1)))
    assert (gates == 1.0).all()                                 # of one choice
    numbers, counts = torch.arange(E, device="cuda"), torch.zeros(E, dtype=torch.int64, device="cuda")
    for lo in range(0, T, part):
        v = x[lo:lo + part]
        first = torch.where(v == v.amax(1, keepdim=True), numbers, E).amin(1)      # ties: the lower one
        assert torch.equal(experts[lo:lo + part].long(), first), lo
        counts += torch.bincount(first, minlength=E)
        # a pair's place holds the pair
        assert torch.equal(order[slots[lo:lo + part].long()].long(), torch.arange(lo, lo + part, device="cuda")), lo
    assert offsets[0] == 0 and torch.equal(offsets[1:].long(), counts.cumsum(0))
    for e in range(E):                                          # places: by expert, those of one in the tokens' order
        own = order[offsets[e]:offsets[e + 1]]
        assert bool((own[1:] > own[:-1]).all()) and bool((experts[own.long()] == e).all()), e


def test_gradient_of_the_logits_of_2_28_tokens(B):
    """16 lanes to a token are 2^32 threads.  In the logits' place, so that a token worked out twice, or not at all, shows."""
    T, E = 1 << 28, 9
    x = torch.empty(T, E, dtype=torch.bfloat16, device="cuda").fill_(7.0)
    experts = torch.arange(T, dtype=torch.int32, device="cuda") % E
    gates, dgates = torch.full((T,), 0.5, device="cuda"), experts.float()
    B.qesgd_route_backward(None, E, T, E, 1, B.GATE_CHOSEN, experts, gates, dgates, x, E)
    # one choice: s = g d, and dlogits = g (d - g d) = d / 4 at the chosen one: exact in bf16
    for lo in range(0, T, 1 << 24):
        part = x[lo:lo + (1 << 24)]
        want = torch.zeros_like(part)
        e = experts[lo:lo + (1 << 24)].long()
        want.scatter_(1, e[:, None], (e.float() / 4).to(torch.bfloat16)[:, None])
        assert torch.equal(part, want), lo


def test_gradient_of_the_gates_of_2_24_long_rows(B):
    """A workgroup to a token of 129 pieces of 16 bytes is 2^32 threads."""
    T, N, R = (1 << 24) + 5, 1032, 6
    dy = torch.empty(T, N, dtype=torch.bfloat16, device="cuda")
    dy.copy_((torch.arange(T, device="cuda") % 3 - 1).to(torch.bfloat16)[:, None].expand(T, N))
    rows = torch.randn(R, N, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(torch.bfloat16)
    slots = (torch.arange(T, dtype=torch.int32, device="cuda") % (R + 1)) - 1
    dgates = torch.full((T,), 9.0, device="cuda")
    B.qesgd_combine_backward(dy, N, rows, N, R, slots, None, T, 1, N, None, 0, dgates)
    sums, size = rows.double().sum(1), rows.double().abs().sum(1)
    pad = torch.zeros(1, dtype=torch.float64, device="cuda")
    want = torch.cat((pad, sums))[slots.long() + 1] * (torch.arange(T, device="cuda") % 3 - 1)
    assert bool(((dgates.double() - want).abs() <= (N + 1) * ONE * torch.cat((pad, size))[slots.long() + 1]).all())
    # and the rows' gradients: rows that a few tokens at either end name
    named = {0: 0, 1: 1, (1 << 23) + 7: 2, (1 << 24) - 2: 3, 1 << 24: 4, T - 1: 5}
    slots.fill_(-1)
    for t, s in named.items():
        slots[t] = s
    gates, drows = torch.full((T,), 2.0, device="cuda"), torch.full((R, N), 9.0, dtype=torch.bfloat16, device="cuda")
    B.qesgd_combine_backward(dy, N, None, 0, R, slots, gates, T, 1, N, drows, N, None)
    for t, s in named.items():
        assert torch.equal(drows[s], 2 * dy[t])
