"""The order of a worker's and the server's calls in the epoch loop of a matrix parameter."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def loop_class():
    from paper_1901_03040_amd.epoch_loop import QesgdMatrixLoop
    assert torch.cuda.is_available()
    return QesgdMatrixLoop


def test_backward_belongs_to_the_parameters_of_its_forward(loop_class):
    """dx is taken with the packed parameters; after a round, or an epoch's start, they are others than the forward pass had."""
    g = torch.Generator().manual_seed(0)
    loop = loop_class(torch.randn(48, 80, generator=g).cuda(), 1, 5)
    x, dy = torch.randn(20, 80, generator=g).cuda(), torch.randn(20, 48, generator=g).cuda()
    _, saved = loop.forward(x)
    dx, dw = loop.backward(dy, saved)
    assert torch.equal(loop.backward(dy, saved)[0], dx)         # as often as one likes before the round
    loop.orthogonal_round(dw[None], 0.1)
    with pytest.raises(AssertionError, match="parameters"):
        loop.backward(dy, saved)
    _, saved = loop.forward(x)
    assert not torch.equal(loop.backward(dy, saved)[0], dx)
    loop.end_epoch()
    loop.begin_epoch()
    with pytest.raises(AssertionError, match="parameters"):
        loop.backward(dy, saved)


@pytest.mark.parametrize("tokens,dtype", [(1, torch.bfloat16), (1, torch.float32), (17, torch.float16), (130, torch.bfloat16)])
def test_a_forward_pass_alone(loop_class, tokens, dtype):
    """Without gradients the same y, bit for bit, and nothing to go back with."""
    g = torch.Generator().manual_seed(tokens)
    loop = loop_class(torch.randn(200, 384, generator=g).cuda(), 1, 5)
    x = torch.randn(tokens, 384, generator=g).to(dtype).cuda()
    y, saved = loop.forward(x, gradients=False)
    assert saved is None and y.dtype == dtype
    assert torch.equal(y, loop.forward(x)[0])
    with pytest.raises(TypeError):
        loop.backward(torch.zeros_like(y), saved)
