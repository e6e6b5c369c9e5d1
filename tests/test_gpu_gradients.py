"""What autograd makes of the training operators."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def g():
    import paper_2208_09151_amd as lib
    return lib


@pytest.mark.parametrize("activation", ["relu", "silu", "gelu"])
@pytest.mark.parametrize("by", ["x", "weight", "router"])
def test_second_derivatives_are_refused(activation, by):
    """The kernels' gradients are no graph: with a term of x beside the layer's, a second derivative would lack the layer's
    part without a word.  So a gradient that is to be differentiated is refused."""
    from paper_2208_09151_amd.experts import ExpertLayer
    torch.manual_seed(1)
    layer = ExpertLayer(64, 32, 4, 2, activation).cuda()
    x = torch.randn((50, 64), device="cuda", requires_grad=True)
    at = {"x": x, "weight": layer.weight, "router": layer.router.weight}[by]
    loss = layer(x).sum() + (at ** 3).sum()
    with pytest.raises(RuntimeError, match="second derivative"):
        first, = torch.autograd.grad(loss, at, create_graph=True)
        torch.autograd.grad(first.sum(), at)
    first, = torch.autograd.grad(layer(x).sum() + (at ** 3).sum(), at)
    assert not first.requires_grad
