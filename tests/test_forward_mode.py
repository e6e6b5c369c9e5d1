"""Tensors that carry a tangent of forward mode are refused: the kernels would lose it without a word (no GPU; the calls
themselves are in test_gpu_forward_mode.py)."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2208_09151_amd import training


class Twice(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x):
        training._no_tangent(x, "x")            # (forward mode is off in here)
        return 2 * x

    @staticmethod
    @training._first_derivative
    def backward(ctx, grad):
        return 2 * grad


def test_a_tensor_with_a_tangent():
    plain = torch.ones(3)
    training._no_tangent(plain, "x")
    with forward_ad.dual_level():
        training._no_tangent(plain, "x")
        training._no_tangent(None, "x")
        dual = forward_ad.make_dual(plain, torch.ones(3))
        for mode in (torch.enable_grad, torch.no_grad):
            with mode(), pytest.raises(RuntimeError, match="x: no tangent of forward mode"):
                training._no_tangent(dual, "x")
        training._no_tangent(forward_ad.unpack_dual(dual).primal, "x")
        with torch.inference_mode():            # (which has no forward mode)
            training._no_tangent(dual, "x")
        with pytest.raises(RuntimeError, match="forward mode"):
            Twice.apply(dual)
    training._no_tangent(dual, "x")             # (the level is gone and the tangent with it)


def test_a_gradient_with_a_tangent():
    x = torch.ones(3, requires_grad=True)
    assert torch.equal(torch.autograd.grad(Twice.apply(x), x, torch.ones(3))[0], torch.full((3,), 2.0))
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(torch.ones(3), torch.ones(3))
        with pytest.raises(RuntimeError, match="no tangent of forward mode"):
            torch.autograd.grad(Twice.apply(x), x, dual)
        assert torch.equal(torch.autograd.grad(Twice.apply(x), x, torch.ones(3))[0], torch.full((3,), 2.0))
