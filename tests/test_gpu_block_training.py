"""Training with residual blocks: every parameter gets a gradient, and all of them are the same bits in every run."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def gradients(blocks, seeds, rows, width):
    from paper_2208_09151_amd.experts import Classifier
    torch.manual_seed(blocks + seeds)
    model = Classifier(width, 32, 6, 5, blocks).cuda()
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn((rows, width), generator=gen, device="cuda")
    count = torch.randint(0, 20, (seeds,), generator=gen, device="cuda")
    count[0] = 0                                # (a seed without neighbours)
    rowptr = torch.cat([count.new_zeros(1), count.cumsum(0)])
    col = torch.randint(0, rows, (int(rowptr[-1]),), generator=gen, device="cuda", dtype=torch.int32)
    loss = torch.nn.functional.cross_entropy(model(x, rowptr, col), torch.randint(0, 6, (seeds,), generator=gen, device="cuda"))
    loss.backward()
    return loss.detach(), {name: p.grad for name, p in model.named_parameters()}


@pytest.mark.parametrize("blocks, seeds, rows, width", [(1, 40, 500, 24), (2, 300, 9000, 64)])
def test_gradients_are_there_and_the_same(blocks, seeds, rows, width):
    loss, first = gradients(blocks, seeds, rows, width)
    assert bool(torch.isfinite(loss))
    for name, grad in first.items():
        assert grad is not None and bool(torch.isfinite(grad).all()) and bool((grad != 0).any()), name
    for _ in range(4):
        again, second = gradients(blocks, seeds, rows, width)
        assert torch.equal(loss, again)
        assert all(torch.equal(first[name], second[name]) for name in first)


def test_losses_of_all_steps_are_the_same():
    """Those after updates, too: they hang on the gradients of every step in front."""
    from paper_2208_09151_amd.experts import train
    first, second = (train(config=1, steps=6, report=None, blocks=1) for _ in range(2))
    assert len(first) == 6 and first == second
