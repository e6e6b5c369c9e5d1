"""The expert layer: its outputs and gradients against the same layer in plain torch and 64 bits, and the
training run over sampled batches.

The layer's products are f32 sums of at most 96 terms (2^-24 each) and the activation's error is 2^-18 of its
value; gradients that go through values kept in 8 bits are compared with the formula at those same values.
Everything is compared at 1e-4 of the largest entry, 16 times 96 2^-24.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def g():
    import paper_2208_09151_amd as lib
    return lib


def near(got, want):
    got, want = got.detach().double().cpu(), want.detach().double().cpu()
    assert got.shape == want.shape
    assert float((got - want).abs().max()) <= 1e-4 * float(want.abs().max())


def slope(x, activation):
    x = x.detach().requires_grad_()
    fn = {"relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[activation]
    return torch.autograd.grad(fn(x).sum(), x)[0], fn


@pytest.mark.parametrize("activation", ["relu", "silu", "gelu"])
@pytest.mark.parametrize("rows, width, out, experts, top, capacity", [
    (1, 64, 32, 4, 2, None), (500, 96, 40, 5, 2, None), (500, 96, 40, 5, 3, 0.7), (64, 33, 17, 64, 4, None)])
def test_layer_and_its_gradients(g, rows, width, out, experts, top, capacity, activation):
    from paper_2208_09151_amd.experts import ExpertLayer
    torch.manual_seed(rows + width)
    layer = ExpertLayer(width, out, experts, top, activation, capacity).cuda()
    x = torch.randn((rows, width), device="cuda", requires_grad=True)
    dy = torch.randn((rows, out), device="cuda")
    y = layer(x)
    y.backward(dy)

    # the same in 64 bits, pair by pair, with the route and the kept values of the layer
    xd, wd = x.detach().double(), layer.weight.detach().double()
    scores = layer.router(x.detach()).float()
    best, chosen = torch.topk(scores, top, dim=1)
    weights = torch.softmax(best.double(), 1)
    most = None if capacity is None else -(-int(rows * top * capacity * 1000) // (experts * 1000))
    r = g.route(chosen, experts, capacity=most)
    kept_x = g.restore(g.compress(x.detach())).double()
    a = torch.einsum("rc,rjcd->rjd", xd, wd[chosen])
    rows_in_slots = g.dispatch(x.detach(), r)
    ends = r.offsets.tolist()
    af = torch.zeros((rows * top, out), device="cuda")
    for e in range(experts):
        torch.mm(rows_in_slots[ends[e]:ends[e + 1]], layer.weight[e].detach(), out=af[ends[e]:ends[e + 1]])
    kept_a = g.restore(g.compress(af)).double()
    has = (r.slot >= 0).double()
    kept_pairs = kept_a[r.slot.clamp(min=0).long()]
    slopes, fn = slope(kept_pairs, activation)
    h = fn(a)
    near(y, (h * (weights * has)[:, :, None]).sum(1))
    dh = dy.double()[:, None, :] * (weights * has)[:, :, None]
    da = dh * slopes
    dw = torch.zeros_like(wd)
    dw.index_add_(0, chosen.reshape(-1), (kept_x[:, None, :, None] * da[:, :, None, :]).reshape(-1, width, out))
    near(layer.weight.grad, dw)
    dweights = (dy.double()[:, None, :] * h).sum(2) * has
    dbest = weights * (dweights - (weights * dweights).sum(1, keepdim=True))
    dscores = torch.zeros((rows, experts), dtype=torch.float64, device="cuda").scatter_(1, chosen, dbest)
    near(layer.router.weight.grad, dscores.t() @ xd)
    dx = torch.einsum("rjd,rjcd->rc", da, wd[chosen]) + dscores @ layer.router.weight.detach().double()
    near(x.grad, dx)


def test_training_on_sampled_batches(g):
    from paper_2208_09151_amd.experts import train
    losses = train(config=1, steps=24, report=None)
    assert len(losses) == 24
    # eight classes: 2.08 is the loss of a guess
    assert sum(losses[-4:]) / 4 < 0.7 * losses[0] and losses[0] > 1.5
