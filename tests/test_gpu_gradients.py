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


def routed(g, rows, top, experts, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    chosen = torch.randint(-1, experts, (rows, top), generator=gen, device="cuda")
    return g.route(chosen, experts, capacity=max(1, rows * top // experts)), gen


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_results_keep_the_graph(g, dtype):
    """dispatch, combine and activate of tensors that require a gradient: the gradients of the calls that are made for it."""
    r, gen = routed(g, 70, 3, 5)
    x = torch.randn((70, 33), generator=gen, device="cuda").to(dtype).requires_grad_()
    w = torch.randn((70, 3), generator=gen, device="cuda").requires_grad_()
    dy = torch.randn((70, 33), generator=gen, device="cuda").to(dtype)
    z = g.dispatch(x, r)
    h, kept = g.activate(z, "silu")
    y = g.combine(h, r, w)
    y.backward(dy)
    with torch.no_grad():
        z2 = g.dispatch(x, r)
        h2, kept2 = g.activate(z2, "silu")
        y2 = g.combine(h2, r, w)
        dh, dw = g.combine_backward(dy, h2, r, w)
        dx = g.dispatch_backward(g.activate_backward(kept2, dh, "silu"), r)
    assert not (z2.requires_grad or h2.requires_grad or y2.requires_grad)
    assert torch.equal(y, y2) and torch.equal(kept.codes, kept2.codes) and torch.equal(kept.scales, kept2.scales)
    assert torch.equal(x.grad, dx) and torch.equal(w.grad, dw)


@pytest.mark.parametrize("needs", ["z", "weights"])
def test_one_of_two_gradients(g, needs):
    r, gen = routed(g, 70, 3, 5)
    z = torch.randn((210, 20), generator=gen, device="cuda").requires_grad_(needs == "z")
    w = torch.randn((70, 3), generator=gen, device="cuda").requires_grad_(needs == "weights")
    g.combine(z, r, w).sum().backward()         # (a gradient of stride 0)
    dz, dw = g.combine_backward(torch.ones((70, 20), device="cuda"), z.detach(), r, w.detach())
    assert torch.equal(z.grad, dz) if needs == "z" else z.grad is None
    assert torch.equal(w.grad, dw) if needs == "weights" else w.grad is None


def test_a_result_that_is_recorded_is_a_new_tensor(g):
    r, gen = routed(g, 70, 3, 5)
    x = torch.randn((70, 20), generator=gen, device="cuda").requires_grad_()
    w = torch.randn((70, 3), generator=gen, device="cuda")
    z = torch.empty((210, 20), device="cuda")
    for call in (lambda: g.dispatch(x, r, out=z), lambda: g.combine(z, r, w.requires_grad_(), out=torch.empty_like(w)),
                 lambda: g.activate(x, "relu", out=x), lambda: g.activate(x, "relu", out=torch.empty_like(x))):
        with pytest.raises(ValueError, match="out"):
            call()
    with torch.no_grad():
        assert g.dispatch(x, r, out=z) is z


def test_what_is_saved_goes_through_the_hooks(g):
    """Codes and routes as well: moved to the host and back between forward and backward pass, they give the same."""
    from paper_2208_09151_amd.experts import ExpertLayer
    torch.manual_seed(2)
    layer = ExpertLayer(64, 32, 4, 2, "gelu", 1.0).cuda()
    x = torch.randn((50, 64), device="cuda", requires_grad=True)
    want = torch.autograd.grad(layer(x).sum(), [x, *layer.parameters()])
    moved = []

    def pack(t):
        moved.append(t.dtype)
        return t.cpu()

    with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t.cuda()):
        loss = layer(x).sum()
    got = torch.autograd.grad(loss, [x, *layer.parameters()])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # codes of the rows and of the activations' inputs, the route of either pass
    assert moved.count(torch.int8) == 2 and moved.count(torch.uint8) == 2 and torch.int32 in moved


def test_codes_and_routes_that_have_changed_are_noticed(g):
    r, gen = routed(g, 70, 3, 5)
    x = torch.randn((70, 20), generator=gen, device="cuda").requires_grad_()
    y, kept = g.activate(x, "relu")
    kept.codes.zero_()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    y = g.dispatch(x, r)
    r.slot.fill_(-1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_a_result_written_into_a_saved_tensor_is_noticed(g):
    """Every call with an output of the caller's counts as one in place."""
    r, gen = routed(g, 70, 3, 5)
    x = torch.randn((70, 20), generator=gen, device="cuda")
    z = torch.randn((210, 20), generator=gen, device="cuda")
    w = torch.randn((70, 3), generator=gen, device="cuda")
    kept = g.compress(x)
    dw = torch.empty((20, 20), device="cuda")
    for call, out in [(lambda t: g.dispatch(x, r, out=t), z), (lambda t: g.combine(z, r, w, out=t), x),
                      (lambda t: g.dispatch_backward(z, r, out=t), x), (lambda t: g.activate(x, "relu", out=t), x),
                      (lambda t: g.restore(kept, out=t), x), (lambda t: g.activate_backward(kept, x, "relu", out=t), x),
                      (lambda t: g.weight_gradient(kept, x, out=t), dw)]:
        by = torch.ones_like(out, requires_grad=True)
        loss = (by * out).sum()                 # keeps `out` for the gradient of `by`
        call(out)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    with torch.inference_mode():
        out = torch.empty_like(z)
        assert g.dispatch(x, r, out=out) is out


def test_a_training_run_leaves_the_random_numbers_alone():
    from paper_2208_09151_amd.experts import train
    torch.manual_seed(3)
    before = torch.get_rng_state(), torch.cuda.get_rng_state()
    first = train(config=1, steps=1, report=None)
    assert torch.equal(torch.get_rng_state(), before[0]) and torch.equal(torch.cuda.get_rng_state(), before[1])
    torch.manual_seed(4)
    # the same weights: the neighbours' sums alone are added up in any order
    assert abs(train(config=1, steps=1, report=None)[0] - first[0]) < 1e-4


@pytest.mark.parametrize("change", [lambda t: t.cpu(), lambda t: t.repeat(2, *[1] * (t.dim() - 1))[::2], lambda t: t[:-1]])
def test_saved_tensors_that_come_back_otherwise_are_refused(g, change):
    """Hooks may return anything: codes and routes are looked at again before the library gets their addresses."""
    r, gen = routed(g, 70, 3, 5)
    x = torch.randn((70, 20), generator=gen, device="cuda").requires_grad_()
    w = torch.randn((70, 3), generator=gen, device="cuda")
    z = torch.randn((210, 20), generator=gen, device="cuda").requires_grad_()
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: change(t) if t.dtype != torch.float32 else t):
        results = [g.dispatch(x, r), g.combine(z, r, w), g.activate(x, "silu")[0]]
    for y in results:
        with pytest.raises((ValueError, g.GinexError)):
            y.sum().backward()
