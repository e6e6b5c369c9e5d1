"""Every call refuses a tensor that carries a tangent of forward mode, with and without the calls' compiled part."""
import pytest
import torch
from torch.autograd import forward_ad

from layer_reference import rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def g():
    import paper_2208_09151_amd as lib
    return lib


@pytest.fixture(params=[True, False], ids=["compiled", "interpreted"])
def way(g, request, monkeypatch):
    from paper_2208_09151_amd import layers
    g.linear(torch.zeros((1, 1), device="cuda"), torch.zeros((1, 1), device="cuda"))
    if not request.param:
        monkeypatch.setattr(layers, "_quick", None)
    elif layers._quick is None:
        pytest.skip("the compiled part is not built for this torch")


def cases(g):
    """(call, its floating arguments)"""
    gen = torch.Generator(device="cuda").manual_seed(1)
    n, width = 9, 8
    x, dy, w = (rows_of(gen, k, width, torch.float32) for k in (n, n, width))
    w3 = rows_of(gen, 3 * width, width, torch.float32).view(3, width, width)
    b, b3 = w[0].clone(), w3[:, 0].contiguous()
    r = g.route(torch.randint(-1, 3, (n, 2), generator=gen, device="cuda"), 3)
    slots, res = rows_of(gen, 2 * n, width, torch.float32), rows_of(gen, 2 * n, width, torch.float32)
    share = torch.rand((n, 2), generator=gen, device="cuda")
    ids = torch.randint(0, n, (n,), generator=gen, device="cuda")
    _, stats = g.layer_norm(x, stats=True)
    kept = g.compress(x)
    return {
        "linear": (lambda x, w, b, res: g.linear(x, w, b, "gelu", res), [x, w, b, dy]),
        "linear, codes": (lambda x, w: g.linear(x, w, None, "silu", keep=True)[0], [x, w]),
        "linear, output": (lambda x, w: g.linear(x, w, out=torch.empty_like(dy)), [x, w]),
        "linear, route": (lambda x, w, b, res: g.linear(x, w, b, "relu", res, r), [x, w3, b3, res]),
        "linear, slots": (lambda x, w: g.linear(x, w, route=r, slots=True), [slots, w3]),
        "linear_backward": (lambda dz, w: g.linear_backward(dz, w), [dy, w]),
        "bias_gradient": (lambda dz: g.bias_gradient(dz), [dy]),
        "expert_layer": (lambda x, s, w, b: g.expert_layer(x, s, w, 2, "silu", b), [x, b3, w3, b3]),
        "layer_norm": (lambda x, w, b: g.layer_norm(x, w, b), [x, b, b3[0].clone()]),
        "layer_norm_backward": (lambda dz, x, s, w: g.layer_norm_backward(dz, x, s, w)[0], [dy, x, stats, b]),
        "lookup": (lambda t: g.lookup(t, ids, 0.5), [x]),
        "lookup_backward": (lambda dz: g.lookup_backward(dz, ids, n), [dy]),
        "dispatch": (lambda x: g.dispatch(x, r), [x]),
        "dispatch_backward": (lambda dz: g.dispatch_backward(dz, r), [slots]),
        "combine": (lambda z, p: g.combine(z, r, p), [slots, share]),
        "combine_backward": (lambda dz, z, p: g.combine_backward(dz, z, r, p)[0], [dy, slots, share]),
        "compress": (lambda x: g.restore(g.compress(x)), [x]),
        "activate": (lambda x: g.activate(x, "gelu")[0], [x]),
        "activate_backward": (lambda dz: g.activate_backward(kept, dz, "relu"), [dy]),
        "weight_gradient": (lambda dz: g.weight_gradient(kept, dz), [dy]),
    }


NAMES = ["linear", "linear, codes", "linear, output", "linear, route", "linear, slots", "linear_backward", "bias_gradient",
         "expert_layer", "layer_norm", "layer_norm_backward", "lookup", "lookup_backward", "dispatch", "dispatch_backward", "combine",
         "combine_backward", "compress", "activate", "activate_backward", "weight_gradient"]


@pytest.mark.parametrize("name", NAMES)
def test_a_tangent_is_refused(g, way, name):
    every = cases(g)
    assert list(every) == NAMES
    call, args = every[name]
    want = call(*args)
    with forward_ad.dual_level():
        assert torch.equal(call(*args), want)                   # (a level alone changes nothing)
        for k, t in enumerate(args):
            dual = [forward_ad.make_dual(a, torch.ones_like(a)) if j == k else a for j, a in enumerate(args)]
            for mode in (torch.enable_grad, torch.no_grad):
                with mode(), pytest.raises(RuntimeError, match="forward mode"):
                    call(*dual)
            with torch.inference_mode():                        # (which has no forward mode)
                assert torch.equal(call(*dual), want)
    assert torch.equal(call(*args), want)


@pytest.mark.parametrize("name", ["linear", "linear, route", "layer_norm", "lookup", "dispatch", "combine", "activate"])
def test_a_tangent_beside_a_gradient(g, way, name):
    """Where autograd records the call, and in a gradient that its backward pass gets."""
    call, args = cases(g)[name]
    leaves = [a.clone().requires_grad_() for a in args]
    y = call(*leaves)
    with forward_ad.dual_level():
        for k in range(len(args)):
            dual = [forward_ad.make_dual(a, torch.ones_like(a)) if j == k else a for j, a in enumerate(leaves)]
            with pytest.raises(RuntimeError, match="forward mode"):
                call(*dual)
        with pytest.raises(RuntimeError, match="forward mode"):
            torch.autograd.grad(y, leaves, forward_ad.make_dual(torch.ones_like(y), torch.ones_like(y)), retain_graph=True)
    assert all(t is not None for t in torch.autograd.grad(y, leaves, torch.ones_like(y)))


def test_sums_of_neighbours(g):
    from paper_2208_09151_amd.experts import Block, ExpertLayer, SumOfRows
    x, of = torch.ones((4, 8), device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x, torch.ones_like(x))
        for call in (lambda: SumOfRows.apply(dual, of, 2), lambda: Block(8, 8, 3).cuda()(dual), lambda: Block(8, 8, 3).cuda().answer(dual),
                     lambda: ExpertLayer(8, 8, 3).cuda()(dual), lambda: ExpertLayer(8, 8, 3).cuda().answer(dual)):
            with pytest.raises(RuntimeError, match="forward mode"):
                call()
