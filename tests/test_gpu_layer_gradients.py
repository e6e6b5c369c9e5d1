"""What autograd makes of the layers: gradients against the formulas in 64 bits, at the values that were kept in 8 bits, and
against differences; a block of all of them together."""
import pytest
import torch

from layer_reference import TYPES, activated, near, random_route, rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def g():
    import paper_2208_09151_amd as lib
    return lib


def slope(z, activation):
    if activation is None:
        return torch.ones_like(z)
    if activation == "relu":
        return (z > 0).double()
    with torch.enable_grad():
        z = z.detach().requires_grad_()
        return torch.autograd.grad(activated(z, activation).sum(), z)[0]


def close(got, want, dtype, terms):
    """Sums of `terms` products in f32 (2^-23 each) of gradients that were rounded to `dtype` twice, against the largest entry."""
    got, want = got.detach().double(), want.double()
    assert got.shape == want.shape
    unit = {torch.float32: 2.0 ** -18, torch.bfloat16: 2.0 ** -6, torch.float16: 2.0 ** -9}[dtype] + terms * 2.0 ** -23
    assert float((got - want).abs().max()) <= unit * max(float(want.abs().max()), 1e-30)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("activation", [None, "relu", "silu", "gelu"])
@pytest.mark.parametrize("rows", [7, 300])
def test_linear(g, rows, activation, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    width, out = 60, 45
    x = rows_of(gen, rows, width, dtype).requires_grad_()
    w = (torch.randn((out, width), generator=gen, device="cuda") / 8).to(dtype).requires_grad_()
    b = torch.randn(out, generator=gen, device="cuda").to(dtype).requires_grad_()
    res = rows_of(gen, rows, out, dtype).requires_grad_()
    dy = rows_of(gen, rows, out, dtype)
    y, kept = g.linear(x, w.t(), b, activation, res, keep=True)
    y.backward(dy)
    with torch.no_grad():
        assert torch.equal(y, g.linear(x, w.t(), b, activation, res))
        z = g.restore(kept).double()
        dz = dy.double() * slope(z, activation)
        close(x.grad, dz @ w.double(), dtype, out)
        close(w.grad, dz.t() @ g.restore(g.compress(x)).double(), dtype, rows)
        close(b.grad, dz.sum(0), dtype, rows)
        assert torch.equal(res.grad, dy)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("slots", [False, True])
@pytest.mark.parametrize("rows", [9, 200])
def test_layers_of_experts(g, rows, slots, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    width, out, experts, top = 40, 33, 5, 3
    r = random_route(g, gen, rows, top, experts, capacity=rows // 2 + 1)
    x = rows_of(gen, rows * top if slots else rows, width, dtype).requires_grad_()
    w = (torch.randn((experts, width, out), generator=gen, device="cuda") / 6).to(dtype).requires_grad_()
    b = torch.randn((experts, out), generator=gen, device="cuda").to(dtype).requires_grad_()
    res = rows_of(gen, rows * top, out, dtype).requires_grad_()
    dy = rows_of(gen, rows * top, out, dtype)
    y, kept = g.linear(x, w, b, "silu", res, route=r, slots=slots, keep=True)
    y.backward(dy)
    with torch.no_grad():
        ends = r.offsets.tolist()
        assert ends[-1] < rows * top
        z = g.restore(kept).double()
        dz = dy.double() * slope(z, "silu")
        xs = g.restore(g.compress(x)).double()
        taken = torch.arange(ends[-1], device="cuda") if slots else r.source[:ends[-1]].long()
        dx = torch.zeros_like(x, dtype=torch.float64)
        dw, db = torch.zeros_like(w, dtype=torch.float64), torch.zeros_like(b, dtype=torch.float64)
        for e in range(experts):
            lo, hi = ends[e], ends[e + 1]
            dx.index_add_(0, taken[lo:hi], dz[lo:hi] @ w[e].double().t())
            dw[e] = xs[taken[lo:hi]].t() @ dz[lo:hi]
            db[e] = dz[lo:hi].sum(0)
        close(x.grad, dx, dtype, out)
        close(w.grad, dw, dtype, rows)
        close(b.grad, db, dtype, rows)
        assert torch.equal(res.grad[:ends[-1]], dy[:ends[-1]]) and bool((res.grad[ends[-1]:] == 0).all())


def differences(f, t, at, step):
    """Central differences of a scalar function at some entries of `t`."""
    got = []
    for i in at:
        flat, keep = t.view(-1), t.view(-1)[i].clone()
        flat[i] = keep + step
        high = f()
        flat[i] = keep - step
        low = f()
        flat[i] = keep
        got.append((high - low) / (2 * step))
    return torch.tensor(got, dtype=torch.float64)


@pytest.mark.parametrize("rows", [6, 100])
def test_against_differences(g, rows):
    """Of what is linear in its argument, or kept as it is.  The value is a sum of f32 numbers of up to some 20, off by 2^-23 of
    that each: over a step of 2^-8 less than 1e-3; layer norm's third derivative counts with the step squared."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    width, out, n = 24, 20, 50
    x, dy = rows_of(gen, rows, width, torch.float32), rows_of(gen, rows, out, torch.float32).double()
    w, b = rows_of(gen, width, out, torch.float32), rows_of(gen, 1, out, torch.float32)[0]
    norm, shift = rows_of(gen, 1, width, torch.float32)[0], rows_of(gen, 1, width, torch.float32)[0]
    table, ids = rows_of(gen, 9, width, torch.float32), torch.randint(-1, 9, (rows,), generator=gen, device="cuda")

    def value():
        rows_of_table = g.lookup(table, ids, 1.5)
        h = g.layer_norm(x, norm, shift, 1e-2)
        return ((g.linear(h, w, b).double() + g.linear(rows_of_table, w).double()) * dy).sum()

    leaves = [x, norm, shift, b, table]
    for t in leaves:
        t.requires_grad_()
    grads = torch.autograd.grad(value(), leaves)
    for t, grad in zip(leaves, grads):
        t.requires_grad_(False)
        at = torch.randint(0, t.numel(), (n,), generator=gen, device="cuda").tolist()
        # (x: layer norm bends, by the step squared)
        step = 2.0 ** -8 if t is x else 2.0 ** -4
        want = differences(lambda: float(value().detach()), t, at, step)
        got = grad.view(-1)[torch.tensor(at, device="cuda")].double().cpu()
        assert float((got - want).abs().max()) <= 2e-3 * float(grad.abs().max()) + 1e-3


@pytest.mark.parametrize("dtype", TYPES)
def test_layer_norm_and_lookup(g, dtype):
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = rows_of(gen, 50, 70, dtype).requires_grad_()
    w, b = (rows_of(gen, 1, 70, dtype)[0].requires_grad_() for _ in range(2))
    dy = rows_of(gen, 50, 70, dtype)
    y, stats = g.layer_norm(x, w, b, stats=True)
    y.backward(dy)
    with torch.no_grad():
        dx, dw, db = g.layer_norm_backward(dy, x, stats, w)
    assert not stats.requires_grad
    assert torch.equal(x.grad, dx) and torch.equal(w.grad, dw.to(dtype)) and torch.equal(b.grad, db.to(dtype))
    only, = torch.autograd.grad(g.layer_norm(x.detach(), w, None).sum(), w)
    assert only.dtype == dtype
    table = rows_of(gen, 20, 70, dtype).requires_grad_()
    ids = torch.randint(-1, 20, (50,), generator=gen, device="cuda")
    g.lookup(table, ids, 0.5).backward(dy)
    assert torch.equal(table.grad, g.lookup_backward(dy, ids, 20, 0.5))


def test_refusals_of_autograd(g):
    x = torch.randn((5, 8), device="cuda", requires_grad=True)
    w = torch.randn((8, 8), device="cuda", requires_grad=True)
    ids = torch.zeros(3, dtype=torch.int64, device="cuda")
    for call in (lambda: g.linear(x, w, out=torch.empty((5, 8), device="cuda")), lambda: g.layer_norm(x, out=torch.empty_like(x)),
                 lambda: g.lookup(w, ids, out=torch.empty((3, 8), device="cuda"))):
        with pytest.raises(ValueError, match="out"):
            call()
    for call, at in ((lambda: g.linear(x, w), x), (lambda: g.linear(x, w, None, "relu"), w), (lambda: g.layer_norm(x), x),
                     (lambda: g.lookup(w, ids), w)):
        with pytest.raises(RuntimeError, match="second derivative"):
            first, = torch.autograd.grad(call().sum() + (at ** 3).sum(), at, create_graph=True)
            torch.autograd.grad(first.sum(), at)


def test_what_is_saved_and_what_is_overwritten(g):
    """Saved tensors go through the hooks; one that has changed is noticed, and so is an output written into one."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = rows_of(gen, 30, 40, torch.float32).requires_grad_()
    w = rows_of(gen, 40, 40, torch.float32).requires_grad_()
    ids = torch.randint(0, 30, (60,), generator=gen, device="cuda")

    def loss():
        return g.lookup(g.layer_norm(g.linear(x, w, None, "gelu"), w.detach()[0]), ids).square().sum()

    want = torch.autograd.grad(loss(), [x, w])
    moved = []

    def pack(t):
        moved.append(t.dtype)
        return t.cpu()

    with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t.cuda()):
        value = loss()
    got = torch.autograd.grad(value, [x, w])
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and moved.count(torch.int8) == 2
    y, kept = g.linear(x, w, None, "gelu", keep=True)
    kept.codes.zero_()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    rows, weight, dw = rows_of(gen, 30, 40, torch.float32), w.detach(), torch.empty(40, device="cuda")
    stats = g.layer_norm(rows, stats=True)[1]
    for call, out in [(lambda t: g.linear(rows, weight, out=t), torch.empty((30, 40), device="cuda")),
                      (lambda t: g.linear_backward(rows, weight, out=t), torch.empty((30, 40), device="cuda")),
                      (lambda t: g.bias_gradient(rows, out=t), dw), (lambda t: g.layer_norm(rows, out=t), torch.empty_like(rows)),
                      (lambda t: g.layer_norm_backward(rows, rows, stats, out=t), torch.empty_like(rows)),
                      (lambda t: g.lookup(rows, ids, out=t), torch.empty((60, 40), device="cuda")),
                      (lambda t: g.lookup_backward(rows, ids[:30], 30, out=t), torch.empty_like(rows)),
                      (lambda t: g.expert_layer(rows, weight[:3], weight[None].expand(3, 40, 40), 2, out=t), torch.empty_like(rows))]:
        by = torch.ones_like(out, requires_grad=True)
        value = (by * out).sum()
        call(out)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            value.backward()


@pytest.mark.parametrize("rows", [1, 40, 64])
def test_a_block_answers_as_it_is_trained(g, rows):
    """The form for a few rows gives what the recorded one gives, to the roundings of f32 sums of at most 96 terms."""
    from paper_2208_09151_amd.experts import Block, ExpertLayer
    torch.manual_seed(rows)
    x = torch.randn((rows, 48), device="cuda")
    block = Block(48, 96, 7, 3).cuda()
    y = block(x)
    assert float((block.answer(x) - y).detach().abs().max()) <= 1e-4 * float(y.detach().abs().max())
    layer = ExpertLayer(48, 30, 9, 2, "silu").cuda()
    y = layer(x)
    assert float((layer.answer(x) - y).detach().abs().max()) <= 1e-4 * float(y.detach().abs().max())


def test_a_blocks_gradients(g):
    """Against the same block in plain torch and 64 bits.  Outputs: 1e-4 of the largest entry.  Rows and pre-activations that are
    kept in 8 bits are off by up to 2^-7 of the largest of 32, a slope or a weight's gradient by twice that: 2^-5 of the largest
    entry for what goes through both."""
    from paper_2208_09151_amd.experts import Block
    torch.manual_seed(11)
    rows, width, hidden, experts, top = 200, 48, 64, 6, 2
    block = Block(width, hidden, experts, top).cuda()
    x = torch.randn((rows, width), device="cuda", requires_grad=True)
    dy = torch.randn((rows, width), device="cuda")
    y = block(x)
    y.backward(dy)
    p = {k: v.detach().double().requires_grad_() for k, v in block.named_parameters()}
    xd = x.detach().double().requires_grad_()
    n = torch.nn.functional.layer_norm(xd, (width,), p["norm_weight"], p["norm_bias"])
    chosen = torch.topk(block.router(g.layer_norm(x.detach(), block.norm_weight.detach(), block.norm_bias.detach())), top, dim=1)[1]
    scores = (n @ p["router.weight"].t()).gather(1, chosen)
    z = torch.stack([(n[:, None, :] @ p["up"][chosen[:, j]])[:, 0] + p["up_bias"][chosen[:, j]] for j in range(top)], 1)
    h = (torch.softmax(scores, 1)[:, :, None] * activated(z, "gelu")).sum(1)
    want = h @ p["down.weight"].t() + p["down.bias"] + xd
    want.backward(dy.double())
    assert float((y.detach() - want.detach()).abs().max()) <= 1e-4 * float(want.detach().abs().max())
    for got, exact in [(x.grad, xd.grad)] + [(v.grad, p[k].grad) for k, v in block.named_parameters()]:
        assert float((got - exact).abs().max()) <= 2.0 ** -5 * float(exact.abs().max())
    assert torch.equal(x.grad, torch.autograd.grad(block(x), x, dy)[0])


def test_training_with_blocks(g):
    """Two steps over sampled batches: every parameter gets a gradient, the same in two runs."""
    from paper_2208_09151_amd.experts import train
    first, second = (train(config=1, steps=3, report=None, blocks=1) for _ in range(2))
    assert len(first) == 3 and all(l == l for l in first) and first[0] == second[0]


@pytest.mark.parametrize("rows", [40, 700])
def test_a_step_with_its_gradients_in_a_graph(g, rows):
    """Lookup, layer norm, a layer of experts and one for all with a residual, captured with their backward passes."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    table = rows_of(gen, 50, 32, torch.float32).requires_grad_()
    gain, shift = (torch.randn(32, generator=gen, device="cuda").requires_grad_() for _ in range(2))
    w3 = (torch.randn((4, 32, 24), generator=gen, device="cuda") / 6).requires_grad_()
    b3 = torch.randn((4, 24), generator=gen, device="cuda").requires_grad_()
    w = (torch.randn((24, 32), generator=gen, device="cuda") / 5).requires_grad_()
    leaves = (table, gain, shift, w3, b3, w)
    ids = torch.randint(0, 50, (rows,), generator=gen, device="cuda")
    chosen = torch.randint(-1, 4, (rows, 2), generator=gen, device="cuda")
    share = torch.rand((rows, 2), generator=gen, device="cuda")
    dy = rows_of(gen, rows, 32, torch.float32)

    def step():
        h = g.lookup(table, ids)
        r = g.route(chosen, 4)
        z = g.linear(g.layer_norm(h, gain, shift), w3, b3, "gelu", route=r)
        y = g.linear(g.combine(z, r, share), w, None, "silu", h)
        return (y.detach(), *torch.autograd.grad(y, leaves, dy))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        ids.copy_(torch.randint(0, 50, (rows,), generator=gen, device="cuda"))
        chosen.copy_(torch.randint(-1, 4, (rows, 2), generator=gen, device="cuda"))
        dy.copy_(rows_of(gen, rows, 32, torch.float32))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, step()))


def test_sums_of_neighbours(g):
    """Sums of rows and their gradients, exact for whole numbers."""
    from paper_2208_09151_amd.experts import SumOfRows
    gen = torch.Generator(device="cuda").manual_seed(3)
    rows = torch.randint(-9, 9, (300, 20), generator=gen, device="cuda").float().requires_grad_()
    of = torch.sort(torch.randint(0, 40, (300,), generator=gen, device="cuda"))[0]
    dy = torch.randint(-9, 9, (41, 20), generator=gen, device="cuda").float()
    y = SumOfRows.apply(rows, of, 41)
    assert torch.equal(y, torch.zeros((41, 20), device="cuda").index_add(0, of, rows.detach()))
    assert torch.equal(torch.autograd.grad(y, rows, dy)[0], dy[of])
