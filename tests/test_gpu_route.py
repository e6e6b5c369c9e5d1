"""Rows sorted by expert and back, against a plain implementation in 64 bits.

Tolerances, per element: a sum of k products in f32 is off by at most (k + 1) 2^-24 sum |terms| (Higham,
"Accuracy and Stability of Numerical Algorithms", 3.1), and rounding to the type by half a unit of it.
Everything else is copied or counted: equal.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
F32 = 2.0 ** -24


@pytest.fixture(scope="module")
def g():
    import paper_2208_09151_amd as lib
    return lib


def plain_route(chosen, experts, capacity=None):
    rows, top = chosen.shape
    flat = chosen.reshape(-1)
    slot = np.full(rows * top, -1, dtype=np.int32)
    source = np.full(rows * top, -1, dtype=np.int32)
    offsets = np.zeros(experts + 1, dtype=np.int64)
    at = 0
    for e in range(experts):
        pairs = np.flatnonzero(flat == e)
        if capacity is not None:
            pairs = pairs[:capacity]
        slot[pairs] = at + np.arange(len(pairs))
        source[at:at + len(pairs)] = pairs // top
        at += len(pairs)
        offsets[e + 1] = at
    return offsets, slot.reshape(rows, top), source


def choices(rows, top, experts, seed=0, absent=0.1):
    r = np.random.default_rng(seed)
    c = r.integers(0, experts, (rows, top))
    c = np.minimum(c, r.integers(0, experts, (rows, top)))         # the first ones are liked more
    c[r.random((rows, top)) < absent] = -1
    return c


def routed(g, chosen, experts, capacity=None, wide=True):
    t = torch.from_numpy(chosen).to(torch.int64 if wide else torch.int32).cuda()
    return g.route(t, experts, capacity=capacity)


def same_route(r, want):
    assert np.array_equal(r.offsets.cpu().numpy(), want[0])
    assert np.array_equal(r.slot.cpu().numpy(), want[1])
    assert np.array_equal(r.source.cpu().numpy(), want[2])


@pytest.mark.parametrize("rows, top, experts", [
    (0, 2, 4), (1, 1, 1), (1, 2, 8), (63, 1, 3), (64, 1, 64), (65, 3, 7), (1000, 8, 256), (4096, 2, 1024),
    (8192, 1, 5), (8193, 1, 5), (4097, 2, 1), (12_289, 1, 2), (3001, 64, 1023), (177_000, 2, 16),
    (100_003, 7, 1024)])
@pytest.mark.parametrize("wide", [True, False])
def test_route(g, rows, top, experts, wide):
    chosen = choices(rows, top, experts, seed=rows + top)
    same_route(routed(g, chosen, experts, None, wide), plain_route(chosen, experts))


@pytest.mark.parametrize("rows", [5, 700, 30_000])
@pytest.mark.parametrize("capacity", [0, 1, 37, 10 ** 12])
def test_route_with_a_capacity(g, rows, capacity):
    chosen = choices(rows, 3, 11, seed=rows)
    same_route(routed(g, chosen, 11, capacity), plain_route(chosen, 11, capacity))


@pytest.mark.parametrize("rows", [100, 20_000])
@pytest.mark.parametrize("value", [-1, 7, 6, 0, 1 << 40, -(1 << 40), (1 << 32) + 3])
def test_route_all_to_one_value(g, rows, value):
    chosen = np.full((rows, 2), value, dtype=np.int64)
    same_route(routed(g, chosen, 7), plain_route(chosen, 7))


@pytest.mark.parametrize("rows, top, experts", [(524_288, 8, 300), (524_289, 8, 300), (2_100_001, 2, 5)])
def test_route_of_many_tiles(g, rows, top, experts):
    chosen = choices(rows, top, experts, seed=rows)
    same_route(routed(g, chosen, experts, 1_000_000, False), plain_route(chosen, experts, 1_000_000))


# on both sides of the sizes from which the tiles' counts are scanned
@pytest.mark.parametrize("rows, top, experts", [
    (32_768, 2, 1024), (32_769, 2, 1024), (16_384, 8, 512), (16_385, 8, 512), (1_048_576, 4, 16), (1_048_577, 4, 16),
    (1_048_577, 4, 1)])
@pytest.mark.parametrize("capacity", [None, 2_000])
def test_route_with_and_without_a_scan(g, rows, top, experts, capacity):
    chosen = choices(rows, top, experts, seed=rows)
    same_route(routed(g, chosen, experts, capacity, False), plain_route(chosen, experts, capacity))


def test_route_refuses_a_workspace_elsewhere(g):
    good = torch.zeros((40_000, 2), dtype=torch.int64, device="cuda")
    with pytest.raises(ValueError, match="GPU memory"):
        g.route(good, 4, workspace=torch.empty(1 << 20, dtype=torch.uint8))
    with pytest.raises(ValueError, match="dtype"):
        g.route(good, 4, workspace=torch.empty(1 << 20, device="cuda"))
    with pytest.raises(ValueError, match="contiguous"):
        g.route(good, 4, workspace=torch.empty(1 << 21, dtype=torch.uint8, device="cuda")[::2])


def test_a_route_elsewhere_is_refused(g):
    r = g.route(torch.zeros((4, 2), dtype=torch.int64, device="cuda"), 4)
    x, z = torch.zeros((4, 8), device="cuda"), torch.zeros((8, 8), device="cuda")
    w = torch.zeros((4, 2), device="cuda")
    there = g.Route._made(r.offsets.cpu(), r.slot.cpu(), r.source.cpu())
    for call in (lambda: g.dispatch(x, there), lambda: g.combine(z, there, w), lambda: g.dispatch_backward(z, there),
                 lambda: g.combine_backward(x, z, there, w), lambda: g.weight_gradient(g.compress(x), z, there)):
        with pytest.raises(ValueError, match="route"):
            call()


def test_route_refusals(g):
    good = torch.zeros((4, 2), dtype=torch.int64, device="cuda")
    with pytest.raises(ValueError):
        g.route(good.float(), 4)
    with pytest.raises(ValueError):
        g.route(good.reshape(-1), 4)
    with pytest.raises(ValueError):
        g.route(good.t(), 4)
    with pytest.raises(ValueError):
        g.route(good, 4, capacity=-1)
    with pytest.raises(g.GinexError):
        g.route(good, 0)
    with pytest.raises(g.GinexError):
        g.route(good, 1025)
    with pytest.raises(g.GinexError):
        g.route(torch.zeros((4, 65), dtype=torch.int64, device="cuda"), 4)
    r = g.route(good, 4)
    with pytest.raises(ValueError):
        g.Route(r.offsets.int(), r.slot, r.source)
    with pytest.raises(ValueError):
        g.Route(r.offsets, r.slot, r.source[:-1])
    x = torch.zeros((4, 8), device="cuda")
    z = torch.zeros((8, 8), device="cuda")
    w = torch.zeros((4, 2), device="cuda")
    with pytest.raises(g.GinexError):
        g.dispatch(x[:3], r)
    with pytest.raises(ValueError):
        g.dispatch(x.double(), r)
    with pytest.raises(ValueError):
        g.dispatch(x.reshape(-1), r)
    with pytest.raises(ValueError):
        g.dispatch(torch.zeros((4, 16), device="cuda")[:, ::2], r)
    with pytest.raises(ValueError):
        g.dispatch(x, r, out=torch.zeros((8, 9), device="cuda"))
    with pytest.raises(g.GinexError):
        g.combine(x, r, w)
    with pytest.raises(ValueError):
        g.combine(z, r, w.half())
    with pytest.raises(ValueError):
        g.combine(z, r, w[:, :1])
    with pytest.raises(g.GinexError):
        g.combine(z, r, w, out=torch.zeros((4, 8), device="cuda")[:1].expand(4, 8))
    with pytest.raises(g.GinexError):
        g.combine_backward(x.half(), z, r, w)


SHAPES = [(1, 1, 1, 1), (1, 256, 2, 8), (5, 3, 1, 2), (130, 64, 3, 4), (257, 100, 5, 7), (64, 333, 4, 3),
          (33, 1025, 8, 16), (2000, 31, 9, 40), (4100, 128, 2, 6), (40, 9001, 1, 3), (300, 2500, 3, 5), (3, 600, 64, 90)]


def random_rows(shape, dtype, seed):
    t = torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float32)
    return t.to(dtype)


def strided(t, pad, shift):
    """The same rows on the GPU, `pad` elements apart and `shift` behind an aligned address."""
    rows, width = t.shape
    base = torch.full((rows * (width + pad) + shift,), float("nan"), dtype=t.dtype, device="cuda")
    view = base[shift:].view(rows, width + pad)[:, :width]
    view.copy_(t)
    return view


def near(got, want, slack, dtype):
    got, want, slack = got.cpu().double(), want.double(), slack.double()
    allowed = slack + UNIT[dtype] * (want.abs() + slack) + LEAST[dtype]
    bad = ~((got - want).abs() <= allowed)
    assert not bad.any(), (int(bad.sum()), float((got - want).abs().max()))


def combined(z, slot, weights):
    total = torch.zeros((slot.shape[0], z.shape[1]), dtype=torch.float64)
    size = torch.zeros_like(total)
    for j in range(slot.shape[1]):
        has = slot[:, j] >= 0
        part = z[slot[has, j].long()].double() * weights[has, j:j + 1].double()
        total[has] += part
        size[has] += part.abs()
    return total, size


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, width, top, experts", SHAPES)
@pytest.mark.parametrize("pad, shift", [(0, 0), (5, 1)])
def test_there_and_back(g, rows, width, top, experts, dtype, pad, shift):
    chosen = choices(rows, top, experts, seed=width)
    capacity = max(1, rows * top // experts)
    r = routed(g, chosen, experts, capacity)
    offsets, slot, source = (torch.from_numpy(a) for a in plain_route(chosen, experts, capacity))
    slots = rows * top
    x, z, dy = (random_rows(s, dtype, i) for i, s in enumerate([(rows, width), (slots, width), (rows, width)]))
    w = random_rows((rows, top), torch.float32, 9)
    hidden = w.clone()
    hidden[slot < 0] = float("nan")             # a weight without a slot does not count, whatever it is
    z[int(offsets[-1]):] = float("nan")         # nor a slot without a row

    found = torch.zeros((slots, width), dtype=dtype)
    found[source >= 0] = x[source[source >= 0].long()]
    assert torch.equal(g.dispatch(strided(x, pad, shift), r).cpu(), found)

    want, size = combined(z, slot, w)
    near(g.combine(strided(z, pad, shift), r, hidden.cuda()), want, (top + 1) * F32 * size, dtype)
    want, size = combined(z, slot, torch.ones_like(w))
    near(g.dispatch_backward(strided(z, pad, shift), r), want, (top + 1) * F32 * size, dtype)

    dz, dw = g.combine_backward(strided(dy, pad, shift), strided(z, pad, shift), r, hidden.cuda())
    kept = slot >= 0
    by = torch.zeros(slots, dtype=torch.float64)
    by[slot[kept].long()] = w[kept].double()
    want = torch.zeros((slots, width), dtype=torch.float64)
    want[source >= 0] = dy[source[source >= 0].long()].double()
    want *= by[:, None]
    near(dz, want, F32 * want.abs(), dtype)
    products = dy[:, None, :].double() * torch.where(kept[:, :, None], z[slot.clamp(min=0).long()].double(), 0.0)
    near(dw, products.sum(2), width * F32 * products.abs().sum(2), torch.float32)


@pytest.mark.parametrize("dtype", TYPES)
def test_written_rows_stay_inside_their_width(g, dtype):
    chosen = choices(50, 2, 5)
    r = routed(g, chosen, 5)
    x = random_rows((50, 37), dtype, 1).cuda()
    out = torch.full((100, 48), 7.0, dtype=dtype, device="cuda")
    g.dispatch(x, r, out=out[:, 3:40])
    assert (out[:, :3] == 7).all() and (out[:, 40:] == 7).all()
    y = torch.full((50, 48), 7.0, dtype=dtype, device="cuda")
    g.dispatch_backward(out[:, 3:40], r, out=y[:, 3:40])
    assert (y[:, :3] == 7).all() and (y[:, 40:] == 7).all()
    count = torch.from_numpy((plain_route(chosen, 5)[1] >= 0).sum(1)).cuda()
    assert torch.equal(y[:, 3:40], (x.double() * count[:, None]).to(dtype))     # 0, 1 or 2 times the row


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [5, 32, 37])
def test_dispatch_copies_bits(g, dtype, width):
    """Whatever a row holds, NaNs of any bits and subnormal numbers among it."""
    words = torch.int32 if dtype == torch.float32 else torch.int16
    low, high = torch.iinfo(words).min, torch.iinfo(words).max
    x = torch.randint(low, high, (200, width), dtype=words, generator=torch.Generator().manual_seed(width))
    r = routed(g, choices(200, 2, 5, absent=0), 5)
    out = g.dispatch(x.cuda().view(dtype), r).view(words).cpu()
    assert torch.equal(out, x[r.source.cpu().long()])


def test_one_row_for_all(g):
    chosen = choices(300, 2, 5, absent=0)
    r = routed(g, chosen, 5)
    x = torch.randn((1, 64), device="cuda")
    assert torch.equal(g.dispatch(x.expand(300, 64), r), x.expand(600, 64))
    dz, _ = g.combine_backward(x.expand(300, 64), torch.zeros((600, 64), device="cuda"), r,
                               torch.ones((300, 2), device="cuda"))
    assert torch.equal(dz, x.expand(600, 64))


@pytest.mark.parametrize("chosen", [np.full((9, 2), -1), np.zeros((0, 2), dtype=np.int64)])
def test_no_slot_at_all(g, chosen):
    n = len(chosen)
    r = routed(g, chosen, 3)
    x = torch.full((n, 20), float("nan"), device="cuda")
    z = torch.full((2 * n, 20), float("inf"), device="cuda")
    w = torch.full((n, 2), float("nan"), device="cuda")
    assert torch.equal(g.dispatch(x, r), torch.zeros((2 * n, 20), device="cuda"))
    assert torch.equal(g.combine(z, r, w), torch.zeros((n, 20), device="cuda"))
    dz, dw = g.combine_backward(x, z, r, w)
    assert torch.equal(dz, torch.zeros((2 * n, 20), device="cuda")) and torch.equal(dw, torch.zeros((n, 2), device="cuda"))


def test_values_that_are_no_numbers_stay_in_their_rows(g):
    chosen = choices(40, 2, 4, absent=0)
    r = routed(g, chosen, 4)
    z = torch.ones((80, 33), device="cuda")
    hit = int(r.slot[7, 1])
    z[hit, 5] = float("inf")
    z[hit, 6] = float("nan")
    y = g.combine(z, r, torch.ones((40, 2), device="cuda"))
    assert y[7, 5] == float("inf") and y[7, 6].isnan()
    y[7, 5:7] = 2
    assert (y == 2).all()


def test_slots_of_a_routing_made_elsewhere_are_checked(g):
    """Slots and offsets that are not there count as none: nothing outside the arrays is touched."""
    big = torch.tensor([[0, 1 << 30], [-5, 1]], dtype=torch.int32, device="cuda")
    source = torch.tensor([0, 1, 1 << 30, -9], dtype=torch.int32, device="cuda")
    r = g.Route(torch.tensor([0, 2, 1 << 50], device="cuda"), big, source)
    x = torch.tensor([[1.0], [2.0]], device="cuda")
    out = g.dispatch(x, r, out=torch.zeros((4, 1), device="cuda"))
    assert out.flatten().tolist() == [1, 2, 0, 0]
    assert g.combine(out, r, torch.ones((2, 2), device="cuda")).flatten().tolist() == [1, 2]


def test_gradients_against_differences(g):
    """combine is linear in z and in the weights: a difference quotient is off by rounding alone.  Sums of
    at most 64 * 128 products of numbers around 1 in f32, steps of 1: below 1e-3 of their size."""
    chosen = choices(60, 3, 5, absent=0.2)
    r = routed(g, chosen, 5, 30)
    gen = torch.Generator(device="cuda").manual_seed(3)
    z, dy, w, dirz, dirw, x, dirx = (torch.randn(s, generator=gen, device="cuda") for s in
                                     [(180, 48), (60, 48), (60, 3), (180, 48), (60, 3), (60, 48), (60, 48)])
    dz, dw = g.combine_backward(dy, z, r, w)
    dot = lambda a, b: float((a.double() * b.double()).sum())
    size = lambda a, b: float((a.double() * b.double()).abs().sum())
    by_z = dot(dy, g.combine(z + dirz, r, w)) - dot(dy, g.combine(z - dirz, r, w))
    assert abs(by_z / 2 - dot(dz, dirz)) < 1e-3 * size(dz, dirz)
    by_w = dot(dy, g.combine(z, r, w + dirw)) - dot(dy, g.combine(z, r, w - dirw))
    assert abs(by_w / 2 - dot(dw, dirw)) < 1e-3 * size(dw, dirw)
    by_x = dot(z, g.dispatch(x + dirx, r)) - dot(z, g.dispatch(x - dirx, r))
    dx = g.dispatch_backward(z, r)
    assert abs(by_x / 2 - dot(dx, dirx)) < 1e-3 * size(dx, dirx)


def test_equal_bits_on_other_streams_and_in_a_graph(g):
    chosen = choices(20_000, 2, 9)
    t = torch.from_numpy(chosen).cuda()
    x = random_rows((20_000, 96), torch.bfloat16, 2).cuda()
    w = torch.randn((20_000, 2), device="cuda")

    def step():
        r = g.route(t, 9, capacity=4000)
        rows = g.dispatch(x, r)
        y = g.combine(rows, r, w)
        return (r.offsets, r.slot, r.source, rows, y, *g.combine_backward(x, rows, r, w))

    first = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        made = step()
    for seed in range(3):
        x.copy_(random_rows((20_000, 96), torch.bfloat16, 10 + seed))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(step(), made))


def test_rows_beyond_2_to_the_31_elements(g):
    """1.2 M rows in 2.4 M slots of 1024: offsets pass 32 bits in elements and in bytes."""
    n, width = 1_200_000, 1024
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty((n, width), dtype=torch.float16, device="cuda").normal_(generator=gen)
    chosen = torch.randint(0, 4, (n, 2), generator=gen, device="cuda")
    r = g.route(chosen, 4)
    rows = g.dispatch(x, r)
    at = torch.randint(0, 2 * n, (5000,), generator=gen, device="cuda")
    at[-1] = 2 * n - 1
    assert torch.equal(rows[at], x[r.source[at].long()])
    y = g.dispatch_backward(rows, r)
    at = torch.cat([at[:-1] // 2, torch.tensor([n - 1], device="cuda")])
    assert torch.equal(y[at], 2 * x[at])
    dz, dw = g.combine_backward(x, rows, r, torch.ones((n, 2), device="cuda"))
    last = torch.arange(2 * n - 1000, 2 * n, device="cuda")
    assert torch.equal(dz[last], rows[last])
    want = x[at].double().square().sum(1)
    assert ((dw[at, 0].double() - want).abs() <= width * F32 * want).all()


def test_gradient_of_more_rows_than_a_launch_has(g):
    """2^25 rows of 33 chunks and up, a wave each, make 2^31 threads; one row for all of dy and of z."""
    n, width = (1 << 25) + 3, 257
    dy = random_rows((1, width), torch.bfloat16, 3).cuda()
    z = random_rows((1, width), torch.bfloat16, 4).cuda()
    chosen = torch.zeros((n, 1), dtype=torch.int32, device="cuda")
    chosen[5] = -1                                                    # the last slot is empty
    r = g.route(chosen, 1)
    w = torch.ones((n, 1), device="cuda")
    w[-2:] = 2
    dz, dw = g.combine_backward(dy.expand(n, width), z.expand(n, width), r, w)
    for at in range(0, n, 1 << 22):
        part = dz[at:at + (1 << 22)]
        want = dy.expand_as(part).clone()
        if at + (1 << 22) >= n:
            want[-3:-1] *= 2
            want[-1] = 0
        assert torch.equal(part, want)
    want = (dy.double() * z.double()).sum()
    bound = (width + 1) * F32 * (dy.double() * z.double()).abs().sum()
    dw = dw[:, 0].double()
    assert float(dw[5]) == 0
    dw[5] = want
    assert float((dw - want).abs().max()) <= float(bound)
