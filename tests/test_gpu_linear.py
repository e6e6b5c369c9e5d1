"""linear, linear_backward and bias_gradient against plain torch in 64 bits."""
import pytest
import torch

from layer_reference import LEAST, ROUND, TYPES, linear as plain, near, random_route, rounded, rows_of

pytestmark = pytest.mark.gpu

# (rows, width, out): one of everything, odd sizes, ends inside chunks, tiles and columns, both sides of 64 rows, and sizes that
# take the largest tiles
SIZES = [(1, 1, 1), (1, 16, 16), (2, 3, 2), (3, 5, 7), (16, 64, 64), (17, 100, 47), (48, 1000, 33), (64, 130, 129), (65, 8, 300),
         (130, 333, 65), (300, 64, 64), (129, 63, 66), (1000, 250, 131), (257, 1027, 3), (8200, 40, 1000), (131200, 24, 40),
         (131100, 9, 63)]


@pytest.fixture(scope="module")
def g():
    import paper_2208_09151_amd as lib
    return lib


def weights_of(gen, shape, dtype, turned, pad=0):
    """[.., width, out] with `pad` elements between rows, turned: between columns."""
    *count, width, out = shape
    dense, other = (width, out) if turned else (out, width)
    w = torch.randn((*count, other, dense + pad), generator=gen, device="cuda")
    w = (w / width ** 0.5).to(dtype)[..., :dense]
    return w.mT if turned else w


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("rows, width, out", SIZES)
def test_sizes(g, rows, width, out, turned, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows + width + out)
    x = rows_of(gen, rows, width, dtype)
    w = weights_of(gen, (width, out), dtype, turned)
    bias = torch.randn(out, generator=gen, device="cuda").to(dtype)
    res = rows_of(gen, rows, out, dtype)
    for activation, b, r in [(None, None, None), ("gelu", bias, res)]:
        want, off, _ = plain(x, w, b, activation, r, dtype)
        near(g.linear(x, w, b, activation, r), want, rounded(want, off, dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("activation", [None, "relu", "silu", "gelu"])
@pytest.mark.parametrize("rows", [5, 200])
def test_activations_strides_and_outputs(g, rows, activation, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    width, out = 77, 91
    x = rows_of(gen, rows, width, dtype, 101)
    bias = torch.randn(out, generator=gen, device="cuda").to(dtype)
    one = rows_of(gen, 1, out, dtype).expand(rows, out)            # one row for all
    for turned in (False, True):
        w = weights_of(gen, (width, out), dtype, turned, pad=5)
        want, off, _ = plain(x, w, bias, activation, one, dtype)
        room = torch.full((rows + 2, 103), 7.0, device="cuda", dtype=dtype)
        to = room[1:1 + rows, 3:3 + out]
        assert g.linear(x, w, bias, activation, one, out=to) is to
        near(to, want, rounded(want, off, dtype))
        room[1:1 + rows, 3:3 + out] = 7.0
        assert bool((room == 7.0).all())                          # nothing beside it is written
        # in place of the residual
        res = rows_of(gen, rows, out, dtype, 103)
        want, off, _ = plain(x, w, None, activation, res.clone(), dtype)
        assert g.linear(x, w, None, activation, res, out=res) is res
        near(res, want, rounded(want, off, dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("rows, top, experts, width, out, capacity", [
    (1, 1, 1, 16, 16, None), (1, 2, 8, 100, 47, None), (20, 3, 5, 64, 70, 4), (30, 2, 1024, 33, 17, None),
    (500, 4, 7, 100, 333, 200), (700, 2, 1000, 40, 64, None), (9000, 8, 3, 24, 129, 20000), (3000, 2, 2, 130, 64, 0)])
def test_layers_of_experts(g, rows, top, experts, width, out, capacity, turned, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows + experts)
    r = random_route(g, gen, rows, top, experts, capacity)
    x = rows_of(gen, rows, width, dtype, width + 3)
    w = weights_of(gen, (experts, width, out), dtype, turned)
    bias = torch.randn((experts, out), generator=gen, device="cuda").to(dtype)
    res = rows_of(gen, rows * top, out, dtype)
    ends = r.offsets.tolist()
    want = torch.zeros((rows * top, out), dtype=torch.float64, device="cuda")
    off = torch.zeros_like(want)
    slots = g.dispatch(x, r)
    for e in range(experts):
        a, b = ends[e], ends[e + 1]
        if b > a:
            want[a:b], off[a:b], _ = plain(slots[a:b], w[e], bias[e], "silu", res[a:b], dtype)
    allowed = rounded(want, off, dtype)
    allowed[ends[-1]:] = 0                      # cleared, whatever the residual
    got = g.linear(x, w, bias, "silu", res, route=r)
    near(got, want, allowed)
    assert torch.equal(g.linear(slots, w, bias, "silu", res, route=r, slots=True), got)
    # gradients of rows and biases
    dz = rows_of(gen, rows * top, out, dtype)
    drows = g.linear_backward(dz, w, route=r)
    want = torch.zeros((rows * top, width), dtype=torch.float64, device="cuda")
    off = torch.zeros_like(want)
    dbias = torch.zeros((experts, out), dtype=torch.float64, device="cuda")
    boff = torch.zeros_like(dbias)
    for e in range(experts):
        a, b = ends[e], ends[e + 1]
        if b > a:
            want[a:b], off[a:b], _ = plain(dz[a:b], w[e].mT, None, None, None, dtype)
            dbias[e] = dz[a:b].double().sum(0)
            boff[e] = (b - a) * 2.0 ** -24 * dz[a:b].double().abs().sum(0)
    allowed = rounded(want, off, dtype)
    allowed[ends[-1]:] = 0
    near(drows, want, allowed)
    near(g.bias_gradient(dz, r), dbias, boff)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, width", [(0, 5), (1, 1), (3, 7), (100, 64), (1000, 333), (300, 5000), (70000, 24), (200000, 8)])
def test_bias_gradient(g, rows, width, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows + width)
    dz = rows_of(gen, rows, width, dtype, width + 1)
    want = dz.double().sum(0)
    near(g.bias_gradient(dz), want, rows * 2.0 ** -24 * dz.double().abs().sum(0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, width, out", [(7, 60, 100), (64, 33, 31), (300, 60, 100), (200, 16, 1)])
def test_kept_is_the_activations_argument(g, rows, width, out, dtype):
    """Codes are off by at most half a step of 2^-6 of the block's exponent, and by a step more where a f32 sum falls on the
    other side of a border; an exponent, too, may be the next one."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = rows_of(gen, rows, width, dtype)
    w = weights_of(gen, (width, out), dtype, False)
    bias = torch.randn(out, generator=gen, device="cuda").to(dtype)
    want, off, z = plain(x, w, bias, "gelu", None, dtype)
    y, kept = g.linear(x, w, bias, "gelu", keep=True)
    near(y, want, rounded(want, off, dtype))
    assert torch.equal(y, g.linear(x, w, bias, "gelu"))
    blocks = -(-out // 32)
    padded = torch.zeros((rows, blocks * 32), dtype=torch.float64, device="cuda")
    padded[:, :out] = z.abs()
    most = padded.view(rows, blocks, 32).amax(2)
    step = torch.exp2(torch.floor(torch.log2(most)) - 6).repeat_interleave(32, 1)[:, :out]
    near(g.restore(kept), z, step * 1.01 + off)       # 127 steps at most: the largest may be a whole step off
    assert bool((kept.codes[:, out:] == 0).all())
    # what compress makes of the same f32 numbers
    if dtype == torch.float32:
        same = g.compress(g.linear(x, w, bias))
        assert torch.equal(kept.codes, same.codes) and torch.equal(kept.scales, same.scales)


def test_kept_of_slots_without_a_row(g):
    gen = torch.Generator(device="cuda").manual_seed(3)
    for rows in (10, 100):
        r = random_route(g, gen, rows, 2, 4, absent=0.5)
        x = rows_of(gen, rows, 40, torch.float32)
        w = weights_of(gen, (4, 40, 50), torch.float32, False)
        y, kept = g.linear(x, w, None, "relu", route=r, keep=True)
        end = int(r.offsets[-1])
        assert end < rows * 2 and bool((y[end:] == 0).all()) and bool((kept.codes[end:] == 0).all())
        assert bool((g.restore(kept)[end:] == 0).all())


@pytest.mark.parametrize("rows", [9, 200])
@pytest.mark.parametrize("dtype", TYPES)
def test_numbers_that_are_none(g, rows, dtype):
    """Infinities and NaN stay in their rows and columns, and their blocks of codes stand for NaN."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = rows_of(gen, rows, 50, dtype)
    w = weights_of(gen, (50, 70), dtype, False)
    clean, kept = g.linear(x, w, keep=True)
    inf, nan = float("inf"), float("nan")
    x[2, 3], x[4, 5] = inf, nan
    y, k = g.linear(x, w, keep=True)
    assert torch.equal(y[2], torch.where(w[3] > 0, inf, -inf).to(dtype)) and bool(torch.isnan(y[4]).all())
    others = [i for i in range(rows) if i not in (2, 4)]
    assert torch.equal(y[others], clean[others]) and torch.equal(k.codes[others], kept.codes[others])
    assert bool((k.scales[[2, 4]] == 255).all()) and bool((k.codes[[2, 4]] == 0).all())
    x[2, 3], x[4, 5] = 1, 1
    clean = g.linear(x, w)
    w[49, 69] = nan                             # the last of the width in the last column
    y = g.linear(x, w)
    assert bool(torch.isnan(y[:, 69]).all()) and torch.equal(y[:, :69], clean[:, :69])


@pytest.mark.parametrize("shape", [(0, 5, 7), (0, 64, 64)])
def test_no_rows(g, shape):
    rows, width, out = shape
    x = torch.zeros((rows, width), device="cuda")
    w = torch.zeros((width, out), device="cuda")
    assert g.linear(x, w, torch.zeros(out, device="cuda"), "relu").shape == (0, out)
    assert g.linear_backward(torch.zeros((0, out), device="cuda"), w).shape == (0, width)
    r = g.route(torch.zeros((0, 2), dtype=torch.int64, device="cuda"), 3)
    assert g.linear(x, w.expand(3, width, out), route=r).shape == (0, out)
    assert bool((g.bias_gradient(torch.zeros((0, out), device="cuda"), r) == 0).all())


@pytest.mark.parametrize("rows", [20, 500])
def test_a_foreign_route_reaches_nothing_else(g, rows):
    """Rows and offsets that do not exist count as none."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = rows_of(gen, rows, 40, torch.float32)
    w = weights_of(gen, (3, 40, 50), torch.float32, False)
    r = g.route(torch.zeros((rows, 1), dtype=torch.int64, device="cuda"), 3)
    clean = g.linear(x, w, route=r)
    source = r.source.clone()
    source[4], source[5], source[6] = -1, rows, 2 ** 31 - 1
    y = g.linear(x, w, route=g.Route(r.offsets, r.slot, source))
    want = clean.clone()
    want[4:7] = 0
    assert torch.equal(y, want)
    for offsets in ([0, -5, 2 ** 40, rows], [0, rows, 3, rows + 100], [-7, 2, -2 ** 60, 5], [2 ** 62, 0, 0, 0]):
        bad = g.Route(torch.tensor(offsets, device="cuda"), r.slot, source)
        room = torch.full((rows + 2, 50), 7.0, device="cuda")
        g.linear(x, w, route=bad, out=room[1:-1])
        torch.cuda.synchronize()
        assert bool((room[0] == 7).all()) and bool((room[-1] == 7).all())
        assert g.bias_gradient(y, bad).shape == (3, 50)


@pytest.mark.parametrize("rows", [30, 1000])
def test_equal_calls_give_equal_bits_on_any_stream_and_in_graphs(g, rows):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    r = random_route(g, gen, rows, 2, 6)
    x = rows_of(gen, rows, 96, torch.bfloat16)
    w = weights_of(gen, (6, 96, 80), torch.bfloat16, False)
    dz = rows_of(gen, 2 * rows, 80, torch.bfloat16)

    def both():
        return g.linear(x, w, None, "gelu", route=r), g.linear_backward(dz, w, r), g.bias_gradient(dz, r)

    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for _ in range(3):
        x.copy_(rows_of(gen, rows, 96, torch.bfloat16))
        dz.copy_(rows_of(gen, 2 * rows, 80, torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, both()))


def test_refusals(g):
    x, w = torch.zeros((9, 4), device="cuda"), torch.zeros((4, 6), device="cuda")
    r = g.route(torch.zeros((9, 2), dtype=torch.int64, device="cuda"), 3)
    w3 = torch.zeros((3, 4, 6), device="cuda")
    for call, says in [(lambda: g.linear(x, w.half()), "dtype"), (lambda: g.linear(x, w3), "weight"),
                       (lambda: g.linear(x, w, route=r), "weight"), (lambda: g.linear(x, w, slots=True), "route"),
                       (lambda: g.linear(x, w, torch.zeros(5, device="cuda")), "bias"),
                       (lambda: g.linear(x, w, torch.zeros(6, device="cuda").half()), "bias"),
                       (lambda: g.linear(x, w, None, "tanh"), "activation"),
                       (lambda: g.linear(x, w, residual=torch.zeros((9, 5), device="cuda")), "residual"),
                       (lambda: g.linear(x, w3, residual=torch.zeros((9, 6), device="cuda"), route=r), "residual"),
                       (lambda: g.linear(x, torch.zeros((8, 12), device="cuda")[::2, ::2]), "dense"),
                       (lambda: g.linear(x, w, out=torch.zeros((9, 5), device="cuda")), "out"),
                       (lambda: g.linear(x.cpu(), w), "GPU"), (lambda: g.linear(x, w.cpu()), "GPU"),
                       (lambda: g.linear(x.double(), w.double()), "float32"),
                       (lambda: g.bias_gradient(x, out=torch.zeros(5, device="cuda")), "out")]:
        with pytest.raises(ValueError, match=says):
            call()
    for call, says in [(lambda: g.linear(x, torch.zeros((5, 6), device="cuda")), "wide"),
                       (lambda: g.linear(x, w3, route=r, slots=True), "slots"),
                       (lambda: g.linear(x[:8], w3, route=r), "rows"),
                       (lambda: g.linear(x, torch.zeros((4, 4, 6), device="cuda"), route=r), "experts"),
                       (lambda: g.bias_gradient(x, r), "slots")]:
        with pytest.raises(g.GinexError, match=says):
            call()
