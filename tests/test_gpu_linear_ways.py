"""linear at the sizes that its rules send to different kernels, against plain torch in 64 bits."""
import pytest
import torch

from layer_reference import TYPES, linear as plain, near, random_route, rounded, rows_of
from test_gpu_linear import weights_of

pytestmark = pytest.mark.gpu

# few workgroups, whose 4, 8 or 16 waves share the width
FEW = [(1000, 30, 130), (300, 200, 64), (300, 1000, 64), (4000, 1000, 100)]
# tiles of 32, 64 and 128 rows, of 64 and of 128 columns
TILES = [(20000, 50, 64), (131040, 20, 40), (131100, 450, 40), (9000, 36, 100), (26000, 40, 100), (40000, 24, 400), (60000, 16, 800)]
# weights in LDS: 1, 2 and 4 times 64 columns of 1, 2 to 3 and more units of 128 bytes, in one, two and more blocks
RESIDENT = [(160001, 8, 8), (160003, 100, 47), (160016, 60, 130), (160040, 300, 70), (160000, 130, 257), (160015, 1000, 65),
            (160100, 520, 100), (160001, 64, 200), (160017, 250, 128)]


@pytest.fixture(scope="module")
def g():
    import paper_2208_09151_amd as lib
    return lib


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("rows, width, out", FEW + TILES + RESIDENT)
def test_sizes(g, rows, width, out, turned, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows + width + out)
    x = rows_of(gen, rows, width, dtype, width + 3)
    w = weights_of(gen, (width, out), dtype, turned, pad=1)
    bias = torch.randn(out, generator=gen, device="cuda").to(dtype)
    want, off, _ = plain(x, w, None, None, None, dtype)
    near(g.linear(x, w), want, rounded(want, off, dtype))
    res = rows_of(gen, rows, out, dtype, out + 5)
    want, off, _ = plain(x, w, bias, "silu", res, dtype)
    got = g.linear(x, w, bias, "silu", res)
    near(got, want, rounded(want, off, dtype))
    assert torch.equal(g.linear(x, w, bias, "silu", res, out=res), got)        # in place of the residual


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, width, out", [FEW[3], TILES[0], TILES[1], TILES[3], TILES[5]] + RESIDENT[:5])
def test_kept_and_numbers_that_are_none(g, rows, width, out, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows + 1)
    x = rows_of(gen, rows, width, dtype)
    w = weights_of(gen, (width, out), dtype, False)
    bias = torch.randn(out, generator=gen, device="cuda").to(dtype)
    clean, kept = g.linear(x, w, bias, "gelu", keep=True)
    assert torch.equal(clean, g.linear(x, w, bias, "gelu"))
    _, off, z = plain(x, w, bias, None, None, dtype)
    blocks = -(-out // 32)
    padded = torch.zeros((rows, blocks * 32), dtype=torch.float64, device="cuda")
    padded[:, :out] = z.abs()
    most = padded.view(rows, blocks, 32).amax(2)
    step = torch.exp2(torch.floor(torch.log2(most)) - 6).repeat_interleave(32, 1)[:, :out]
    near(g.restore(kept), z, step * 1.01 + off)
    assert bool((kept.codes[:, out:] == 0).all())
    x[2, 3], x[rows - 1, width - 1] = float("inf"), float("nan")
    y, k = g.linear(x, w, bias, keep=True)
    clean, kept = g.linear(torch.nan_to_num(x, 1.0, 1.0), w, bias, keep=True)
    assert torch.equal(y[2], torch.where(w[3] > 0, float("inf"), -float("inf")).to(dtype)) and bool(torch.isnan(y[-1]).all())
    assert bool((k.scales[[2, rows - 1]] == 255).all()) and bool((k.codes[[2, rows - 1]] == 0).all())
    others = torch.ones(rows, dtype=torch.bool, device="cuda")
    others[2] = others[-1] = False
    assert torch.equal(y[others], clean[others]) and torch.equal(k.codes[others], kept.codes[others])
    x[2, 3], x[rows - 1, width - 1] = 1, 1
    clean = g.linear(x, w)
    w[width - 1, out - 1] = float("nan")
    y = g.linear(x, w)
    assert bool(torch.isnan(y[:, -1]).all()) and torch.equal(y[:, :-1], clean[:, :-1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("rows, top, experts, width, out, capacity", [
    (150, 2, 40, 300, 64, None), (20000, 2, 3, 60, 64, None), (20000, 2, 40, 60, 130, 900), (40001, 4, 5, 100, 47, None),
    (40001, 4, 1, 60, 200, None), (20011, 8, 40, 300, 70, 3000), (20011, 8, 2, 130, 300, 60000), (20011, 8, 300, 60, 40, None)])
def test_layers_of_experts(g, rows, top, experts, width, out, capacity, turned, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows + experts)
    r = random_route(g, gen, rows, top, experts, capacity)
    x = rows_of(gen, rows, width, dtype, width + 1)
    w = weights_of(gen, (experts, width, out), dtype, turned, pad=2)
    bias = torch.randn((experts, out), generator=gen, device="cuda").to(dtype)
    res = rows_of(gen, rows * top, out, dtype)
    ends = r.offsets.tolist()
    want = torch.zeros((rows * top, out), dtype=torch.float64, device="cuda")
    off = torch.zeros_like(want)
    slots = g.dispatch(x, r)
    for e in range(experts):
        a, b = ends[e], ends[e + 1]
        if b > a:
            want[a:b], off[a:b], _ = plain(slots[a:b], w[e], bias[e], "relu", res[a:b], dtype)
    allowed = rounded(want, off, dtype)
    allowed[ends[-1]:] = 0
    y, kept = g.linear(x, w, bias, "relu", res, r, keep=True)
    near(y, want, allowed)
    assert torch.equal(g.linear(slots, w, bias, "relu", res, r, slots=True), y)
    assert bool((kept.codes[ends[-1]:] == 0).all()) and bool((kept.codes[:, out:] == 0).all())
    room = torch.full((rows * top + 2, out + 8), 7.0, device="cuda", dtype=dtype)
    g.linear(x, w, bias, "relu", res, r, out=room[1:-1, 4:-4])
    assert torch.equal(room[1:-1, 4:-4], y)
    room[1:-1, 4:-4] = 7.0
    assert bool((room == 7.0).all())
    # rows and offsets that do not exist count as none
    source = r.source.clone()
    source[0], source[1], source[2] = -1, rows, 2 ** 31 - 1
    room = torch.full((rows * top + 2, out), 7.0, device="cuda", dtype=dtype)
    g.linear(x, w, route=g.Route(r.offsets, r.slot, source), out=room[1:-1])
    assert bool((room[1:4] == 0).all())
    bad = r.offsets.clone()
    bad[0], bad[-1] = -2 ** 60, 2 ** 61
    g.linear(x, w, route=g.Route(bad, r.slot, source), out=room[1:-1])
    assert bool((room[0] == 7).all()) and bool((room[-1] == 7).all())


@pytest.mark.parametrize("rows, width, out", [FEW[3], TILES[1], TILES[4], RESIDENT[2]])
def test_graphs(g, rows, width, out):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = rows_of(gen, rows, width, torch.float32)
    w = weights_of(gen, (width, out), torch.float32, False)
    graph = torch.cuda.CUDAGraph()
    g.linear(x, w, None, "gelu")
    with torch.cuda.graph(graph):
        got = g.linear(x, w, None, "gelu")
    for _ in range(3):
        x.copy_(rows_of(gen, rows, width, torch.float32))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, g.linear(x, w, None, "gelu"))


@pytest.mark.parametrize("rows, width, out", [FEW[2], TILES[3], TILES[6], RESIDENT[2], RESIDENT[6]])
def test_f32_of_all_magnitudes(g, rows, width, out):
    """Products of large and small numbers, and rows whose parts are beyond bf16's ends: a factor loses less than 2^-133."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    for of_x, of_w in [(2.0 ** -118, 2.0 ** 60), (2.0 ** 118, 2.0 ** -100), (2.0 ** 60, 2.0 ** -120)]:
        x = rows_of(gen, rows, width, torch.float32, by=of_x)
        w = weights_of(gen, (width, out), torch.float32, False) * of_w
        want, off, _ = plain(x, w, None, None, None, torch.float32)
        lost = 2.0 ** -133 * (x.double().abs().sum(1, keepdim=True) + w.double().abs().sum(0))
        near(g.linear(x, w), want, rounded(want, off + lost, torch.float32))
    # the largest numbers, which are none in bf16
    most = torch.finfo(torch.float32).max
    x = rows_of(gen, rows, width, torch.float32)
    w = weights_of(gen, (width, out), torch.float32, False) * 2.0 ** -20
    x[3, width // 2] = x[rows - 1, 0] = most
    want, off, _ = plain(x, w, None, None, None, torch.float32)
    near(g.linear(x, w), want, rounded(want, off, torch.float32))
