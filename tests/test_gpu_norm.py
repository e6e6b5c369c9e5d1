"""layer_norm and its gradients against plain torch in 64 bits.

With u = 2^-24 and n numbers a row, a mean in f32 is off by n u of the mean magnitude at most; the kernel adds lanes up in a tree
and takes away what is left of the mean, so that what remains is (n / 64 + 12) u of the mean distance, counted as n u + 32 u.
unit is then off by (2 n + 64) u (1 + |unit|), y by that times |weight| and a few roundings more.
"""
import pytest
import torch

from layer_reference import LEAST, ROUND, TYPES, near, rounded, rows_of

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
WIDTHS = [1, 2, 3, 7, 8, 31, 64, 100, 256, 333, 512, 1000, 1025, 2048, 2500, 4096, 8200, 20000]


@pytest.fixture(scope="module")
def g():
    import paper_2208_09151_amd as lib
    return lib


def plain(x, weight, bias, eps):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + eps)
    unit = (x - mean) * rstd
    w = torch.ones_like(unit) if weight is None else weight.double().expand_as(unit)
    y = unit * w + (0 if bias is None else bias.double())
    return y, unit, rstd, w, mean


def off_of_unit(unit, rstd, mean, width):
    """x - mean loses nothing but the rounding of the difference (|x| u of what is far from 0 is in x already)."""
    return (2 * width + 64) * U * (1 + unit.abs()) + 2 * U * rstd * mean.abs() * 2.0 ** -20


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("rows", [1, 37])
def test_forward_and_backward(g, rows, width, dtype):
    gen = torch.Generator(device="cuda").manual_seed(width + rows)
    x = rows_of(gen, rows, width, dtype, width + 3) * 3 + 1
    weight = (torch.randn(width, generator=gen, device="cuda") * 0.2 + 1).to(dtype)
    bias = torch.randn(width, generator=gen, device="cuda").to(dtype)
    dy = rows_of(gen, rows, width, dtype)
    eps = 1e-3
    for w, b in [(weight, bias), (None, None)]:
        want, unit, rstd, wd, mean = plain(x, w, b, eps)
        y, stats = g.layer_norm(x, w, b, eps, stats=True)
        off = off_of_unit(unit, rstd, mean, width)
        near(y, want, rounded(want, off * wd.abs() + 4 * U * (want.abs() + (unit * wd).abs()), dtype))
        near(stats, torch.cat([mean, rstd], 1), torch.cat([(width * U) * x.double().abs().mean(1, keepdim=True) + U,
                                                           (2 * width + 64) * U * rstd], 1))
        d = dy.double()
        a = d * wd
        am, aum = a.mean(1, keepdim=True), (a * unit).mean(1, keepdim=True)
        dx = rstd * (a - am - unit * aum)
        got, dw, db = g.layer_norm_backward(dy, x, stats, w)
        size = a.abs().mean(1, keepdim=True) + a.abs() + (1 + unit.abs()) * (a * unit).abs().mean(1, keepdim=True) \
            + (1 + unit.abs()) * a.abs().mean(1, keepdim=True)
        near(got, dx, rounded(dx, 4 * (2 * width + 64) * U * rstd * size, dtype))
        near(dw, (d * unit).sum(0), (rows * U * (d * unit).abs() + d.abs() * (off + 4 * U * unit.abs())).sum(0))
        near(db, d.sum(0), rows * U * d.abs().sum(0))
        alone = g.layer_norm_backward(dy, x, stats, w, vectors=False)
        assert torch.equal(alone[0], got) and alone[1] is None and alone[2] is None


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, width", [(0, 64), (5000, 24), (70001, 16), (3000, 300), (1500, 1030), (40, 9000)])
def test_many_rows(g, rows, width, dtype):
    gen = torch.Generator(device="cuda").manual_seed(width)
    x, dy = rows_of(gen, rows, width, dtype), rows_of(gen, rows, width, dtype)
    weight = torch.randn(width, generator=gen, device="cuda").to(dtype)
    want, unit, rstd, wd, mean = plain(x, weight, None, 1e-5)
    y, stats = g.layer_norm(x, weight, stats=True)
    off = off_of_unit(unit, rstd, mean, width)
    near(y, want, rounded(want, off * wd.abs() + 8 * U * want.abs(), dtype))
    _, dw, db = g.layer_norm_backward(dy, x, stats, weight)
    d = dy.double()
    near(dw, (d * unit).sum(0), (rows * U * (d * unit).abs() + d.abs() * (off + 4 * U * unit.abs())).sum(0))
    near(db, d.sum(0), rows * U * d.abs().sum(0))


@pytest.mark.parametrize("width", [64, 300, 1500, 6000, 20000])
def test_rows_far_from_zero(g, width):
    """x = 10 000 + noise: half a unit of the mean is 2^-11, which a unit of the noise would show."""
    gen = torch.Generator(device="cuda").manual_seed(width)
    x = torch.randn((20, width), generator=gen, device="cuda") + 10000
    dy = torch.randn((20, width), generator=gen, device="cuda")
    want, unit, rstd, _, _ = plain(x, None, None, 1e-5)
    y, stats = g.layer_norm(x, stats=True)
    near(y, want, (2 * width + 64) * U * (1 + unit.abs()))
    d = dy.double()
    dx = rstd * (d - d.mean(1, keepdim=True) - unit * (d * unit).mean(1, keepdim=True))
    got, _, _ = g.layer_norm_backward(dy, x, stats)
    size = (1 + unit.abs()) * (d.abs().mean(1, keepdim=True) + (d * unit).abs().mean(1, keepdim=True)) + d.abs()
    near(got, dx, 4 * (2 * width + 64) * U * rstd * size)


@pytest.mark.parametrize("width", [5, 64, 700, 3000, 17000])
def test_rows_of_one_value_and_no_numbers(g, width):
    x = torch.randn((6, width), device="cuda")
    x[1] = 3.25
    x[2, -1] = float("nan")
    x[3, 0] = float("inf")
    y, stats = g.layer_norm(x, eps=1e-5, stats=True)
    assert bool((y[1] == 0).all()) and bool(torch.isnan(y[2]).all()) and bool(torch.isnan(y[3]).all())
    assert bool(torch.isnan(stats[2]).all()) and bool(torch.isfinite(y[[0, 4, 5]]).all())
    y, _ = g.layer_norm(x, eps=0.0, stats=True)
    assert bool(torch.isnan(y[1]).all())        # 0 times infinity
    dx, dw, _ = g.layer_norm_backward(torch.ones_like(x), x, stats)
    assert bool(torch.isnan(dx[2]).all()) and bool(torch.isfinite(dx[[0, 1, 4, 5]]).all()) and bool(torch.isnan(dw).any())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, width", [(50, 33), (3, 5000), (20, 40000)])
def test_in_place_and_strides(g, rows, width, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x, dy = rows_of(gen, rows, width, dtype, width + 5), rows_of(gen, rows, width, dtype, width + 5)
    y, stats = g.layer_norm(x, stats=True)
    dx, dw, db = g.layer_norm_backward(dy, x, stats)
    kept = x.clone()
    assert g.layer_norm(x, out=x) is x and torch.equal(x, y)
    dx2, dw2, db2 = g.layer_norm_backward(dy, kept, stats, out=dy)
    assert dx2 is dy and torch.equal(dx2, dx) and torch.equal(dw2, dw) and torch.equal(db2, db)
    one = rows_of(gen, 1, width, dtype).expand(rows, width)         # one row for all
    assert torch.equal(g.layer_norm(one), g.layer_norm(one.contiguous()))


def test_streams_and_graphs(g):
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, dy = rows_of(gen, 3000, 200, torch.bfloat16), rows_of(gen, 3000, 200, torch.bfloat16)
    weight = torch.randn(200, generator=gen, device="cuda").bfloat16()

    def both():
        y, stats = g.layer_norm(x, weight, stats=True)
        return y, *g.layer_norm_backward(dy, x, stats, weight)

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
        x.copy_(rows_of(gen, 3000, 200, torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, both()))


def test_refusals(g):
    x = torch.zeros((3, 8), device="cuda")
    stats = torch.zeros((3, 2), device="cuda")
    for call, says in [(lambda: g.layer_norm(x, torch.zeros(7, device="cuda")), "weight"),
                       (lambda: g.layer_norm(x, None, torch.zeros(8, device="cuda").half()), "bias"),
                       (lambda: g.layer_norm(x, out=torch.zeros((3, 7), device="cuda")), "out"),
                       (lambda: g.layer_norm_backward(x, x, stats[:2]), "stats"),
                       (lambda: g.layer_norm_backward(x, x, stats.double()), "stats")]:
        with pytest.raises(ValueError, match=says):
            call()
    for call, says in [(lambda: g.layer_norm(x, eps=-1.0), "eps"), (lambda: g.layer_norm(x, eps=float("nan")), "eps"),
                       (lambda: g.layer_norm_backward(x.half(), x, stats), "type"),
                       (lambda: g.layer_norm_backward(x[:2], x, stats), "rows"),
                       (lambda: g.layer_norm_backward(x[:, :7], x, stats), "width")]:
        with pytest.raises(g.GinexError, match=says):
            call()
