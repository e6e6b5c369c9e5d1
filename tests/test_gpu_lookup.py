"""lookup and its gradient against plain torch in 64 bits."""
import pytest
import torch

from layer_reference import LEAST, ROUND, TYPES, near, rounded, rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def g():
    import paper_2208_09151_amd as lib
    return lib


def check(g, table, dy, ids, scale):
    rows, width = table.shape
    dtype = table.dtype
    there = ((ids >= 0) & (ids < rows))[:, None]
    at = ids.clamp(0, max(rows - 1, 0)).long()
    scale32 = float(torch.tensor(scale, dtype=torch.float32))
    found = table[at].double() * scale32 if rows else torch.zeros((ids.numel(), width), dtype=torch.float64, device="cuda")
    want = torch.where(there, found, torch.zeros_like(found))
    near(g.lookup(table, ids, scale), want, rounded(want, 2.0 ** -24 * want.abs(), dtype) * (want != 0))
    want = torch.zeros((rows + 1, width), dtype=torch.float64, device="cuda")
    size, count = torch.zeros_like(want), torch.zeros(rows + 1, dtype=torch.float64, device="cuda")
    to = torch.where(there[:, 0], ids.long(), torch.full_like(at, rows))
    want.index_add_(0, to, dy.double() * scale32)
    size.index_add_(0, to, dy.double().abs() * abs(scale32))
    count.index_add_(0, to, torch.ones(ids.numel(), dtype=torch.float64, device="cuda"))
    got = g.lookup_backward(dy, ids, rows, scale)
    want, off = want[:rows], ((count[:, None] + 1) * 2.0 ** -24 * size)[:rows]
    near(got, want, rounded(want, off, dtype) * (count[:rows, None] > 0))
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("rows, ids, width", [
    (1, 1, 1), (1, 100, 5), (7, 0, 33), (0, 9, 8), (5, 31, 64), (5, 32, 7), (40, 33, 100), (300, 5000, 128), (3000, 200, 16),
    (70000, 20000, 24), (17, 9000, 300), (100, 3000, 1000), (2, 40000, 9),
    (50, 64, 8), (50, 65, 8), (1000, 4096, 8), (9, 4097, 16), (3000, 8192, 8), (3000, 8193, 8),
    (3_000_000, 5, 3), (2_000_003, 700, 2)])
def test_sizes(g, rows, ids, width, wide, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows + ids + width)
    at = torch.randint(-1, rows + 1, (ids,), generator=gen, device="cuda")
    at = at if wide else at.to(torch.int32)
    check(g, rows_of(gen, rows, width, dtype, width + 1), rows_of(gen, ids, width, dtype, width + 2), at, 1.7)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [12_800, 4_500])
@pytest.mark.parametrize("kind", ["equal", "sorted", "reversed", "runs", "long runs", "no row", "far"])
def test_orders(g, kind, n, dtype):
    """Ids whose places in sorted order begin and end with a run, in it, or many runs apart."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    rows, width = 400, 40
    place = torch.arange(n, device="cuda")
    ids = {"equal": torch.full((n,), 123, device="cuda"), "sorted": place // 32, "reversed": (n - 1 - place) // 32,
           "runs": place // 31, "long runs": place // 3000 * 7, "no row": torch.full((n,), -5, device="cuda"),
           "far": place % 3 * (2 ** 62) - 2 ** 61}[kind]
    check(g, rows_of(gen, rows, width, dtype), rows_of(gen, n, width, dtype), ids, -0.5)


def test_long_runs_of_long_rows(g):
    gen = torch.Generator(device="cuda").manual_seed(6)
    ids = torch.zeros(20_000, dtype=torch.int32, device="cuda")
    ids[:3000] = 2
    check(g, rows_of(gen, 3, 600, torch.float32), rows_of(gen, 20_000, 600, torch.float32), ids, 1.0)


@pytest.mark.parametrize("dtype", TYPES)
def test_outputs_are_written_where_they_are(g, dtype):
    gen = torch.Generator(device="cuda").manual_seed(7)
    table, dy = rows_of(gen, 50, 33, dtype), rows_of(gen, 900, 33, dtype)
    ids = torch.randint(0, 40, (900,), generator=gen, device="cuda")
    for make, n in [(lambda out: g.lookup(table, ids, 2.0, out=out), 900), (lambda out: g.lookup_backward(dy, ids, 50, out=out), 50)]:
        room = torch.full((n + 2, 40), 7.0, device="cuda", dtype=dtype)
        to = room[1:1 + n, 3:36]
        assert make(to) is to
        assert torch.equal(to, make(None))
        room[1:1 + n, 3:36] = 7
        assert bool((room == 7).all())


def test_numbers_that_are_none(g):
    """They reach the rows that are asked for, and no padded one."""
    table = torch.ones((4, 20), device="cuda")
    table[1] = float("nan")
    table[0] = float("inf")
    ids = torch.tensor([-1, 1, 2, 0, 4], device="cuda")
    y = g.lookup(table, ids, 3.0)
    assert bool((y[0] == 0).all()) and bool(torch.isnan(y[1]).all()) and bool((y[2] == 3).all())
    assert bool((y[3] == float("inf")).all()) and bool((y[4] == 0).all())
    dy = torch.ones((5, 20), device="cuda")
    dy[0] = dy[4] = float("nan")
    dy[2] = float("inf")
    d = g.lookup_backward(dy, ids, 4)
    assert d[:, 0].tolist() == [1.0, 1.0, float("inf"), 0.0]


def test_streams_and_graphs(g):
    gen = torch.Generator(device="cuda").manual_seed(8)
    ids = torch.randint(0, 300, (20_000,), generator=gen, device="cuda")
    table, dy = rows_of(gen, 300, 70, torch.float16), rows_of(gen, 20_000, 70, torch.float16)
    ws = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")

    def both():
        return g.lookup(table, ids, 1.5), g.lookup_backward(dy, ids, 300, 1.5, workspace=ws)

    want = both()
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(both(), want))
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
        ids.copy_(torch.randint(0, 250, (20_000,), generator=gen, device="cuda"))
        dy.copy_(rows_of(gen, 20_000, 70, torch.float16))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, both()))


def test_refusals(g):
    table, ids = torch.zeros((4, 8), device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    for call in [lambda: g.lookup(table, ids.float()), lambda: g.lookup(table, ids[None]), lambda: g.lookup(table, ids.cpu()),
                 lambda: g.lookup(table, torch.zeros(6, dtype=torch.int64, device="cuda")[::2]),
                 lambda: g.lookup_backward(table, ids, 5)]:
        with pytest.raises(ValueError, match="ids"):
            call()
    with pytest.raises(ValueError, match="out"):
        g.lookup(table, ids, out=torch.zeros((2, 8), device="cuda"))
    with pytest.raises(g.GinexError, match="rows"):
        g.lookup_backward(table[:3], ids, -1)
