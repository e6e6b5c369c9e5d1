"""expert_layer, a whole layer of experts for few rows, against plain torch in 64 bits."""
import pytest
import torch

from layer_reference import TYPES, linear as plain, near, rounded, rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def g():
    import paper_2208_09151_amd as lib
    return lib


def reference(x, router, w, top, activation, bias, dtype):
    scores = x.double() @ router.double().t()
    best, chosen = torch.sort(scores, dim=1, descending=True, stable=True)
    best, chosen = best[:, :top], chosen[:, :top]
    share = torch.softmax(best, 1)
    want = torch.zeros((x.shape[0], w.shape[2]), dtype=torch.float64, device="cuda")
    off = torch.zeros_like(want)
    for r in range(x.shape[0]):
        for j in range(top):
            e = int(chosen[r, j])
            y, o, _ = plain(x[r:r + 1], w[e], None if bias is None else bias[e], activation, None, dtype)
            want[r] += share[r, j] * y[0]
            # shares and sums of `top` terms in f32
            off[r] += share[r, j] * (o[0] + (top + 2) * 2.0 ** -23 * y[0].abs())
    return want, off


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("rows, width, out, experts, top, activation", [
    (1, 1, 1, 1, 1, None), (1, 64, 64, 8, 2, "silu"), (1, 1000, 70, 20, 1, "gelu"), (1, 100, 200, 3, 2, None), (1, 600, 70, 300, 2, "relu"), (1, 333, 70, 64, 16, "gelu"), (2, 5, 3, 3, 3, "relu"),
    (7, 100, 130, 1024, 4, "gelu"), (17, 1000, 33, 5, 2, "silu"), (48, 200, 65, 2, 2, "gelu"), (64, 96, 40, 70, 16, None)])
def test_sizes(g, rows, width, out, experts, top, activation, turned, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows + width + experts)
    x = rows_of(gen, rows, width, dtype, width + 1)
    router = rows_of(gen, experts, width, dtype, width + 2, width ** -0.5)
    shape = (experts, out, width) if turned else (experts, width, out)
    w = (torch.randn(shape, generator=gen, device="cuda") / width ** 0.5).to(dtype)
    w = w.mT if turned else w
    bias = torch.randn((experts, out), generator=gen, device="cuda").to(dtype)
    for b in (None, bias):
        want, off = reference(x, router, w, top, activation, b, dtype)
        near(g.expert_layer(x, router, w, top, activation, b), want, rounded(want, off, dtype))


def test_equal_scores_take_the_first_experts(g):
    x = torch.ones((3, 8), device="cuda")
    router = torch.zeros((70, 8), device="cuda")
    router[5] = router[69] = router[11] = 1
    x[1] = 0                                    # all scores 0
    x[2] = -0.0
    w = torch.arange(70, device="cuda", dtype=torch.float32)[:, None, None].expand(70, 8, 4).contiguous()
    b = torch.arange(70, device="cuda", dtype=torch.float32)[:, None].expand(70, 4).contiguous()
    y = g.expert_layer(x, router, w, 2, None, b)
    assert torch.equal(y, torch.tensor([[9 * 8.0], [0.5], [0.5]], device="cuda").expand(3, 4))


@pytest.mark.parametrize("dtype", TYPES)
def test_scores_that_are_no_numbers(g, dtype):
    """NaN counts as the largest and leaves NaN; an infinite score takes all; a row is nobody else's business."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = rows_of(gen, 5, 40, dtype)
    router = rows_of(gen, 9, 40, dtype)
    w = rows_of(gen, 9 * 40, 30, dtype).view(9, 40, 30)
    clean = g.expert_layer(x, router, w, 3, "relu")
    router[4, 0] = float("nan")
    y = g.expert_layer(x, router, w, 3, "relu")
    assert bool(torch.isnan(y).all())
    router[4, 0] = 0
    clean = g.expert_layer(x, router, w, 3, "relu")
    x[2, 7] = float("nan")
    y = g.expert_layer(x, router, w, 3, "relu")
    others = [0, 1, 3, 4]
    assert bool(torch.isnan(y[2]).all()) and torch.equal(y[others], clean[others])
    # all scores -inf: there is no softmax of them
    x[2] = 1
    router[:] = -float("inf")
    assert bool(torch.isnan(g.expert_layer(x.abs() + 1, router, w, 3)).all())


def test_calls_graphs_and_streams(g):
    """Equal bits in any call, with one workspace call after call, captured and replayed between eager calls."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = rows_of(gen, 40, 128, torch.bfloat16)
    router = rows_of(gen, 16, 128, torch.bfloat16)
    w = rows_of(gen, 16 * 128, 192, torch.bfloat16).view(16, 128, 192)
    ws = torch.full((4 << 20,), 255, dtype=torch.uint8, device="cuda")

    def call():
        return g.expert_layer(x, router, w, 4, "gelu", workspace=ws)

    want = call()
    for _ in range(20):
        assert torch.equal(call(), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = g.expert_layer(x, router, w, 4, "gelu")
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for _ in range(3):
        x.copy_(rows_of(gen, 40, 128, torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, call())


def test_no_rows_and_refusals(g):
    x, router = torch.zeros((3, 4), device="cuda"), torch.zeros((5, 4), device="cuda")
    w = torch.zeros((5, 4, 6), device="cuda")
    assert g.expert_layer(x[:0], router, w, 2).shape == (0, 6)
    for call, says in [(lambda: g.expert_layer(x, router.half(), w, 2), "router"),
                       (lambda: g.expert_layer(x, router, w.half(), 2), "dtype"),
                       (lambda: g.expert_layer(x, router, w[0], 2), "weight"),
                       (lambda: g.expert_layer(x, router, w, 2, bias=torch.zeros(6, device="cuda")), "bias"),
                       (lambda: g.expert_layer(x, router, w, 2, "tanh"), "activation"),
                       (lambda: g.expert_layer(x.requires_grad_(), router, w, 2), "gradient")]:
        with pytest.raises(ValueError, match=says):
            call()
    x = x.detach()
    for call, says in [(lambda: g.expert_layer(x, router, w, 6), "top"), (lambda: g.expert_layer(x, router, w, 0), "top"),
                       (lambda: g.expert_layer(x, router[:4], w, 2), "experts"),
                       (lambda: g.expert_layer(torch.zeros((65, 4), device="cuda"), router, w, 2), "rows"),
                       (lambda: g.expert_layer(x[:, :3], router[:, :3], w, 2), "wide")]:
        with pytest.raises(g.GinexError, match=says):
            call()
