"""The layers' calls with and without their compiled part: equal results, equal refusals."""
import pytest
import torch

from layer_reference import rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def g():
    import paper_2208_09151_amd as lib
    return lib


def calls(g, x, w3, bias3, r, ids):
    w, b = w3[0], bias3[0]
    stats = torch.stack([torch.zeros(x.shape[0], device="cuda"), torch.ones(x.shape[0], device="cuda")], 1)
    out = w.shape[1]
    res = x[:, :out].contiguous()
    return [lambda: g.linear(x, w), lambda: g.linear(x, w, b, "gelu", res), lambda: g.linear(x, w3, bias3, "relu", route=r),
            lambda: g.linear(g.dispatch(x, r), w3, route=r, slots=True), lambda: g.linear_backward(x, w.mT),
            lambda: g.bias_gradient(x), lambda: g.bias_gradient(g.dispatch(x, r), r),
            lambda: g.expert_layer(x[:20], w3[:, :, 0].contiguous(), w3, 2, "silu", bias3),
            lambda: g.layer_norm(x), lambda: g.layer_norm(x[:, :out], b, b, 1e-3, stats=True),
            lambda: g.layer_norm_backward(x, x, stats), lambda: g.lookup(x, ids, 0.5), lambda: g.lookup(x, ids.int()),
            lambda: g.lookup_backward(x, ids, 40, 2.0)]


def both(g, monkeypatch, call):
    from paper_2208_09151_amd import layers
    outcomes = []
    for quick in (layers._quick, None):
        with monkeypatch.context() as m:
            m.setattr(layers, "_quick", quick)
            try:
                y = call()
                outcomes.append(y if isinstance(y, tuple) else (y,))
            except Exception as e:                  # noqa: BLE001 (the same on both sides is what counts)
                outcomes.append((type(e), str(e)))
    return outcomes


@pytest.fixture(scope="module")
def quick(g):
    from paper_2208_09151_amd import layers
    g.linear(torch.zeros((1, 1), device="cuda"), torch.zeros((1, 1), device="cuda"))
    if layers._quick is None:
        pytest.skip("the compiled part is not built for this torch")
    return layers._quick


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows", [1, 33])
def test_equal(g, quick, monkeypatch, rows, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = rows_of(gen, rows, 24, dtype, 31)
    w3 = torch.randn((5, 24, 16), generator=gen, device="cuda").to(dtype)
    bias3 = torch.randn((5, 16), generator=gen, device="cuda").to(dtype)
    r = g.route(torch.randint(-1, 5, (rows, 2), generator=gen, device="cuda"), 5)
    ids = torch.randint(0, rows, (rows,), generator=gen, device="cuda")
    for call in calls(g, x, w3, bias3, r, ids):
        a, b = both(g, monkeypatch, call)
        assert all(isinstance(t, torch.Tensor) for t in a), a
        assert len(a) == len(b) and all(torch.equal(s, t) and s.dtype == t.dtype for s, t in zip(a, b))


def test_it_takes_the_plain_case_alone(g, quick):
    """Whatever else there is, is left to the Python names: None, and no error that is pending."""
    x, w = torch.zeros((3, 4), device="cuda"), torch.zeros((4, 6), device="cuda")
    w3, none = torch.zeros((2, 4, 6), device="cuda"), (None, None, None)
    r = g.route(torch.zeros((3, 2), dtype=torch.int64, device="cuda"), 2)
    ids = torch.zeros(3, dtype=torch.int64, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream

    def linear(x=x, w=w, bias=None, activation=0, residual=None, route=none, slots=False):
        return quick.linear(0, stream, x, w, bias, activation, residual, *route, slots)

    assert linear() is not None and linear(w=w3, route=r._tensors()) is not None
    learned = w.clone().requires_grad_()
    with torch.no_grad():
        assert linear(w=learned) is not None
    o, s, f = r._tensors()
    for got in [linear(x=x.cpu()), linear(w=w.cpu()), linear(x="x"), linear(w=None), linear(x=x.double(), w=w.double()),
                linear(w=w.half()), linear(w=learned), linear(w=w3), linear(bias=torch.zeros(5, device="cuda")),
                linear(bias=torch.zeros((1, 6), device="cuda")), linear(residual=torch.zeros((3, 5), device="cuda")),
                linear(residual=x), linear(slots=True), linear(x=x[0]), linear(x=torch.zeros((3, 8), device="cuda")[:, ::2]),
                linear(w=torch.zeros((8, 12), device="cuda")[::2, ::2]), linear(activation=2 ** 70), linear(activation=None),
                linear(w=w3, route=(o, s, f[:-1])), linear(w=w3, route=(o.int(), s, f)), linear(w=w3, route=(o[:1], s, f)),
                linear(w=w3, route=(o, s.flatten(), f)), linear(w=w3, route=(o, s, None)), quick.linear(0, stream, x),
                linear(x=x.to_sparse()), quick.linear(1, stream, x, w, None, 0, None, None, None, None, False),
                quick.bias_gradient(0, stream, x.cpu(), *none), quick.bias_gradient(0, stream, x.long(), *none),
                quick.expert_layer(0, stream, x, x[:2], w3, None, 2 ** 32 + 1, 0),
                quick.expert_layer(0, stream, x, x[:2], w3, None, 1.5, 0), quick.expert_layer(0, stream, x, x[:2], w3, None, -1, 0),
                quick.expert_layer(0, stream, x, x[:2].half(), w3, None, 1, 0),
                quick.layer_norm(0, stream, x, None, None, 1, False), quick.layer_norm(0, stream, x, w[0], None, 1e-5, False),
                quick.layer_norm_backward(0, stream, x, x, x, None),
                quick.layer_norm_backward(0, stream, x, x, torch.zeros((3, 2), device="cuda").double(), None),
                quick.lookup(0, stream, x, ids.float(), 1.0), quick.lookup(0, stream, x, ids, 1),
                quick.lookup(0, stream, x, ids[::2], 1.0), quick.lookup_backward(0, stream, x, ids[:2], 5, 1.0),
                quick.lookup_backward(0, stream, x, ids, -1, 1.0), quick.lookup_backward(0, stream, x, ids, 2 ** 70, 1.0),
                quick.lookup_backward(0, stream, x, ids, 5.0, 1.0)]:
        assert got is None


def test_equal_refusals(g, quick, monkeypatch):
    x, w3 = torch.zeros((9, 4), device="cuda"), torch.zeros((3, 4, 6), device="cuda")
    w = w3[0]
    r = g.route(torch.zeros((9, 2), dtype=torch.int64, device="cuda"), 3)
    ids = torch.zeros(9, dtype=torch.int64, device="cuda")
    stats = torch.zeros((9, 2), device="cuda")
    for call in [lambda: g.linear(x, w.half()), lambda: g.linear(x, w3), lambda: g.linear(x, w3[:2], route=r),
                 lambda: g.linear(x, torch.zeros((5, 6), device="cuda")), lambda: g.linear(x[:8], w3, route=r),
                 lambda: g.linear(x, w3, route=r, slots=True), lambda: g.linear(x, w, torch.zeros(6)),
                 lambda: g.bias_gradient(x, r), lambda: g.expert_layer(x, x[:3], w3, 4), lambda: g.expert_layer(x, x[:3], w3, 2 ** 32 + 1),
                 lambda: g.expert_layer(x, x[:2], w3, 1), lambda: g.expert_layer(x.expand(9, 4), x[:3, :3], w3, 1),
                 lambda: g.layer_norm(x, eps=-1.0), lambda: g.layer_norm(x, eps=float("nan")),
                 lambda: g.layer_norm_backward(x[:8], x, stats), lambda: g.layer_norm_backward(x.half(), x, stats),
                 lambda: g.layer_norm_backward(x, x, stats[:8]), lambda: g.lookup(x, ids.cpu()),
                 lambda: g.lookup_backward(x, ids, -1), lambda: g.lookup_backward(x, ids, 2 ** 40), lambda: g.lookup(x, ids, float("nan"))]:
        a, b = both(g, monkeypatch, call)
        if isinstance(b[0], type):
            assert a == b
        else:
            assert torch.equal(torch.nan_to_num(a[0]), torch.nan_to_num(b[0]))
