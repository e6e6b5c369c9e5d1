"""Weight gradients in every workgroup shape of the kernel, on experts of uneven sizes that ranges share.

All results are exact, whatever the order of the sums.  Rows and gradients of small whole numbers: the sum of the terms'
magnitudes stays below 2^24.  Rows of powers of two and gradients of full significands, one slot of an expert in a column:
one product each, whose parts (8 bits at a time) add up without rounding.
"""
import pytest
import torch

import weight_shapes

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def g():
    import paper_2208_09151_amd as lib
    return lib


def strided(t, pad, shift):
    rows, width = t.shape
    base = torch.full((rows * (width + pad) + shift,), float("nan"), dtype=t.dtype, device="cuda")
    view = base[shift:].view(rows, width + pad)[:, :width]
    view.copy_(t)
    return view


class Slots:
    """A route by which expert e has sizes[e] slots, rows in any order; the last pairs have no expert."""

    def __init__(self, g, sizes, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        chosen = torch.repeat_interleave(torch.arange(len(sizes), device="cuda"), torch.tensor(sizes, device="cuda"))
        chosen = torch.cat([chosen, torch.full((weight_shapes.EMPTY,), -1, device="cuda")])
        self.rows = self.slots = chosen.numel()
        self.route = g.route(chosen[torch.randperm(self.slots, generator=gen, device="cuda")].view(-1, 1), len(sizes))
        self.ends = self.route.offsets.tolist()
        assert self.ends == [0] + torch.tensor(sizes).cumsum(0).tolist()
        self.source = self.route.source.long()
        self.gen = gen

    def whole(self, shape, most):
        return torch.randint(-most, most + 1, shape, generator=self.gen, device="cuda").float()

    def spoil(self, dy):
        """Slots without a row are not read."""
        dy[self.ends[-1]:] = float("nan")
        return dy


@pytest.mark.parametrize("shape, sizes, width, out, dtype", weight_shapes.PARAMS, ids=weight_shapes.IDS)
@pytest.mark.parametrize("pad, shift", [(0, 0), (3, 1)])
def test_sums_of_whole_numbers(g, shape, sizes, width, out, dtype, pad, shift):
    s = Slots(g, sizes, width + out)
    x = s.whole((s.rows, width), 3)
    dy = s.spoil(s.whole((s.slots, out), 7)).to(TYPES[dtype])
    got = g.weight_gradient(g.compress(x), strided(dy, pad, shift), s.route)
    for e, (a, b) in enumerate(zip(s.ends[:-1], s.ends[1:])):
        want = x[s.source[a:b]].double().t().contiguous() @ dy[a:b].double()
        assert torch.equal(got[e].double(), want), (e, a, b)


@pytest.mark.parametrize("shape, sizes, width, out, dtype", weight_shapes.PARAMS, ids=weight_shapes.IDS)
def test_single_products_of_full_significands(g, shape, sizes, width, out, dtype):
    s = Slots(g, sizes, width)
    x = torch.exp2(s.whole((s.rows, width), 2)) * (1 - 2 * (s.whole((s.rows, width), 3) > 0).float())
    dy = torch.zeros((s.slots, out), dtype=TYPES[dtype], device="cuda")
    want = torch.zeros((len(sizes), width, out), device="cuda")
    column = torch.arange(out, device="cuda")
    for e, (a, b) in enumerate(zip(s.ends[:-1], s.ends[1:])):
        if a == b:
            continue
        at = torch.randint(a, b, (out,), generator=s.gen, device="cuda")
        at[:2], at[-2:] = a, b - 1              # the first and the last slot among them
        values = torch.randn(out, generator=s.gen, device="cuda").to(dy.dtype)
        dy[at, column] = values
        want[e] = x[s.source[at]].t() * values.float()
    got = g.weight_gradient(g.compress(x), s.spoil(dy), s.route)
    assert torch.equal(got, want)


@pytest.mark.parametrize("shape, sizes, width, out, dtype", weight_shapes.PARAMS, ids=weight_shapes.IDS)
def test_values_that_are_no_numbers_stay_with_their_expert(g, shape, sizes, width, out, dtype):
    """A block without numbers spoils its 32 channels of its expert, an infinite gradient its column where the row is not 0."""
    s = Slots(g, sizes, width + 1)
    x = s.whole((s.rows, width), 1) * 2 + 1     # no zeros
    dy = s.whole((s.slots, out), 7)
    bad, hot = 1, len(sizes) - 2                # the experts that are hit
    if sizes[hot] == 0:
        hot -= 1
    slot = s.ends[bad] + sizes[bad] // 2
    at = s.ends[hot + 1] - 1
    assert sizes[bad] and sizes[hot] and bad != hot
    clean = g.weight_gradient(g.compress(x), s.spoil(dy).to(TYPES[dtype]), s.route)
    x[s.source[slot], width - 1] = float("nan")
    dy[at, out - 1] = float("inf")
    got = g.weight_gradient(g.compress(x), s.spoil(dy).to(TYPES[dtype]), s.route)
    block = (width - 1) // 32 * 32
    assert got[bad, block:].isnan().all()
    assert torch.equal(got[hot, :, out - 1], torch.copysign(torch.full((width,), float("inf"), device="cuda"),
                                                            x[s.source[at]]))
    got[bad, block:] = clean[bad, block:]
    got[hot, :, out - 1] = clean[hot, :, out - 1]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("shape, sizes, width, out, dtype", weight_shapes.PARAMS, ids=weight_shapes.IDS)
def test_equal_bits_again(g, shape, sizes, width, out, dtype):
    s = Slots(g, sizes, width + 2)
    kept = g.compress(torch.randn((s.rows, width), generator=s.gen, device="cuda"))
    dy = torch.randn((s.slots, out), generator=s.gen, device="cuda").to(TYPES[dtype])
    first = g.weight_gradient(kept, dy, s.route)
    for _ in range(3):
        assert torch.equal(g.weight_gradient(kept, dy, s.route), first)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows, width, out", [(270_000, 256, 256), (270_001, 130, 140), (270_001, 100, 130)])
def test_one_layer_of_many_rows(g, rows, width, out, dtype):
    """Without a route, in the large shapes."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randint(-3, 4, (rows, width), generator=gen, device="cuda").float()
    dy = torch.randint(-7, 8, (rows, out), generator=gen, device="cuda").to(TYPES[dtype])
    got = g.weight_gradient(g.compress(x), dy)
    assert torch.equal(got.double(), x.double().t().contiguous() @ dy.double())
