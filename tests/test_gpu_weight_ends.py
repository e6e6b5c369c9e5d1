"""f32 gradients at the lower end of their range: what the three bf16 numbers that stand for one leave out.

Each takes the upper 16 bits of what the ones before it left, so a remainder that is a normal number loses nothing, and one
below 2^-126 loses what lies below bf16's least bit, 2^-133.  From 2^-110 on a gradient's 24 bits end above that: exact.
Beneath, a product is off by less than 2^-133 |x|, and a sum by that and by n 2^-24 of its terms' sizes.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def g():
    import paper_2208_09151_amd as lib
    return lib


@pytest.mark.parametrize("exponent", [-80, -100, -109, -110, -111, -118, -125, -126, -130, -140, -148])
@pytest.mark.parametrize("width, out, rows", [(32, 40, 1), (100, 200, 1), (64, 64, 50), (256, 256, 270_000)])
def test_small_gradients_of_large_rows(g, exponent, width, out, rows):
    gen = torch.Generator(device="cuda").manual_seed(1 - exponent)
    x = torch.exp2(torch.randint(96, 101, (rows, width), generator=gen, device="cuda").float())
    dy = torch.zeros((rows, out), device="cuda")
    some = min(rows, 40)
    at = torch.randperm(rows, generator=gen, device="cuda")[:some]
    bits = 1 + torch.randint(0, 1 << 23, (some, out), generator=gen, device="cuda").double() * 2.0 ** -23
    dy[at] = (bits * 2.0 ** exponent).float()
    got = g.weight_gradient(g.compress(x), dy).double()
    xt, d = x[at].double().t().contiguous(), dy[at].double()
    want, size = xt @ d, xt.sum(1, keepdim=True)
    allowed = (3 * some if some > 1 else 2) * 2.0 ** -24 * want
    if exponent < -110:
        allowed = allowed + 2.0 ** -133 * size
    elif some == 1:
        allowed = torch.zeros_like(want)        # one product, a power of two times 24 bits
    assert ((got - want).abs() <= allowed).all()
