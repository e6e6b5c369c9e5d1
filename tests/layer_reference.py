"""The layers on gathered rows in plain torch and 64 bits, and how far f32 arithmetic may be from that.

A rounding is off by half a step at most: 2^-24 (f32), 2^-8 (bf16), 2^-11 (f16) of the value, or half of the least number.  A
sum of n products in f32 is off by n 2^-23 of the sum of their magnitudes at most, whichever way the matrix cores round an
addition.  The activations are good to what ginex_train.h says.
"""
import torch

ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def activated(z, activation):
    if activation == "relu":
        return z.clamp(min=0)
    if activation == "silu":
        return z * torch.sigmoid(z)
    if activation == "gelu":
        return z * torch.special.ndtr(z)
    return z


def activation_error(z, activation, dtype):
    """Of the value: 2^-20 (silu) and 2^-18 + z^2 2^-22 (gelu) in f32, the larger of those and 16 bits' everywhere."""
    if activation in (None, "relu"):
        return torch.zeros_like(z)
    return activated(z, activation).abs() * (2.0 ** -18 + z * z * 2.0 ** -22) + 2.0 ** -119


def linear(x, w, bias, activation, residual, dtype):
    """(result, allowed error) of rows x [n, width] through one layer's w [width, out]."""
    x, w = x.double(), w.double()
    z = x @ w
    size = x.abs() @ w.abs()
    if bias is not None:
        z, size = z + bias.double(), size + bias.double().abs()
    y = activated(z, activation)
    # the slope of silu and gelu is below 1.13
    off = 1.13 * (x.shape[1] + 2) * 2.0 ** -23 * size + activation_error(z, activation, dtype)
    if residual is not None:
        y = y + residual.double()
        off = off + 2.0 ** -24 * y.abs()
    return y, off, z


def rounded(y, off, dtype):
    """The allowed error after one more rounding to `dtype`."""
    return off * (1 + ROUND[dtype]) + ROUND[dtype] * y.abs() + LEAST[dtype]


def near(got, want, allowed):
    got = got.detach().double()
    assert got.shape == want.shape
    bad = ~((got - want).abs() <= allowed)
    if bool(bad.any()):
        at = tuple(int(v) for v in torch.nonzero(bad)[0])
        raise AssertionError(f"{int(bad.sum())} of {bad.numel()} are off, first {at}: got {float(got[at])}, want "
                             f"{float(want[at])} within {float(allowed[at])}")


def rows_of(gen, n, width, dtype, stride=None, by=1.0):
    """Random rows, `stride` elements apart."""
    stride = stride or width
    flat = (torch.randn(max(n, 1) * stride, generator=gen, device="cuda") * by).to(dtype)
    return flat.as_strided((n, width), (stride, 1))


def random_route(g, gen, rows, top, experts, capacity=None, absent=0.2):
    chosen = torch.randint(0, experts, (rows, top), generator=gen, device="cuda")
    gone = torch.rand((rows, top), generator=gen, device="cuda") < absent
    return g.route(torch.where(gone, -torch.ones_like(chosen), chosen), experts, capacity=capacity)
