"""layer_norm and its gradients on rows far from zero, at every width's kernel: the mean that f32 rounds is taken away twice.

With u = 2^-24 and D additions one after the other at most (D = width / 256 + 32: a thread's numbers of a row beyond 16 KB, or at most
32, then lanes and waves), mean m, a the mean of |x - m| and v the variance + eps:

  the first mean is off by s <= (D + 2) u |m|; what is taken from it, d = x - mean, is exact (the two are within a factor of 2), and
  the mean of d is off by (D + 2) u (a + s) at most.  The variance, mean(d^2) - mean(d)^2, is off by (D + 4) u (v + s^2) +
  2 s (D + 2) u (a + s), rstd by half of that over v and 4 u more, of itself: R.  unit is off by
  (D + 4) u (a + s) / sqrt v + |unit| (R + 6 u).

The gradients take the mean as it was kept, rounded to f32: for them s is u |m| + (D + 2) u (a + s) instead.  A mean that was not
taken away twice would be off by up to u |m|, 2^-11 of x = 10 000, which is 2^-8 of a unit of 0.1.
"""
import pytest
import torch

from layer_reference import near, rounded, rows_of

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EPS = 1e-5
# (type, where the rows are, how far their numbers lie from there); in f16 numbers of 2000 are 1 apart
FAR = [(torch.float32, 10000.0, 1.0), (torch.float32, 10000.0, 0.1), (torch.float32, -3000.0, 0.1), (torch.float16, 1500.0, 3.0)]
WIDTHS = [64, 300, 1030, 4096, 4097, 6000, 8192, 8200, 20000]


@pytest.fixture(scope="module")
def g():
    import paper_2208_09151_amd as lib
    return lib


def exact(x, dy, weight):
    """Results in 64 bits and what they may be off by before they are rounded."""
    width = x.shape[1]
    D = width / 256 + 32
    x, d, w = x.double(), dy.double(), 1.0 if weight is None else weight.double()
    m = x.mean(1, keepdim=True)
    v = ((x - m) ** 2).mean(1, keepdim=True) + EPS
    unit, near_by, a = (x - m) / v.sqrt(), (x - m).abs().mean(1, keepdim=True), d * w

    def off_of_unit(s, r):
        return (D + 4) * U * (near_by + s) / v.sqrt() + unit.abs() * (r + 6 * U)

    s = (D + 2) * U * m.abs()
    r = ((D + 4) * U * (v + s * s) / 2 + s * (D + 2) * U * (near_by + s)) / v + 4 * U
    off = off_of_unit(s, r)
    y = unit * w
    t = U * m.abs() + (D + 2) * U * (near_by + s)
    off_b = off_of_unit(t, r)
    mean_a, size_a = a.mean(1, keepdim=True), a.abs().mean(1, keepdim=True)
    mean_au, size_au = (a * unit).mean(1, keepdim=True), (a * unit).abs().mean(1, keepdim=True)
    off_au = (D + 6) * U * (size_au + 2 * t / v.sqrt() * size_a) + (D + 4) * U * (near_by + t) / v.sqrt() * size_a + (r + 4 * U) * size_au
    dx = (a - mean_a - unit * mean_au) / v.sqrt()
    off_dx = ((D + 4) * U * size_a + off_b * mean_au.abs() + (unit.abs() + off_b) * off_au
              + 4 * U * (a.abs() + size_a + unit.abs() * size_au)) / v.sqrt() + (r + 4 * U) * dx.abs()
    dw, db = (d * unit).sum(0), d.sum(0)
    rows = x.shape[0]
    off_dw = ((rows + 4) * U * (d * unit).abs() + d.abs() * off_b).sum(0)
    return (y, off * abs(w) + 4 * U * y.abs()), (dx, off_dx), (dw, off_dw), (db, rows * U * d.abs().sum(0))


@pytest.mark.parametrize("dtype, at, by", FAR)
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("rows", [5, 150])
def test_rows_far_from_zero(g, rows, width, dtype, at, by):
    gen = torch.Generator(device="cuda").manual_seed(width + rows)
    x = rows_of(gen, rows, width, torch.float32, width + 3, by)
    x = (x + at).to(dtype)
    dy = (rows_of(gen, rows, width, torch.float32) + 0.5).to(dtype)
    weight = (torch.randn(width, generator=gen, device="cuda") * 0.2 + 1).to(dtype)
    for w in (None, weight):
        (y, off), (dx, off_dx), (dw, off_dw), (db, off_db) = exact(x, dy, w)
        got, stats = g.layer_norm(x, w, stats=True, eps=EPS)
        near(got, y, rounded(y, off, dtype))
        got, got_w, got_b = g.layer_norm_backward(dy, x, stats, w)
        near(got, dx, rounded(dx, off_dx, dtype))
        near(got_w, dw, off_dw)
        near(got_b, db, off_db)
        alone = g.layer_norm_backward(dy, x, stats, w, vectors=False)[0]
        assert torch.equal(alone, got)
        again = dy.clone()
        in_place = g.layer_norm_backward(again, x, stats, w, out=again)
        assert all(torch.equal(s, t) for s, t in zip(in_place, (got, got_w, got_b)))
