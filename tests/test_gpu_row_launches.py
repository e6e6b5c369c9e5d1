"""Rows of more chunks than a launch numbers: dispatch and combine take two launches, and rows on both sides of the seam
are right."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_rows_beyond_2_to_the_31_chunks():
    """2048 f16 are 256 chunks of 16 bytes: 8 388 607 rows are all that one launch has.  Copies, and sums of one: equal."""
    import paper_2208_09151_amd as g
    seam, width = ((1 << 31) - 256) // 256, 2048
    n = seam + 100
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty((n, width), dtype=torch.float16, device="cuda").normal_(generator=gen)
    chosen = torch.randint(0, 4, (n, 1), generator=gen, device="cuda", dtype=torch.int32)
    gone = torch.tensor([0, 5, seam - 1, seam + 1, n - 2], device="cuda")
    chosen[gone] = -1
    r = g.route(chosen, 4)
    rows = torch.full((n, width), float("nan"), dtype=torch.float16, device="cuda")
    g.dispatch(x, r, out=rows)
    assert (rows[-len(gone):] == 0).all()
    at = torch.cat([torch.randint(0, n, (2000,), generator=gen, device="cuda"), torch.arange(seam - 50, n, device="cuda")])
    slot = r.slot[at, 0].long()
    has = slot >= 0
    assert int((~has[2000:]).sum()) == 3
    assert torch.equal(rows[slot[has]], x[at[has]])
    y = g.combine(rows, r, torch.full((n, 1), 2.0, device="cuda"))
    x[gone] = 0
    for a in range(0, n, 1 << 20):
        assert torch.equal(y[a:a + (1 << 20)], 2 * x[a:a + (1 << 20)])
