"""Routes that were not made by route(): slots, offsets and sources that are not there count as none, and nothing
outside the arrays is read or written."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def g():
    import paper_2208_09151_amd as lib
    return lib


# 2^50 rows of 2^13 chunks are 2^63 chunks
@pytest.mark.parametrize("end", [1 << 50, (1 << 63) - 1, 1 << 48, 5, 4, 2, -1, -(1 << 63)])
@pytest.mark.parametrize("width", [1, 4, 100, 32_768])
def test_rows_from_an_end_that_is_not_there(g, width, end):
    slot = torch.tensor([[0, 1 << 30], [-5, 1]], dtype=torch.int32, device="cuda")
    source = torch.tensor([0, 1, 1 << 30, -9], dtype=torch.int32, device="cuda")
    r = g.Route(torch.tensor([0, 2, end], device="cuda"), slot, source)
    x = torch.randn((2, width), device="cuda")
    around = torch.full((68, width), 7.0, device="cuda")
    out = g.dispatch(x, r, out=around[32:36])
    # (with an end in front of them the two rows may be cleared as well as written)
    cleared = max(min(end, 4), 0)
    if end >= 2:
        assert torch.equal(out[:2], x)
    assert (out[max(cleared, 2):] == 0).all() and (out[2:max(cleared, 2)] == 7).all()
    assert (around[:32] == 7).all() and (around[36:] == 7).all()
    w = torch.tensor([[2.0, 3.0], [4.0, 5.0]], device="cuda")
    z = torch.randn((4, width), device="cuda")
    dz, dw = g.combine_backward(x, z, r, w)
    if end >= 2:
        assert torch.equal(dz[:2], x * torch.tensor([[2.0], [5.0]], device="cuda"))
    assert (dz[max(cleared, 2):] == 0).all()
    assert dw[0, 1] == 0 and dw[1, 0] == 0


@pytest.mark.parametrize("offsets", [
    [0, 1000, 2000, 16], [0, 2048, 0, 2048, 5], [0, 1 << 50, 1 << 50, 1 << 50], [-5, 100, 50, 2048],
    [0, 700, (1 << 63) - 1, -1], [0, 100, 1000, 1800]])
@pytest.mark.parametrize("width, out", [(128, 256), (64, 64), (33, 5)])
def test_weight_gradient_by_offsets_that_are_not_there(g, offsets, width, out):
    """Sums of offsets that ascend are right, sources that are not there count as zeros; the rest is only bounded."""
    slots, experts = 2048, len(offsets) - 1
    kept = g.compress(torch.randn((slots, width), device="cuda"))
    dy = torch.randn((slots, out), device="cuda")
    source = torch.arange(slots, dtype=torch.int32, device="cuda")
    source[::7] = (1 << 31) - 1                 # rows that are not there
    source[1::7] = -3
    r = g.Route(torch.tensor(offsets, device="cuda"), source.view(-1, 1), source)
    need = g._lib.load().ginex_weight_gradient_workspace_bytes(slots, experts, width, out)
    around = torch.zeros(need + 2048, dtype=torch.uint8, device="cuda")
    dw = g.weight_gradient(kept, dy, r, workspace=around[1024:1024 + need])
    assert dw.shape == (experts, width, out) and (around[:1024] == 0).all() and (around[1024 + need:] == 0).all()
    if offsets == [0, 100, 1000, 1800]:
        x = g.restore(kept).double()
        x[(source < 0) | (source >= slots)] = 0
        for e in range(3):
            a, b = offsets[e], offsets[e + 1]
            size = x[a:b].abs().t().contiguous() @ dy[a:b].double().abs()
            want = x[a:b].t().contiguous() @ dy[a:b].double()
            # (a sum of n products in f32 is off by at most n 2^-24 of their size)
            assert ((dw[e].double() - want).abs() <= (b - a + 1) * 2.0 ** -24 * size + 2.0 ** -126).all()
