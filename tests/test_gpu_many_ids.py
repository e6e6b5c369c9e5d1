"""Lookup's gradient of as many ids as it takes: 2^30, whose runs are more workgroups than one launch has threads for."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fewer", [0, 77])
def test_most_ids(fewer):
    """One row of ones for all of them: every sum is its count, below 2^24 and so exact in f32."""
    import paper_2208_09151_amd as g
    n, names, width = 2 ** 30 - fewer, 2 ** 14, 129
    ids = torch.arange(n, dtype=torch.int32, device="cuda")
    ids.bitwise_and_(names - 1).mul_(7919).bitwise_and_(names - 1)
    dy = torch.ones((1, width), device="cuda").expand(n, width)
    got = g.lookup_backward(dy, ids, names + 3)
    left_out = torch.bincount(torch.arange(n, 2 ** 30) * 7919 % names, minlength=names)
    count = torch.cat([2 ** 16 - left_out, torch.zeros(3, dtype=torch.int64)]).cuda()
    assert torch.equal(got, count.float()[:, None].expand(names + 3, width))
    del ids, dy, got
    torch.cuda.empty_cache()
