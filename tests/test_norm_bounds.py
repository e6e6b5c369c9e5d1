"""The allowance of test_gpu_norm_far.py shows what it is for (no GPU)."""
import torch

from test_gpu_norm_far import EPS, WIDTHS, exact


def test_a_mean_taken_away_once():
    """With the mean as f32 rounds it, dweight of rows at 10 000 is off by more than the allowance, at all widths."""
    for width in WIDTHS:
        gen = torch.Generator().manual_seed(width)
        x = torch.randn((20, width), generator=gen) * 0.1 + 10000
        dy = torch.randn((20, width), generator=gen) + 0.5
        _, _, (dw, off), _ = exact(x, dy, None)
        rounded_mean = x.double().mean(1, keepdim=True).float().double()
        spread = (x.double().var(1, keepdim=True, unbiased=False) + EPS).sqrt()
        once = (dy.double() * (x.double() - rounded_mean) / spread).sum(0)
        assert float(((once - dw).abs() / off).median()) > 2
