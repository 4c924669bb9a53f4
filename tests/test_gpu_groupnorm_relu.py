"""Group norm with ReLU: the border between values that are let through and values that are not, in both passes (pytest -m gpu)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("affine", [True, False])
@pytest.mark.parametrize("pixels,channels,groups", [(1, 512, 4), (64, 480, 8), (50, 495, 5), (1024, 512, 16), (16384, 512, 8), (9000, 495, 3)])
def test_relus_border_is_the_same_in_both_passes(pixels, channels, groups, affine):
    """A value that the forward pass lets through has a gradient, and one that it does not let through has none, also where the argument is a
    rounding away from 0: each channel's bias is minus what one pixel of it has there."""
    from paper_2204_08211_amd import binding as B
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(pixels + channels)
    x = torch.randn(2, pixels, channels, generator=gen, device="cuda:0") + 0.3
    weight = 1 + 0.3 * torch.randn(channels, generator=gen, device="cuda:0") if affine else None
    _, mean, rstd = B.co3_groupnorm(x, groups, weight)
    at = torch.randint(0, pixels, (channels,), generator=gen, device="cuda:0")
    c = torch.arange(channels, device="cuda:0")
    for sample in (0, 1):
        g = c // (channels // groups)
        xh = (x[sample, at, c].double() - mean[sample, g].double()) * rstd[sample, g].double()
        bias = (-xh * (1 if weight is None else weight.double())).float()
        y, m, r = B.co3_groupnorm(x, groups, weight, bias, activation=B.ACT_RELU)
        assert torch.equal(m, mean) and torch.equal(r, rstd)
        dy = torch.zeros_like(x)
        dy[sample, at, c] = 1.0
        grad = torch.full((1, channels), 5.0, device="cuda:0")
        B.co3_groupnorm_backward(dy, x, groups, weight, bias, mean, rstd, activation=B.ACT_RELU, dbias=grad)
        assert torch.equal(grad[0], (y[sample, at, c] > 0).float())
        assert bool((y[sample, at, c] <= 2.0 ** -20 * (1 + xh.abs())).all())
