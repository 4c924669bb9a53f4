"""Group norm's statistics where a group's mean is far larger than its spread, where values are infinite or small (pytest -m gpu).

Tolerance of rstd.  In one launch the squared distances are taken from a mean m that is off by at most T 2^-25 |mean|, T the fp32 terms one
behind the other in its sums, 64 at most, and the mean distance's square is taken off again.  Distances are exact here, and their sums,
whole multiples of the values' step below 2^24 of them, too; squares' sums are of multiples of the step's square and exact
as well while below 2^24.  What is left are fp64's roundings and rstd's own, 2^-24, and where sums of squares pass 2^24 steps at most 32 roundings of
2^-24 of a sum that is (1 + (m's error / spread)^2) times the variance, here at most 5 times: 160 2^-24 of the variance, 80 2^-24 < 2^-17 of rstd.
By slices everything is fp64, off by far less.  The mean's tolerance is half its step for fp64 sums and one for what they are rounded to: 2^-23."""
import pytest
import torch

pytestmark = pytest.mark.gpu

# pixels, channels, groups: one launch of whole packs, of partial ones, of one and of sixteen packs a thread; by slices
SIZES = [(1, 64, 1), (50, 16, 2), (50, 15, 5), (256, 64, 8), (1000, 64, 8), (1024, 256, 32), (700, 30, 5), (20000, 16, 2), (20000, 15, 5), (9, 2048, 1)]


def statistics(x, groups, eps):
    n, p, c = x.shape
    g = x.double().view(n, p, groups, c // groups)
    mean = g.mean(dim=(1, 3))
    return mean, ((g - mean[:, None, :, None]).square().mean(dim=(1, 3)) + eps) ** -0.5


@pytest.mark.parametrize("steps", [3, 28, 1000])     # the mean is some 2^23, 2^20, 2^15 times the spread
@pytest.mark.parametrize("pixels,channels,groups", SIZES)
def test_means_far_larger_than_the_spread(pixels, channels, groups, steps):
    """The same rstd whatever way the size takes."""
    from paper_2204_08211_amd import binding as B
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(pixels + channels + steps)
    k = torch.randint(0, steps + 1, (3, pixels, channels), generator=gen, device="cuda:0")
    k[:, 0, ::channels // groups], k[:, 0, channels // groups - 1::channels // groups] = 0, steps       # a spread in every group
    for first, step in ((1.0, 2.0 ** -23), (-4096.0, 2.0 ** -11), (1e30, None)):
        x = (first + k.double() * (step if step else 2.0 ** 76)).float()
        mean, rstd = statistics(x, groups, 0.0)
        y, m, r = B.co3_groupnorm(x, groups, eps=0.0)
        assert float((r.double() / rstd - 1).abs().max()) <= 2.0 ** -17
        assert float((m.double() / mean - 1).abs().max()) <= 2.0 ** -23


@pytest.mark.parametrize("pixels,channels,groups", SIZES)
def test_one_value_apart(pixels, channels, groups):
    """All of a group alike but for one, also where that one is the first, and where it is far away."""
    from paper_2204_08211_amd import binding as B
    per = channels // groups
    for base, other in ((1.0, 1.0 + 2.0 ** -23), (3.0, -5.0), (1.0, 1e6), (1e-3, 0.0)):
        for at in (0, pixels - 1):
            x = torch.full((2, pixels, channels), base, device="cuda:0")
            x[:, at, at % per::per] = other
            mean, rstd = statistics(x, groups, 0.0)
            y, m, r = B.co3_groupnorm(x, groups, eps=0.0)
            if pixels * per > 1:
                assert float((r.double() / rstd - 1).abs().max()) <= 2.0 ** -17, (base, other, at)
                assert float((m.double() - mean).abs().max()) <= 2.0 ** -23 * max(abs(base), float(mean.abs().max())), (base, other, at)


@pytest.mark.parametrize("pixels,channels,groups", SIZES)
def test_infinities_leave_their_mean(pixels, channels, groups):
    """An infinity anywhere in a group, the first value too, makes its mean infinite; a NaN makes it NaN."""
    from paper_2204_08211_amd import binding as B
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(pixels)
    per = channels // groups
    for name in (torch.float32, torch.bfloat16):
        for at in (0, pixels - 1):
            x = torch.randn(3, pixels, channels, generator=gen, device="cuda:0")
            x[0, at, 0], x[1, at, per - 1], x[2, at, 0] = float("inf"), -float("inf"), float("nan")
            y, m, r = B.co3_groupnorm(x.to(name), groups)
            assert float(m[0, 0]) == float("inf") and float(m[1, 0]) == -float("inf") and bool(m[2, 0].isnan())
            assert bool(r[:, 0].isnan().all()) and bool(r[:, 1:].isfinite().all()) and bool(y[:, :, :per].isnan().all()) and bool(y[:, :, per:].isfinite().all())


@pytest.mark.parametrize("scale", [2.0 ** -24, 2.0 ** -20, 2.0 ** -15])
@pytest.mark.parametrize("pixels,channels,groups", SIZES)
def test_small_numbers_of_fp16(pixels, channels, groups, scale):
    """Numbers below 2^-14, which fp16 holds with fewer bits, count as what they are."""
    from paper_2204_08211_amd import binding as B
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(pixels + channels)
    x = (torch.randint(-9, 10, (3, pixels, channels), generator=gen, device="cuda:0") * scale).half()
    x[:, 0, ::channels // groups] = 9 * scale
    x[:, 0, channels // groups - 1::channels // groups] = -4 * scale
    mean, rstd = statistics(x, groups, 1e-13)
    y, m, r = B.co3_groupnorm(x, groups, eps=1e-13)
    assert float((r.double() / rstd - 1).abs().max()) <= 2.0 ** -17
    assert float((m.double() - mean).abs().max()) <= 2.0 ** -20 * 9 * scale
    g = x.double().view(3, pixels, groups, -1)
    want = ((g - mean[:, None, :, None]) * rstd[:, None, :, None]).view(x.shape)
    assert float((y.double() - want).abs().max()) <= (2.0 ** -11 + 2.0 ** -17) * float(want.abs().max())
