"""Group norm with an activation, both passes, against a plain implementation in 64 bits (pytest -m gpu): types, activations, widths of a
group, sizes around every form's limits, strides, users, x in 8 bits, accumulation, in place, extreme values, other streams, a replayed
graph; gradients against differences.

Tolerances: a result of 16 bits is rounded once, by at most half a step (2^-8 of a bfloat16, 2^-11 of a float16); fp32 ones go through some
twenty roundings of 2^-24 and the sigmoid's, in which the exponent's rounding is |z| 2^-24 (|z| < 16 here), and sums whose errors grow as
the square root of their length: 2^-19 of the result's 2-norm in all.  Gradients of weights are sums of dz and of dz xh: 2^-19 of the sum of |dy|, of
|dy xh|.  (Not of |dz|: SiLU's slope p (1 + z (1 - p)) is 0 near z = -1.28, where what is left is roundings of p, z (1 - p) and the sum, each 2^-24
of something below 1.3, and z's own, 2^-23 |z|, times a slope of the slope of 0.5 at most, |z slope''| < 0.6: 2^-21 in all, whatever dz is.)  Where ReLU's argument is within 2^-20 of 0 either side may be right: inputs that have such a
place are made without it."""
import pytest
import torch

import blocks8_util as bu

pytestmark = pytest.mark.gpu

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
TOL = {torch.float32: 2.0 ** -19, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
ACTS = ["none", "relu", "silu"]


def act_of(name):
    from paper_2204_08211_amd import binding as B
    return {"none": B.ACT_NONE, "relu": B.ACT_RELU, "silu": B.ACT_SILU}[name]


def rel(x, y):
    d, n = (x.double() - y.double()).norm(), y.double().norm()
    return float(d / n) if n > 0 else float(d)


def activated(z, act):
    return z.clamp(min=0) if act == "relu" else z * torch.sigmoid(z) if act == "silu" else z


def slope(z, act):
    s = torch.sigmoid(z)
    return (z > 0).double() if act == "relu" else s * (1 + z * (1 - s)) if act == "silu" else torch.ones_like(z)


def plain_forward(x, groups, weight, bias, eps, act):
    n, p, c = x.shape
    g = x.double().view(n, p, groups, c // groups)
    mean = g.mean(dim=(1, 3))
    rstd = ((g - mean[:, None, :, None]).square().mean(dim=(1, 3)) + eps) ** -0.5
    z = ((g - mean[:, None, :, None]) * rstd[:, None, :, None]).view(n, p, c)
    z = z * (1 if weight is None else weight.double()) + (0 if bias is None else bias.double())
    return activated(z, act), mean, rstd


def plain_backward(dy, x, groups, weight, bias, mean, rstd, act, users):
    n, p, c = x.shape
    per = c // groups
    wide = lambda v: v.double().repeat_interleave(per, dim=1)[:, None, :]  # noqa: E731
    w = torch.ones(c, dtype=torch.float64, device=x.device) if weight is None else weight.double()
    xh = (x.double() - wide(mean)) * wide(rstd)
    dz = dy.double() * slope(xh * w + (0 if bias is None else bias.double()), act)
    t = dz * w
    over = lambda v: v.view(n, p, groups, per).mean(dim=(1, 3))  # noqa: E731
    dx = wide(rstd) * (t - wide(over(t)) - xh * wide(over(t * xh)))
    of = lambda v: v.view(users, -1, c).sum(dim=1)  # noqa: E731
    return dx, of(dz * xh), of(dz), of((dy.double() * xh).abs()), of(dy.double().abs())


def make(n, p, c, groups, t, seed, act, affine=True):
    """x, dy, weight, bias; no argument of the activation next to 0."""
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(seed)
    x = (2 * torch.randn(n, p, c, generator=gen, device="cuda:0") + torch.randn(n, 1, c, generator=gen, device="cuda:0")).to(t)
    dy = torch.randn(n, p, c, generator=gen, device="cuda:0").to(t)
    weight = 1 + 0.3 * torch.randn(c, generator=gen, device="cuda:0") if affine else None
    bias = torch.randn(c, generator=gen, device="cuda:0") if affine else None
    return x, dy, weight, bias


def quiet(dy, x, groups, weight, bias, mean, rstd):
    """dy with zeros where ReLU's argument is next to 0."""
    per = x.shape[2] // groups
    wide = lambda v: v.double().repeat_interleave(per, dim=1)[:, None, :]  # noqa: E731
    z = (x.double() - wide(mean)) * wide(rstd) * (1 if weight is None else weight.double()) + (0 if bias is None else bias.double())
    return torch.where(z.abs() < 2.0 ** -20 * 16, torch.zeros_like(dy), dy)


def check_backward(dy, x, groups, weight, bias, mean, rstd, act, users, seen=None, **how):
    """seen: what x's numbers are, where it is in 8 bits."""
    from paper_2204_08211_amd import binding as B
    n, p, c = dy.shape
    dw, db = torch.full((users, c), 7.0, device="cuda:0"), torch.full((users, c), 7.0, device="cuda:0")
    dx = B.co3_groupnorm_backward(dy, x, groups, weight, bias, mean, rstd, activation=act_of(act), users=users, dweight=dw, dbias=db, **how)
    edx, edw, edb, sw, sb = plain_backward(dy, x if seen is None else seen, groups, weight, bias, mean, rstd, act, users)
    if p * (c // groups) > 2:
        assert rel(dx, edx) <= TOL[dy.dtype]
    else:    # a difference that leaves only roundings
        limit = 16 * TOL[dy.dtype] * float((dy.double().abs().amax() * (1 if weight is None else weight.abs().amax()) * rstd.max() * 2))
        assert float((dx.double() - edx).abs().max()) <= limit
    assert bool(((dw.double() - edw).abs() <= 2.0 ** -19 * sw + 1e-30).all()) and bool(((db.double() - edb).abs() <= 2.0 ** -19 * sb + 1e-30).all())
    return dx, dw, db


# pixels, channels, groups: one of all; groups of one channel, of odd numbers, wider than a workgroup; each form's limits
SIZES = [(1, 1, 1), (1, 8, 8), (2, 6, 3), (1, 64, 1), (49, 64, 8), (64, 60, 4), (100, 33, 11), (257, 40, 5), (1024, 64, 32), (1025, 96, 3),
         (4096, 16, 2), (9, 2048, 1), (5, 3001, 1), (1, 32768, 4), (700, 333, 37), (8200, 24, 3)]


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("name", sorted(TYPES))
@pytest.mark.parametrize("pixels,channels,groups", SIZES)
def test_both_passes(pixels, channels, groups, name, act):
    from paper_2204_08211_amd import binding as B
    t = TYPES[name]
    x, dy, weight, bias = make(4, pixels, channels, groups, t, pixels + channels, act)
    y, mean, rstd = B.co3_groupnorm(x, groups, weight, bias, eps=1e-3, activation=act_of(act))
    ey, emean, erstd = plain_forward(x, groups, weight, bias, 1e-3, act)
    assert rel(y, ey) <= TOL[t]
    assert rel(rstd, erstd) <= 2.0 ** -20 and float((mean.double() - emean).abs().max()) <= 2.0 ** -20 * float(x.double().abs().max())
    check_backward(quiet(dy, x, groups, weight, bias, mean, rstd), x, groups, weight, bias, mean, rstd, act, 2)


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("name", sorted(TYPES))
@pytest.mark.parametrize("pixels,channels,groups", [(1, 16, 2), (64, 60, 4), (100, 33, 11), (300, 200, 8), (1030, 257, 1), (5000, 130, 13), (3, 1500, 5)])
def test_x_kept_in_8_bits(pixels, channels, groups, name, block_rows):
    from paper_2204_08211_amd import binding as B
    x, dy, weight, bias = make(6, pixels, channels, groups, TYPES[name], channels, "silu")
    _, mean, rstd = B.co3_groupnorm(x, groups, weight, bias, activation=B.ACT_SILU)
    for users, batch in ((3, 3), (2, 1), (1, 1)):
        kept = B.co3_quantize8(x.view(batch, 6 // batch * pixels, channels), block_rows=block_rows)
        seen = bu.numbers(kept.values, kept.scales, channels, block_rows).view(6, pixels, channels)
        check_backward(dy, kept, groups, weight, bias, mean, rstd, "silu", users, seen=seen)


@pytest.mark.parametrize("pixels,channels,groups", [(60, 64, 8), (3000, 30, 5)])
def test_without_weight_bias_or_gradients(pixels, channels, groups):
    from paper_2204_08211_amd import binding as B
    x, dy, weight, bias = make(4, pixels, channels, groups, torch.float32, 5, "silu")
    for w, b in ((None, None), (weight, None), (None, bias)):
        y, mean, rstd = B.co3_groupnorm(x, groups, w, b, activation=B.ACT_SILU)
        assert rel(y, plain_forward(x, groups, w, b, 1e-5, "silu")[0]) <= TOL[torch.float32]
        dx, dw, db = check_backward(dy, x, groups, w, b, mean, rstd, "silu", 2)
        only = torch.zeros_like(dw)
        call = lambda **k: B.co3_groupnorm_backward(dy, x, groups, w, b, mean, rstd, activation=B.ACT_SILU, users=2, **k)  # noqa: E731
        assert torch.equal(call(dweight=only), dx) and torch.equal(only, dw)
        assert torch.equal(call(dbias=only), dx) and torch.equal(only, db)
        assert torch.equal(call(), dx)


@pytest.mark.parametrize("pixels,channels,groups", [(60, 64, 8), (3000, 30, 5)])
def test_gradients_of_users_in_their_rows(pixels, channels, groups):
    from paper_2204_08211_amd import binding as B
    users = 3
    x, dy, weight, bias = make(6, pixels, channels, groups, torch.bfloat16, 6, "silu")
    _, mean, rstd = B.co3_groupnorm(x, groups, weight, bias, activation=B.ACT_SILU)
    buffer = torch.full((users, 5 + 2 * channels + 3), -3.0, device="cuda:0")
    dw, db = buffer[:, 5:5 + channels], buffer[:, 5 + channels:5 + 2 * channels]
    call = lambda **k: B.co3_groupnorm_backward(dy, x, groups, weight, bias, mean, rstd, activation=B.ACT_SILU, users=users, dweight=dw, dbias=db, **k)  # noqa: E731
    call()
    first = buffer.clone()
    call()
    assert torch.equal(first, buffer)
    for u in range(users):      # a user alone has the same gradients
        part = slice(2 * u, 2 * u + 2)
        own = torch.zeros(2, channels, device="cuda:0")
        B.co3_groupnorm_backward(dy[part], x[part], groups, weight, bias, mean[part], rstd[part], activation=B.ACT_SILU, dweight=own[0], dbias=own[1])
        assert rel(own[0], first[u, 5:5 + channels]) <= 2.0 ** -19 and rel(own[1], first[u, 5 + channels:5 + 2 * channels]) <= 2.0 ** -19
    call(accumulate=True)
    assert rel(dw, 2 * first[:, 5:5 + channels].double()) <= 2.0 ** -22 and rel(db, 2 * first[:, 5 + channels:5 + 2 * channels].double()) <= 2.0 ** -22
    assert bool((buffer[:, :5] == -3).all()) and bool((buffer[:, 5 + 2 * channels:] == -3).all())


@pytest.mark.parametrize("name", sorted(TYPES))
@pytest.mark.parametrize("pixels,channels,groups", [(20, 14, 2), (40, 64, 8), (5000, 21, 3)])
def test_pixels_apart_at_any_element_and_in_place(pixels, channels, groups, name):
    from paper_2204_08211_amd import binding as B
    t = TYPES[name]

    def apart(pad, shift, v):
        whole = torch.full((3 * pixels * (channels + pad) + 64,), 5.0, device="cuda:0").to(t)
        view = whole[shift:shift + 3 * pixels * (channels + pad)].view(3, pixels, channels + pad)[:, :, :channels]
        view.copy_(v)
        return whole, view

    x, dy, weight, bias = make(3, pixels, channels, groups, t, 4, "silu")
    want, mean, rstd = B.co3_groupnorm(x, groups, weight, bias, activation=B.ACT_SILU)
    _, xs = apart(3, 1, x)
    y_all, ys = apart(7, 3, torch.zeros_like(x))
    keep = torch.ones_like(y_all, dtype=torch.bool)
    keep[3:3 + 3 * pixels * (channels + 7)].view(3, pixels, channels + 7)[:, :, :channels] = False
    _, m2, r2 = B.co3_groupnorm(xs, groups, weight, bias, activation=B.ACT_SILU, y=ys)
    assert torch.equal(ys, want) and torch.equal(mean, m2) and torch.equal(rstd, r2) and bool((y_all[keep] == 5).all())
    dx = B.co3_groupnorm_backward(dy, x, groups, weight, bias, mean, rstd, activation=B.ACT_SILU)
    _, ds = apart(2, 5, dy)
    out_all, outs = apart(7, 3, torch.zeros_like(x))
    B.co3_groupnorm_backward(ds, xs, groups, weight, bias, mean, rstd, activation=B.ACT_SILU, dx=outs)
    assert torch.equal(outs, dx) and bool((out_all[keep] == 5).all())
    grads = torch.zeros(2, channels, device="cuda:0")
    B.co3_groupnorm_backward(dy, x, groups, weight, bias, mean, rstd, activation=B.ACT_SILU, dweight=grads[0], dbias=grads[1])
    for place in (0, 1):        # dx in dy's place, and in x's
        xc, dc, own = x.clone(), dy.clone(), torch.zeros(2, channels, device="cuda:0")
        B.co3_groupnorm_backward(dc, xc, groups, weight, bias, mean, rstd, activation=B.ACT_SILU, dx=xc if place else dc, dweight=own[0], dbias=own[1])
        assert torch.equal(xc if place else dc, dx) and torch.equal(own, grads)
    xc = x.clone()
    B.co3_groupnorm(xc, groups, weight, bias, activation=B.ACT_SILU, y=xc)
    assert torch.equal(xc, want)


@pytest.mark.parametrize("pixels", [50, 20000])
def test_values_far_from_zero_and_at_the_ends(pixels):
    from paper_2204_08211_amd import binding as B
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(pixels)
    x = torch.randn(2, pixels, 16, generator=gen, device="cuda:0") + 4096          # a mean of 4096 times the spread
    y, mean, rstd = B.co3_groupnorm(x, 2)
    ey, emean, erstd = plain_forward(x, 2, None, None, 1e-5, "none")
    # x itself is rounded at 2^-12 of the spread: the mean's rounding of 2^-12.5 is in every y of a group alike
    assert rel(y, ey) <= 2.0 ** -12 and rel(rstd, erstd) <= 2.0 ** -18 and rel(mean, emean) <= 2.0 ** -23
    x = torch.full((2, pixels, 16), 3.0, device="cuda:0")                          # no spread at all
    y, mean, rstd = B.co3_groupnorm(x, 2, eps=1e-5)
    assert float(y.abs().max()) <= 1e-3 and rel(rstd, torch.full_like(rstd, 1e-5 ** -0.5)) <= 2.0 ** -20
    x = torch.randn(2, pixels, 16, generator=gen, device="cuda:0")
    x[0, 7, 3], x[1, 0, 12] = float("nan"), float("inf")
    for act in ACTS:
        y, mean, rstd = B.co3_groupnorm(x, 2, activation=act_of(act))
        bad = torch.zeros(2, 2, dtype=torch.bool, device="cuda:0")
        bad[0, 0], bad[1, 1] = True, True
        assert torch.equal(rstd.isnan(), bad)
        assert torch.equal(y.isnan(), bad[:, None, :].expand(2, pixels, 2).repeat_interleave(8, dim=2))


@pytest.mark.parametrize("scale", [1e37, 1e25, 1e-25, 1e-36])
@pytest.mark.parametrize("pixels,channels,groups", [(50, 16, 2), (50, 15, 5), (1000, 64, 8), (20000, 16, 2)])
def test_squares_beyond_the_type(pixels, channels, groups, scale):
    """Values whose squares leave fp32 at either end are normed as others are, beside a group of ordinary ones; scale is in every term alike, so
    the tolerance is that of ordinary values."""
    from paper_2204_08211_amd import binding as B
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(pixels + channels)
    x = torch.randn(2, pixels, channels, generator=gen, device="cuda:0") + 0.5
    x[..., channels // groups:] *= scale
    for t in (torch.float32, torch.bfloat16):
        y, mean, rstd = B.co3_groupnorm(x.to(t), groups, eps=0.0)
        ey, emean, erstd = plain_forward(x.to(t), groups, None, None, 0.0, "none")
        per = channels // groups
        for part in (slice(0, per), slice(per, None)):
            assert rel(y[..., part], ey[..., part]) <= TOL[t]
        for part in (slice(0, 1), slice(1, None)):
            assert rel(rstd[:, part], erstd[:, part]) <= TOL[torch.float32] and rel(mean[:, part], emean[:, part]) <= TOL[torch.float32]


def test_large_activations():
    """The sigmoid at its ends: no NaN, and the activation's limits."""
    from paper_2204_08211_amd import binding as B
    x = torch.linspace(-1, 1, 4 * 64 * 32, device="cuda:0").view(4, 64, 32)
    weight = torch.full((32,), 200.0, device="cuda:0")
    y, mean, rstd = B.co3_groupnorm(x, 4, weight, None, activation=B.ACT_SILU)
    want, _, _ = plain_forward(x, 4, weight, None, 1e-5, "silu")
    assert bool(y.isfinite().all()) and float((y.double() - want).abs().max()) <= 2.0 ** -19 * float(want.abs().max())
    check_backward(torch.ones_like(x), x, 4, weight, None, mean, rstd, "silu", 1)


@pytest.mark.parametrize("act", ["none", "silu"])
def test_gradients_against_differences(act):
    """(f(v + h) - f(v - h)) / 2h of the plain form in 64 bits along random directions of x, weight and bias."""
    from paper_2204_08211_amd import binding as B
    x, dy, weight, bias = make(2, 30, 12, 3, torch.float32, 9, act)
    _, mean, rstd = B.co3_groupnorm(x, 3, weight, bias, activation=act_of(act))
    dw, db = torch.zeros(1, 12, device="cuda:0"), torch.zeros(1, 12, device="cuda:0")
    dx = B.co3_groupnorm_backward(dy, x, 3, weight, bias, mean, rstd, activation=act_of(act), dweight=dw, dbias=db)
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(1)
    f = lambda x_, w_, b_: float((plain_forward(x_, 3, w_, b_, 1e-5, act)[0] * dy.double()).sum())  # noqa: E731
    at = [x.double(), weight.double(), bias.double()]
    for k, grad in enumerate((dx, dw[0], db[0])):
        v = torch.randn(at[k].shape, generator=gen, device="cuda:0", dtype=torch.float64)
        h = 1e-5
        up, down = list(at), list(at)
        up[k], down[k] = at[k] + h * v, at[k] - h * v
        want = (f(*up) - f(*down)) / (2 * h)
        # the differences are off by h^2 of a third derivative, some 1e-8; the gradient by 2^-19 of its norm
        assert abs(float((grad.double() * v).sum()) - want) <= 1e-6 * abs(want) + 2.0 ** -19 * float(grad.double().norm() * v.norm())


def test_no_samples():
    from paper_2204_08211_amd import binding as B
    x = torch.zeros(0, 5, 8, device="cuda:0")
    y, mean, rstd = B.co3_groupnorm(x, 2)
    assert y.shape == (0, 5, 8) and mean.shape == (0, 2)
    dw, db = torch.full((2, 8), 3.0, device="cuda:0"), torch.full((2, 8), 3.0, device="cuda:0")
    B.co3_groupnorm_backward(x, x, 2, None, None, mean, rstd, users=2, dweight=dw, dbias=db, accumulate=True)
    assert bool((dw == 3).all())
    B.co3_groupnorm_backward(x, x, 2, None, None, mean, rstd, users=2, dweight=dw, dbias=db)
    assert bool((dw == 0).all()) and bool((db == 0).all())


def test_many_samples_and_many_users():
    """More samples than a dimension of a launch takes, a user for each."""
    from paper_2204_08211_amd import binding as B
    x, dy, weight, bias = make(70000, 3, 8, 2, torch.float16, 3, "silu")
    y, mean, rstd = B.co3_groupnorm(x, 2, weight, bias, activation=B.ACT_SILU)
    assert rel(y, plain_forward(x, 2, weight, bias, 1e-5, "silu")[0]) <= TOL[torch.float16]
    check_backward(dy, x, 2, weight, bias, mean, rstd, "silu", 35000)


@pytest.mark.parametrize("pixels", [40, 3000])
def test_other_streams_and_a_replayed_graph(pixels):
    from paper_2204_08211_amd import binding as B
    channels, groups = 24, 3
    x, dy, weight, bias = make(4, pixels, channels, groups, torch.bfloat16, 2, "silu")
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(4, groups, device="cuda:0"), torch.empty(4, groups, device="cuda:0")
    grad = torch.zeros(2, 2 * channels, device="cuda:0")
    ws = torch.empty(max(B.co3_groupnorm_workspace_bytes(4, pixels, channels, groups, x.dtype),
                         B.co3_groupnorm_backward_workspace_bytes(2, 4, pixels, channels, groups, x.dtype)), dtype=torch.uint8, device="cuda:0")

    def step(stream=None):
        B.co3_groupnorm(x, groups, weight, bias, activation=B.ACT_SILU, y=y, mean=mean, rstd=rstd, workspace=ws, stream=stream)
        B.co3_groupnorm_backward(dy, x, groups, weight, bias, mean, rstd, activation=B.ACT_SILU, users=2, dx=dx, dweight=grad[:, :channels],
                                 dbias=grad[:, channels:], workspace=ws, stream=stream)

    outs = (y, mean, rstd, dx, grad)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    first = [o.clone() for o in outs]
    assert rel(y, plain_forward(x, groups, weight, bias, 1e-5, "silu")[0]) <= TOL[torch.bfloat16]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (5, 6, 2):
        a, b, _, _ = make(4, pixels, channels, groups, torch.bfloat16, seed, "silu")
        x.copy_(a)
        dy.copy_(b)
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        step()
        assert all(torch.equal(p, q) for p, q in zip(got, outs))
    assert all(torch.equal(p, q) for p, q in zip(first, outs))


@pytest.mark.parametrize("pixels", [60, 1500])     # in one launch, and by slices
def test_offsets_beyond_32_bits(pixels):
    """Pixels 2^22 elements apart, more than 2^32 in all: the bits of the same call on pixels next to each other."""
    from paper_2204_08211_amd import binding as B
    far, n, c = 1 << 22, -(-1500 // pixels), 30
    x, dy, weight, bias = make(n, pixels, c, 5, torch.bfloat16, 7, "silu")
    at = [torch.empty(n * pixels * far, dtype=torch.bfloat16, device="cuda:0").as_strided((n, pixels, c), (pixels * far, far, 1)) for _ in range(4)]
    at[0].copy_(x)
    at[1].copy_(dy)
    y, mean, rstd = B.co3_groupnorm(x, 5, weight, bias, activation=B.ACT_SILU)
    far_y, far_mean, far_rstd = B.co3_groupnorm(at[0], 5, weight, bias, activation=B.ACT_SILU, y=at[2])
    assert torch.equal(far_y, y) and torch.equal(far_mean, mean) and torch.equal(far_rstd, rstd)
    grads, far_grads = torch.zeros(2, 1, c, device="cuda:0"), torch.zeros(2, 1, c, device="cuda:0")
    dx = B.co3_groupnorm_backward(dy, x, 5, weight, bias, mean, rstd, activation=B.ACT_SILU, dweight=grads[0], dbias=grads[1])
    far_dx = B.co3_groupnorm_backward(at[1], at[0], 5, weight, bias, mean, rstd, activation=B.ACT_SILU, dx=at[3], dweight=far_grads[0], dbias=far_grads[1])
    assert torch.equal(far_dx, dx) and torch.equal(far_grads, grads)
