"""Layer norm's forward and backward pass against a plain implementation in 64 bits (pytest -m gpu): types, row lengths
around every form's limits, strides, users, accumulation, in place, extreme values, other streams, a replayed graph.

Tolerances, all of the difference's 2-norm over the result's: a result of 16 bits is rounded once, by at most half a unit in the
last place (2^-8 of a bfloat16 of 8 significant bits, 2^-11 of a float16 of 11); one of fp32 goes through some ten roundings of 2^-24 and sums whose
errors grow as the square root of their length, 2^-20 in all.  A single value may be a whole rounding off, plus as much."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

TOL = {"float32": 2.0 ** -20, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


def dtype_of(name):
    import torch
    return getattr(torch, name)


def rel(x, y):
    d = (x.double() - y).norm()
    n = y.norm()
    return float(d / n) if n > 0 else float(d)


def plain_forward(x, weight, bias, eps):
    x = x.double()
    mean = x.mean(dim=-1, keepdim=True)
    rstd = ((x - mean).square().mean(dim=-1, keepdim=True) + eps) ** -0.5
    y = (x - mean) * rstd
    if weight is not None:
        y = y * weight.double()
    if bias is not None:
        y = y + bias.double()
    return y, mean[..., 0], rstd[..., 0]


def plain_backward(dy, x, weight, mean, rstd):
    dy, x = dy.double(), x.double()
    xh = (x - mean.double()[..., None]) * rstd.double()[..., None]
    t = dy if weight is None else dy * weight.double()
    dx = rstd.double()[..., None] * (t - t.mean(dim=-1, keepdim=True) - xh * (t * xh).mean(dim=-1, keepdim=True))
    return dx, (dy * xh).sum(dim=-2), dy.sum(dim=-2)


# one and two elements; the limits of 8, 16, 32 and 64 lanes a row, of two, four and eight packs a lane, of the larger workgroups, each
# for 8 elements of 16 bits and 4 of 32 in a pack; odd lengths in between
COLS = [1, 2, 3, 31, 32, 33, 64, 65, 127, 128, 129, 256, 257, 511, 513, 1001, 1024, 2047, 2048, 2049, 4096, 4099, 8192, 8193, 16384, 16387, 32768]


@pytest.mark.parametrize("name", sorted(TOL))
@pytest.mark.parametrize("cols", COLS)
def test_both_passes(cols, name):
    import torch
    from paper_2204_08211_amd import binding as B
    dt, dev = dtype_of(name), "cuda:0"
    gen = torch.Generator(device=dev)
    gen.manual_seed(cols)
    users, rows = 3, (37 if cols < 4096 else 5)
    x = (2 * torch.randn(users, rows, cols, generator=gen, device=dev) + torch.randn(users, rows, 1, generator=gen, device=dev)).to(dt)
    dy = torch.randn(users, rows, cols, generator=gen, device=dev).to(dt)
    weight, bias = 1 + 0.3 * torch.randn(cols, generator=gen, device=dev), torch.randn(cols, generator=gen, device=dev)
    y, mean, rstd = B.co3_layernorm(x, weight, bias, eps=1e-5)
    ey, emean, erstd = plain_forward(x, weight, bias, 1e-5)
    assert rel(y, ey) <= TOL[name] and rel(rstd, erstd) <= 2.0 ** -20
    assert float((mean.double() - emean).abs().max()) <= 2.0 ** -20 * float(x.double().abs().max())
    dweight, dbias = torch.full((users, cols), 7.0, device=dev), torch.full((users, cols), 7.0, device=dev)
    dx = B.co3_layernorm_backward(dy, x, weight, mean, rstd, dweight=dweight, dbias=dbias)
    edx, edw, edb = plain_backward(dy, x, weight, mean, rstd)
    if cols > 2:     # the gradient of rows of one or two elements is a difference that leaves only roundings
        assert rel(dx, edx) <= TOL[name]
    else:
        assert float((dx.double() - edx).abs().max()) <= 8 * TOL[name] * float((dy.double().abs().amax() * weight.abs().amax() * rstd.max()))
    assert rel(dbias, edb) <= 2.0 ** -20
    assert float((dweight.double() - edw).abs().max()) <= 2.0 ** -20 * float(dy.double().abs().max()) * 2 * rows


@pytest.mark.parametrize("users,rows", [(1, 1), (1, 15), (1, 17), (1, 4097), (5, 64), (16, 333), (600, 40)])
@pytest.mark.parametrize("cols", [48, 300, 2500])
def test_gradients_of_users_are_their_own(users, rows, cols):
    import torch
    from paper_2204_08211_amd import binding as B
    dev = "cuda:0"
    gen = torch.Generator(device=dev)
    gen.manual_seed(users * rows)
    x = torch.randn(users, rows, cols, generator=gen, device=dev).bfloat16()
    dy = torch.randn(users, rows, cols, generator=gen, device=dev).bfloat16()
    _, mean, rstd = B.co3_layernorm(x)
    buffer = torch.full((users, 3 + 2 * cols + 5), -3.0, device=dev)      # a layer's weight and bias within the users' gradients
    dw, db = buffer[:, 3:3 + cols], buffer[:, 3 + cols:3 + 2 * cols]
    B.co3_layernorm_backward(dy, x, None, mean, rstd, dweight=dw, dbias=db)
    _, edw, edb = plain_backward(dy, x, None, mean, rstd)
    limit = 2.0 ** -20 * 6 * rows ** 0.5 + 2.0 ** -20
    assert float((dw.double() - edw).abs().max()) <= limit * 4 and float((db.double() - edb).abs().max()) <= limit * 4
    first = buffer.clone()
    B.co3_layernorm_backward(dy, x, None, mean, rstd, dweight=dw, dbias=db)
    assert torch.equal(first, buffer)                                      # the same order every time
    B.co3_layernorm_backward(dy, x, None, mean, rstd, dweight=dw, dbias=db, accumulate=True)
    assert rel(dw, 2 * first[:, 3:3 + cols].double()) <= 2.0 ** -22
    assert bool((buffer[:, :3] == -3).all()) and bool((buffer[:, 3 + 2 * cols:] == -3).all())


def test_one_gradient_or_none():
    import torch
    from paper_2204_08211_amd import binding as B
    x = torch.randn(2, 600, 70, device="cuda:0")
    dy = torch.randn_like(x)
    _, mean, rstd = B.co3_layernorm(x)
    dw, db = torch.zeros(2, 70, device="cuda:0"), torch.zeros(2, 70, device="cuda:0")
    both = B.co3_layernorm_backward(dy, x, None, mean, rstd, dweight=dw, dbias=db)
    only = torch.zeros_like(dw)
    assert torch.equal(B.co3_layernorm_backward(dy, x, None, mean, rstd, dweight=only), both) and torch.equal(only, dw)
    only.zero_()
    assert torch.equal(B.co3_layernorm_backward(dy, x, None, mean, rstd, dbias=only), both) and torch.equal(only, db)
    assert torch.equal(B.co3_layernorm_backward(dy, x, None, mean, rstd), both)


@pytest.mark.parametrize("name", sorted(TOL))
@pytest.mark.parametrize("cols", [5, 100, 1500, 9000])
def test_rows_apart_at_any_element_and_in_place(cols, name):
    import torch
    from paper_2204_08211_amd import binding as B
    dt, dev = dtype_of(name), "cuda:0"
    gen = torch.Generator(device=dev)
    gen.manual_seed(cols)

    def rows_of(pad, shift):
        whole = torch.full((29 * (cols + pad) + 64,), 5.0, device=dev).to(dt)
        view = whole[shift:shift + 29 * (cols + pad)].view(29, cols + pad)[:, :cols]
        view.copy_(torch.randn(29, cols, generator=gen, device=dev))
        return whole, view

    flat = torch.randn(2 * cols + 1, generator=gen, device=dev)
    weight, bias = flat[1:1 + cols], flat[1 + cols:]
    _, x = rows_of(3, 1)
    y_all, y = rows_of(7, 3)
    before = y_all.clone()
    B.co3_layernorm(x, weight, bias, y=y)
    want, _, _ = plain_forward(x, weight, bias, 1e-5)
    assert rel(y, want) <= TOL[name]
    y.fill_(5.0)
    before[3:3 + 29 * (cols + 7)].view(29, cols + 7)[:, :cols] = 5.0
    assert torch.equal(y_all, before)                                      # nothing but the rows was written
    _, mean, rstd = B.co3_layernorm(x, weight, bias)
    _, dy = rows_of(2, 5)
    want = B.co3_layernorm_backward(dy, x, weight, mean, rstd, dx=torch.empty(29, cols, device=dev, dtype=dt))
    for target in (dy, x):
        d, xx = dy.clone(), x.clone()
        if target is dy:
            assert torch.equal(B.co3_layernorm_backward(d, xx, weight, mean, rstd, dx=d), want)
        else:
            assert torch.equal(B.co3_layernorm_backward(d, xx, weight, mean, rstd, dx=xx), want)
    xx = x.clone()
    assert torch.equal(B.co3_layernorm(xx, weight, bias, y=xx)[0], B.co3_layernorm(x, weight, bias)[0])


@pytest.mark.parametrize("name", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows", [9, 70])
@pytest.mark.parametrize("cols", [700, 12000, 20000])
def test_gradients_where_dx_takes_the_place_of_dy_or_x(cols, rows, name):
    import torch
    from paper_2204_08211_amd import binding as B
    x = torch.randn(2, rows, cols, device="cuda:0").to(dtype_of(name))
    dy = torch.randn(2, rows, cols, device="cuda:0").to(dtype_of(name))
    _, mean, rstd = B.co3_layernorm(x)
    want = [torch.empty(2, cols, device="cuda:0") for _ in range(2)]
    dx = B.co3_layernorm_backward(dy, x, None, mean, rstd, dweight=want[0], dbias=want[1])
    _, edw, edb = plain_backward(dy, x, None, mean, rstd)
    assert float((want[0].double() - edw).abs().max()) <= 2.0 ** -18 * rows and float((want[1].double() - edb).abs().max()) <= 2.0 ** -18 * rows
    for place in ("dy", "x"):
        t = dict(dy=dy.clone(), x=x.clone())
        got = [torch.empty(2, cols, device="cuda:0") for _ in range(2)]
        B.co3_layernorm_backward(t["dy"], t["x"], None, mean, rstd, dx=t[place], dweight=got[0], dbias=got[1])
        assert torch.equal(t[place], dx) and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_rows_far_from_zero_constant_and_not_finite():
    import torch
    from paper_2204_08211_amd import binding as B
    dev = "cuda:0"
    x = torch.randn(6, 777, device=dev)
    x[0] = 3.0                                     # no variance: rstd = eps^-1/2, y = bias
    x[1] += 4096.0                                 # a mean far larger than the spread
    x[2] *= 1e-18
    x[3, 5] = float("nan")
    x[4, 7] = float("inf")
    bias = torch.randn(777, device=dev)
    y, mean, rstd = B.co3_layernorm(x, None, bias)
    ey, _, erstd = plain_forward(x, None, bias, 1e-5)
    assert float((y[0] - bias).abs().max()) == 0.0
    assert float((rstd[[0, 2]].double() - 1e-5 ** -0.5).abs().max()) <= 1e-3
    assert rel(y[1], ey[1]) <= 4096 * 2.0 ** -22   # the mean is rounded to 2^-12 of the spread
    assert rel(y[5], ey[5]) <= TOL["float32"]
    assert bool(torch.isnan(y[3]).all()) and bool(torch.isnan(y[4]).all()) and bool(torch.isfinite(y[[0, 1, 2, 5]]).all())
    dy = torch.randn_like(x)
    dx = B.co3_layernorm_backward(dy, x, None, mean, rstd)
    assert bool(torch.isnan(dx[3]).all()) and bool(torch.isfinite(dx[[0, 1, 2, 5]]).all())


@pytest.mark.parametrize("cols", [17, 640])
def test_gradients_against_differences(cols):
    import torch
    from paper_2204_08211_amd import binding as B
    dev = "cuda:0"
    gen = torch.Generator(device=dev)
    gen.manual_seed(cols)
    draw = lambda *s: torch.randn(*s, generator=gen, device=dev)  # noqa: E731
    x, dy, weight, bias = draw(4, 9, cols), draw(4, 9, cols), 1 + 0.3 * draw(cols), draw(cols)
    vx, vw, vb = draw(4, 9, cols), draw(cols), draw(cols)
    _, mean, rstd = B.co3_layernorm(x, weight, bias)
    dw, db = torch.zeros(4, cols, device=dev), torch.zeros(4, cols, device=dev)
    dx = B.co3_layernorm_backward(dy, x, weight, mean, rstd, dweight=dw, dbias=db)
    loss = lambda a, b, c: float((B.co3_layernorm(a, b, c)[0].double() * dy.double()).sum())  # noqa: E731
    h = 2.0 ** -7
    for along, slope in ((lambda s: (x + s * vx, weight, bias), (dx.double() * vx.double()).sum()),
                         (lambda s: (x, weight + s * vw, bias), (dw.double().sum(0) * vw.double()).sum()),
                         (lambda s: (x, weight, bias + s * vb), (db.double().sum(0) * vb.double()).sum())):
        difference = (loss(*along(h)) - loss(*along(-h))) / (2 * h)
        # third derivatives leave h^2 of a sum of 4 9 cols terms of about 1, roundings 2^-24 / h of each
        terms = (36 * cols) ** 0.5
        assert abs(difference - float(slope)) <= (4 * h * h + 2.0 ** -22 / h) * 4 * terms


def test_no_rows_and_no_users_rows():
    import torch
    from paper_2204_08211_amd import binding as B
    x = torch.zeros(0, 16, device="cuda:0")
    y, mean, rstd = B.co3_layernorm(x)
    assert y.shape == (0, 16) and mean.shape == (0,)
    e = torch.zeros(3, 0, 16, device="cuda:0")
    m = torch.zeros(3, 0, device="cuda:0")
    dw, db = torch.ones(3, 16, device="cuda:0"), torch.ones(3, 16, device="cuda:0")
    B.co3_layernorm_backward(e, e, None, m, m, dweight=dw, dbias=db, accumulate=True)
    assert bool((dw == 1).all()) and bool((db == 1).all())
    B.co3_layernorm_backward(e, e, None, m, m, dweight=dw, dbias=db)
    assert bool((dw == 0).all()) and bool((db == 0).all())


def test_many_short_rows_past_32_bits_of_bytes():
    import torch
    from paper_2204_08211_amd import binding as B
    rows, cols, stride = 70001, 24, 40000                                  # 5.6e9 bytes from the first row to the last
    whole = torch.zeros(rows * stride, dtype=torch.bfloat16, device="cuda:0")
    x = whole.view(rows, stride)[:, :cols]
    x.copy_(torch.randn(rows, cols, device="cuda:0"))
    y, mean, rstd = B.co3_layernorm(x)
    ey, _, _ = plain_forward(x, None, None, 1e-5)
    assert rel(y, ey) <= TOL["bfloat16"]
    dy = torch.randn(rows, cols, device="cuda:0").bfloat16()
    dx = B.co3_layernorm_backward(dy, x, None, mean, rstd, dx=torch.empty_like(dy))
    assert rel(dx, plain_backward(dy, x, None, mean, rstd)[0]) <= TOL["bfloat16"]


def test_another_stream_and_a_replayed_graph():
    import torch
    from paper_2204_08211_amd import binding as B
    dev = "cuda:0"
    x, dy = torch.randn(2, 900, 300, device=dev).half(), torch.randn(2, 900, 300, device=dev).half()
    w, b = torch.randn(300, device=dev), torch.randn(300, device=dev)
    y, mean, rstd = torch.empty_like(x), torch.empty(2, 900, device=dev), torch.empty(2, 900, device=dev)
    dx, grad = torch.empty_like(x), torch.zeros(2, 600, device=dev)
    ws = torch.empty(B.co3_layernorm_backward_workspace_bytes(2, 900, 300), dtype=torch.uint8, device=dev)

    def step():
        B.co3_layernorm(x, w, b, y=y, mean=mean, rstd=rstd)
        B.co3_layernorm_backward(dy, x, w, mean, rstd, dx=dx, dweight=grad[:, :300], dbias=grad[:, 300:], workspace=ws)

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    for it in range(4):
        x.copy_(torch.randn(2, 900, 300, device=dev) * (it + 1))
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (y, mean, rstd, dx, grad)]
        for t in (y, mean, rstd, dx, grad):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for t, e in zip((y, mean, rstd, dx, grad), want):
            assert torch.equal(t, e)


def test_stream_argument_and_refused_devices():
    import torch
    from paper_2204_08211_amd import binding as B
    dev = "cuda:0"
    x, dy = torch.randn(2, 700, 300, device=dev), torch.randn(2, 700, 300, device=dev)
    w, grad, want_grad = torch.randn(300, device=dev), torch.zeros(2, 600, device=dev), torch.zeros(2, 600, device=dev)
    want = B.co3_layernorm(x, w)
    want_dx = B.co3_layernorm_backward(dy, x, w, *want[1:], dweight=want_grad[:, :300], dbias=want_grad[:, 300:])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = B.co3_layernorm(x, w, stream=side)
    dx = B.co3_layernorm_backward(dy, x, w, *got[1:], dweight=grad[:, :300], dbias=grad[:, 300:], stream=side)
    for _ in range(8):   # memory that a call let go of is not the current stream's to write
        torch.full((B.co3_layernorm_backward_workspace_bytes(2, 700, 300),), 255, dtype=torch.uint8, device=dev)
    torch.cuda.synchronize()
    for t, e in zip((*got, dx, grad), (*want, want_dx, want_grad)):
        assert torch.equal(t, e)
    for bad in (dict(x=x.cpu()), dict(weight=w.cpu()), dict(y=torch.empty(2, 700, 300)), dict(mean=torch.empty(2, 700)), dict(x=x.cpu(), weight=w.cpu())):
        with pytest.raises(ValueError):
            B.co3_layernorm(**{"x": x, "weight": w, **bad})
    for bad in (dict(dy=dy.cpu()), dict(mean=want[1].cpu()), dict(dx=torch.empty(2, 700, 300)), dict(dweight=torch.empty(2, 300)),
                dict(workspace=torch.empty(1 << 20, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            B.co3_layernorm_backward(**{"dy": dy, "x": x, "weight": w, "mean": want[1], "rstd": want[2], **bad})
