"""Group norms, tensors in 8 bits and their products together, as a user's training step calls them (pytest -m gpu): every intermediate
tensor against 64 bits from the ones it was made of, with no synchronisation in between, also replayed from a graph; the example's network against
automatic differentiation, and a few iterations of its training, which have to repeat themselves.

Tolerances: of a single call, those of its own tests.  The network's gradients come through products whose operands are rounded to three bits
behind the leading one: at most 2^-4 of a value, 2^-4 / sqrt(3) of it on average over even steps, in either operand, and independently in
every term, so that a product is off by sqrt(2 / 3) 2^-4 = 5.1e-2 of its norm; the norms pass errors on with about their size.  A weight's gradient
behind b blocks is made by b + 1 products forward and b + 1 back, and itself: at b = 2 at most seven errors of 5.1e-2, 0.14 together; 0.2 is
allowed."""
import pytest
import torch

import blocks8_util as bu

pytestmark = pytest.mark.gpu


def numbers(x):
    return bu.numbers(x.values, x.scales, x.cols, x.block_rows)


def rel(x, y):
    return float((x.double() - y).norm() / y.norm())


def silu_slope(z):
    s = torch.sigmoid(z)
    return s * (1 + z * (1 - s))


class Step:
    """A layer's training step on its own buffers: y = silu(group norm(x)) W^T and back."""

    def __init__(self, users, samples, pixels, channels, outs, groups, dtype, seed):
        from paper_2204_08211_amd import binding as B
        self.dims, self.gen = (users, samples, pixels, channels, outs, groups), torch.Generator(device="cuda:0")
        self.gen.manual_seed(seed)
        r = lambda *shape: torch.randn(*shape, generator=self.gen, device="cuda:0")  # noqa: E731
        rows = samples * pixels
        self.x, self.dy = r(users * samples, pixels, channels).to(dtype), (1e-3 * r(users, rows, outs)).to(dtype)
        self.weight, self.bias, self.w = 1 + 0.3 * r(channels), r(channels), r(1, outs, channels).to(dtype)
        self.n, self.y, self.dn, self.dx = torch.zeros_like(self.x), torch.zeros_like(self.dy), torch.zeros(users, rows, channels, dtype=dtype, device="cuda:0"), torch.zeros_like(self.x)
        self.mean, self.rstd = torch.zeros(users * samples, groups, device="cuda:0"), torch.zeros(users * samples, groups, device="cuda:0")
        e = lambda *shape: B.Blocks8.empty(*shape, device="cuda:0")  # noqa: E731
        self.x8, self.n8, self.w8, self.dy8 = e(users, rows, channels), e(users, rows, channels), e(1, outs, channels), e(users, rows, outs)
        self.g = torch.zeros(users, 3 + 2 * channels + outs * channels, device="cuda:0")
        need = [B.co3_matmul8_workspace_bytes(self.n8, self.w8, transpose_b=True), B.co3_matmul8_workspace_bytes(self.dy8, self.w8),
                B.co3_matmul8_workspace_bytes(self.dy8, self.n8, transpose_a=True), B.co3_groupnorm_workspace_bytes(users * samples, pixels, channels, groups, dtype),
                B.co3_groupnorm_backward_workspace_bytes(users, users * samples, pixels, channels, groups, dtype)]
        self.ws = torch.empty(max(need), dtype=torch.uint8, device="cuda:0")   # one after the other: one for all

    def parts(self):
        _, _, _, channels, outs, _ = self.dims
        g = self.g
        return g[:, 3:3 + channels], g[:, 3 + channels:3 + 2 * channels], g[:, 3 + 2 * channels:].unflatten(1, (outs, channels))

    def run(self, stream=None):
        from paper_2204_08211_amd import binding as B
        users, samples, pixels, channels, outs, groups = self.dims
        k = dict(stream=stream)
        dweight, dbias, dw = self.parts()
        B.co3_quantize8(self.x.view(users, -1, channels), out=self.x8, **k)
        B.co3_groupnorm(self.x, groups, self.weight, self.bias, activation=B.ACT_SILU, y=self.n, mean=self.mean, rstd=self.rstd, workspace=self.ws, **k)
        B.co3_quantize8(self.n.view(users, -1, channels), out=self.n8, **k)
        B.co3_quantize8(self.w, out=self.w8, **k)
        B.co3_matmul8(self.n8, self.w8, out=self.y, transpose_b=True, workspace=self.ws, **k)
        B.co3_quantize8(self.dy, out=self.dy8, **k)
        B.co3_matmul8(self.dy8, self.w8, out=self.dn, workspace=self.ws, **k)
        B.co3_matmul8(self.dy8, self.n8, out=dw, transpose_a=True, workspace=self.ws, **k)
        B.co3_groupnorm_backward(self.dn.view(self.x.shape), self.x8, groups, self.weight, self.bias, self.mean, self.rstd, activation=B.ACT_SILU, users=users, dx=self.dx,
                                 dweight=dweight, dbias=dbias, workspace=self.ws, **k)

    def outputs(self):
        return [self.x8.values, self.n, self.mean, self.rstd, self.n8.values, self.w8.values, self.y, self.dy8.values, self.dn, self.dx, self.g]

    def check(self):
        users, samples, pixels, channels, outs, groups = self.dims
        half = torch.finfo(self.x.dtype).eps / 2
        exact = self.x.dtype is torch.float32
        for t, kept in ((self.x, self.x8), (self.n, self.n8), (self.w, self.w8), (self.dy, self.dy8)):
            values, _ = bu.stored(t.double().view(kept.shape), 128)
            assert (kept.values.cpu().numpy() == values).all()
        per = channels // groups
        wide = lambda v: v.double().repeat_interleave(per, dim=1)[:, None, :]  # noqa: E731
        z = (self.x.double() - wide(self.mean)) * wide(self.rstd) * self.weight.double() + self.bias.double()
        assert rel(self.n, z * torch.sigmoid(z)) <= (2.0 ** -19 if exact else half)
        n8, w8, dy8, x8 = (numbers(t) for t in (self.n8, self.w8, self.dy8, self.x8))
        product = 1e-6 if exact else 2e-4 + half
        assert rel(self.y, torch.stack([torch.mm(a, w8[0].t()) for a in n8])) <= product
        assert rel(self.dn, torch.stack([torch.mm(a, w8[0]) for a in dy8])) <= product
        dweight, dbias, dw = self.parts()
        assert rel(dw, torch.stack([torch.mm(a.t(), b) for a, b in zip(dy8, n8)])) <= 1e-6
        xh = (x8.view(self.x.shape) - wide(self.mean)) * wide(self.rstd)
        d = self.dn.double().view(self.x.shape)
        dz = d * silu_slope(xh * self.weight.double() + self.bias.double())
        over = lambda v: v.view(-1, pixels, groups, per).mean(dim=(1, 3))  # noqa: E731
        t = dz * self.weight.double()
        assert rel(self.dx, wide(self.rstd) * (t - wide(over(t)) - xh * wide(over(t * xh)))) <= (2.0 ** -19 if exact else half)
        of = lambda v: v.view(users, -1, channels).sum(dim=1)  # noqa: E731
        assert bool(((dweight.double() - of(dz * xh)).abs() <= 2.0 ** -19 * of((d * xh).abs())).all())
        assert bool(((dbias.double() - of(dz)).abs() <= 2.0 ** -19 * of(d.abs())).all())
        assert bool((self.g[:, :3] == 0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dims", [(3, 2, 49, 40, 24, 5), (2, 3, 1030, 64, 200, 8), (1, 1, 1, 8, 3, 2)])
def test_a_layers_step(dims, dtype):
    step = Step(*dims, dtype, 3)
    if dims[0] == 1:        # one pixel: no means to speak of, but a step all the same
        step.run()
        assert bool(step.dx.isfinite().all())
        return
    step.run()
    step.check()


def test_a_layers_step_on_another_stream_and_replayed():
    dims, dtype = (2, 2, 1030, 40, 24, 5), torch.bfloat16
    step = Step(*dims, dtype, 4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step.run(side)
    side.synchronize()
    step.check()
    first = [o.clone() for o in step.outputs()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.run()
    x, dy = step.x.clone(), step.dy.clone()
    for scale in (0.5, 3.0, 1.0):
        step.x.copy_(x * scale)
        step.dy.copy_(dy * scale)
        for o in step.outputs():
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        step.check()
        got = [o.clone() for o in step.outputs()]
        step.run()
        assert all(torch.equal(p, q) for p, q in zip(got, step.outputs()))
    assert all(torch.equal(p, q) for p, q in zip(first, step.outputs()))


def test_the_networks_gradients():
    from paper_2204_08211_amd.examples.local_training import ImageNetwork
    users, samples, pixels, width = 3, 4, 36, 48
    net = ImageNetwork(width, 2, 12, pixels, groups=6)
    w = net.start(3, "cuda:0")
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(5)
    w += 0.1 * torch.randn(net.d, generator=gen, device="cuda:0")
    x = torch.randn(users, samples * pixels, width, generator=gen, device="cuda:0")
    dy = torch.randn(users, samples * pixels, 12, generator=gen, device="cuda:0")
    g = torch.zeros(users, net.d + 5, device="cuda:0")
    out, kept = net.forward(w, x)
    net.backward(w, dy, kept, g)
    for u in range(users):
        p = w.double().cpu().requires_grad_()
        part = lambda name: net.part(p, name)  # noqa: E731
        h = x[u].double().cpu().view(samples, pixels, width)

        def norm(h, k):
            v = h.view(samples, pixels, 6, width // 6)
            v = (v - v.mean(dim=(1, 3), keepdim=True)) / (v.var(dim=(1, 3), unbiased=False, keepdim=True) + 1e-5).sqrt()
            v = v.view(h.shape) * part(f"weight{k}") + part(f"bias{k}")
            return v * torch.sigmoid(v)
        for k in range(2):
            h = h + norm(h, k) @ part(f"mix{k}").t()
        want = norm(h, "_out") @ part("out").t()
        assert rel(out[u].cpu(), want.detach().view(-1, 12)) <= 0.2
        (want.view(-1, 12) * dy[u].double().cpu()).sum().backward()
        for name, (o, shape) in net.at.items():
            n = torch.Size(shape).numel()
            assert rel(g[u, o:o + n].cpu(), p.grad[o:o + n]) <= 0.2, name
    assert bool((g[:, net.d:] == 0).all())


def test_training_on_images_repeats_itself():
    from paper_2204_08211_amd.examples.local_training import ImageNetwork, train
    net = ImageNetwork(64, 2, 16, 64)
    errors, bits = train(net, users=3, rows=256, iters=6)
    again, _ = train(net, users=3, rows=256, iters=6)
    assert all(e == e and e < 1e3 for e in errors) and 1.0 < bits < 9.0
    assert errors[:1] == again[:1] and all(abs(a - b) <= 1e-3 * a for a, b in zip(errors, again))


@pytest.mark.parametrize("images", [True, False])
def test_training_gives_the_same_bits(images):
    """All sums are formed in a fixed order, the codec's and the update's too: another run has the same errors and sends as many bits."""
    from paper_2204_08211_amd.examples.local_training import ImageNetwork, Network, train
    net = ImageNetwork(64, 2, 16, 64) if images else Network(64, 128, 2, 16)
    assert train(net, users=3, rows=256, iters=6) == train(net, users=3, rows=256, iters=6)


def test_the_networks_gradients_have_the_same_bits():
    from paper_2204_08211_amd.examples.local_training import ImageNetwork
    net = ImageNetwork(64, 2, 16, 64)
    w = net.start(3, "cuda:0")
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(9)
    x, dy = (torch.randn(3, 1024, n, generator=gen, device="cuda:0") for n in (64, 16))
    first = None
    for _ in range(8):
        g = torch.zeros(3, net.d, device="cuda:0")
        out, kept = net.forward(w, x)
        net.backward(w, dy, kept, g)
        first = (out, g) if first is None else first
        assert torch.equal(out, first[0]) and torch.equal(g, first[1])
