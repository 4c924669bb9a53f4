"""Orthogonalised matrices and Muon's update against the iteration in 64 bits (pytest -m gpu): types, shapes around every form's
limits, matrices side by side and at odd offsets, sums in slices, spectra with one dominant direction, zeros and values that are
not finite, in place, other streams, a replayed graph.

Tolerances, of the difference's 2-norm over the result's.  Pairs of fp16 hold 22 bits: every step rounds X, A and B by 2^-23 of
themselves at most, and B X, up to 2.8 X, takes each of them up; six steps of some 8 such roundings stay below 2^-17.  High parts alone
are rounded by 2^-12: A, X and B together up to 2.8 sqrt(3) 2^-12 a step where singular values are near one, three steps long, 2^-9 in all,
before the result is rounded to bfloat16 (2^-9 in the mean).  One dominant direction takes the rounding of the
pairs, spread over all others, up by a^steps = 485: 485 2^-23 = 2^-14."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

PAIR, HIGH = 2.0 ** -17, 2.0 ** -8
DOMINANT = 2.0 ** -13


def steps_of(g, steps=5, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7):
    x = g.double()
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    x = x / (x.norm() + eps)
    for k in range(steps):
        a, b, c = coefficients if not isinstance(coefficients[0], tuple) else coefficients[k]
        gram = x @ x.t()
        x = a * x + (b * gram + c * gram @ gram) @ x
    return x.t() if tall else x


def rel(x, y):
    return float((x.double() - y).norm() / y.norm())


def tolerance(dtype):
    import torch
    return HIGH if dtype == torch.bfloat16 else 2.0 ** -11 if dtype == torch.float16 else PAIR


def lay_out(shapes, gap=3):
    """Matrices one behind the other, `gap` elements before each."""
    out, at = [], 0
    for rows, cols in shapes:
        out.append((at + gap, rows, cols))
        at += gap + rows * cols
    return out, at + gap


def check(shapes, dtype, make, tol, **kw):
    import torch
    from paper_2204_08211_amd import binding as B
    matrices, n = lay_out(shapes)
    g = torch.full((n,), 9.0, device="cuda:0").to(dtype)
    for k, (at, rows, cols) in enumerate(matrices):
        g[at:at + rows * cols] = make(k, rows, cols).reshape(-1).to(dtype)
    scales = [1.0 + 0.5 * k for k in range(len(matrices))]
    plan = B.MatrixPlan(matrices, dtype=dtype, scales=scales)
    out = torch.full_like(g, 4.0)
    status = torch.zeros(B.STATUS_WORDS, dtype=torch.int64, device="cuda:0")
    B.co3_orthogonalize(plan, g, out, status=status, **kw)
    again = torch.full_like(g, 4.0)
    B.co3_orthogonalize(plan, g, again, **kw)
    assert torch.equal(out, again)                        # the same order every time
    mask = torch.ones(n, dtype=torch.bool, device="cuda:0")
    for (at, rows, cols), scale in zip(matrices, scales):
        mask[at:at + rows * cols] = False
        err = rel(out[at:at + rows * cols].view(rows, cols), scale * steps_of(g[at:at + rows * cols].view(rows, cols), **kw))
        assert err <= tol, (rows, cols, err)
    assert bool((out[mask] == 4.0).all())                 # the elements between them are left alone
    assert int(status.sum()) == 0


def noise(k, rows, cols):
    import torch
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(100 * k + rows + cols)
    return torch.randn(rows, cols, generator=gen, device="cuda:0") * 10.0 ** (k % 7 - 5)


def falling(k, rows, cols):
    import torch
    r = min(8, rows, cols)
    left = noise(k, rows, r) * torch.arange(1, r + 1, device="cuda:0") ** -1.0
    return left @ noise(k + 1, r, cols) / r + 0.5 * noise(k, rows, cols)


SHAPES = {
    "one launch": [(1, 1), (1, 5), (7, 1), (2, 3), (16, 16), (31, 33), (32, 32), (64, 64), (64, 128), (128, 64), (63, 127), (128, 1), (33, 100)],
    "past one launch": [(65, 65), (64, 129), (129, 1), (1, 129), (2, 700)],
    "around tiles": [(63, 300), (128, 128), (129, 257), (255, 256), (300, 70), (512, 513)],
    "long sums": [(3, 9000), (33, 4097), (64, 8192), (5000, 17), (100, 6000)],
    "large": [(1000, 2048), (2100, 900)],
}


@pytest.mark.parametrize("name", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("what", sorted(SHAPES))
def test_shapes(what, name):
    import torch
    dtype = getattr(torch, name)
    check(SHAPES[what], dtype, noise, tolerance(dtype))
    check(SHAPES[what], dtype, falling, tolerance(dtype))


@pytest.mark.parametrize("name,rows,cols", [("bfloat16", 4096, 4096), ("float32", 2304, 4100), ("float32", 4096, 1500)])
def test_largest_tiles(name, rows, cols):
    import torch
    dtype = getattr(torch, name)
    check([(rows, cols)], dtype, falling, tolerance(dtype))


@pytest.mark.parametrize("shape", [(48, 96), (200, 700), (1024, 1024)])
@pytest.mark.parametrize("name", ["float32", "bfloat16"])
def test_one_dominant_direction(shape, name):
    import torch

    def make(k, rows, cols):
        return noise(0, rows, 1) @ noise(1, 1, cols) + 1e-3 * noise(0, rows, 1).abs().mean() * noise(1, rows, cols) / 10

    check([shape], getattr(torch, name), make, max(DOMINANT, tolerance(getattr(torch, name))) if name == "bfloat16" else DOMINANT)


@pytest.mark.parametrize("shapes", [[(40, 60)], [(150, 260), (40, 60)]])
def test_coefficients_of_their_own_for_every_step(shapes):
    import torch
    cubic, quintic = (1.5, -0.5, 0.0), (3.4445, -4.7750, 2.0315)
    for kw in (dict(steps=1), dict(steps=6), dict(steps=12, coefficients=cubic), dict(steps=3, coefficients=(quintic, quintic, cubic))):
        check(shapes, torch.float32, noise, PAIR * (2 if kw["steps"] > 6 else 1), **kw)


def test_eps_bounds_small_matrices():
    import torch
    from paper_2204_08211_amd import binding as B
    for shape in ((30, 40), (90, 200)):
        g = (torch.randn(shape, device="cuda:0") * 1e-6).reshape(-1)
        plan = B.MatrixPlan([(0,) + shape])
        out = B.co3_orthogonalize(plan, g, eps=1e-3)
        assert rel(out.view(shape), steps_of(g.view(shape), eps=1e-3)) <= PAIR * 4     # far from the working range of the pairs
        for size in (1e-30, 1e30, 1e-42):
            out = B.co3_orthogonalize(plan, g * 1e6 * size, eps=0.0)
            assert rel(out.view(shape), steps_of((g * 1e6 * size).view(shape), eps=0.0)) <= PAIR


@pytest.mark.parametrize("name", ["float32", "bfloat16"])
@pytest.mark.parametrize("bad", [(60, 30), (70, 200)])
def test_zeros_and_values_that_are_not_finite(bad, name):
    import torch
    from paper_2204_08211_amd import binding as B
    dtype = getattr(torch, name)
    shapes = [bad, bad, bad, (64, 100)]
    matrices, n = lay_out(shapes, gap=0)
    g = torch.randn(n, device="cuda:0").to(dtype)
    size = bad[0] * bad[1]
    g[:size] = 0
    g[size + 5] = float("nan")
    g[2 * size + 7] = float("-inf")
    plan = B.MatrixPlan(matrices, dtype=dtype)
    status = torch.zeros(B.STATUS_WORDS, dtype=torch.int64, device="cuda:0")
    for eps in (1e-7, 0.0):
        out = B.co3_orthogonalize(plan, g, eps=eps, status=status)
        assert bool((out[:size] == 0).all()) and bool(torch.isnan(out[size:3 * size]).all())
        at, rows, cols = matrices[3]
        assert rel(out[at:].view(rows, cols), steps_of(g[at:].view(rows, cols), eps=eps)) <= tolerance(dtype)
    assert status.tolist() == [4, 0, 0, 0, 0, 0, 0, 0]


@pytest.mark.parametrize("sizes", [(20, 30, 100), (70, 90, 300)])
def test_matrices_side_by_side_and_in_place(sizes):
    import torch
    from paper_2204_08211_amd import binding as B
    rows, cols, ld = sizes
    g = torch.randn(rows * ld, device="cuda:0")
    matrices = [(0, rows, cols, ld), (cols, rows, cols, ld), (2 * cols + 1, rows, 7, ld)]
    plan = B.MatrixPlan(matrices)
    want = g.view(rows, ld).clone().double()
    for at, _, c, _ in matrices:
        want[:, at:at + c] = steps_of(g.view(rows, ld)[:, at:at + c])
    out = B.co3_orthogonalize(plan, g, g.clone())
    assert rel(out.view(rows, ld), want) <= PAIR
    assert bool((out.view(rows, ld)[:, 2 * cols] == g.view(rows, ld)[:, 2 * cols]).all())
    assert bool((out.view(rows, ld)[:, 2 * cols + 8:] == g.view(rows, ld)[:, 2 * cols + 8:]).all())
    inplace = g.clone()
    B.co3_orthogonalize(plan, inplace, inplace)
    assert torch.equal(inplace, out)


@pytest.mark.parametrize("shapes", [[(64, 100), (10, 64), (1, 30)], [(256, 300), (1000, 70), (10, 64)], [(1024, 2048), (513, 512)]])
@pytest.mark.parametrize("nesterov", [True, False])
def test_update(shapes, nesterov):
    import torch
    from paper_2204_08211_amd import binding as B
    matrices, n = lay_out(shapes, gap=5)
    dev = "cuda:0"
    g, m, w = (torch.randn(n, device=dev) * s for s in (1e-3, 3e-3, 1.0))
    scales = [max(1.0, r / c) ** 0.5 for _, r, c in matrices]
    plan = B.MatrixPlan(matrices, scales=scales)
    ms, ws = [m.clone()], [w.clone()]
    em, ew = m.double(), w.double()
    for _ in range(3):
        B.co3_muon_update(plan, g, m, w, eta=0.05, beta=0.9, nesterov=nesterov, weight_decay=0.1)
        ms.append(m.clone())
        for (at, rows, cols), scale in zip(matrices, scales):
            s = slice(at, at + rows * cols)
            em[s] = 0.9 * em[s] + g[s].double()
            u = g[s].double() + 0.9 * em[s] if nesterov else em[s]
            ew[s] = ew[s] * (1 - 0.05 * 0.1) - 0.05 * scale * steps_of(u.view(rows, cols)).reshape(-1)
    assert rel(m, em) <= 2.0 ** -22 and rel(w, ew) <= 2.0 ** -21      # three steps of a few fp32 roundings each
    outside = torch.ones(n, dtype=torch.bool, device=dev)
    for at, rows, cols in matrices:
        outside[at:at + rows * cols] = False
    assert torch.equal(m[outside], ms[0][outside]) and torch.equal(w[outside], ws[0][outside])


def test_update_counts_and_spreads_what_is_not_finite():
    import torch
    from paper_2204_08211_amd import binding as B
    for shape in ((30, 40), (80, 130)):
        n = shape[0] * shape[1]
        g, m, w = torch.randn(2 * n, device="cuda:0"), torch.zeros(2 * n, device="cuda:0"), torch.ones(2 * n, device="cuda:0")
        g[3] = float("inf")
        plan = B.MatrixPlan([(0,) + shape, (n,) + shape])
        status = torch.zeros(B.STATUS_WORDS, dtype=torch.int64, device="cuda:0")
        B.co3_muon_update(plan, g, m, w, eta=0.1, status=status)
        assert int(status[B.STAT_NONFINITE]) == 1
        assert bool(torch.isnan(w[:n]).all()) and bool(torch.isfinite(w[n:]).all())
        assert int((~torch.isfinite(m)).sum()) == 1


def test_high_products_on_request():
    import torch
    from paper_2204_08211_amd import binding as B
    for shape in ((64, 64), (300, 500)):
        g = torch.randn(shape, device="cuda:0").reshape(-1)
        out = B.co3_orthogonalize(B.MatrixPlan([(0,) + shape], products=B.PRODUCTS_HIGH), g)
        assert rel(out.view(shape), steps_of(g.view(shape))) <= 2.0 ** -9
        b = g.bfloat16()
        out = B.co3_orthogonalize(B.MatrixPlan([(0,) + shape], dtype=torch.bfloat16, products=B.PRODUCTS_PAIR), b)
        assert rel(out.view(shape), steps_of(b.view(shape))) <= 2.0 ** -9


def test_refusals():
    import ctypes as C
    import torch
    from paper_2204_08211_amd import binding as B
    L = B.lib()
    g = torch.zeros(4096, device="cuda:0")
    plan, half = B.MatrixPlan([(0, 48, 64)]), B.MatrixPlan([(0, 48, 64)], dtype=torch.bfloat16)
    ws = torch.zeros(max(plan.workspace_bytes, half.workspace_bytes) + 256, dtype=torch.uint8, device="cuda:0")
    coef = np.tile(np.float32([3.4445, -4.775, 2.0315]), (32, 1))

    def ortho(p=plan, **change):
        f = dict(g=g.data_ptr(), out=g.data_ptr(), coefficients=coef.ctypes.data, steps=5, eps=1e-7, status=None, workspace=ws.data_ptr(),
                 workspace_bytes=p.workspace_bytes)
        f.update(change)
        return L.co3_orthogonalize(p.handle, C.byref(B.OrthogonalizeArgs(**f)), None)

    assert ortho() == B.OK
    torch.cuda.synchronize()
    for change in (dict(g=None), dict(out=None), dict(coefficients=None), dict(steps=0), dict(steps=33), dict(eps=-1.0), dict(eps=float("nan")),
                   dict(workspace=None), dict(workspace=ws.data_ptr() + 8), dict(g=g.data_ptr() + 2), dict(out=g.data_ptr() + 1),
                   dict(status=ws.data_ptr() + 4)):
        assert ortho(**change) == B.ERR_ARG, change
    assert ortho(workspace_bytes=plan.workspace_bytes - 1) == B.ERR_CAPACITY
    for bad in ((3.0, 0.0, 0.0), (1.5, -0.5, 5.0), (float("nan"), 0.0, 0.0), (3.4445, -4.775, float("inf")), (0.5, 8.0, -8.0), (2.0, 0.0, 0.01)):
        c = np.tile(np.float32(bad), (32, 1))
        assert ortho(coefficients=c.ctypes.data) == B.ERR_ARG, bad
    for good in ((1.5, -0.5, 0.0), (2.0, -1.5, 0.5), (1.0, 0.0, 0.0), (0.0, 0.0, 0.0), (2.0, -1.0, 0.0)):
        c = np.tile(np.float32(good), (32, 1))
        assert ortho(coefficients=c.ctypes.data, steps=32) == B.OK, good

    def muon(p=plan, **change):
        f = dict(g=g.data_ptr(), momentum=g.data_ptr() + 4, model=g.data_ptr() + 8, coefficients=coef.ctypes.data, steps=5, eps=1e-7, eta=0.1,
                 beta=0.9, weight_decay=0.0, nesterov=1, status=None, workspace=ws.data_ptr(), workspace_bytes=p.workspace_bytes)
        f.update(change)
        return L.co3_muon_update(p.handle, C.byref(B.MuonArgs(**f)), None)

    for change in (dict(g=None), dict(momentum=None), dict(model=None), dict(momentum=g.data_ptr()), dict(model=g.data_ptr()),
                   dict(model=g.data_ptr() + 4), dict(model=g.data_ptr() + 2), dict(eta=float("nan")), dict(beta=float("inf")),
                   dict(weight_decay=float("nan")), dict(steps=0), dict(p=half)):
        assert muon(**change) == B.ERR_ARG, change
    with pytest.raises(ValueError):
        B.co3_orthogonalize(plan, g.half())
    with pytest.raises(ValueError):
        B.co3_orthogonalize(plan, g[:100])
    with pytest.raises(ValueError):
        B.co3_orthogonalize(plan, g[::2])
    torch.cuda.synchronize()


@pytest.mark.parametrize("shapes", [[(50, 100), (64, 64)], [(33, 4097), (300, 700)]])
def test_another_stream_and_a_replayed_graph(shapes):
    import torch
    from paper_2204_08211_amd import binding as B
    matrices, n = lay_out(shapes)
    dev = "cuda:0"
    plan = B.MatrixPlan(matrices)
    ws = torch.empty(plan.workspace_bytes, dtype=torch.uint8, device=dev)
    g, m, w = torch.randn(n, device=dev), torch.zeros(n, device=dev), torch.ones(n, device=dev)

    def step(m, w):
        B.co3_muon_update(plan, g, m, w, eta=0.1, workspace=ws)

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(m.clone(), w.clone())
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            step(m, w)
    torch.cuda.synchronize()
    for it in range(4):
        g.copy_(torch.randn(n, device=dev) * (it + 1))
        em, ew = m.clone(), w.clone()
        step(em, ew)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(m, em) and torch.equal(w, ew)


def test_stream_argument_and_refused_devices():
    import torch
    from paper_2204_08211_amd import binding as B
    dev = "cuda:0"
    plan = B.MatrixPlan([(3, 50, 100), (6000, 200, 70)])
    g = torch.randn(21000, device=dev)
    want = B.co3_orthogonalize(plan, g)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(50_000_000)   # the current stream is some milliseconds behind: what is made for the call is made on its stream
    out = B.co3_orthogonalize(plan, g, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    with pytest.raises(ValueError):
        B.co3_orthogonalize(plan, g.cpu())
    with pytest.raises(ValueError):
        B.co3_orthogonalize(plan, g, out=torch.empty(21000))
    with pytest.raises(ValueError):
        B.co3_orthogonalize(plan, g, workspace=torch.empty(plan.workspace_bytes, dtype=torch.uint8))
    for status in (torch.zeros(8, dtype=torch.int64), torch.zeros(7, dtype=torch.int64, device=dev), torch.zeros(8, dtype=torch.int32, device=dev)):
        with pytest.raises(ValueError):
            B.co3_orthogonalize(plan, g, status=status)
    with pytest.raises(ValueError):
        B.co3_muon_update(plan, g, g.cpu(), g.clone(), eta=0.1)


# Matrices of up to 64 rows or columns, 128 of the others at a time: one, two and many such strips, the last one of a single column,
# sums of 32 x 32 and 64 x 64, and just beyond what is taken that way (64 x 40000).
FEW_ROWS = [[(64, 129)], [(1, 129), (129, 1), (33, 128), (128, 33)], [(32, 256), (256, 32), (2, 777), (64, 700), (5, 5)], [(17, 20000)], [(20000, 17)],
            [(64, 8192), (31, 1000)], [(40, 300)] * 40, [(64, 40000)]]


@pytest.mark.parametrize("name", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("shapes", FEW_ROWS)
def test_few_rows(shapes, name):
    import torch
    dtype = getattr(torch, name)
    check(shapes, dtype, noise, tolerance(dtype))
    check(shapes, dtype, falling, tolerance(dtype))
    for steps in (1, 2):
        check(shapes[:5], dtype, noise, tolerance(dtype), steps=steps)


@pytest.mark.parametrize("name", ["float32", "bfloat16"])
def test_few_rows_with_one_dominant_direction(name):
    test_one_dominant_direction((48, 900), name)


def test_few_rows_zeros_and_values_that_are_not_finite():
    for name in ("float32", "bfloat16"):
        for bad in ((40, 300), (300, 20)):
            test_zeros_and_values_that_are_not_finite(bad, name)


def test_few_rows_coefficients_in_place_update_and_graph():
    test_coefficients_of_their_own_for_every_step([(50, 260), (40, 60)])
    test_matrices_side_by_side_and_in_place((50, 60, 300))
    for nesterov in (True, False):
        test_update([(64, 300), (1000, 10), (10, 64)], nesterov)
    test_another_stream_and_a_replayed_graph([(33, 500), (300, 64)])
