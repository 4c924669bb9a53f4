"""How far orthogonalised matrices are from the iteration in 64 bits, in every form (pytest -m gpu): a workgroup's, a launch a step, tiles.

Tolerances, of the difference's 2-norm over the result's.  A result y + e, where e is what the iteration is off, is rounded to the
nearest number of the type: that is no further from y + e than y's own rounding is + |e|, so it is off by at most y's rounding + 2 |e|.
Pairs leave |e| <= 2^-17, as derived in test_gpu_orthogonalize.py for six steps.  High parts are rounded by 2^-11 at most and 2^-12 in the mean;
a step takes that up to six times, from its three factors.  Over hundreds of elements the roundings come to their mean, three such steps long:
2^-8.  Those of a few elements need not: 6 2^-11 a step, five steps long, 2^-6, and twice that as small directions grow."""
import pytest

from test_gpu_orthogonalize import SHAPES, falling, lay_out, noise, rel, steps_of

pytestmark = pytest.mark.gpu

FORMS = {"a workgroup": [(64, 64), (33, 100), (128, 64), (1, 5)], "a launch a step": [(64, 1024), (700, 40), (1, 777)],
         "tiles": [(1000, 2048), (257, 1023), (33, 4097), (1, 777)], "large tiles": [(2304, 2304)]}


def results(shapes, dtype, make, **plan_args):
    """(result, the iteration in 64 bits) of every matrix, with the plan's own choice of products unless one is given."""
    import torch
    from paper_2204_08211_amd import binding as B
    matrices, n = lay_out(shapes)
    g = torch.zeros(n, device="cuda:0", dtype=dtype)
    for k, (at, rows, cols) in enumerate(matrices):
        g[at:at + rows * cols] = make(k, rows, cols).reshape(-1).to(dtype)
    out = B.co3_orthogonalize(B.MatrixPlan(matrices, dtype=dtype, **plan_args), g)
    for at, rows, cols in matrices:
        s = slice(at, at + rows * cols)
        yield out[s].view(rows, cols), steps_of(g[s].view(rows, cols))


@pytest.mark.parametrize("name", ["bfloat16", "float16"])
@pytest.mark.parametrize("what", sorted(FORMS))
def test_results_of_16_bits_are_rounded_once(what, name):
    import torch
    dtype = getattr(torch, name)
    for make in (noise, falling):
        for out, want in results(FORMS[what], dtype, make):
            assert rel(out, want) <= rel(want.to(dtype), want) + 2 * 2.0 ** -17, tuple(out.shape)


@pytest.mark.parametrize("name", ["float32", "bfloat16"])
@pytest.mark.parametrize("what", sorted(FORMS))
def test_high_parts_alone_on_request(what, name):
    import torch
    from paper_2204_08211_amd import binding as B
    dtype = getattr(torch, name)
    for make in (noise, falling):
        for out, want in results(FORMS[what], dtype, make, products=B.PRODUCTS_HIGH):
            off = 2.0 ** -8 if out.numel() >= 256 else 2.0 ** -5
            assert rel(out, want) <= (off if name == "float32" else rel(want.to(dtype), want) + 2 * off), tuple(out.shape)


@pytest.mark.parametrize("what", sorted(FORMS))
def test_pairs_keep_their_bits(what):
    """fp32 results of hundreds of elements and more.  A pair is rounded by 2^-22 at most and about 2^-24 in the root mean square; five such
    roundings a step (X, A, B, and the products of low parts that two sums leave out), each taken up to 2.8 times, five steps long, come to
    sqrt(25) 2.8 2^-24 = 2^-20.2 where they are independent: 2^-19.  Three bits less in any of them would be past it."""
    import torch
    for make in (noise, falling):
        for out, want in results(FORMS[what], torch.float32, make):
            if out.numel() >= 256:
                assert rel(out, want) <= 2.0 ** -19, tuple(out.shape)


@pytest.mark.parametrize("what", sorted(SHAPES))
def test_high_parts_around_every_forms_limits(what):
    import torch
    from paper_2204_08211_amd import binding as B
    for make in (noise, falling):
        for out, want in results(SHAPES[what], torch.float16, make, products=B.PRODUCTS_HIGH):
            off = 2.0 ** -8 if out.numel() >= 256 else 2.0 ** -5
            assert rel(out, want) <= rel(want.half(), want) + 2 * off, tuple(out.shape)


@pytest.mark.parametrize("bad", [(60, 30), (40, 300), (70, 200)])
def test_high_parts_of_zeros_and_values_that_are_not_finite(bad):
    import torch
    from paper_2204_08211_amd import binding as B
    size = bad[0] * bad[1]
    g = torch.randn(4 * size, device="cuda:0").bfloat16()
    g[:size] = 0
    g[size + 5] = float("nan")
    g[2 * size + 7] = float("inf")
    status = torch.zeros(B.STATUS_WORDS, dtype=torch.int64, device="cuda:0")
    plan = B.MatrixPlan([(k * size,) + bad for k in range(4)], dtype=torch.bfloat16, products=B.PRODUCTS_HIGH)
    out = B.co3_orthogonalize(plan, g, status=status)
    assert bool((out[:size] == 0).all()) and bool(torch.isnan(out[size:3 * size]).all()) and int(status[B.STAT_NONFINITE]) == 2
    want = steps_of(g[3 * size:].view(bad))
    assert rel(out[3 * size:].view(bad), want) <= rel(want.bfloat16(), want) + 2 * 2.0 ** -8
