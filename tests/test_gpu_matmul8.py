"""Products in 8 bits against 64 bits (pytest -m gpu): the four forms, types, sizes around tiles and blocks, batches, broadcast, strides,
accumulation, NaN in and behind the operands.

Tolerances, of a single result against sum |a| |b| = S: fp32 results are sums of exact products, each addition off by 2^-24 of a partial
sum, at most S; there are fewer than k / 4 + 8 of them one behind the other in a sum's accumulator and its slices, so (k / 4 + 8) 2^-24 S, and
2^-24 of the result.  Results of 16 bits: sixteen products are cut off 2^-13 of the largest of them at worst (the instructions' own
sums, some 2^-16 measured), so 16 2^-13 max |a b| for each sixteen, which is 2^-9 times the sum of these maxima, itself at most S: 2^-9 S,
and half a step of the type (2^-25 of the smallest fp16 numbers).  Over all of a matrix these errors average out: the 2-norm of the difference over the result's is at
most 1e-6 (fp32) and 2e-4 beside the rounding's 2^-8 or 2^-11."""
import pytest
import torch

import blocks8_util as bu

pytestmark = pytest.mark.gpu

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
HALF_STEP = {t: torch.finfo(t).eps / 2 for t in TYPES.values()}


def operand(batch, rows, cols, block_rows, gen):
    """A Blocks8 of any bytes that are numbers, scales of 2^-13 to 2^-3; what lies behind the columns' sixteens, and in scales that no row has, is NaN."""
    from paper_2204_08211_amd import binding as B
    dev = "cuda:0"
    wide = (cols + 15) // 16 * 16
    values = torch.full((batch, rows, wide + 32), 127, dtype=torch.uint8, device=dev)
    x = torch.randn(batch, rows, cols, generator=gen, device=dev) * torch.exp(torch.randn(batch, rows, 1, generator=gen, device=dev))
    values[:, :, :wide] = 0
    values[:, :, :cols] = (x * 8).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    n, c = -(-rows // block_rows), -(-cols // 128)
    scales = torch.full((batch, c, (n + 15) // 16 * 16), 255, dtype=torch.uint8, device=dev)
    scales[:, :, :n] = torch.randint(114, 125, (batch, c, n), generator=gen, device=dev, dtype=torch.uint8)
    return B.Blocks8(values, scales, cols, block_rows)


def numbers(x):
    return bu.numbers(x.values, x.scales, x.cols, x.block_rows)


def op(x, transposed):
    return x.mT.contiguous() if transposed else x


def product(a, b):
    return torch.stack([torch.mm(a[i if a.shape[0] > 1 else 0], b[i if b.shape[0] > 1 else 0]) for i in range(max(a.shape[0], b.shape[0]))])


def compare(out, a, b, ta, tb, add=None):
    x, y = op(numbers(a), ta), op(numbers(b), tb)
    want, size = product(x, y), product(x.abs(), y.abs())
    if add is not None:
        want = want + add.double()
        size = size + add.double().abs()
    k, t = x.shape[2], out.dtype
    share = (k / 4 + 8) * 2.0 ** -24 if t is torch.float32 else 2.0 ** -9
    err = (out.double() - want).abs()
    assert bool((err <= HALF_STEP[t] * want.abs() + share * size + 2.0 ** -25 * (t is torch.float16)).all())
    if want.numel() and float(want.norm()) > 0:
        assert float((out.double() - want).norm()) <= (1e-6 if t is torch.float32 else 2e-4 + HALF_STEP[t]) * float(want.norm())


FORMS = [(False, True), (False, False), (True, False), (True, True)]
SIZES = [(1, 1, 1), (1, 64, 128), (1, 40, 5000), (15, 65, 1040), (17, 33, 4000), (3, 5, 129), (31, 33, 127), (128, 128, 128), (129, 127, 16), (130, 257, 300), (16, 1000, 640), (255, 256, 1000), (300, 17, 2049)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("ta,tb", FORMS)
@pytest.mark.parametrize("name", sorted(TYPES))
def test_forms(name, ta, tb, m, n, k):
    from paper_2204_08211_amd import binding as B
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(m * n + k)
    for block_rows in ((128,) if ta and not tb else (128, 1)):
        a = operand(1, *((k, m) if ta else (m, k)), 128 if ta else block_rows, gen)
        b = operand(1, *((n, k) if tb else (k, n)), block_rows if tb else 128, gen)
        out = B.co3_matmul8(a, b, dtype=TYPES[name], transpose_a=ta, transpose_b=tb)
        assert out.shape == (1, m, n)
        compare(out, a, b, ta, tb)


@pytest.mark.parametrize("m,n,k", [(4001, 4100, 270), (4000, 4090, 1100), (700, 900, 5000)])
@pytest.mark.parametrize("ta,tb", FORMS)
@pytest.mark.parametrize("name", ["float32", "bfloat16"])
def test_large_tiles(name, ta, tb, m, n, k):
    """Enough tiles of 128 and of 256 for all CUs, ragged at every end; long sums in slices."""
    from paper_2204_08211_amd import binding as B
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(7)
    a, b = operand(1, *((k, m) if ta else (m, k)), 128 if ta else 1, gen), operand(1, *((n, k) if tb else (k, n)), 128, gen)
    compare(B.co3_matmul8(a, b, dtype=TYPES[name], transpose_a=ta, transpose_b=tb), a, b, ta, tb)


@pytest.mark.parametrize("ta,tb", FORMS)
@pytest.mark.parametrize("batch_a,batch_b", [(3, 3), (3, 1), (1, 3)])
def test_batches_and_one_for_all(batch_a, batch_b, ta, tb):
    from paper_2204_08211_amd import binding as B
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(batch_a)
    m, n, k = 150, 90, 260
    a, b = operand(batch_a, *((k, m) if ta else (m, k)), 128, gen), operand(batch_b, *((n, k) if tb else (k, n)), 128, gen)
    for t in (torch.float32, torch.float16):
        out = B.co3_matmul8(a, b, dtype=t, transpose_a=ta, transpose_b=tb)
        assert out.shape == (3, m, n)
        compare(out, a, b, ta, tb)


@pytest.mark.parametrize("k", [40, 3000])      # in one piece, and in slices
@pytest.mark.parametrize("name", sorted(TYPES))
def test_into_a_part_of_the_users_gradients(name, k):
    """Users' rows apart at odd places, written and then added to, and nothing beside them touched."""
    from paper_2204_08211_amd import binding as B
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(k)
    m, n, users, t = 70, 45, 3, TYPES[name]
    a, b = operand(users, k, m, 128, gen), operand(users, k, n, 128, gen)
    buffer = torch.full((users, 7 + m * n + 6), 5.0, device="cuda:0").to(t)
    out = buffer[:, 7:7 + m * n].unflatten(1, (m, n))
    B.co3_matmul8(a, b, out=out, transpose_a=True)
    compare(out, a, b, True, False)
    first = buffer.clone()
    B.co3_matmul8(a, b, out=out, transpose_a=True)
    assert torch.equal(first, buffer)                          # the same order every time
    B.co3_matmul8(a, b, out=out, transpose_a=True, accumulate=True)
    compare(out, a, b, True, False, add=first[:, 7:7 + m * n].unflatten(1, (m, n)))
    assert bool((buffer[:, :7] == 5).all()) and bool((buffer[:, 7 + m * n:] == 5).all())
    side = torch.full((m, users, n + 1), 2.0, device="cuda:0").to(t)          # users side by side in the same rows
    B.co3_matmul8(a, b, out=side.transpose(0, 1)[:, :, :n], transpose_a=True)
    assert torch.equal(side.transpose(0, 1)[:, :, :n], first[:, 7:7 + m * n].unflatten(1, (m, n))) and bool((side[:, :, n] == 2).all())


def test_sums_of_nothing():
    from paper_2204_08211_amd import binding as B
    a, b = B.Blocks8.empty(2, 0, 30, device="cuda:0"), B.Blocks8.empty(2, 0, 20, device="cuda:0")
    out = torch.full((2, 30, 20), 4.0, device="cuda:0")
    B.co3_matmul8(a, b, out=out, transpose_a=True, accumulate=True)
    assert bool((out == 4).all())
    B.co3_matmul8(a, b, out=out, transpose_a=True)
    assert bool((out == 0).all())
    w = B.Blocks8.empty(1, 20, 30, device="cuda:0")
    assert B.co3_matmul8(B.Blocks8.empty(2, 0, 30, device="cuda:0"), w, transpose_b=True).shape == (2, 0, 20)


@pytest.mark.parametrize("ta,tb", FORMS)
@pytest.mark.parametrize("name", ["float32", "bfloat16"])
def test_nan_stays_in_its_row_and_column(name, ta, tb):
    from paper_2204_08211_amd import binding as B
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(11)
    m, n, k = 140, 150, 200
    a, b = operand(1, *((k, m) if ta else (m, k)), 128, gen), operand(1, *((n, k) if tb else (k, n)), 128, gen)
    (a.values[0].t() if ta else a.values[0])[139, 199] = 127
    (b.values[0].t() if tb else b.values[0])[3, 149] = 255
    out = B.co3_matmul8(a, b, dtype=TYPES[name], transpose_a=ta, transpose_b=tb)[0]
    want = torch.zeros(m, n, dtype=torch.bool, device="cuda:0")
    want[139], want[:, 149] = True, True
    assert torch.equal(out.isnan(), want)


def test_scales_at_their_ends():
    """Products of the smallest and the largest scales, and of those whose product leaves fp32's range.  Numbers below 2^-126 may count as
    zeros where the result is fp32: there the smallest scale is 2^-117."""
    from paper_2204_08211_amd import binding as B
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(2)
    a, b = operand(1, 64, 128, 1, gen), operand(1, 64, 128, 1, gen)
    a.scales[0, 0], b.scales[0, 0] = 1, 247
    compare(B.co3_matmul8(a, b, dtype=torch.bfloat16, transpose_b=True), a, b, False, True)
    compare(B.co3_matmul8(b, a, dtype=torch.bfloat16, transpose_b=True), b, a, False, True)
    a.scales[0, 0] = 10
    compare(B.co3_matmul8(a, b, dtype=torch.float32, transpose_b=True), a, b, False, True)
    compare(B.co3_matmul8(b, a, dtype=torch.float32, transpose_b=True), b, a, False, True)
    a.scales[0, 0] = 247
    out = B.co3_matmul8(a, b, dtype=torch.float32, transpose_b=True)
    assert bool((out.abs() > 1e38).all() | (~out.isfinite()).any())
    a.scales[0, 0], b.scales[0, 0] = 1, 1
    assert float(B.co3_matmul8(a, b, dtype=torch.float32, transpose_b=True).abs().max()) == 0.0


def test_other_streams_and_a_replayed_graph():
    from paper_2204_08211_amd import binding as B
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(4)
    dy, x, w = operand(2, 700, 130, 128, gen), operand(2, 700, 260, 128, gen), operand(1, 130, 260, 128, gen)
    dx, dw = torch.zeros(2, 700, 260, device="cuda:0").bfloat16(), torch.zeros(2, 130, 260, device="cuda:0")
    ws = torch.empty(max(B.co3_matmul8_workspace_bytes(dy, w), B.co3_matmul8_workspace_bytes(dy, x, transpose_a=True)), dtype=torch.uint8, device="cuda:0")

    def step(stream=None):
        B.co3_matmul8(dy, w, out=dx, workspace=ws, stream=stream)
        B.co3_matmul8(dy, x, out=dw, transpose_a=True, workspace=ws, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    compare(dx, dy, w, False, False)
    compare(dw, dy, x, True, False)
    first = (dx.clone(), dw.clone())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        dy.values.copy_(operand(2, 700, 130, 128, gen).values)
        dx.zero_()
        dw.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = (dx.clone(), dw.clone())
        step()
        assert torch.equal(got[0], dx) and torch.equal(got[1], dw) and not torch.equal(got[1], first[1])
        compare(dw, dy, x, True, False)


@pytest.mark.parametrize("ta,tb", FORMS)
@pytest.mark.parametrize("m", [7, 300])     # few rows, and tiles
def test_offsets_beyond_32_bits(m, ta, tb):
    """Rows 2^22 bytes and elements apart, 1100 and more of them: the bits of the same product of rows next to each other."""
    from paper_2204_08211_amd import binding as B
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(m)
    far, k, n = 1 << 22, 1100, 1100
    shape = (1, n, 130) if tb else (1, k, 130)
    x = torch.randn(shape, generator=gen, device="cuda:0").bfloat16()
    near = B.co3_quantize8(x)
    apart = torch.empty(shape[1] * far, dtype=torch.bfloat16, device="cuda:0").as_strided(shape, (0, far, 1))
    apart.copy_(x)
    values = torch.empty(shape[1] * far, dtype=torch.uint8, device="cuda:0").as_strided((1, shape[1], 144), (shape[1] * far, far, 1))
    b = B.Blocks8(values, torch.empty_like(near.scales), 130)
    B.co3_quantize8(apart, out=b)
    assert torch.equal(b.values, near.values) and torch.equal(b.scales[:, :, :9], near.scales[:, :, :9])
    assert torch.equal(B.co3_dequantize8(b), B.co3_dequantize8(near))
    inner = 130 if tb else k
    a = B.co3_quantize8(torch.randn((1, inner, m) if ta else (1, m, inner), generator=gen, device="cuda:0"))
    want = B.co3_matmul8(a, near, transpose_a=ta, transpose_b=tb)
    assert torch.equal(B.co3_matmul8(a, b, transpose_a=ta, transpose_b=tb), want)
    # b in the place of the first operand, results far apart
    c = B.co3_quantize8(torch.randn(1, 40, 130, generator=gen, device="cuda:0"))
    out = torch.empty(shape[1] * far, dtype=torch.bfloat16, device="cuda:0").as_strided((1, shape[1], 40), (0, far, 1))
    assert torch.equal(B.co3_matmul8(b, c, out=out, transpose_b=True), B.co3_matmul8(near, c, transpose_b=True))
