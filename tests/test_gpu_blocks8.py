"""Tensors in 8 bits against their definition (pytest -m gpu): every byte of what is stored and every number that comes back has to be
equal.  Sizes around the blocks' limits, types, strides, batches, values at the format's ends and such that are not finite."""
import numpy as np
import pytest
import torch

import blocks8_util as bu

pytestmark = pytest.mark.gpu

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def inputs(shape, dtype, seed):
    """Rows of sizes of their own, ties of the format among them."""
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(seed)
    x = torch.randn(shape, generator=gen, device="cuda:0")
    x *= torch.exp(3 * torch.randn(shape[:-1] + (1,), generator=gen, device="cuda:0"))
    ties = torch.randint(0, 64, shape, generator=gen, device="cuda:0").float() / 16
    return torch.where(torch.rand(shape, generator=gen, device="cuda:0") < 0.3, ties, x).to(dtype)


def check(x, kept):
    values, scales = bu.stored(x.double(), kept.block_rows)
    blocks = -(-x.shape[1] // kept.block_rows)
    assert np.array_equal(kept.scales.cpu().numpy()[:, :, :blocks], scales[:, :, :blocks])
    assert np.array_equal(kept.values.cpu().numpy()[:, :, :values.shape[2]], values)


@pytest.mark.parametrize("name", sorted(TYPES))
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 3, 16), (2, 127, 17), (1, 128, 128), (3, 129, 129), (1, 31, 300), (2, 33, 255), (1, 257, 1001)])
def test_bytes_and_back(shape, block_rows, name):
    from paper_2204_08211_amd import binding as B
    x = inputs(shape, TYPES[name], sum(shape))
    kept = B.co3_quantize8(x, block_rows=block_rows)
    assert kept.shape == shape
    check(x, kept)
    want = bu.numbers(kept.values, kept.scales, shape[2], block_rows)
    for t in TYPES.values():
        back = B.co3_dequantize8(kept, dtype=t)
        most = torch.finfo(t).max
        # fp16 rounds numbers below its own smallest normal one, and those beyond its range are at its ends
        assert torch.equal(back, want.clamp(-most, most).to(t))


@pytest.mark.parametrize("block_rows", [1, 128])
def test_ends_of_the_format(block_rows):
    """Blocks of the largest and the smallest numbers, of zeros, next to the turns of the scale (448 2^e and the numbers beside it)."""
    from paper_2204_08211_amd import binding as B
    big = torch.finfo(torch.float32).max
    ends = [0.0, big, 2.0 ** -149, 2.0 ** -126, 1e-38, 448 * 2.0 ** -126, 448 * 2.0 ** -126 * (1 + 2.0 ** -23), 2.0 ** -120]
    for e in (-100, -20, -1, 0, 3, 60, 118):
        ends += [448 * 2.0 ** e, 448 * 2.0 ** e * (1 + 2.0 ** -23), 448 * 2.0 ** e * (1 - 2.0 ** -24), 2.0 ** e]
    x = torch.zeros(len(ends), 1, 130, device="cuda:0")
    for k, v in enumerate(ends):
        x[k, 0, 5] = -v
        x[k, 0, 6:20] = torch.tensor([v * 2.0 ** -i for i in range(1, 15)])
        x[k, 0, 129] = v
    kept = B.co3_quantize8(x, block_rows=block_rows)
    check(x, kept)
    back = B.co3_dequantize8(kept, dtype=torch.float32)
    assert torch.equal(back, bu.numbers(kept.values, kept.scales, 130, block_rows).clamp(-big, big).float())
    assert float(back[1, 0, 129]) == big            # rounded to 2^128, which is beyond fp32


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("name", sorted(TYPES))
def test_not_finite(block_rows, name):
    from paper_2204_08211_amd import binding as B
    x = inputs((2, 40, 200), TYPES[name], 3)
    x[0, 3, 7], x[0, 3, 150], x[1, 39, 199], x[1, 0, 0] = float("nan"), float("inf"), -float("inf"), float("nan")
    x[0, 20] = float("nan")
    status = torch.zeros(B.STATUS_WORDS, dtype=torch.int64, device="cuda:0")
    status[B.STAT_NONFINITE] = 5
    kept = B.co3_quantize8(x, block_rows=block_rows, status=status)
    check(x, kept)
    assert int(status[B.STAT_NONFINITE]) == 5 + 204 and int(status.sum()) == 5 + 204
    back = B.co3_dequantize8(kept, dtype=TYPES[name])
    assert torch.equal(back.isnan(), ~x.isfinite())


def test_strides_and_what_lies_between():
    from paper_2204_08211_amd import binding as B
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(1)
    whole = torch.randn(2, 50, 3, 77, generator=gen, device="cuda:0").bfloat16()
    x = whole[:, :, 1, 3:73]                                   # rows 231 elements apart, at odd addresses
    values = torch.full((2, 60, 96), 200, dtype=torch.uint8, device="cuda:0")
    scales = torch.full((2, 1, 16), 9, dtype=torch.uint8, device="cuda:0")
    kept = B.Blocks8(values[:, 5:55], scales, 70)
    assert B.co3_quantize8(x, out=kept) is kept
    check(x, kept)
    assert bool((values[:, :5] == 200).all()) and bool((values[:, 55:] == 200).all()) and bool((values[:, :, 80:] == 200).all())
    assert bool((scales[:, :, 1:] == 9).all())
    assert torch.equal(B.co3_quantize8(x.contiguous()).values[:, :, :80], values[:, 5:55, :80])
    out = torch.full((50, 2, 75), 3.0, device="cuda:0")        # matrices side by side in the same rows
    B.co3_dequantize8(kept, out=out.transpose(0, 1)[:, :, 2:72])
    assert torch.equal(out.transpose(0, 1)[:, :, 2:72], bu.numbers(values[:, 5:55], scales, 70, 128).float())
    assert bool((out[:, :, :2] == 3).all()) and bool((out[:, :, 72:] == 3).all())


def test_nothing():
    from paper_2204_08211_amd import binding as B
    kept = B.co3_quantize8(torch.zeros(2, 0, 5, device="cuda:0"))
    assert kept.shape == (2, 0, 5) and B.co3_dequantize8(kept).shape == (2, 0, 5)


def test_other_streams_and_a_replayed_graph():
    from paper_2204_08211_amd import binding as B
    x = inputs((2, 300, 200), torch.bfloat16, 8)
    kept, back = B.Blocks8.empty(2, 300, 200, device="cuda:0"), torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.co3_dequantize8(B.co3_quantize8(x, out=kept, stream=side), out=back, stream=side)
    side.synchronize()
    first = back.clone()
    check(x, kept)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.co3_quantize8(x, out=kept)
        B.co3_dequantize8(kept, out=back)
    for seed in (9, 10, 8):
        x.copy_(inputs((2, 300, 200), torch.bfloat16, seed))
        graph.replay()
        torch.cuda.synchronize()
        check(x, kept)
        assert torch.equal(back, B.co3_dequantize8(B.co3_quantize8(x)))
    assert torch.equal(back, first)
