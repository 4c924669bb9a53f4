"""Products in 8 bits whose sums are cut into slices, in tiles of every size (pytest -m gpu): against 64 bits, with the workspace that a call
allots and with one of exactly the bytes that are asked for.  Tolerances are test_gpu_matmul8.py's."""
import pytest
import torch

from test_gpu_matmul8 import FORMS, TYPES, compare, operand
from test_matmul8_plans import CUTS

pytestmark = pytest.mark.gpu

SLICED = [(sizes, name) for sizes in sorted(CUTS) for name in sorted(TYPES) if name != "float16" or sizes[1] * sizes[2] < 1 << 19]


@pytest.mark.parametrize("ta,tb", FORMS)
@pytest.mark.parametrize("sizes,name", SLICED)
def test_slices(sizes, name, ta, tb):
    from paper_2204_08211_amd import binding as B
    batch, m, n, k = sizes
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(m + n + k)
    a = operand(batch, *((k, m) if ta else (m, k)), 128 if ta else 1, gen)
    b = operand(batch, *((n, k) if tb else (k, n)), 128, gen)
    out = B.co3_matmul8(a, b, dtype=TYPES[name], transpose_a=ta, transpose_b=tb)
    compare(out, a, b, ta, tb)
    need = B.co3_matmul8_workspace_bytes(a, b, ta, tb, dtype=TYPES[name])
    room = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda:0")       # NaN in what no slice has written
    again = B.co3_matmul8(a, b, out=torch.empty_like(out), transpose_a=ta, transpose_b=tb, workspace=room[:need])
    assert torch.equal(again, out) and bool((room[need:] == 255).all())
    if need:
        with pytest.raises(RuntimeError):
            B.co3_matmul8(a, b, out=again, transpose_a=ta, transpose_b=tb, workspace=room[:need - 1])


def test_one_workspace_for_every_type():
    """What is said without a type does for all of them."""
    from paper_2204_08211_amd import binding as B
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(3)
    a, b = operand(1, 512, 4096, 1, gen), operand(1, 4096, 4096, 128, gen)
    ws = torch.empty(B.co3_matmul8_workspace_bytes(a, b, transpose_b=True), dtype=torch.uint8, device="cuda:0")
    for t in TYPES.values():
        compare(B.co3_matmul8(a, b, dtype=t, transpose_b=True, workspace=ws), a, b, False, True)
