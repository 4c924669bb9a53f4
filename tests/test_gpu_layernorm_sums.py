"""Layer norm's weight gradients of many rows, whose terms have one sign (pytest -m gpu).

Tolerance: an accumulator of fp32 takes 512 rows at most.  Its k-th addition is off by 2^-24 of the k terms in it at most, 512 / 2 of
2^-24 over the sum of all; the up to 32 rows that a workgroup has on their way at a time are added up after that, 2^-24 a time, and the
slices' sums in fp64 with a rounding at the end: (256 + 32 + 1) 2^-24 of the sum."""
import pytest

pytestmark = pytest.mark.gpu


# many users, whose slices are few: a row by a workgroup, 32 rows of 8 lanes each; one user of many rows
@pytest.mark.parametrize("users,rows,cols", [(300, 8192, 1100), (300, 32 * 8192, 24), (1, 1 << 22, 600)])
def test_sums_of_many_rows_keep_what_is_added(users, rows, cols):
    import torch
    from paper_2204_08211_amd import binding as B
    dev, term = "cuda:0", 1 + 2.0 ** -12 + 2.0 ** -20      # half an ulp of sums between 4096 and 8192, and a little more
    x, dy = (torch.full((users, rows, cols), v, device=dev) for v in (1.0, term))
    mean, rstd = torch.zeros(users, rows, device=dev), torch.ones(users, rows, device=dev)   # of rows, the norm's 1
    dweight, dbias = torch.empty(users, cols, device=dev), torch.empty(users, cols, device=dev)
    B.co3_layernorm_backward(dy, x, None, mean, rstd, dx=x, dweight=dweight, dbias=dbias)
    for got in (dweight, dbias):
        assert float((got.double() / (rows * term) - 1).abs().max()) <= 289 * 2.0 ** -24
