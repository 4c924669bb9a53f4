"""Layer norm of more rows than a launch takes (pytest -m gpu): the forward pass, all rows against 64 bits."""
import pytest

from test_gpu_layernorm import TOL, plain_backward, plain_forward, rel

pytestmark = pytest.mark.gpu


def test_more_rows_than_a_launch_takes():
    import torch
    from paper_2204_08211_amd import binding as B
    dev, rows, cols = "cuda:0", (1 << 29) + 77, 3          # 2^29 rows of eight threads
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device=dev).normal_()
    weight, bias = torch.randn(cols, device=dev), torch.randn(cols, device=dev)
    y, mean, rstd = B.co3_layernorm(x, weight, bias)
    dy = torch.empty_like(x).normal_()
    dx = B.co3_layernorm_backward(dy, x, weight, mean, rstd)
    for at in list(range(0, rows, 1 << 26)) + [rows - 200]:
        s = slice(at, at + (1 << 26))
        ey, emean, erstd = plain_forward(x[s], weight, bias, 1e-5)
        assert rel(y[s], ey) <= TOL["bfloat16"] and rel(rstd[s], erstd) <= 2.0 ** -20
        assert float((mean[s].double() - emean).abs().max()) <= 2.0 ** -20 * 8
        assert rel(dx[s], plain_backward(dy[s], x[s], weight, mean[s], rstd[s])[0]) <= TOL["bfloat16"]
