"""Matrices whose rows lie apart (pytest -m gpu): of few columns among others, against 64 bits, in about the time of the same ones side by side
in memory; past 2^32 elements of a vector."""
import pytest

from test_gpu_orthogonalize import PAIR, rel, steps_of

pytestmark = pytest.mark.gpu

# one pack a line and less, several lines a wavefront, a wavefront and more a line; for 4 and 8 elements a pack
COLS = [1, 3, 4, 5, 8, 9, 31, 64, 65, 250, 600, 1025, 2049]


@pytest.mark.parametrize("name", ["float32", "bfloat16"])
@pytest.mark.parametrize("cols", COLS)
def test_few_columns_among_others(cols, name):
    import torch
    from paper_2204_08211_amd import binding as B
    dtype, rows, ld = getattr(torch, name), 1500, cols + 7
    g = torch.randn(rows * ld, device="cuda:0").to(dtype)
    g.view(rows, ld)[:, cols:] = float("nan")                          # what lies between is not read
    out = B.co3_orthogonalize(B.MatrixPlan([(0, rows, cols, ld)], dtype=dtype), g)
    got, want = out.view(rows, ld)[:, :cols], steps_of(g.view(rows, ld)[:, :cols])
    assert rel(got, want) <= rel(want.to(dtype), want) + 2 * PAIR and bool((out.view(rows, ld)[:, cols:] == 0).all())
    momentum, model = torch.full((rows * ld,), 2.0, device="cuda:0"), torch.zeros(rows * ld, device="cuda:0")
    g = g.float()
    B.co3_muon_update(B.MatrixPlan([(0, rows, cols, ld)]), g, momentum, model, eta=1.0, beta=0.5)
    assert torch.equal(momentum.view(rows, ld)[:, :cols], 1 + g.view(rows, ld)[:, :cols])
    assert bool((momentum.view(rows, ld)[:, cols:] == 2).all()) and bool((model.view(rows, ld)[:, cols:] == 0).all())


def test_few_columns_among_others_take_no_longer():
    import torch
    from paper_2204_08211_amd import binding as B

    def time_of(cols, ld):
        g = torch.randn(65536 * ld, device="cuda:0")
        plan = B.MatrixPlan([(0, 65536, cols, ld)])
        out, ws = torch.empty_like(g), torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda:0")
        times = []
        for _ in range(6):
            ends = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
            ends[0].record()
            B.co3_orthogonalize(plan, g, out, workspace=ws)
            ends[1].record()
            torch.cuda.synchronize()
            times.append(ends[0].elapsed_time(ends[1]))
        return min(times)

    for cols in (1, 7):   # one line after the other: ten and three times as long
        assert time_of(cols, cols + 1) <= 2 * time_of(cols, cols)


def test_matrices_past_32_bits_of_elements():
    import torch
    from paper_2204_08211_amd import binding as B
    for name in ("bfloat16", "float32"):
        dtype, n = getattr(torch, name), (1 << 32) + 200000
        g = torch.zeros(n, dtype=dtype, device="cuda:0")
        # one behind the last 32-bit number, one whose rows pass it, and one by tiles, whose rows lie 40 million apart
        for matrices in ([((1 << 32) + 7, 60, 90)], [((1 << 32) - 3000, 64, 500)], [(11, 107, 300, 40 * 10 ** 6)]):
            views = [g.as_strided((m[1], m[2]), (m[3] if len(m) > 3 else m[2], 1), m[0]) for m in matrices]
            for v in views:
                v.copy_(torch.randn(v.shape, device="cuda:0"))
            want = [steps_of(v) for v in views]
            B.co3_orthogonalize(B.MatrixPlan(matrices, dtype=dtype), g, g)
            for v, w in zip(views, want):
                assert rel(v, w) <= rel(w.to(dtype), w) + 2 * PAIR
                v.zero_()
            assert int(torch.count_nonzero(g)) == 0
        del g
