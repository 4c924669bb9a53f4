"""The workspace of products in 8 bits: what the binding says and allots against what the library asks for each type of result (CPU only).
A product is cut by its type too, so that results of 16 bits may need more than fp32's, or less."""
import ctypes as C
import random

import pytest
import torch

from paper_2204_08211_amd import binding as B
from test_train8_host import Calls
from test_train_devices import OnGpu1

TYPES = {torch.float32: B.F32, torch.bfloat16: B.BF16, torch.float16: B.F16}
FORMS = [(False, True), (False, False), (True, False), (True, True)]
# products whose results of 16 bits are cut into more slices than fp32's, one row among them, and others
SIZES = [(256, 8192, 4096), (512, 4096, 4096), (1024, 2048, 4096), (4096, 512, 4096), (1024, 1024, 8192), (1, 4096, 8192), (512, 5120, 8192), (320, 4096, 5120),
         (1271, 1484, 7966), (256, 256, 4096), (1, 1, 1), (17, 33, 4000), (1, 5, 1 << 17), (8192, 4096, 4096), (0, 4, 9), (5, 7, 0)]


class Sizes:
    """Stands for a Blocks8 where only sizes are asked for."""

    def __init__(self, batch, rows, cols):
        columns, blocks = (cols + 127) // 128, (rows + 127) // 128
        self.batch, self.rows, self.cols, self.gpu = batch, rows, cols, 1
        ld = (cols + 15) // 16 * 16
        self._fields = (4096, 4096, rows, ld, rows * ld, cols, batch, 128, (blocks + 15) // 16 * 16)


def operands(batch, m, n, k, ta, tb):
    return Sizes(batch, *((k, m) if ta else (m, k))), Sizes(batch, *((n, k) if tb else (k, n)))


def asked(a, b, ta, tb, kind):
    return B.lib().co3_matmul8_workspace_bytes(C.byref(B.Matmul8Args(B.Blocks8Struct(*a._fields), B.Blocks8Struct(*b._fields), None, 0, 0, kind, ta, tb, 0, None, 0)))


def check(batch, m, n, k):
    """Whether any type asks for more than fp32 does."""
    more = False
    for ta, tb in FORMS:
        if min(m if ta else k, k if tb else n) == 0:
            continue                                        # a matrix has a column at least
        a, b = operands(batch, m, n, k, ta, tb)
        of = {t: asked(a, b, ta, tb, kind) for t, kind in TYPES.items()}
        assert B.co3_matmul8_workspace_bytes(a, b, ta, tb) == max(of.values()), (batch, m, n, k, ta, tb)
        for t, need in of.items():
            assert B.co3_matmul8_workspace_bytes(a, b, ta, tb, dtype=t) == need
            more = more or need > of[torch.float32]
    return more


@pytest.mark.parametrize("batch", [1, 3])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_enough_for_every_type(m, n, k, batch):
    check(batch, m, n, k)


def test_enough_for_every_type_at_drawn_sizes():
    rng = random.Random(8)
    size = lambda low, high: int(2 ** rng.uniform(low, high))  # noqa: E731
    more = sum(check(rng.choice([1, 1, 2, 3, 8, 16]), size(0, 13), size(0, 13), size(0, 15)) for _ in range(600))
    assert more > 0                                         # such products were among them
    assert check(1, 256, 8192, 4096)


class Planned(Calls):
    """Records calls, with the sizes that the library asks for."""

    def __init__(self):
        super().__init__()
        self.co3_matmul8_workspace_bytes = B.lib().co3_matmul8_workspace_bytes


@pytest.mark.parametrize("ta,tb", FORMS)
@pytest.mark.parametrize("m,n,k", [(256, 8192, 4096), (512, 4096, 4096), (1, 4096, 8192), (1271, 1484, 7966)])
def test_what_a_call_allots(monkeypatch, m, n, k, ta, tb):
    """The workspace of a call that is given none is its product's, with the type of `out`, of `dtype`, and of neither."""
    s, empty = Planned(), torch.empty
    monkeypatch.setattr(B, "_torch_c", s)
    monkeypatch.setattr(B, "lib", lambda: s)
    monkeypatch.setattr(torch, "empty", lambda *size, **how: empty(*size, **how).as_subclass(OnGpu1))
    s.current = 1
    a, b = operands(1, m, n, k, ta, tb)
    a.values = b.values = empty(0)

    def made(**how):
        out = B.co3_matmul8(a, b, transpose_a=ta, transpose_b=tb, **how)
        args = B.Matmul8Args.from_buffer_copy(s.kept[-1][:C.sizeof(B.Matmul8Args)])
        assert args.type == TYPES[out.dtype]
        assert args.workspace_bytes == s.co3_matmul8_workspace_bytes(C.byref(args)) and (args.workspace or args.workspace_bytes == 0)
        return out.dtype

    assert made() is torch.bfloat16
    for t in TYPES:
        assert made(dtype=t) is t
        assert made(out=empty(1, m, n, dtype=t).as_subclass(OnGpu1)) is t
