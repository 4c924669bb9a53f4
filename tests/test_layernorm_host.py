"""What layer norm launches, without a GPU: its host side compiled for the CPU, its launches written down (CPU only)."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2204_08211_amd import binding as B
from paper_2204_08211_amd import build as hip_build

HERE = os.path.dirname(os.path.abspath(__file__))


class Launch(C.Structure):
    _fields_ = [("grid", C.c_uint32 * 3), ("block", C.c_uint32 * 3), ("args", C.c_ubyte * C.sizeof(B.LayernormBackwardArgs))]


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    so = tmp_path_factory.mktemp("layernorm") / "layernorm.so"
    flags = [f for f in hip_build.FLAGS if not f.startswith("--offload-arch")]
    flags = [f for f in flags if f not in ("-Xclang", "-target-feature", "-packed-fp32-ops")]
    subprocess.run([hip_build.HIPCC, "-x", "hip", "--cuda-host-only", "-fuse-cuid=none", "-shared", "-Wl,-Bsymbolic", os.path.join(HERE, "layernorm_host.cpp"),
                    "-o", str(so)] + flags, check=True)
    L = C.CDLL(str(so))
    L.backward_workspace.argtypes, L.backward_workspace.restype = [C.c_uint32, C.c_uint64, C.c_uint32], C.c_size_t
    L.one_not_launched.restype = C.c_char_p
    return L


def launches(call, args):
    room = (Launch * 4096)()
    n = call(C.byref(args), room, 4096)
    assert n <= 4096
    return [(tuple(l.grid), tuple(l.block), type(args).from_buffer_copy(bytes(l.args)[:C.sizeof(args)])) for l in room[:n]]


COLS = [1, 17, 33, 64, 129, 257, 1025, 2049, 4096, 4097, 8193, 16384, 16385, 32768]


@pytest.mark.parametrize("kind", [B.F32, B.BF16, B.F16])
@pytest.mark.parametrize("cols", COLS)
def test_forward_launches_fit_and_have_every_row_once(host, cols, kind):
    size = 4 if kind == B.F32 else 2
    for rows in (1, 5, 70001, 1 << 24, (1 << 26) + 1, (1 << 28) - 1, 1 << 29, (1 << 31) - 1):
        a = B.LayernormArgs(x=1 << 20, y=1 << 50, weight=None, bias=None, mean=1 << 58, rstd=None, rows=rows, x_stride=cols + 3, y_stride=cols + 5, cols=cols,
                            type=kind, eps=1e-5, reserved=0)
        at = 0
        for grid, block, part in launches(host.forward_launches, a):
            assert all(g * b < 1 << 32 for g, b in zip(grid, block))          # HIP refuses more
            assert part.x == a.x + at * size * (cols + 3) and part.y == a.y + at * size * (cols + 5)
            assert part.mean == a.mean + 4 * at and not part.rstd and part.cols == cols and part.x_stride == cols + 3
            assert 8 * part.rows <= grid[0] * block[0] and grid[0] <= part.rows and grid[1:] == (1, 1)   # 8 lanes a row at least
            at += part.rows
        assert at == rows


def backward_args(users, rows, cols, kind, grad):
    return B.LayernormBackwardArgs(dy=1 << 20, x=1 << 30, dx=1 << 35, weight=None, mean=1 << 20, rstd=1 << 20, dweight=grad, dbias=grad, grad_stride=cols,
                                   rows_per_user=rows, dy_stride=cols, x_stride=cols, dx_stride=cols, U=users, cols=cols, type=kind, accumulate=0,
                                   workspace=1 << 20, workspace_bytes=1 << 50)


@pytest.mark.parametrize("kind", [B.F32, B.BF16])
@pytest.mark.parametrize("cols", COLS)
def test_backward_launches_fit(host, cols, kind):
    for users, rows in ((1, 0), (1, 1), (3, 70001), (300, 1 << 20), (65535, 1), (65535, 32768), (1, (1 << 31) - 1)):
        for grad in (None, 1 << 40):
            a = backward_args(users, rows, cols, kind, grad)
            for grid, block, _ in launches(host.backward_launches, a):
                assert all(0 < g and g * b < 1 << 32 for g, b in zip(grid, block)) and max(grid[1:]) <= 65535


@pytest.mark.parametrize("cols", COLS + [32, 65, 128, 1024])
def test_an_accumulator_takes_512_rows_at_most(host, cols):
    at_once = 32 if cols <= 32 else 16 if cols <= 64 else 8 if cols <= 128 else 4 if cols <= 1024 else 1   # with accumulators of their own
    for users in (1, 2, 16, 256, 257, 300, 65535):
        for rows in (1, 512, 513, 8192, 32768, 100003, (1 << 31) // users - 1):
            slices = max(1, host.backward_workspace(users, rows, cols) // (users * 2 * cols * 4))
            assert -(-rows // slices) <= 512 * at_once


def test_every_kernel_is_launched_by_some_call(host):
    for kind in (B.F32, B.BF16, B.F16):
        for cols in [1 << k for k in range(16)]:
            launches(host.forward_launches, B.LayernormArgs(x=1 << 20, y=1 << 50, rows=9, x_stride=cols, y_stride=cols, cols=cols, type=kind, eps=1e-5))
            launches(host.backward_launches, backward_args(2, 900, cols, kind, 1 << 40))
    assert host.not_launched() == 0, host.one_not_launched().decode()
