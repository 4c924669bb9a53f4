"""Tensors and products in 8 bits, group norm: what the library refuses before it touches a GPU, the layout of the argument
structures, the binding's own checks, which GPU a call is made on (CPU only)."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

import blocks8_util as bu
from paper_2204_08211_amd import binding as B
from test_train_devices import OnGpu1, State, Stream

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = {"co3_blocks8": B.Blocks8Struct, "co3_quantize8_args": B.Quantize8Args, "co3_dequantize8_args": B.Dequantize8Args,
           "co3_matmul8_args": B.Matmul8Args, "co3_groupnorm_args": B.GroupnormArgs, "co3_groupnorm_backward_args": B.GroupnormBackwardArgs}


def test_struct_layouts_match_the_header(tmp_path):
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "co3.h"', 'int main(void){']
    for cname, st in STRUCTS.items():
        lines.append(f'printf("{cname} %zu\\n", sizeof({cname}));')
        for fname, _ in st._fields_:
            lines.append(f'printf("{cname}.{fname} %zu\\n", offsetof({cname}, {fname}));')
    lines.append('printf("cols %u\\nld %u\\nacts %d\\n", CO3_MAX_BLOCKS8_COLS, CO3_MAX_BLOCKS8_LD, CO3_ACT_NONE + 10 * CO3_ACT_RELU + 100 * CO3_ACT_SILU); return 0;}')
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = dict(l.split() for l in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines())
    for cname, st in STRUCTS.items():
        assert int(out[cname]) == C.sizeof(st), cname
        for fname, _ in st._fields_:
            assert int(out[f"{cname}.{fname}"]) == getattr(st, fname).offset, (cname, fname)
    assert (int(out["cols"]), int(out["ld"])) == (B.MAX_BLOCKS8_COLS, B.MAX_BLOCKS8_LD)
    assert int(out["acts"]) == B.ACT_NONE + 10 * B.ACT_RELU + 100 * B.ACT_SILU


BUF = np.zeros(1 << 16, np.uint8)
AT = (BUF.ctypes.data + 255) // 256 * 256


def blocks(**change):
    f = dict(values=AT, scales=AT, rows=200, ld=48, batch_stride=200 * 48, cols=40, batch=2, block_rows=128, scale_ld=16)
    f.update(change)
    return B.Blocks8Struct(**f)


BAD_BLOCKS = [dict(values=None), dict(scales=None), dict(values=AT + 8), dict(scales=AT + 4), dict(cols=0), dict(cols=49), dict(ld=40), dict(ld=56),
              dict(ld=B.MAX_BLOCKS8_LD + 16, batch_stride=1 << 40), dict(rows=1 << 31, scale_ld=1 << 25, batch_stride=1 << 40), dict(batch=0), dict(batch=65536),
              dict(batch_stride=200 * 48 + 8), dict(batch_stride=199 * 48), dict(batch_stride=32), dict(batch_stride=1 << 50), dict(block_rows=64),
              dict(block_rows=0), dict(scale_ld=8), dict(scale_ld=0), dict(block_rows=1, scale_ld=192)]


@pytest.mark.parametrize("change", BAD_BLOCKS)
def test_every_call_refuses_such_tensors(change):
    bad, L = blocks(**change), B.lib()
    assert L.co3_quantize8(C.byref(B.Quantize8Args(AT, bad, 64, 1 << 20, None, B.BF16, 0)), None) == B.ERR_ARG
    assert L.co3_dequantize8(C.byref(B.Dequantize8Args(bad, AT, 64, 1 << 20, B.BF16, 0)), None) == B.ERR_ARG
    for a, b in ((bad, blocks()), (blocks(), bad)):
        args = B.Matmul8Args(a, b, AT, 4096, 1 << 30, B.BF16, 1, 0, 0, AT, 1 << 40)
        assert L.co3_matmul8(C.byref(args), None) == B.ERR_ARG and L.co3_matmul8_workspace_bytes(C.byref(args)) == 0
    assert L.co3_groupnorm_backward(C.byref(backward_args(x=None, x8=bad, U=2, samples_per_user=2, pixels=100, channels=40, groups=4, grad_stride=40, dy_stride=40,
                                                          dx_stride=40)), None) == B.ERR_ARG


def test_rows_side_by_side_are_taken():
    """Matrices in the same rows do not share a byte: the refusals above are not of them.  (Nothing runs: the product has no rows.)"""
    side = blocks(rows=0, ld=96, batch_stride=48)
    assert B.lib().co3_quantize8(C.byref(B.Quantize8Args(AT, side, 64, 0, None, B.F32, 0)), None) == B.OK
    n, m = blocks(cols=48, rows=200), blocks(rows=0, cols=200, ld=208, values=None, scales=None)
    assert B.lib().co3_matmul8(C.byref(B.Matmul8Args(m, n, None, 48, 0, B.F32, 0, 0, 0, None, 0)), None) == B.OK


@pytest.mark.parametrize("change", [dict(x=None), dict(x=AT + 1), dict(type=B.F32, x=AT + 2), dict(type=3), dict(x_stride=39), dict(x_stride=1 << 33),
                                    dict(x_batch_stride=1 << 50), dict(status=AT + 4)])
def test_quantize8_refuses(change):
    f = dict(x=AT, out=blocks(), x_stride=40, x_batch_stride=8000, status=None, type=B.F16, reserved=0)
    f.update(change)
    assert B.lib().co3_quantize8(C.byref(B.Quantize8Args(**f)), None) == B.ERR_ARG


@pytest.mark.parametrize("change", [dict(out=None), dict(out=AT + 1), dict(type=B.F32, out=AT + 2), dict(type=-1), dict(out_stride=39),
                                    dict(out_batch_stride=7999), dict(out_batch_stride=39, out_stride=100), dict(out_batch_stride=60, out_stride=99)])
def test_dequantize8_refuses(change):
    f = dict(x=blocks(), out=AT, out_stride=40, out_batch_stride=8000, type=B.F16, reserved=0)
    f.update(change)
    assert B.lib().co3_dequantize8(C.byref(B.Dequantize8Args(**f)), None) == B.ERR_ARG


def product_args(**change):
    f = dict(a=blocks(), b=blocks(cols=48), out=AT, out_stride=48, out_batch_stride=48 * 40, type=B.F32, transpose_a=1, transpose_b=0, accumulate=0,
             workspace=AT, workspace_bytes=1 << 40)
    f.update(change)
    return B.Matmul8Args(**f)


@pytest.mark.parametrize("change", [
    dict(out=None), dict(out=AT + 2), dict(type=5), dict(out_stride=47), dict(out_stride=1 << 33), dict(out_batch_stride=48 * 40 - 1),
    dict(out_batch_stride=47, out_stride=200), dict(b=blocks(rows=199, cols=48)), dict(transpose_a=0), dict(transpose_b=1),
    dict(a=blocks(block_rows=1, scale_ld=208)), dict(b=blocks(block_rows=1, scale_ld=208)), dict(b=blocks(batch=3, cols=48)),
    # sums in slices: the workspace is looked at
    dict(a=blocks(rows=3000, batch_stride=3000 * 48, scale_ld=32), b=blocks(rows=3000, batch_stride=3000 * 48, scale_ld=32), workspace=None),
    dict(a=blocks(rows=3000, batch_stride=3000 * 48, scale_ld=32), b=blocks(rows=3000, batch_stride=3000 * 48, scale_ld=32), workspace=AT + 8)])
def test_matmul8_refuses(change):
    assert B.lib().co3_matmul8(C.byref(product_args(**change)), None) == B.ERR_ARG


def test_matmul8_refuses_a_small_workspace():
    long = blocks(rows=3000, batch_stride=3000 * 48, scale_ld=32)
    args = product_args(a=long, b=long)
    need = B.lib().co3_matmul8_workspace_bytes(C.byref(args))
    assert need > 0 and B.lib().co3_matmul8_workspace_bytes(C.byref(product_args())) == 0
    assert B.lib().co3_matmul8(C.byref(product_args(a=long, b=long, workspace_bytes=need - 1)), None) == B.ERR_CAPACITY


def test_matmul8_refuses_what_a_launch_cannot_hold():
    rows = (1 << 31) - 1
    a = blocks(rows=rows, cols=16, ld=16, batch=1, batch_stride=0, scale_ld=1 << 25)
    assert B.lib().co3_matmul8(C.byref(product_args(a=a, b=a, transpose_a=0, transpose_b=1, out_stride=1 << 31)), None) == B.ERR_CAPACITY


def forward_args(**change):
    f = dict(x=AT, y=AT, weight=AT, bias=AT, mean=AT, rstd=AT, samples=3, pixels=10, x_stride=12, y_stride=12, channels=12, groups=3, type=B.BF16,
             activation=B.ACT_SILU, eps=1e-5, reserved=0, workspace=None, workspace_bytes=0)
    f.update(change)
    return B.GroupnormArgs(**f)


BAD_SIZES = [dict(channels=0), dict(channels=B.MAX_NORM_COLS + 1, groups=1), dict(groups=0), dict(groups=5), dict(groups=24), dict(pixels=0), dict(pixels=1 << 31), dict(type=3),
             dict(activation=3), dict(activation=-1)]


@pytest.mark.parametrize("change", BAD_SIZES + [
    dict(samples=1 << 31), dict(samples=1 << 28), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(x=None), dict(y=None), dict(x=AT + 1), dict(type=B.F32, y=AT + 2),
    dict(weight=AT + 2), dict(bias=AT + 1), dict(mean=AT + 3), dict(rstd=AT + 2), dict(x_stride=11), dict(y_stride=11), dict(y_stride=13), dict(x_stride=1 << 33),
    dict(pixels=100000), dict(pixels=100000, workspace=AT + 8, workspace_bytes=1 << 40)])
def test_groupnorm_refuses(change):
    assert B.lib().co3_groupnorm(C.byref(forward_args(**change)), None) == B.ERR_ARG


def backward_args(**change):
    f = dict(dy=AT, x=AT + 4096, dx=AT + 8192, x8=B.Blocks8Struct(), weight=AT, bias=AT, mean=AT, rstd=AT, dweight=AT, dbias=AT, grad_stride=12, samples_per_user=3,
             pixels=10, dy_stride=12, x_stride=12, dx_stride=12, U=2, channels=12, groups=3, type=B.F32, activation=B.ACT_RELU, accumulate=0,
             workspace=AT, workspace_bytes=1 << 40)
    f.update(change)
    return B.GroupnormBackwardArgs(**f)


KEPT = dict(values=AT, scales=AT, rows=30, ld=16, batch_stride=480, cols=12, batch=2, block_rows=128, scale_ld=16)


@pytest.mark.parametrize("change", BAD_SIZES + [
    dict(U=0), dict(U=65536), dict(samples_per_user=1 << 31), dict(samples_per_user=1 << 27), dict(dy=None), dict(dx=None), dict(mean=None), dict(rstd=None), dict(dy=AT + 2),
    dict(x=AT + 2), dict(dx=AT + 2), dict(weight=AT + 1), dict(bias=AT + 1), dict(dweight=AT + 2), dict(dbias=AT + 2), dict(grad_stride=11), dict(grad_stride=1 << 33),
    dict(dy_stride=11), dict(x_stride=11), dict(dx_stride=11), dict(dx=AT, dx_stride=13), dict(x=AT + 8192, x_stride=13), dict(workspace=None), dict(workspace=AT + 4),
    dict(x=None), dict(x=None, x8=B.Blocks8Struct(**{**KEPT, "cols": 11})), dict(x=None, x8=B.Blocks8Struct(**{**KEPT, "rows": 29})),
    dict(x=None, x8=B.Blocks8Struct(**{**KEPT, "batch": 3, "rows": 20, "batch_stride": 320}))])
def test_groupnorm_backward_refuses(change):
    assert B.lib().co3_groupnorm_backward(C.byref(backward_args(**change)), None) == B.ERR_ARG


def test_groupnorm_refuses_a_small_workspace():
    need = B.co3_groupnorm_workspace_bytes(3, 100000, 12, 3, torch.bfloat16)
    assert need > 0 and B.co3_groupnorm_workspace_bytes(3, 10, 12, 3, torch.bfloat16) == 0
    assert B.lib().co3_groupnorm(C.byref(forward_args(pixels=100000, workspace=AT, workspace_bytes=need - 1)), None) == B.ERR_CAPACITY
    for pixels in (10, 100000):
        need = B.co3_groupnorm_backward_workspace_bytes(2, 6, pixels, 12, 3, torch.float32)
        assert need > 0
        assert B.lib().co3_groupnorm_backward(C.byref(backward_args(pixels=pixels, workspace_bytes=need - 1)), None) == B.ERR_CAPACITY
    assert B.lib().co3_groupnorm_workspace_bytes(3, 10, 12, 5, 0) == 0 and B.lib().co3_groupnorm_backward_workspace_bytes(0, 1, 10, 12, 3, 0) == 0


def test_calls_refuse_null_and_nothing_to_do_needs_no_gpu():
    L = B.lib()
    for call in (L.co3_quantize8, L.co3_dequantize8, L.co3_matmul8, L.co3_groupnorm, L.co3_groupnorm_backward):
        assert call(None, None) == B.ERR_ARG
    assert L.co3_matmul8_workspace_bytes(None) == 0
    none = blocks(rows=0, values=None, scales=None)
    assert L.co3_quantize8(C.byref(B.Quantize8Args(None, none, 0, 0, None, B.F32, 0)), None) == B.OK
    assert L.co3_dequantize8(C.byref(B.Dequantize8Args(none, None, 0, 0, B.F32, 0)), None) == B.OK
    assert L.co3_groupnorm(C.byref(forward_args(samples=0, x=None, y=None)), None) == B.OK
    assert L.co3_groupnorm_backward(C.byref(backward_args(samples_per_user=0, dweight=None, dbias=None, dy=None, x=None, dx=None, workspace=None)), None) == B.OK


def test_blocks8_refuses_memory_that_does_not_fit():
    values, scales = torch.zeros(2, 200, 48, dtype=torch.uint8), torch.zeros(2, 1, 16, dtype=torch.uint8)
    ok = B.Blocks8(values, scales, 40)
    assert ok.shape == (2, 200, 40)
    for bad in (lambda: B.Blocks8(values, scales, 49), lambda: B.Blocks8(values, scales, 0), lambda: B.Blocks8(values, scales, 40, block_rows=64),
                lambda: B.Blocks8(values, scales, 40, block_rows=1), lambda: B.Blocks8(values[:, :, :40], scales, 40), lambda: B.Blocks8(values.int(), scales, 40),
                lambda: B.Blocks8(values[0], scales, 40), lambda: B.Blocks8(values, scales[:, :, :8], 40), lambda: B.Blocks8(values, scales[:1], 40),
                lambda: B.Blocks8(values.transpose(1, 2), scales, 40), lambda: B.Blocks8(values[:, :, 1:], scales, 40),
                lambda: B.Blocks8(torch.zeros(2, 200, 160, dtype=torch.uint8), scales, 150), lambda: B.Blocks8(values[:, :1].expand(2, 200, 48), scales, 40),
                lambda: B.Blocks8.empty(1, 4, 5, block_rows=2, device="cpu")):
        with pytest.raises(ValueError):
            bad()


def test_binding_refuses_what_does_not_fit():
    x = torch.zeros(2, 6, 8)
    for bad in (lambda: B.co3_quantize8(torch.zeros(8)), lambda: B.co3_quantize8(x.transpose(1, 2)), lambda: B.co3_quantize8(x),
                lambda: B.co3_groupnorm(x[0], 2), lambda: B.co3_groupnorm(x, 3), lambda: B.co3_groupnorm(x, 0), lambda: B.co3_groupnorm(x.transpose(1, 2), 2),
                lambda: B.co3_groupnorm(torch.zeros(2, 7, 8)[:, :6], 2), lambda: B.co3_groupnorm(x, 2, torch.zeros(7)),
                lambda: B.co3_groupnorm(x, 2, y=torch.zeros(2, 6, 9)), lambda: B.co3_groupnorm(x, 2, mean=torch.zeros(2, 3)),
                lambda: B.co3_groupnorm_backward(x, x, 2, None, None, torch.zeros(2, 2), torch.zeros(2, 2), users=3),
                lambda: B.co3_groupnorm_backward(x, x[:1], 2, None, None, torch.zeros(2, 2), torch.zeros(2, 2)),
                lambda: B.co3_groupnorm_backward(x, x, 2, None, None, torch.zeros(2, 2), torch.zeros(2, 2), dweight=torch.zeros(2, 8)),
                lambda: B.co3_groupnorm_backward(x, x, 2, None, None, torch.zeros(2, 2), torch.zeros(2, 2), users=2, dweight=torch.zeros(2, 8),
                                                 dbias=torch.zeros(2, 9)[:, :8]),
                lambda: B.co3_groupnorm_backward(x, B.Blocks8.empty(2, 5, 8, device="cpu"), 2, None, None, torch.zeros(2, 2), torch.zeros(2, 2))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        B.co3_quantize8(x.double())
    with pytest.raises(TypeError):
        B.co3_groupnorm(x.double(), 2)
    a, b = B.Blocks8.empty(2, 10, 20, device="cpu"), B.Blocks8.empty(2, 30, 20, device="cpu")
    for bad in (lambda: B.co3_matmul8(a, b), lambda: B.co3_matmul8(a, b, transpose_b=True), lambda: B.co3_matmul8(a, b, transpose_a=True)):
        with pytest.raises(ValueError):   # lengths of the sums; tensors on the host
            bad()


class Calls(State):
    """Records the GPU that is current in every call, its stream and its arguments."""

    def __init__(self):
        super().__init__()
        self.kept = []

    def _made(self, args, stream):
        self.calls.append((self.current, stream))
        self.kept.append(bytes(args))
        return B.OK

    co3_quantize8 = co3_dequantize8 = co3_matmul8 = co3_groupnorm = co3_groupnorm_backward = _made

    def co3_matmul8_workspace_bytes(self, args):
        return 0


@pytest.fixture
def state(monkeypatch):
    s = Calls()
    monkeypatch.setattr(B, "_torch_c", s)
    monkeypatch.setattr(B, "lib", lambda: s)
    monkeypatch.setattr(torch.cuda, "device", s.device)
    return s


def on_gpu_1(*shape, dtype=torch.float32):
    whole = torch.zeros(torch.Size(shape).numel() + 16 // dtype.itemsize, dtype=dtype)
    skip = -whole.data_ptr() % 16 // dtype.itemsize
    return whole[skip:skip + torch.Size(shape).numel()].view(shape).as_subclass(OnGpu1)


def kept_on_gpu_1(batch, rows, cols):
    return B.Blocks8(on_gpu_1(batch, rows, (cols + 15) // 16 * 16, dtype=torch.uint8), on_gpu_1(batch, -(-cols // 128), 16, dtype=torch.uint8), cols)


def calls(stream):
    x, kept, w, ws = on_gpu_1(2, 6, 8), kept_on_gpu_1(2, 6, 8), kept_on_gpu_1(1, 4, 8), on_gpu_1(64, dtype=torch.uint8)
    B.co3_quantize8(x, out=kept, stream=stream)
    B.co3_dequantize8(kept, out=x, stream=stream)
    B.co3_matmul8(kept, w, out=on_gpu_1(2, 6, 4), transpose_b=True, workspace=ws, stream=stream)
    m = on_gpu_1(2, 2)
    B.co3_groupnorm(x, 2, y=x, mean=m, rstd=m, workspace=ws, stream=stream)
    B.co3_groupnorm_backward(x, kept, 2, None, None, m, m, users=2, dx=x, workspace=ws, stream=stream)


@pytest.mark.parametrize("handle", [0, 77])
def test_calls_run_on_the_streams_gpu(state, handle):
    calls(Stream(1, handle))
    assert state.calls == [(1, handle)] * 5 and state.current == 0


def test_calls_on_the_current_gpu(state):
    with pytest.raises(ValueError):
        calls(None)
    with pytest.raises(ValueError):
        calls(Stream(0, 0))
    state.current = 1
    calls(None)
    assert state.calls == [(1, 101)] * 5


def test_memory_that_is_not_there_is_refused(state):
    state.current = 1
    x, kept, w, m = on_gpu_1(2, 6, 8), kept_on_gpu_1(2, 6, 8), kept_on_gpu_1(1, 4, 8), on_gpu_1(2, 2)
    for bad in (torch.zeros(1, dtype=torch.uint8).expand(64).as_subclass(OnGpu1), on_gpu_1(128, dtype=torch.uint8)[::2], torch.zeros(64, dtype=torch.uint8)):
        for call in (lambda: B.co3_matmul8(kept, w, out=on_gpu_1(2, 6, 4), transpose_b=True, workspace=bad),
                     lambda: B.co3_groupnorm(x, 2, y=x, mean=m, rstd=m, workspace=bad),
                     lambda: B.co3_groupnorm_backward(x, x, 2, None, None, m, m, dx=x, workspace=bad)):
            with pytest.raises(ValueError):
                call()
    with pytest.raises(ValueError):
        B.co3_quantize8(x, out=kept, status=torch.zeros(1, dtype=torch.int64).expand(B.STATUS_WORDS).as_subclass(OnGpu1))
    with pytest.raises(ValueError):
        B.co3_quantize8(x, out=kept_on_gpu_1(2, 6, 9))
    with pytest.raises(ValueError):
        B.co3_matmul8(kept, w, out=on_gpu_1(2, 6, 5), transpose_b=True, workspace=on_gpu_1(64, dtype=torch.uint8))
    with pytest.raises(ValueError):
        B.co3_matmul8(kept, w, transpose_b=True, accumulate=True, workspace=on_gpu_1(64, dtype=torch.uint8))
    assert state.calls == []


def test_the_definition_of_the_tests():
    """The helper that the GPU's bytes are compared with, against torch's own conversion."""
    assert torch.equal(bu.NUMBERS[:127], torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double())
    gen = torch.Generator().manual_seed(0)
    x = torch.randn(2, 150, 200, generator=gen)
    values, scales = bu.stored(x.double(), 128)
    back = bu.numbers(torch.from_numpy(values), torch.from_numpy(scales), 200, 128)
    e = torch.from_numpy(scales).double().sub(127).exp2()
    for b, i, j in ((0, 0, 0), (1, 1, 1)):
        t = x[b, i * 128:(i + 1) * 128, j * 128:(j + 1) * 128].double()
        assert 224 < float(t.abs().max() / e[b, j, i]) <= 448
        assert torch.equal(back[b, i * 128:(i + 1) * 128, j * 128:(j + 1) * 128], (t / e[b, j, i]).float().to(torch.float8_e4m3fn).double() * e[b, j, i])
