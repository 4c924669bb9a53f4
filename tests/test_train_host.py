"""Layer norm, orthogonalised matrices and Muon's update: what the library refuses before it touches a GPU, the layout of
the argument structures, the binding's own checks (CPU only)."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

from paper_2204_08211_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = {"co3_matrix": B.Matrix, "co3_orthogonalize_args": B.OrthogonalizeArgs, "co3_muon_args": B.MuonArgs,
           "co3_layernorm_args": B.LayernormArgs, "co3_layernorm_backward_args": B.LayernormBackwardArgs}


def test_struct_layouts_match_the_header(tmp_path):
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "co3.h"', 'int main(void){']
    for cname, st in STRUCTS.items():
        lines.append(f'printf("{cname} %zu\\n", sizeof({cname}));')
        for fname, _ in st._fields_:
            lines.append(f'printf("{cname}.{fname} %zu\\n", offsetof({cname}, {fname}));')
    lines.append('printf("steps %u\\n", CO3_MAX_NS_STEPS); printf("cols %u\\n", CO3_MAX_NORM_COLS); return 0;}')
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = dict(l.split() for l in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines())
    for cname, st in STRUCTS.items():
        assert int(out[cname]) == C.sizeof(st), cname
        for fname, _ in st._fields_:
            assert int(out[f"{cname}.{fname}"]) == getattr(st, fname).offset, (cname, fname)
    assert int(out["steps"]) == B.MAX_NS_STEPS and int(out["cols"]) == B.MAX_NORM_COLS


def create(matrices, type_=B.F32, products=B.PRODUCTS_PAIR, count=None):
    table = (B.Matrix * max(1, len(matrices)))(*[B.Matrix(*m) for m in matrices])
    out = C.c_void_p(1)
    rc = B.lib().co3_matrix_plan_create(len(matrices) if count is None else count, C.cast(table, C.c_void_p), type_, products, C.byref(out))
    return rc, out


REFUSED = {
    "no rows": [(0, 8, 0, 8, 1.0, 0)],
    "no columns": [(0, 8, 8, 0, 1.0, 0)],
    "too many rows": [(0, 8, (1 << 20) + 1, 8, 1.0, 0)],
    "rows closer than they are long": [(0, 7, 8, 8, 1.0, 0)],
    "a scale that is not finite": [(0, 8, 8, 8, float("inf"), 0)],
    "an offset beyond all memory": [((1 << 60) + 1, 8, 8, 8, 1.0, 0)],
    "the same matrix twice": [(0, 8, 8, 8, 1.0, 0), (0, 8, 8, 8, 1.0, 0)],
    "a matrix that begins in another's last row": [(0, 8, 8, 8, 1.0, 0), (63, 8, 8, 8, 1.0, 0)],
    "side by side with a column shared": [(0, 16, 8, 9, 1.0, 0), (8, 16, 8, 8, 1.0, 0)],
    "side by side beyond the row's end": [(0, 16, 8, 8, 1.0, 0), (9, 16, 8, 8, 1.0, 0)],
    "interleaved at another distance": [(0, 16, 8, 8, 1.0, 0), (8, 17, 8, 8, 1.0, 0)],
}


@pytest.mark.parametrize("what", sorted(REFUSED))
def test_plans_refuse(what):
    rc, out = create(REFUSED[what])
    assert rc == B.ERR_ARG and not out.value


def test_plans_refuse_types_products_and_counts():
    ok = [(0, 8, 8, 8, 1.0, 0)]
    assert create(ok, type_=3)[0] == B.ERR_ARG and create(ok, type_=-1)[0] == B.ERR_ARG
    assert create(ok, products=2)[0] == B.ERR_ARG
    assert create(ok, count=0)[0] == B.ERR_ARG and create(ok, count=65537)[0] == B.ERR_ARG
    assert B.lib().co3_matrix_plan_create(1, None, 0, 0, C.byref(C.c_void_p())) == B.ERR_ARG
    assert B.lib().co3_matrix_plan_create(1, None, 0, 0, None) == B.ERR_ARG
    assert B.lib().co3_matrix_plan_workspace_bytes(None) == 0 and B.lib().co3_matrix_plan_elements(None) == 0
    B.lib().co3_matrix_plan_destroy(None)


def test_calls_refuse_null():
    L = B.lib()
    assert L.co3_orthogonalize(None, C.byref(B.OrthogonalizeArgs()), None) == B.ERR_ARG
    assert L.co3_muon_update(None, C.byref(B.MuonArgs()), None) == B.ERR_ARG
    assert L.co3_layernorm(None, None) == B.ERR_ARG and L.co3_layernorm_backward(None, None) == B.ERR_ARG


BUF = np.zeros(4096, np.float32)
AT = (BUF.ctypes.data + 255) // 256 * 256


def forward_args(**change):
    f = dict(x=AT, y=AT, weight=AT, bias=AT, mean=AT, rstd=AT, rows=4, x_stride=16, y_stride=16, cols=16, type=B.BF16, eps=1e-5, reserved=0)
    f.update(change)
    return B.LayernormArgs(**f)


@pytest.mark.parametrize("change", [dict(cols=0), dict(cols=B.MAX_NORM_COLS + 1, x_stride=1 << 20, y_stride=1 << 20), dict(rows=1 << 31), dict(type=3),
                                    dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(x=None), dict(y=None),
                                    dict(x=AT + 1), dict(type=B.F32, x=AT + 2), dict(weight=AT + 2), dict(bias=AT + 1), dict(mean=AT + 3),
                                    dict(rstd=AT + 2), dict(x_stride=15), dict(y_stride=15), dict(y_stride=17)])
def test_layernorm_refuses(change):
    assert B.lib().co3_layernorm(C.byref(forward_args(**change)), None) == B.ERR_ARG


def backward_args(**change):
    f = dict(dy=AT, x=AT + 1024, dx=AT + 2048, weight=AT, mean=AT, rstd=AT, dweight=AT, dbias=AT, grad_stride=16, rows_per_user=4, dy_stride=16,
             x_stride=16, dx_stride=16, U=2, cols=16, type=B.F32, accumulate=0, workspace=None, workspace_bytes=0)
    f.update(change)
    return B.LayernormBackwardArgs(**f)


@pytest.mark.parametrize("change", [dict(cols=0), dict(U=0), dict(U=65536), dict(rows_per_user=1 << 31), dict(rows_per_user=1 << 30), dict(type=7),
                                    dict(dy=None), dict(x=None), dict(dx=None), dict(mean=None), dict(rstd=None), dict(dy=AT + 2),
                                    dict(weight=AT + 1), dict(dweight=AT + 2), dict(dbias=AT + 2), dict(grad_stride=15), dict(dy_stride=15),
                                    dict(x_stride=15), dict(dx_stride=15), dict(dx=AT, dx_stride=17),
                                    dict(rows_per_user=4096, workspace=None), dict(rows_per_user=4096, workspace=AT + 4, workspace_bytes=1 << 40)])
def test_layernorm_backward_refuses(change):
    assert B.lib().co3_layernorm_backward(C.byref(backward_args(**change)), None) == B.ERR_ARG


def test_layernorm_backward_refuses_a_small_workspace():
    need = B.co3_layernorm_backward_workspace_bytes(2, 4096, 16)
    assert need > 0 and B.co3_layernorm_backward_workspace_bytes(2, 4, 16) == 0
    a = backward_args(rows_per_user=4096, workspace=AT, workspace_bytes=need - 1)
    assert B.lib().co3_layernorm_backward(C.byref(a), None) == B.ERR_CAPACITY


def test_nothing_to_do_needs_no_gpu():
    assert B.lib().co3_layernorm(C.byref(forward_args(rows=0, x=None, y=None)), None) == B.OK
    a = backward_args(rows_per_user=0, dweight=None, dbias=None, dy=None, x=None, dx=None, mean=None, rstd=None)
    assert B.lib().co3_layernorm_backward(C.byref(a), None) == B.OK


def test_binding_refuses_what_does_not_fit():
    import torch
    x = torch.zeros(2, 3, 8)
    with pytest.raises(ValueError):
        B.co3_layernorm(torch.zeros(8))
    with pytest.raises(ValueError):
        B.co3_layernorm(x.transpose(1, 2))
    with pytest.raises(ValueError):
        B.co3_layernorm(torch.zeros(3, 4, 8)[:, :3])          # users further apart than their rows
    with pytest.raises(ValueError):
        B.co3_layernorm(x, torch.zeros(7))
    with pytest.raises(ValueError):
        B.co3_layernorm(x, torch.zeros(8, dtype=torch.float64))
    with pytest.raises(ValueError):
        B.co3_layernorm(x, y=torch.zeros(2, 3, 9))
    with pytest.raises(TypeError):
        B.co3_layernorm(x.double())
    m = torch.zeros(2, 3)
    with pytest.raises(ValueError):
        B.co3_layernorm_backward(x, x, None, m, m, dweight=torch.zeros(3, 8))
    with pytest.raises(ValueError):
        B.co3_layernorm_backward(x, x, None, m, m, dweight=torch.zeros(2, 8), dbias=torch.zeros(2, 9)[:, :8])
    with pytest.raises(ValueError):
        B.co3_layernorm_backward(x[:, :, :4], x, None, m, m)
    with pytest.raises(TypeError):
        B.MatrixPlan([(0, 8, 8)], dtype=torch.float64)
    with pytest.raises(B.Co3Error):
        B.MatrixPlan([(0, 8, 0)])
