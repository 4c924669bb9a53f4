"""How products in 8 bits are cut: the library's host side compiled for the CPU (CPU only).  CUTS are the products whose slices
test_gpu_matmul8_slices.py runs: a change of the rule's rates that cuts them otherwise fails here."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2204_08211_amd import binding as B
from paper_2204_08211_amd import build as hip_build
from test_matmul8_workspace import FORMS, operands

HERE = os.path.dirname(os.path.abspath(__file__))
KINDS = {"float32": B.F32, "bfloat16": B.BF16, "float16": B.F16}
# batch, m, n, k: tile and slices of results of fp32, of 16 bits
CUTS = {(1, 256, 8192, 4096): ((128, 1), (128, 2)),
        (1, 512, 4096, 4096): ((128, 1), (128, 2)),
        (1, 1024, 1024, 8192): ((128, 3), (128, 4)),
        (1, 1271, 1484, 7966): ((128, 2), (128, 3)),
        (3, 717, 1009, 4266): ((128, 1), (128, 2)),
        (3, 318, 1159, 6753): ((64, 1), (128, 3)),
        (1, 512, 512, 16384): ((128, 13), (128, 13)),
        (1, 2048, 2048, 16384): ((128, 1), (256, 3)),
        (3, 150, 3460, 11860): ((256, 3), (128, 2)),
        (1, 149, 1665, 94173): ((256, 19), (256, 28)),
        (1, 19, 22, 3471): ((64, 28), (64, 28)),
        (1, 256, 256, 4096): ((64, 9), (64, 9))}


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    so = tmp_path_factory.mktemp("plans") / "plans.so"
    flags = [f for f in hip_build.FLAGS if not f.startswith("--offload-arch") and f not in ("-Xclang", "-target-feature", "-packed-fp32-ops")]
    subprocess.run([hip_build.HIPCC, "-x", "hip", "--cuda-host-only", "-shared", os.path.join(HERE, "matmul8_plan_host.cpp"), "-o", str(so)] + flags, check=True)
    L = C.CDLL(str(so))
    L.plan_of.argtypes = [C.c_void_p, C.POINTER(C.c_uint32), C.POINTER(C.c_uint32)]
    L.co3_matmul8_workspace_bytes.argtypes, L.co3_matmul8_workspace_bytes.restype = [C.c_void_p], C.c_size_t
    return L


@pytest.mark.parametrize("sizes", sorted(CUTS))
def test_cuts(host, sizes):
    batch, m, n, _ = sizes
    for ta, tb in FORMS:
        a, b = operands(*sizes, ta, tb)
        for name, kind in KINDS.items():
            args = B.Matmul8Args(B.Blocks8Struct(*a._fields), B.Blocks8Struct(*b._fields), None, 0, 0, kind, ta, tb, 0, None, 0)
            form, slices = C.c_uint32(), C.c_uint32()
            assert host.plan_of(C.byref(args), C.byref(form), C.byref(slices)) == B.OK
            assert (form.value, slices.value) == CUTS[sizes][name != "float32"]
            need = slices.value * batch * m * ((n + 3) // 4 * 4) * 4 if slices.value > 1 else 0
            assert need == host.co3_matmul8_workspace_bytes(C.byref(args)) == B.lib().co3_matmul8_workspace_bytes(C.byref(args))
