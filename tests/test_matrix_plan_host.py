"""Plans of matrices and the checks of their calls without a GPU: the library's host side compiled for the CPU, where a launch does
nothing (CPU only)."""
import ctypes as C
import os
import subprocess
import time

import numpy as np
import pytest

from paper_2204_08211_amd import binding as B
from paper_2204_08211_amd import build as hip_build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    so = tmp_path_factory.mktemp("plans") / "plans.so"
    flags = [f for f in hip_build.FLAGS if not f.startswith("--offload-arch")]
    flags = [f for f in flags if f not in ("-Xclang", "-target-feature", "-packed-fp32-ops")]
    subprocess.run([hip_build.HIPCC, "-x", "hip", "--cuda-host-only", "-shared", os.path.join(HERE, "matrix_plan_host.cpp"), "-o", str(so)] + flags,
                   check=True)
    L = C.CDLL(str(so))
    L.co3_matrix_plan_create.argtypes = [C.c_uint32, C.c_void_p, C.c_int32, C.c_int32, C.POINTER(C.c_void_p)]
    L.co3_matrix_plan_destroy.argtypes, L.co3_matrix_plan_destroy.restype = [C.c_void_p], None
    L.co3_matrix_plan_workspace_bytes.argtypes, L.co3_matrix_plan_workspace_bytes.restype = [C.c_void_p], C.c_size_t
    L.co3_orthogonalize.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]
    return L


def plan_of(host, matrices, type_=B.F32, products=B.PRODUCTS_PAIR):
    """The plan's handle and what its creation returned, of matrices (offset, ld, rows, cols)."""
    table = (B.Matrix * len(matrices))(*[B.Matrix(*m, 1.0, 0) for m in matrices])
    out = C.c_void_p()
    rc = host.co3_matrix_plan_create(len(matrices), C.cast(table, C.c_void_p), type_, products, C.byref(out))
    return out, rc


def orthogonalize(host, plan, coefficients):
    """What co3_orthogonalize returns for these coefficients, one triple a step."""
    c = np.ascontiguousarray(coefficients, np.float32).reshape(-1, 3)
    a = B.OrthogonalizeArgs(g=4096, out=4096, coefficients=c.ctypes.data, steps=len(c), eps=1e-7, status=None, workspace=4096,
                            workspace_bytes=host.co3_matrix_plan_workspace_bytes(plan))
    return host.co3_orthogonalize(plan, C.byref(a), None)


def bounded(coefficients):
    """The largest |a s + b s^3 + c s^5| and |b s^2 + c s^4| of all steps, over a fine grid of every step's range."""
    top, most, factor = 1.0, 0.0, 0.0
    for a, b, c in np.asarray(np.float32(coefficients), np.float64).reshape(-1, 3):
        s = np.linspace(0.0, top, 200001)
        t = s * s
        top = np.abs(s * (a + t * (b + t * c))).max()
        most, factor = max(most, top), max(factor, np.abs(t * (b + t * c)).max())
    return most, factor


def test_coefficients_are_taken_by_what_their_polynomials_reach(host):
    plan, rc = plan_of(host, [(0, 64, 48, 64)])
    assert rc == B.OK
    cases = [[(6, -6, c)] for c in (0, 1e-30, -1e-30, 1e-12, 1e-6, 1e-3)]                    # 2.31 at s = 0.58, 0 at s = 1
    cases += [[(4, -4, c)] for c in (0, 1e-30, -1e-30, 1e-9)]                                # 1.54
    cases += [[(6, -6, 1e-30), (1000, 0, 0)], [(4, -4, 1e-30), (1000, 0, 0)], [(3.4445, -4.775, 2.0315)] * 5, [(1.5, -0.5, 1e-40)] * 12]
    rng = np.random.default_rng(3)
    for _ in range(400):
        cases.append([(rng.uniform(0, 6), rng.uniform(-6, 2), rng.choice([0, 1, 1e-20, 1e-37, -1e-8]) * rng.uniform(-4, 4))
                      for _ in range(rng.integers(1, 4))])
    for c in cases:
        most, factor = bounded(c)
        if abs(most - 2) < 1e-4 or abs(factor - 7) < 1e-4:
            continue   # nearer to a limit than the grid is fine
        assert orthogonalize(host, plan, c) == (B.OK if most < 2 and factor < 7 else B.ERR_ARG), (c, most, factor)
    host.co3_matrix_plan_destroy(plan)


def elements(matrices):
    """Every matrix's elements, as a set each."""
    return [{offset + r * ld + c for r in range(rows) for c in range(cols)} for offset, ld, rows, cols in matrices]


def taken(host, matrices):
    plan, rc = plan_of(host, matrices)
    assert rc in (B.OK, B.ERR_ARG) and (rc == B.OK) == bool(plan.value)
    host.co3_matrix_plan_destroy(plan)
    return rc == B.OK


@pytest.mark.parametrize("matrices,there", [
    ([(0, 20, 10, 5), (10, 5, 1, 5)], True),                # a single row in another's gap, whatever its ld
    ([(0, 20, 10, 5), (10, 5, 2, 5)], True),
    ([(0, 20, 10, 5), (10, 5, 3, 5)], False),               # its third row is the other's second
    ([(0, 16, 8, 8), (8, 32, 4, 8)], True),                 # every second gap
    ([(0, 16, 8, 8), (8, 24, 4, 8)], False),
    ([(0, 16, 8, 8), (8, 17, 8, 8)], False),
    ([(0, 16, 1 << 20, 8), (8, 48, 1 << 18, 8)], True),
    ([(0, 16, 1 << 20, 8), (8, 48, 1 << 18, 9)], False),
    ([(0, 16, 1 << 20, 8), (8, 16 * ((1 << 20) - 2) + 1, 2, 8)], False),   # its last row ends in the other's last
    ([(0, 16, 1 << 20, 8), (8, 16 * ((1 << 20) - 2) + 1, 2, 7)], True),
    ([(5, (1 << 40) - 1, 1 << 20, 3), (0, 1 << 40, 3, 4)], False),         # one element nearer a row
    ([(5, (1 << 40) - 1, 1 << 20, 3), (0, 1 << 40, 2, 4)], True),
])
def test_matrices_in_each_others_gaps(host, matrices, there):
    assert taken(host, matrices) == there
    assert taken(host, matrices[::-1]) == there


def test_overlaps_against_sets_of_elements(host):
    rng = np.random.default_rng(7)
    seen = [0, 0]
    for _ in range(3000):
        matrices = []
        for _ in range(rng.integers(2, 5)):
            rows, cols = int(rng.integers(1, 9)), int(rng.integers(1, 7))
            ld = cols + int(rng.choice([0, rng.integers(0, 40), 12 - cols if cols < 12 else 0, 24 - cols]))
            matrices.append((int(rng.integers(0, 120)), ld, rows, cols))
        every = elements(matrices)
        apart = sum(map(len, every)) == len(set().union(*every))
        assert taken(host, matrices) == apart, matrices
        seen[apart] += 1
    assert min(seen) > 200


def test_many_matrices_side_by_side(host):
    """65536 columns of one row distance, and half as many beside rows of their own: in the order of n log n steps, far below a second
    (every pair looked at takes several)."""
    n = 65536
    for matrices in ([(k, n, 4, 1) for k in range(n)], [(2 * k, n, 4, 1) for k in range(n // 2)] + [(4 * n + k, 1, 1, 1) for k in range(n // 2)]):
        for there in (True, False):
            if not there:
                matrices = matrices[:-1] + [matrices[7]]
            begin = time.process_time()
            assert taken(host, matrices) == there
            assert time.process_time() - begin < 1.5


def test_plans_beyond_what_a_launch_takes_are_refused(host):
    """A launch has fewer than 2^32 threads: 2^24 workgroups of 256 lay matrices out by blocks of 64 x 64."""
    plan, rc = plan_of(host, [(0, 1 << 17, 1 << 20, 1 << 17)])
    host.co3_matrix_plan_destroy(plan)
    assert rc == B.ERR_CAPACITY
    plan, rc = plan_of(host, [(0, 1 << 13, 1 << 18, 1 << 13)])
    host.co3_matrix_plan_destroy(plan)
    assert rc == B.OK
