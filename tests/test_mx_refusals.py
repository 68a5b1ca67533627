"""What the microscaled entry points refuse although every argument is valid by itself (no GPU: nothing is launched; a call that got as far
as a launch would return SPARQ_ELAUNCH here)."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

sq = pytest.importorskip("paper_2105_11010_amd")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, EINVAL, EUNSUPPORTED, EWORKSPACE, ELAUNCH = 0, 1, 2, 3, 4
P = ctypes.c_void_p
A = P(0x10000)                   # never dereferenced: the checks come first
I64, SZ = ctypes.c_int64, ctypes.c_size_t
BF16, F32 = 2, 0
MUCH = SZ(1 << 62)


def test_more_tiles_of_weights_gradients_than_a_launch_counts():
    N, K = 1 << 24, 1 << 20
    assert sq.lib.sparq_mx_linear_dw(A, BF16, I64(N), A, A, A, BF16, I64(K), None, I64(512), N, K, A, MUCH, None) == EUNSUPPORTED


def test_weights_gradients_are_refused_before_the_bias_is_begun():
    N, K = 1 << 24, 1 << 20
    assert sq.lib.sparq_mx_linear_dw(A, BF16, I64(N), A, A, A, BF16, I64(K), A, I64(512), N, K, A, MUCH, None) == EUNSUPPORTED


def test_a_product_is_refused_before_its_rows_are_quantised():
    M, N, K = 1 << 30, 1 << 28, 64
    assert sq.lib.sparq_mx_linear(A, BF16, I64(K), A, A, None, A, BF16, I64(N), I64(M), N, K, A, MUCH, None) == EUNSUPPORTED
    assert sq.lib.sparq_mx_gemm(A, A, A, A, None, A, BF16, I64(N), I64(M), N, K, A, MUCH, None) == EUNSUPPORTED


@pytest.mark.skipif(torch.cuda.device_count() > 0, reason="the addresses are made up")
def test_gradients_of_no_rows_take_no_dy():
    """The gradients are zeros then and dy is not looked at: NULL and a distance of 0 will do.  In a process of its own, which a division by that
    distance would end (without a GPU the launch is what fails)."""
    code = """
import ctypes, sys
import paper_2105_11010_amd as sq
A, I64, SZ, n, z = ctypes.c_void_p(0x10000), ctypes.c_int64, ctypes.c_size_t, None, ctypes.c_int64(0)
big = SZ(1 << 40)
got = [sq.lib.sparq_mx_linear_dw(n, t, z, n, n, A, 0, I64(64), db, z, N, 64, A, big, n) for t in (0, 1, 2) for db in (n, A) for N in (8, 5, 300)]
got.append(sq.lib.sparq_mx_norm_grad(n, z, n, n, n, n, n, n, z, 2, A, A, z, 64, n, SZ(0), n))
print(set(got))
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=ROOT)
    assert r.returncode == 0 and r.stdout.strip() == "{%d}" % ELAUNCH, (r.returncode, r.stdout, r.stderr)


# One byte less than the query names, everything else valid: EWORKSPACE and nothing else; sizes whose plan takes a workspace.
def _workspaces():
    M, N, K = 300, 8, 64
    yield "linear", (A, BF16, I64(K), A, A, None, A, BF16, I64(N), I64(M), N, K), (M, N, K)
    yield "linear", (A, F32, I64(8300), A, A, A, A, F32, I64(100), I64(70), 100, 8300), (70, 100, 8300)
    yield "gemm", (A, A, A, A, None, A, BF16, I64(100), I64(70), 100, 8300), (70, 100, 8300)
    yield "linear_dx", (A, F32, I64(3008), A, A, A, F32, I64(49), I64(24), 3008, 49), (24, 3008, 49)
    yield "linear_dw", (A, F32, I64(1234), A, A, A, F32, I64(114), A, I64(1757), 1234, 114), (1757, 1234, 114)
    yield "norm_grad", (A, I64(64), A, A, A, A, A, A, I64(64), BF16, A, A, I64(3), 64), (3, 64)


@pytest.mark.parametrize("name,args,sizes", list(_workspaces()), ids=lambda v: v if isinstance(v, str) else "x".join(map(str, v)) if isinstance(v[0], int) else "")
def test_a_workspace_one_byte_short(name, args, sizes):
    f, need = getattr(sq.lib, "sparq_mx_" + name), getattr(sq, "sparq_mx_%s_workspace_bytes" % name)(*sizes)
    assert need > 0
    for short in (0, need - 1):
        assert f(*args, A, SZ(short), None) == EWORKSPACE
    for bad in (None, P(0x10010)):
        assert f(*args, bad, SZ(need), None) == EINVAL


# The argument lists that test_mx_abi.py varies are valid: with more rows than a call counts each is refused for that alone.
MANY = I64(1 << 31)


@pytest.mark.parametrize("name,args", [
    ("quantize", (A, BF16, I64(64), MANY, 64, A, A, None, None, None)),
    ("quantize", (A, BF16, I64(64), MANY, 64, A, A, A, A, None)),
    ("dequantize", (A, A, 8, A, F32, I64(64), MANY, 64, None)),
    ("act", (0, A, I64(64), A, I64(64), A, I64(64), BF16, A, A, A, A, MANY, 64, None)),
    ("act_grad", (1, A, I64(64), A, A, A, A, A, I64(64), A, I64(64), BF16, MANY, 64, None)),
    ("norm", (A, I64(64), A, None, ctypes.c_float(1e-5), A, I64(64), BF16, A, A, A, A, MANY, 64, None)),
    ("norm_grad", (A, I64(64), A, A, A, A, A, A, I64(64), BF16, A, A, MANY, 64, A, MUCH, None)),
    ("linear", (A, BF16, I64(64), A, A, None, A, BF16, I64(8), MANY, 8, 64, A, MUCH, None)),
], ids=lambda v: v if isinstance(v, str) else "")
def test_valid_but_for_the_number_of_rows(name, args):
    assert getattr(sq.lib, "sparq_mx_" + name)(*args) == EUNSUPPORTED
