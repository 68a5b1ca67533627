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
