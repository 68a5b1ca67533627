"""What the microscaled entry points refuse although every argument is valid by itself (no GPU: nothing is launched; a call that got as far
as a launch would return SPARQ_ELAUNCH here)."""
import ctypes

import pytest

sq = pytest.importorskip("paper_2105_11010_amd")

OK, EINVAL, EUNSUPPORTED, EWORKSPACE = 0, 1, 2, 3
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
