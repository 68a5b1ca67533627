"""The microscaled entry points without a GPU: what the header declares is exported and bound, sizes, and refusals -- by the library
(nothing is launched) and by the binding before the library is called."""
import ctypes
import os
import re

import pytest
import torch

sq = pytest.importorskip("paper_2105_11010_amd")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, EINVAL, EUNSUPPORTED, EWORKSPACE = 0, 1, 2, 3
P = ctypes.c_void_p
A = P(0x10000)                   # never dereferenced: the checks come first
I64, F32 = ctypes.c_int64, ctypes.c_float


def declared():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "sparq_mx.h")).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(sparq_mx_[a-z0-9_]+)\s*\(", text)))


def test_declared_exported_and_bound():
    names = declared()
    assert len(names) == 17
    for n in names:
        assert hasattr(sq.lib, n) and hasattr(sq, n) and n in sq.__all__, n


def test_row_sizes():
    for K, c4, c8, s in ((1, 64, 128, 16), (128, 64, 128, 16), (129, 128, 256, 16), (512, 256, 512, 16), (513, 320, 640, 32), (4096, 2048, 4096, 128)):
        assert (sq.sparq_mx_code_bytes(K, 4), sq.sparq_mx_code_bytes(K, 8), sq.sparq_mx_scale_bytes(K)) == (c4, c8, s)
    assert sq.sparq_mx_code_bytes(0, 4) == sq.sparq_mx_code_bytes(64, 5) == sq.sparq_mx_code_bytes((1 << 28) + 1, 8) == sq.sparq_mx_scale_bytes(0) == 0


def _calls():
    """Name, a valid argument list, and which positions may not be changed to what."""
    n = None
    big = ctypes.c_size_t(1 << 40)
    quantize = [A, 2, I64(64), I64(3), 64, A, A, n, n, n]
    yield "quantize", quantize, {0: (n, P(0x10001)), 1: (3, -1), 2: (I64(63),), 3: (I64(-1),), 4: (0, (1 << 28) + 1), 5: (n, P(0x10008)), 6: (n,), 7: (A,), 8: (A,)}
    yield "dequantize", [A, A, 8, A, 1, I64(64), I64(3), 64, n], {0: (n, P(0x10004)), 1: (n,), 2: (5,), 3: (n, P(0x10001)), 4: (7,), 5: (I64(1),), 6: (I64(-1),), 7: (0,)}
    yield "gemm", [A, A, A, A, n, A, 2, I64(8), I64(3), 8, 64, A, big, n], {0: (n,), 1: (n,), 2: (n,), 3: (n, P(0x10002)), 4: (P(0x10002),), 5: (n,), 6: (3,), 7: (I64(7),), 8: (I64(-1),), 9: (0,), 10: (0,)}
    yield "linear", [A, 2, I64(64), A, A, n, A, 2, I64(8), I64(3), 8, 64, A, big, n], {0: (n,), 1: (9,), 2: (I64(63),), 3: (n,), 4: (n,), 6: (n,), 7: (9,), 8: (I64(7),), 9: (I64(-2),), 10: (0,), 11: (-4,)}
    yield "linear_dx", [A, 2, I64(8), A, A, A, 2, I64(64), I64(3), 8, 64, A, big, n], {0: (n,), 1: (4,), 2: (I64(7),), 3: (n,), 4: (n,), 5: (n,), 6: (4,), 7: (I64(63),), 8: (I64(-1),), 9: (0,), 10: (0,)}
    yield "linear_dw", [A, 2, I64(8), A, A, A, 0, I64(64), n, I64(3), 8, 64, A, big, n], {0: (n,), 1: (4,), 2: (I64(7),), 3: (n,), 4: (n,), 5: (n,), 6: (4,), 7: (I64(63),), 8: (P(0x10001),), 9: (I64(-1),), 10: (0,), 11: (0,)}
    yield "act", [0, A, I64(64), A, I64(64), A, I64(64), 2, A, A, A, A, I64(3), 64, n], {0: (2, -1), 1: (n,), 2: (I64(63),), 3: (n,), 4: (I64(1),), 5: (n,), 6: (I64(1),), 7: (3,), 8: (n,), 9: (n,), 10: (n,), 12: (I64(-1),), 13: (0,)}
    yield "act_grad", [1, A, I64(64), A, A, A, A, A, I64(64), A, I64(64), 2, I64(3), 64, n], {0: (2,), 1: (n,), 2: (I64(1),), 3: (n,), 4: (n,), 5: (n,), 6: (n,), 7: (n,), 8: (I64(3),), 9: (n,), 10: (I64(3),), 11: (5,), 12: (I64(-1),), 13: (0,)}
    yield "norm", [A, I64(64), A, n, F32(1e-5), A, I64(64), 2, A, A, A, A, I64(3), 64, n], {0: (n,), 1: (I64(63),), 2: (n, P(0x10001)), 3: (P(0x10001),), 4: (F32(-1), F32(float("nan"))), 5: (n,), 6: (I64(63),), 7: (5,), 8: (n,), 9: (n,), 10: (n,), 11: (n,), 12: (I64(-1),), 13: (0,)}
    yield "norm_grad", [A, I64(64), A, A, A, A, A, A, I64(64), 2, A, A, I64(3), 64, A, big, n], {0: (n,), 1: (I64(3),), 2: (n,), 3: (n,), 4: (n,), 5: (n,), 6: (n,), 7: (n,), 8: (I64(3),), 9: (3,), 10: (P(0x10001),), 11: (P(0x10002),), 12: (I64(-1),), 13: (0,), 14: (n, P(0x10010))}


@pytest.mark.parametrize("name,valid,changes", list(_calls()), ids=lambda v: v if isinstance(v, str) else "")
def test_library_refuses(name, valid, changes):
    f = getattr(sq.lib, "sparq_mx_" + name)
    for at, values in changes.items():
        for v in values:
            args = list(valid)
            args[at] = v
            assert f(*args) == EINVAL, (at, v)


def test_small_workspaces_are_refused():
    f = sq.lib
    small = ctypes.c_size_t(16)
    assert f.sparq_mx_linear(A, 2, I64(64), A, A, None, A, 2, I64(8), I64(300), 8, 64, A, small, None) in (EWORKSPACE, EINVAL)
    assert f.sparq_mx_norm_grad(A, I64(64), A, A, A, A, A, A, I64(64), 2, A, A, I64(3), 64, A, small, None) == EWORKSPACE


def test_no_rows_are_no_work():
    f, n, z = sq.lib, None, I64(0)
    assert f.sparq_mx_quantize(n, 2, I64(64), z, 64, n, n, n, n, n) == OK
    assert f.sparq_mx_dequantize(n, n, 4, n, 2, I64(64), z, 64, n) == OK
    assert f.sparq_mx_gemm(n, n, n, n, n, n, 2, I64(8), z, 8, 64, n, ctypes.c_size_t(0), n) == OK
    assert f.sparq_mx_linear(n, 2, I64(64), n, n, n, n, 2, I64(8), z, 8, 64, n, ctypes.c_size_t(0), n) == OK
    assert f.sparq_mx_linear_dx(n, 2, I64(8), n, n, n, 2, I64(64), z, 8, 64, n, ctypes.c_size_t(0), n) == OK
    assert f.sparq_mx_act(0, n, I64(64), n, z, n, I64(64), 2, n, n, n, n, z, 64, n) == OK
    assert f.sparq_mx_act_grad(0, n, I64(64), n, n, n, n, n, I64(64), n, z, 2, z, 64, n) == OK
    assert f.sparq_mx_norm(n, I64(64), n, n, F32(0), n, I64(64), 2, n, n, n, n, z, 64, n) == OK


def test_more_rows_than_a_launch_counts():
    many = I64(1 << 31)
    assert sq.lib.sparq_mx_quantize(A, 2, I64(64), many, 64, A, A, None, None, None) == EUNSUPPORTED
    assert sq.lib.sparq_mx_norm(A, I64(64), A, None, F32(0), A, I64(64), 2, None, None, None, None, many, 64, None) == EUNSUPPORTED


X = torch.zeros(4, 64, dtype=torch.bfloat16)


@pytest.mark.parametrize("error,text,call", [
    (TypeError, "missing", lambda: sq.sparq_mx_quantize()),
    (TypeError, "unexpected keyword", lambda: sq.sparq_mx_quantize(X, z=1)),
    (TypeError, "must be a tensor", lambda: sq.sparq_mx_quantize(3)),
    (TypeError, "x must be a device tensor", lambda: sq.sparq_mx_quantize(X, X, X)),
    (ValueError, "positive", lambda: sq.sparq_mx_gemm(X, X, X, X, 0, X)),
    (ValueError, "bits must be 4 or 8", lambda: sq.sparq_mx_dequantize(X, X, 5, X)),
    (ValueError, "silu", lambda: sq.sparq_mx_act("relu", X, X)),
    (ValueError, "silu", lambda: sq.sparq_mx_act_grad(0, X, X, X, X)),
    (TypeError, "x must be a device tensor", lambda: sq.sparq_mx_norm(X, X, X, 1e-5, X)),
    (TypeError, "dy must be a device tensor", lambda: sq.sparq_mx_linear_dw(X, X, X, X)),
], ids=lambda v: v.__name__ if isinstance(v, type) else None)
def test_binding_refuses(error, text, call):
    with pytest.raises(error, match=text):
        call()
