"""The entry points of a block with experts without a GPU: what the header declares is exported and bound, workspaces, and refusals -- by the
library (nothing is launched; a call that got as far as a launch would return SPARQ_ELAUNCH here) and by the binding before the library is called."""
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
ODD1, ODD2, ODD4, ODD8 = P(0x10001), P(0x10002), P(0x10004), P(0x10008)
I64, F64, U64, SZ = ctypes.c_int64, ctypes.c_double, ctypes.c_uint64, ctypes.c_size_t
BIG = SZ(1 << 60)
n = None


def declared():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "sparq_mx_experts.h")).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(sparq_mx_[a-z0-9_]+)\s*\(", text)))


def test_declared_exported_and_bound():
    names = declared()
    assert len(names) == 14
    for name in names:
        assert hasattr(sq.lib, name) and hasattr(sq, name) and name in sq.__all__, name


# Name, a valid argument list, and which positions may not be changed to what.
CALLS = [
    ("sort", [A, I64(8), 4, A, A, n, n, SZ(0), n], {0: (n, ODD2), 1: (I64(-1),), 2: (0, -3), 3: (n, ODD2), 4: (n, ODD2), 5: (ODD1,)}),
    ("gather", [A, 2, I64(64), I64(3), 64, A, 2, A, I64(64), A, A, A, A, I64(6), n],
     {0: (n, ODD1), 1: (3, -1), 2: (I64(63),), 3: (I64(-1),), 4: (0, (1 << 28) + 1), 5: (n, ODD2), 6: (0,), 7: (ODD1,), 8: (I64(63),), 9: (n, ODD8), 10: (n,),
      11: (n, ODD8), 12: (n,), 13: (I64(-1),)}),
    ("gather", [A, 2, I64(64), I64(3), 64, A, 2, A, I64(64), n, n, n, n, I64(6), n], {7: (n,), 9: (A,), 11: (A,), 12: (A,)}),
    ("combine", [A, I64(64), I64(6), A, A, 2, A, I64(64), A, I64(64), 2, I64(3), 64, n],
     {0: (n, ODD1), 1: (I64(63),), 2: (I64(-1),), 3: (n, ODD2), 4: (ODD2,), 5: (0,), 6: (ODD1,), 7: (I64(63),), 8: (n, ODD1), 9: (I64(63),), 10: (3,), 11: (I64(-1),), 12: (0,)}),
    ("combine_grad", [A, I64(64), A, A, 2, A, I64(64), A, I64(64), I64(6), A, 2, I64(3), 64, n],
     {0: (n, ODD1), 1: (I64(63),), 2: (n, ODD2), 3: (n, ODD2), 4: (0,), 5: (ODD1,), 6: (I64(63),), 7: (n, ODD1), 8: (I64(63),), 9: (I64(-1),), 10: (ODD2,), 11: (7,), 12: (I64(-1),),
      13: (0,)}),
    ("combine_grad", [A, I64(64), A, n, 2, n, I64(0), A, I64(64), I64(6), A, 2, I64(3), 64, n], {5: (A,), 10: (n,)}),
    ("experts_gemm", [A, A, A, 100, A, A, A, 0, A, I64(8), A, 2, I64(8), A, A, I64(3000), 8, 64, A, BIG, n],
     {0: (n, ODD8), 1: (n,), 2: (n, ODD2), 3: (0, -1), 4: (n,), 5: (n,), 6: (ODD2,), 7: (-2, 2), 8: (ODD1,), 9: (I64(7),), 10: (n, ODD1), 11: (3,), 12: (I64(7),), 13: (n, ODD8),
      14: (n,), 15: (I64(-1),), 16: (0,), 17: (0, (1 << 23) + 1), 18: (n, P(0x10010))}),
    ("experts_linear", [A, 2, I64(64), A, 4, A, A, A, 1, A, I64(8), A, 2, I64(8), A, A, I64(300), 8, 64, A, BIG, n],
     {0: (n, ODD1), 1: (5,), 2: (I64(63),), 3: (n, ODD2), 4: (0,), 5: (n,), 6: (n,), 7: (ODD2,), 8: (-2, 2), 9: (ODD1,), 10: (I64(7),), 11: (n,), 12: (3,), 13: (I64(7),), 14: (n,),
      15: (n,), 16: (I64(-1),), 17: (0,), 18: (0,), 19: (n, P(0x10010))}),
    ("experts_dx", [A, 2, I64(8), A, 100, A, A, A, 2, I64(64), I64(300), 8, 64, A, BIG, n],
     {0: (n, ODD1), 1: (4,), 2: (I64(7),), 3: (n, ODD2), 4: (0,), 5: (n,), 6: (n,), 7: (n,), 8: (1, 4), 9: (I64(63),), 10: (I64(-1),), 11: (0,), 12: (0,), 13: (n, P(0x10010))}),
    ("experts_dw", [A, 2, I64(8), A, 4, A, A, A, 0, I64(64), A, I64(300), 8, 64, n, SZ(0), n],
     {0: (n, ODD1), 1: (4,), 2: (I64(7),), 3: (n, ODD2), 4: (0,), 5: (n,), 6: (n,), 7: (n, ODD2), 8: (1, 4), 9: (I64(63),), 10: (ODD2,), 11: (I64(-1),), 12: (0,), 13: (0,)}),
    ("dropout", [A, I64(64), F64(0.5), U64(1), U64(2), A, A, I64(64), A, I64(64), 2, I64(3), 64, n],
     {0: (n, ODD1), 1: (I64(63),), 2: (F64(-0.1), F64(1.1), F64(float("nan"))), 5: (ODD4,), 6: (ODD1,), 7: (I64(63),), 8: (n,), 9: (I64(63),), 10: (3,), 11: (I64(-1),), 12: (0,)}),
]


@pytest.mark.parametrize("name,valid,changes", CALLS, ids=lambda v: v if isinstance(v, str) else "")
def test_library_refuses(name, valid, changes):
    f = getattr(sq.lib, "sparq_mx_" + name)
    for at, values in changes.items():
        for v in values:
            args = list(valid)
            args[at] = v
            assert f(*args) == EINVAL, (at, v)


# The same argument lists with more of something than a call counts: refused for that alone, so that all else is valid.
@pytest.mark.parametrize("call,at,value", [(0, 1, I64((1 << 30) + 1)), (0, 2, 1025), (1, 3, I64(1 << 31)), (2, 3, I64(1 << 31)), (3, 11, I64(1 << 31)), (4, 12, I64(1 << 31)), (5, 12, I64(1 << 31)),
                                           (6, 15, I64(1 << 31)), (6, 3, 1025), (7, 16, I64(1 << 31)), (7, 4, 1025), (8, 10, I64(1 << 31)), (8, 4, 1025), (9, 11, I64(1 << 31)), (9, 4, 1025),
                                           (10, 11, I64(1 << 31))])
def test_more_than_a_call_counts(call, at, value):
    name, args, _ = CALLS[call]
    args = list(args)
    args[at] = value
    assert getattr(sq.lib, "sparq_mx_" + name)(*args) == EUNSUPPORTED


@pytest.mark.parametrize("call,at", [(1, 6), (2, 6), (3, 5), (4, 4), (5, 4)])
def test_more_slots_a_token_than_a_call_counts(call, at):
    """Their number and four more have to fit 32 bits."""
    name, args, _ = CALLS[call]
    for per in ((1 << 30) + 1, (1 << 31) - 1):
        args = list(args)
        args[at] = per
        assert getattr(sq.lib, "sparq_mx_" + name)(*args) == EUNSUPPORTED


def test_an_expert_without_offsets_is_alone():
    name, args, _ = CALLS[6]
    args = list(args)
    args[2], args[3] = n, 2
    assert sq.lib.sparq_mx_experts_gemm(*args) == EINVAL
    args[3], args[15] = 1, I64(1 << 31)
    assert sq.lib.sparq_mx_experts_gemm(*args) == EUNSUPPORTED


def test_more_results_than_a_launch_counts():
    M, N, K, E = 1 << 30, 1 << 20, 64, 4
    assert sq.lib.sparq_mx_experts_gemm(A, A, A, E, A, A, n, -1, n, I64(0), A, 2, I64(N), n, n, I64(M), N, K, A, BIG, n) == EUNSUPPORTED
    assert sq.lib.sparq_mx_experts_linear(A, 2, I64(K), A, E, A, A, n, -1, n, I64(0), A, 2, I64(N), n, n, I64(M), N, K, A, BIG, n) == EUNSUPPORTED
    assert sq.lib.sparq_mx_experts_dx(A, 2, I64(64), A, E, A, A, A, 2, I64(1 << 24), I64(M), 64, 1 << 24, A, BIG, n) == EUNSUPPORTED
    assert sq.lib.sparq_mx_experts_dw(A, 2, I64(1 << 28), A, 4, A, A, A, 0, I64(1 << 20), n, I64(300), 1 << 28, 1 << 20, n, SZ(0), n) == EUNSUPPORTED
    assert sq.lib.sparq_mx_experts_gemm(A, A, A, 16, A, A, n, -1, n, I64(0), A, 2, I64(1 << 28), n, n, I64(4), 1 << 28, K, A, BIG, n) == EUNSUPPORTED


# One byte less than the query names, everything else valid: EWORKSPACE and nothing else; sizes whose plan takes all of it.
def _workspaces():
    yield "sort", (A, I64(300000), 256, A, A, n), (300000, 256)
    yield "experts_gemm", (A, A, A, 100, A, A, n, -1, n, I64(0), A, 2, I64(8), n, n, I64(3000), 8, 1 << 20), (3000, 8, 1 << 20, 100)
    yield "experts_gemm", (A, A, n, 1, A, A, n, -1, n, I64(0), A, 2, I64(100), n, n, I64(70), 100, 8300), (70, 100, 8300, 1)
    yield "experts_linear", (A, 2, I64(1 << 20), A, 4, A, A, n, -1, n, I64(0), A, 2, I64(8), n, n, I64(3000), 8, 1 << 20), (3000, 8, 1 << 20, 4)
    yield "experts_dx", (A, 2, I64(8), A, 100, A, A, A, 2, I64(64), I64(300), 8, 64), (300, 8, 64, 100)


@pytest.mark.parametrize("name,args,sizes", list(_workspaces()), ids=lambda v: v if isinstance(v, str) else "")
def test_a_workspace_one_byte_short(name, args, sizes):
    f, need = getattr(sq.lib, "sparq_mx_" + name), getattr(sq, "sparq_mx_%s_workspace_bytes" % name)(*sizes)
    assert need > 0
    for short in (0, need - 1):
        assert f(*args, A, SZ(short), None) == EWORKSPACE
    for bad in (None, P(0x10010)):
        assert f(*args, bad, SZ(need), None) == EINVAL


def test_no_rows_are_no_work():
    f, z, zero = sq.lib, I64(0), SZ(0)
    assert f.sparq_mx_gather(n, 2, I64(64), z, 64, n, 2, n, z, n, n, n, n, I64(5), n) == OK
    assert f.sparq_mx_gather(A, 2, I64(64), I64(3), 64, A, 2, n, z, n, n, n, n, z, n) == OK
    assert f.sparq_mx_combine(n, z, z, n, n, 2, n, z, n, z, 2, z, 64, n) == OK
    assert f.sparq_mx_combine_grad(n, z, n, n, 2, n, z, n, z, z, n, 2, z, 64, n) == OK
    assert f.sparq_mx_combine_grad(A, I64(64), A, A, 2, n, z, n, z, z, n, 2, I64(3), 64, n) == OK
    assert f.sparq_mx_experts_gemm(n, n, A, 4, n, n, n, -1, n, z, n, 2, z, n, n, z, 8, 64, n, zero, n) == OK
    assert f.sparq_mx_experts_linear(n, 2, z, A, 4, n, n, n, -1, n, z, n, 2, z, n, n, z, 8, 64, n, zero, n) == OK
    assert f.sparq_mx_experts_dx(n, 2, z, A, 4, n, n, n, 2, z, z, 8, 64, n, zero, n) == OK
    assert f.sparq_mx_dropout(n, z, F64(0.5), U64(0), U64(0), n, n, z, n, z, 2, z, 64, n) == OK


def test_workspaces_of_wrong_sizes_are_none():
    assert sq.sparq_mx_sort_workspace_bytes(-1, 4) == sq.sparq_mx_sort_workspace_bytes(4, 0) == sq.sparq_mx_sort_workspace_bytes(1 << 40, 4) == 0
    for f in (sq.sparq_mx_experts_gemm_workspace_bytes, sq.sparq_mx_experts_linear_workspace_bytes, sq.sparq_mx_experts_dx_workspace_bytes, sq.sparq_mx_experts_dw_workspace_bytes):
        for sizes in ((-1, 64, 64, 4), (64, 0, 64, 4), (64, 64, 0, 4), (64, 64, 64, 0)):
            assert f(*sizes) == 0


X = torch.zeros(4, 64, dtype=torch.bfloat16)


@pytest.mark.parametrize("error,text,call", [
    (TypeError, "missing", lambda: sq.sparq_mx_sort(X)),
    (TypeError, "unexpected keyword", lambda: sq.sparq_mx_gather(X, X, z=1)),
    (TypeError, "must be a tensor", lambda: sq.sparq_mx_combine(X, 3, 4)),
    (TypeError, "expert must be a device tensor", lambda: sq.sparq_mx_sort(X, X, X)),
    (TypeError, "x must be a device tensor", lambda: sq.sparq_mx_gather(X, X, X)),
    (TypeError, "dy must be a device tensor", lambda: sq.sparq_mx_combine_grad(X, X, X, X)),
    (ValueError, "positive", lambda: sq.sparq_mx_experts_gemm(X, X, X, X, 0, X)),
    (TypeError, "x must be a device tensor", lambda: sq.sparq_mx_experts_linear(X, X, X, X)),
    (TypeError, "dy must be a device tensor", lambda: sq.sparq_mx_experts_dx(X, X, X, X, X)),
    (TypeError, "dy must be a device tensor", lambda: sq.sparq_mx_experts_dw(X, X, X, X, X)),
    (TypeError, "x must be a device tensor", lambda: sq.sparq_mx_dropout(X, 0.5, 1, X)),
], ids=lambda v: v.__name__ if isinstance(v, type) else None)
def test_binding_refuses(error, text, call):
    with pytest.raises(error, match=text):
        call()
