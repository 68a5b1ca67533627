"""The microscaled operators on the GPU against the plain reference in 64 bits (tests/mx_reference.py).

Tolerances, fixed before any run.  u = 2^-24 is fp32's unit roundoff, U the result type's (2^-24, 2^-11, 2^-8), and every result is
rounded once: U |ref|, for fp16 at least half a subnormal step (2^-25).
  codec         to the bit
  products      a sum of n exact products made in any order and rounded at most once an addition: (n + 2) u sum|a||b|; twice that
                for an adder that truncates where it aligns
  activations   a few roundings of fp32 and an exponential of a relative error of (2 + |v|) u: stated at the test
  norm          statistics from sums of depth d = K / 64 + 16
"""
import numpy as np
import pytest
import torch

import mx_reference as R

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
u = 2.0 ** -24


@pytest.fixture(scope="module")
def sq():
    assert torch.cuda.is_available(), "GPU tests need a device"
    import paper_2105_11010_amd as sq_
    return sq_


R_quantised = R.quantised


def rng(*seed):
    return np.random.default_rng([20210511, *seed])


def values(g, rows, K, t, spread=1.0):
    """Values that a tensor of type t holds, as float64: channels of different spread."""
    x = g.standard_normal((rows, K)) * np.exp(0.7 * g.standard_normal(K)) * spread
    return torch.from_numpy(x).to(TYPES[t]).double().numpy()


def matrix(x, t, pad=0, at=0, fill=None):
    """x on the device as columns `at` and on of a wider tensor (a row stride of x's width + pad + at)."""
    rows, K = x.shape
    wide = torch.full((rows, K + pad + at), float("nan") if fill is None else fill, dtype=TYPES[t], device=DEV)
    v = wide[:, at: at + K]
    v.copy_(torch.from_numpy(np.ascontiguousarray(x)).to(TYPES[t]))
    return v


class Result:
    """A result tensor inside a wider one whose other elements have to stay as they are."""

    def __init__(self, rows, K, t, pad=0, at=0):
        self.wide = torch.full((rows + 1, K + pad + at), 77.0, dtype=TYPES[t], device=DEV)
        self.view = self.wide[:rows, at: at + K]
        self.view.fill_(-55.0)

    def get(self):
        torch.cuda.synchronize()
        rows, K = self.view.shape
        mask = torch.ones_like(self.wide, dtype=torch.bool)
        at = self.view.storage_offset()
        mask[:rows, at: at + K] = False
        assert bool((self.wide[mask] == 77).all()), "written outside the result"
        return self.view.double().cpu().numpy()


class Bytes:
    """A buffer of bytes with a guard behind it."""

    def __init__(self, rows, pitch):
        self.all = torch.full((rows * pitch + 256,), 0xA5, dtype=torch.uint8, device=DEV)
        self.t = self.all[: rows * pitch].view(rows, pitch)

    def get(self):
        torch.cuda.synchronize()
        assert bool((self.all[self.t.numel():] == 0xA5).all()), "written past the buffer"
        return self.t.cpu().numpy()


def coded_buffers(sq, rows, K, bits):
    return Bytes(rows, sq.sparq_mx_code_bytes(K, bits)), Bytes(rows, sq.sparq_mx_scale_bytes(K))


def stored(sq, x, bits):
    """x encoded by the reference, as device buffers."""
    rows, K = x.shape
    c, s = R.store(*R.encode(x, bits), bits, sq.sparq_mx_code_bytes(K, bits), sq.sparq_mx_scale_bytes(K))
    return torch.from_numpy(c).to(DEV), torch.from_numpy(s).to(DEV)


def workspace(nbytes):
    ws = torch.full((nbytes + 256,), 0x5A, dtype=torch.uint8, device=DEV)
    return ws, ws[:nbytes]


def guard(ws, view):
    torch.cuda.synchronize()
    assert bool((ws[view.numel():] == 0x5A).all()), "written past the workspace"


def close(got, ref, bound, t):
    bound = bound + UNIT[t] * np.abs(ref) * (1 + 2 ** -7) + (2.0 ** -25 if t == "f16" else 0.0)
    wrong = ~(np.abs(got - ref) <= bound)
    assert not wrong.any(), f"{wrong.sum()} of {wrong.size} off, worst {np.nanmax(np.abs(got - ref) / np.maximum(bound, 1e-300))} of the bound, first at {np.argwhere(wrong)[0]}"


# ---- codec -----------------------------------------------------------------------------------------------------------
CODEC = [(1, 1), (3, 31), (2, 32), (5, 33), (4, 127), (3, 128), (2, 129), (3, 504), (2, 511), (2, 512), (3, 513), (7, 1000), (1, 4096), (2, 2057)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows,K", CODEC)
@pytest.mark.parametrize("pad,at", [(0, 0), (5, 3)])
def test_codec(sq, t, rows, K, pad, at):
    x = values(rng(1, rows, K), rows, K, t)
    xd = matrix(x, t, pad, at)
    both = coded_buffers(sq, rows, K, 4) + coded_buffers(sq, rows, K, 8)
    sq.sparq_mx_quantize(xd, *[b.t for b in both])
    for bits in (4, 8):
        ref = R.encode(x, bits)
        c, s = R.store(*ref, bits, sq.sparq_mx_code_bytes(K, bits), sq.sparq_mx_scale_bytes(K))
        one = coded_buffers(sq, rows, K, bits)
        sq.sparq_mx_quantize(xd, **{f"codes{bits}": one[0].t, f"scales{bits}": one[1].t})
        for got in (one, both[:2] if bits == 4 else both[2:]):
            assert np.array_equal(got[0].get(), c) and np.array_equal(got[1].get(), s)
        y = Result(rows, K, t, pad, at)
        sq.sparq_mx_dequantize(one[0].t, one[1].t, bits, y.view)
        want = torch.from_numpy(R.decode(*ref, bits)).to(TYPES[t]).double().numpy()
        assert np.array_equal(y.get(), want)


@pytest.mark.parametrize("bits", (4, 8))
def test_codec_at_the_edges(sq, bits):
    """Ties, saturation, zeros of either sign, subnormal and largest blocks, NaN and infinity: a block each."""
    g = rng(2)
    blocks = [np.array([6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -.75, -5, 7, 7.9, 0.5, 0, -0.0] * 2),
              np.zeros(32), -np.zeros(32), np.array([1.0] + [(2 * i + 1) / 128 for i in range(31)]),
              g.standard_normal(32) * 2.0 ** -127, g.standard_normal(32) * 2.0 ** -140, np.array([2.0 ** -149] + [0.0] * 31),
              np.array([2.0 ** -126] + [2.0 ** -133] * 31), np.array([1.999 * 2.0 ** 127] + [1.0] * 31), np.array([-(2.0 ** 127)] * 32),
              np.array([np.inf] + [1.0] * 31), np.array([1.0] * 31 + [-np.inf]), np.array([1.0] * 15 + [np.nan] + [1.0] * 16), np.arange(32) - 15.5]
    x = torch.from_numpy(np.concatenate(blocks)[None]).float()
    c, s = coded_buffers(sq, 1, x.shape[1], bits)
    sq.sparq_mx_quantize(x.to(DEV), **{f"codes{bits}": c.t, f"scales{bits}": s.t})
    codes, scales = R.encode(x.double().numpy(), bits)
    rc, rs = R.store(codes, scales, bits, c.t.shape[1], s.t.shape[1])
    assert np.array_equal(s.get(), rs) and np.array_equal(c.get(), rc)
    y = torch.empty_like(x, device=DEV)
    sq.sparq_mx_dequantize(c.t, s.t, bits, y)
    assert np.array_equal(y.double().cpu().numpy(), R.decode(codes, scales, bits).astype(np.float32).astype(np.float64), equal_nan=True)


# ---- product -----------------------------------------------------------------------------------------------------------
# sizes of one, around the tiles' and the steps' edges, and rows that no tile divides
PRODUCT = [(1, 1, 1), (1, 16, 33), (1, 300, 1000), (2, 64, 128), (5, 130, 257), (16, 48, 512), (17, 33, 640), (31, 257, 129), (33, 1000, 384),
           (64, 64, 64), (65, 129, 1300), (130, 70, 2100), (257, 255, 511), (300, 520, 1024), (1, 513, 4224), (8, 96, 8200), (600, 700, 96)]


@pytest.mark.parametrize("M,N,K", PRODUCT)
@pytest.mark.parametrize("t,bias,pad,at", [("bf16", False, 0, 0), ("f32", True, 3, 1), ("f16", True, 0, 0), ("bf16", True, 8, 5)])
def test_product(sq, M, N, K, t, bias, pad, at):
    g = rng(3, M, N, K)
    x, w = values(g, M, K, t), values(g, N, K, "f32", K ** -0.5)
    b = g.standard_normal(N).astype(np.float32) if bias else None
    X, W = R.quantised(x, 4), R.quantised(w, 4)
    ref = X @ W.T + (b if bias else 0.0)
    bound = 2 * (K + 3) * u * (np.abs(X) @ np.abs(W).T + (np.abs(b) if bias else 0.0))
    wd, bd = stored(sq, w, 4), torch.from_numpy(b).to(DEV) if bias else None
    xd = stored(sq, x, 4)
    y = Result(M, N, t, pad, at)
    ws, view = workspace(sq.sparq_mx_gemm_workspace_bytes(M, N, K))
    sq.sparq_mx_gemm(*xd, *wd, K, y.view, bias=bd, workspace=view)
    close(y.get(), ref, bound, t)
    guard(ws, view)
    y = Result(M, N, t, pad, at)
    ws, view = workspace(sq.sparq_mx_linear_workspace_bytes(M, N, K))
    sq.sparq_mx_linear(matrix(x, t, pad, at), *wd, y.view, bias=bd, workspace=view)
    close(y.get(), ref, bound, t)
    guard(ws, view)


# many results, so that the largest tiles are used: whole ones, cut ones, and reductions that end inside a step or before the first ends
@pytest.mark.parametrize("M,N,K", [(4100, 3300, 100), (4096, 3328, 640), (3333, 4001, 1500), (1500, 1300, 700), (1409, 1300, 129), (2001, 960, 1100)])
@pytest.mark.parametrize("t,bias", [("bf16", True), ("f32", False)])
def test_product_in_large_tiles(sq, M, N, K, t, bias):
    test_product(sq, M, N, K, t, bias, 0, 0)


# few results of a long reduction, which is divided; few rows whose weights are too many for x to be quantised on the way; most of the few rows
@pytest.mark.parametrize("M,N,K", [(70, 100, 8300), (130, 65, 9000), (16, 3000, 3000), (64, 515, 2056), (49, 2000, 1100), (15, 53, 128), (7, 40, 5), (13, 65, 735), (6, 33, 1031)])
@pytest.mark.parametrize("t,bias,pad,at", [("bf16", True, 0, 0), ("f32", False, 3, 1)])
def test_product_of_other_shapes(sq, M, N, K, t, bias, pad, at):
    test_product(sq, M, N, K, t, bias, pad, at)


@pytest.mark.parametrize("M,N,K", [(1, 40, 300), (40, 70, 300), (300, 300, 700)])
def test_product_of_what_is_not_finite(sq, M, N, K):
    """A NaN or an infinity makes its row (of x) or column (of w) NaN and nothing else."""
    g = rng(4, M, N, K)
    x, w = values(g, M, K, "bf16"), values(g, N, K, "f32")
    x[M // 2, K - 1] = np.inf
    w[N - 1, 0] = np.nan
    y = Result(M, N, "f32")
    ws = workspace(sq.sparq_mx_linear_workspace_bytes(M, N, K))[1]
    sq.sparq_mx_linear(matrix(x, "bf16"), *stored(sq, w, 4), y.view, workspace=ws)
    got = y.get()
    nan = np.zeros((M, N), bool)
    nan[M // 2], nan[:, N - 1] = True, True
    assert np.array_equal(np.isnan(got), nan)
    X, W = R.quantised(x, 4), R.quantised(w, 4)
    keep = [m for m in range(M) if m != M // 2]
    ref = X[keep] @ W[:-1].T
    close(got[keep][:, :-1], ref, 2 * (K + 3) * u * (np.abs(X[keep]) @ np.abs(W[:-1]).T), "f32")


# ---- the product's gradients ---------------------------------------------------------------------------------------------
GRAD = [(1, 1, 1), (3, 5, 33), (17, 64, 128), (64, 33, 100), (40, 129, 257), (130, 96, 640), (257, 300, 130), (515, 70, 200), (96, 1030, 64), (1300, 40, 72),
        (256, 512, 512), (2100, 70, 96), (70, 2100, 96)]


@pytest.mark.parametrize("M,N,K", GRAD)
@pytest.mark.parametrize("t,o,pad,at", [("bf16", "bf16", 0, 0), ("f16", "f32", 3, 1), ("f32", "f32", 0, 0), ("bf16", "f16", 8, 5), ("f32", "bf16", 1, 0)])
def test_product_gradients(sq, M, N, K, t, o, pad, at):
    g = rng(5, M, N, K)
    x, w, dy = values(g, M, K, "bf16"), values(g, N, K, "f32", K ** -0.5), values(g, M, N, t, 0.1)
    X, W = R.quantised(x, 8), R.quantised(w, 4)
    dyd = matrix(dy, t, pad, at)
    parts = {"bf16": 1, "f16": 2, "f32": 3}[t]
    dx = Result(M, K, o, pad, at)
    ws, view = workspace(sq.sparq_mx_linear_dx_workspace_bytes(M, N, K))
    sq.sparq_mx_linear_dx(dyd, *stored(sq, w, 4), dx.view, workspace=view)
    close(dx.get(), dy @ W, 2 * (parts * N + 2) * u * (np.abs(dy) @ np.abs(W)), o)
    guard(ws, view)
    dw, db = Result(N, K, o, pad, at), torch.full((N + 64,), 9.0, device=DEV)
    ws, view = workspace(sq.sparq_mx_linear_dw_workspace_bytes(M, N, K))
    sq.sparq_mx_linear_dw(dyd, *stored(sq, x, 8), dw.view, db=db[:N], workspace=view)
    close(dw.get(), dy.T @ X, 2 * (parts * M + 2) * u * (np.abs(dy).T @ np.abs(X)), o)
    close(db[:N].double().cpu().numpy(), dy.sum(0), (M + 2) * u * np.abs(dy).sum(0), "f32")
    assert bool((db[N:] == 9).all())
    guard(ws, view)


@pytest.mark.parametrize("J,R,K", [(4100, 205, 3300), (4096, 64, 3328), (4104, 40, 3201), (3336, 512, 4000), (4104, 333, 3400), (2056, 205, 1700), (264, 3300, 3000), (4099, 257, 3201), (2049, 129, 1730), (261, 3300, 3000), (1600, 4100, 1700)])
@pytest.mark.parametrize("o,pad,at", [("bf16", 0, 0), ("f32", 6, 2), ("f16", 4, 1)])
def test_product_gradients_in_large_tiles(sq, J, R, K, o, pad, at, t="bf16"):
    """dx [J][K] over R outputs, dw [J][K] over R rows."""
    g = rng(13, J, R, K)
    V, d = values(g, R, K, "bf16"), values(g, J, R, t, 0.1)
    parts = {"bf16": 1, "f16": 2, "f32": 3}[t]
    for bits in (4, 8):
        ref = R_quantised(V, bits)
        out = Result(J, K, o, pad, at)
        if bits == 4:
            ws, view = workspace(sq.sparq_mx_linear_dx_workspace_bytes(J, R, K))
            sq.sparq_mx_linear_dx(matrix(d, t, pad, at), *stored(sq, V, 4), out.view, workspace=view)
        else:
            ws, view = workspace(sq.sparq_mx_linear_dw_workspace_bytes(R, J, K))
            sq.sparq_mx_linear_dw(matrix(d.T, t, pad, at), *stored(sq, V, 8), out.view, workspace=view)
        close(out.get(), d @ ref, 2 * (parts * R + 2) * u * (np.abs(d) @ np.abs(ref)), o)
        guard(ws, view)


@pytest.mark.parametrize("J,R,K", [(2056, 205, 1700), (2049, 129, 1730), (264, 3300, 3000), (261, 3299, 3000), (2048, 64, 1664), (1600, 4100, 1700)])
@pytest.mark.parametrize("t,o,pad,at", [("f16", "f32", 0, 0), ("f32", "f32", 0, 0), ("f16", "f16", 5, 1), ("f32", "bf16", 3, 2)])
def test_product_gradients_of_wider_types(sq, J, R, K, t, o, pad, at):
    test_product_gradients_in_large_tiles(sq, J, R, K, o, pad, at, t)


# fewer columns of dy than a read takes, whose reads run on into the next rows; bias gradients of a few rows, of slabs, and of many elements
@pytest.mark.parametrize("M,N,K", [(700, 1, 300), (577, 2, 128), (640, 5, 64), (131, 7, 100), (900, 9, 130), (1000, 200, 333), (24, 3008, 49), (1757, 300, 114), (2100, 2100, 64), (1040, 4101, 33)])
@pytest.mark.parametrize("t,o,pad,at", [("bf16", "f32", 0, 0), ("f16", "f16", 1, 0), ("f32", "f32", 0, 0)])
def test_product_gradients_of_few_columns(sq, M, N, K, t, o, pad, at):
    test_product_gradients(sq, M, N, K, t, o, pad, at)


def test_product_gradients_are_the_differences(sq):
    """The loss sum(y * dy) is linear in the codes' values: its differences are exact, so the kernel's gradients are held to them."""
    g = rng(6)
    M, N, K = 7, 9, 40
    X, W, dy = R.quantised(g.standard_normal((M, K)), 8), R.quantised(g.standard_normal((N, K)), 4), values(g, M, N, "f32")
    dx, dw = Result(M, K, "f32"), Result(N, K, "f32")
    dyd = matrix(dy, "f32")
    sq.sparq_mx_linear_dx(dyd, *stored(sq, W, 4), dx.view, workspace=workspace(sq.sparq_mx_linear_dx_workspace_bytes(M, N, K))[1])
    sq.sparq_mx_linear_dw(dyd, *stored(sq, X, 8), dw.view, workspace=workspace(sq.sparq_mx_linear_dw_workspace_bytes(M, N, K))[1])
    loss = lambda X, W: ((X @ W.T) * dy).sum()      # noqa: E731
    dx, dw, base = dx.get(), dw.get(), loss(X, W)
    for i, j in ((0, 0), (M - 1, K - 1), (3, 31), (4, 32)):
        e = np.zeros_like(X)
        e[i, j] = 1.0
        assert abs(loss(X + e, W) - base - dx[i, j]) < 1e-5
    for i, j in ((0, 0), (N - 1, K - 1), (3, 31), (4, 32)):
        e = np.zeros_like(W)
        e[i, j] = 1.0
        assert abs(loss(X, W + e) - base - dw[i, j]) < 1e-5


@pytest.mark.parametrize("M,N,K", [(40, 70, 130), (300, 260, 300)])
def test_product_gradients_of_what_is_not_finite(sq, M, N, K):
    g = rng(7, M, N, K)
    x, w, dy = values(g, M, K, "f32"), values(g, N, K, "f32"), values(g, M, N, "f32")
    w[N - 1, K - 1], x[M - 1, 0] = np.nan, np.inf
    dx, dw = Result(M, K, "f32"), Result(N, K, "f32")
    sq.sparq_mx_linear_dx(matrix(dy, "f32"), *stored(sq, w, 4), dx.view, workspace=workspace(sq.sparq_mx_linear_dx_workspace_bytes(M, N, K))[1])
    sq.sparq_mx_linear_dw(matrix(dy, "f32"), *stored(sq, x, 8), dw.view, workspace=workspace(sq.sparq_mx_linear_dw_workspace_bytes(M, N, K))[1])
    nan = np.zeros(K, bool)
    nan[(K - 1) // 32 * 32:] = True
    assert np.array_equal(np.isnan(dx.get()), np.broadcast_to(nan, (M, K)))
    nan = np.zeros(K, bool)
    nan[:32] = True
    assert np.array_equal(np.isnan(dw.get()), np.broadcast_to(nan, (N, K)))
    dy[M // 2, N // 2] = np.inf
    w[N - 1, K - 1], x[M - 1, 0] = 1.0, 1.0
    sq.sparq_mx_linear_dx(matrix(dy, "f32"), *stored(sq, w, 4), dx.view, workspace=workspace(sq.sparq_mx_linear_dx_workspace_bytes(M, N, K))[1])
    got = dx.get()
    assert not np.isfinite(got[M // 2][R.quantised(w, 4)[N // 2] != 0]).any() and np.isfinite(np.delete(got, M // 2, 0)).all()


def test_no_rows_give_gradients_of_zero(sq):
    N, K = 70, 90
    dy, e = torch.empty(0, N, dtype=torch.bfloat16, device=DEV), torch.empty(0, dtype=torch.uint8, device=DEV)
    dw, db = Result(N, K, "f32"), torch.full((N,), 9.0, device=DEV)
    ws = workspace(sq.sparq_mx_linear_dw_workspace_bytes(0, N, K))[1]
    sq.sparq_mx_linear_dw(dy, e, e, dw.view, db=db, workspace=ws)
    assert not dw.get().any() and not db.any()
    dgamma, dbeta, none = torch.full((K,), 9.0, device=DEV), torch.full((K,), 9.0, device=DEV), torch.empty(0, device=DEV)
    x = torch.empty(0, K, device=DEV)
    sq.sparq_mx_norm_grad(x, e, e, none, none, torch.ones(K, device=DEV), x, dgamma, dbeta)
    assert not dgamma.any() and not dbeta.any()


# ---- activations -----------------------------------------------------------------------------------------------------------
ROWS = [(1, 1), (3, 31), (2, 129), (5, 511), (3, 512), (2, 513), (4, 2049), (130, 96), (1, 9000)]


@pytest.mark.parametrize("name", ("silu", "gelu"))
@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows,K", ROWS)
@pytest.mark.parametrize("pad,at", [(0, 0), (7, 1)])
def test_act(sq, name, t, rows, K, pad, at):
    """The value: exponential and quotient are off by (2 + |v|) u and a few u, relatively; the 16-bit tensors' gelu goes through
    1 + erf, whose error is 4 u absolutely.  The slope: the same, times 1 + |v|."""
    g = rng(8, rows, K)
    gate, up, dy = values(g, rows, K, t, 2.0), values(g, rows, K, t), values(g, rows, K, t, 0.1)
    gc, uc = coded_buffers(sq, rows, K, 8), coded_buffers(sq, rows, K, 8)
    y, plain = Result(rows, K, t, pad, at), Result(rows, K, t)
    gd, ud = matrix(gate, t, pad, at), matrix(up, t, pad, at)
    sq.sparq_mx_act(name, gd, y.view, up=ud, gate_codes=gc[0].t, gate_scales=gc[1].t, up_codes=uc[0].t, up_scales=uc[1].t)
    sq.sparq_mx_act(name, gd, plain.view)
    f = R.function(name, gate)
    error = lambda v, f: 16 * u * ((2 + np.abs(v)) * np.abs(f) + (np.abs(v) if name == "gelu" else 0) + 2.0 ** -126)      # noqa: E731
    close(y.get(), f * up, error(gate, f) * np.abs(up), t)
    close(plain.get(), f, error(gate, f), t)
    for got, x in ((gc, gate), (uc, up)):
        c, s = R.store(*R.encode(x, 8), 8, got[0].t.shape[1], got[1].t.shape[1])
        assert np.array_equal(got[0].get(), c) and np.array_equal(got[1].get(), s)
    G, U = R.quantised(gate, 8), R.quantised(up, 8)
    f, d = R.function(name, G), R.slope(name, G)
    dg, du, dp = Result(rows, K, t, pad, at), Result(rows, K, t, pad, at), Result(rows, K, t)
    dyd = matrix(dy, t, pad, at)
    sq.sparq_mx_act_grad(name, dyd, gc[0].t, gc[1].t, dg.view, up_codes=uc[0].t, up_scales=uc[1].t, dup=du.view)
    sq.sparq_mx_act_grad(name, dyd, gc[0].t, gc[1].t, dp.view)
    off = 16 * u * (2 + np.abs(G)) * (1 + np.abs(G))
    close(dg.get(), dy * U * d, off * np.abs(dy * U), t)
    close(du.get(), dy * f, (error(G, f) + 4 * u * np.abs(f)) * np.abs(dy), t)
    close(dp.get(), dy * d, off * np.abs(dy), t)


def test_act_at_the_edges(sq):
    """Far out both functions are 0 and v, without NaN on the way; checkpoints of what is not finite are NaN, block by block."""
    v = np.array([[-1e4, -200, -88, -20, 0, 20, 88, 200, 1e4] + [0.0] * 23 + [np.inf] + [1.0] * 31 + [2.0] * 32])
    for name in ("silu", "gelu"):
        for t in ("f32", "bf16"):
            c, s = coded_buffers(sq, 1, 96, 8)
            y = Result(1, 96, t)
            sq.sparq_mx_act(name, matrix(v, t), y.view, gate_codes=c.t, gate_scales=s.t)
            got = y.get()[0]
            x = torch.from_numpy(v).to(TYPES[t]).double().numpy()[0]
            assert np.all(np.abs(got[:3]) < 1e-30) and np.array_equal(got[6:9], x[6:9]) and got[4] == 0
            dg = Result(1, 96, t)
            sq.sparq_mx_act_grad(name, matrix(np.ones((1, 96)), t), c.t, s.t, dg.view)
            d = dg.get()[0]
            assert np.isfinite(d[:32]).all() and np.isnan(d[32:64]).all() and np.isfinite(d[64:]).all()
            assert d[8] == 1 and d[0] == 0


# ---- norm --------------------------------------------------------------------------------------------------------------------
NORM = ROWS + [(9, 1000), (5, 1025), (3, 4096), (70, 4100), (300, 520), (3, 8191), (2, 20000)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows,K", NORM)
@pytest.mark.parametrize("pad,at", [(0, 0), (7, 1)])
def test_norm(sq, t, rows, K, pad, at):
    g = rng(9, rows, K)
    eps = 1e-5
    x, dy = values(g, rows, K, t) + 0.5, values(g, rows, K, t, 0.1)
    x = torch.from_numpy(x).to(TYPES[t]).double().numpy()
    gamma, beta = (1 + 0.2 * g.standard_normal(K)).astype(np.float32), g.standard_normal(K).astype(np.float32)
    gd, bd = torch.from_numpy(gamma).to(DEV), torch.from_numpy(beta).to(DEV)
    c, s = coded_buffers(sq, rows, K, 8)
    mean, rstd = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    y, bare = Result(rows, K, t, pad, at), Result(rows, K, t)
    xd = matrix(x, t, pad, at)
    sq.sparq_mx_norm(xd, gd, bd, eps, y.view, mean=mean, rstd=rstd, codes=c.t, scales=s.t)
    sq.sparq_mx_norm(xd, gd, None, eps, bare.view)
    ref, mu, r = R.norm(x, gamma, beta, eps)
    d = K / 64 + 16
    off_mean = d * u * np.abs(x).mean(1, keepdims=True)
    off_r = r * (d * u + (off_mean * r) ** 2)                        # (the squares' sum is off by d u, and by the mean's error squared)
    off = np.abs(gamma) * (r * off_mean + np.abs(x - mu) * off_r) + 6 * u * (np.abs((x - mu) * r * gamma) + np.abs(ref))
    assert np.all(np.abs(mean.double().cpu().numpy() - mu[:, 0]) <= off_mean[:, 0] + u * np.abs(mu[:, 0]))
    assert np.all(np.abs(rstd.double().cpu().numpy() - r[:, 0]) <= off_r[:, 0] + 4 * u * r[:, 0])
    close(y.get(), ref, off, t)
    close(bare.get(), ref - beta, off + u * np.abs(beta), t)
    rc, rs = R.store(*R.encode(x, 8), 8, c.t.shape[1], s.t.shape[1])
    assert np.array_equal(c.get(), rc) and np.array_equal(s.get(), rs)
    # backward, from the statistics the forward pass wrote
    X, mu, r = R.quantised(x, 8), mean.double().cpu().numpy()[:, None], rstd.double().cpu().numpy()[:, None]
    dx_ref, dgamma_ref, dbeta_ref = R.norm_grad(dy, X, mu, r, gamma)
    dx, dgamma, dbeta = Result(rows, K, t, pad, at), torch.full((K + 64,), 9.0, device=DEV), torch.full((K + 64,), 9.0, device=DEV)
    ws, view = workspace(sq.sparq_mx_norm_grad_workspace_bytes(rows, K))
    sq.sparq_mx_norm_grad(matrix(dy, t, pad, at), c.t, s.t, mean, rstd, gd, dx.view, dgamma=dgamma[:K], dbeta=dbeta[:K], workspace=view)
    guard(ws, view)
    h, e = np.abs(X - mu) * r + 2 * u * r * (np.abs(X) + np.abs(mu)), np.abs(dy * gamma)
    off = r * u * (8 * (e + h * (e * h).mean(1, keepdims=True)) + (d + 8) * (e.mean(1, keepdims=True) + h * (e * h).mean(1, keepdims=True)))
    close(dx.get(), dx_ref, off, t)
    close(dgamma[:K].double().cpu().numpy(), dgamma_ref, (rows + 6) * u * (np.abs(dy) * h).sum(0), "f32")
    close(dbeta[:K].double().cpu().numpy(), dbeta_ref, (rows + 2) * u * np.abs(dy).sum(0), "f32")
    assert bool((dgamma[K:] == 9).all()) and bool((dbeta[K:] == 9).all())
    for one in ("dgamma", "dbeta", None):                            # either gradient alone, and neither: the others do not change
        out, dx2 = torch.empty(K, device=DEV), Result(rows, K, t, pad, at)
        sq.sparq_mx_norm_grad(matrix(dy, t, pad, at), c.t, s.t, mean, rstd, gd, dx2.view, workspace=view, **({one: out} if one else {}))
        assert np.array_equal(dx2.get(), dx.get())
        assert one is None or torch.equal(out, (dgamma if one == "dgamma" else dbeta)[:K])


def test_norm_grad_is_the_differences(sq):
    """On an input that its checkpoint holds exactly the gradient is the layer norm's own: central differences in 64 bits, whose
    truncation and rounding stay under 1e-6 here."""
    g = rng(10)
    rows, K, eps, h = 3, 40, 1e-5, 1e-5
    x = R.quantised(g.standard_normal((rows, K)), 8)
    dy, gamma, beta = values(g, rows, K, "f32"), values(g, 1, K, "f32")[0], values(g, 1, K, "f32")[0]
    c, s = coded_buffers(sq, rows, K, 8)
    mean, rstd, y, dx = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), Result(rows, K, "f32"), Result(rows, K, "f32")
    gd, bd, dgamma, dbeta = torch.from_numpy(gamma).float().to(DEV), torch.from_numpy(beta).float().to(DEV), torch.empty(K, device=DEV), torch.empty(K, device=DEV)
    sq.sparq_mx_norm(matrix(x, "f32"), gd, bd, eps, y.view, mean=mean, rstd=rstd, codes=c.t, scales=s.t)
    sq.sparq_mx_norm_grad(matrix(dy, "f32"), c.t, s.t, mean, rstd, gd, dx.view, dgamma, dbeta, workspace(sq.sparq_mx_norm_grad_workspace_bytes(rows, K))[1])
    loss = lambda x, gamma: (R.norm(x, gamma, beta, eps)[0] * dy).sum()      # noqa: E731
    got, dgamma = dx.get(), dgamma.double().cpu().numpy()
    for i in range(rows):
        for j in range(0, K, 7):
            e = np.zeros_like(x)
            e[i, j] = h
            assert abs((loss(x + e, gamma) - loss(x - e, gamma)) / (2 * h) - got[i, j]) < 2e-5 * (1 + abs(got[i, j]))
    for j in range(0, K, 7):
        e = np.zeros(K)
        e[j] = h
        assert abs((loss(x, gamma + e) - loss(x, gamma - e)) / (2 * h) - dgamma[j]) < 2e-5 * (1 + abs(dgamma[j]))


# ---- how they are called -----------------------------------------------------------------------------------------------------
def _block(sq, seed, M=70, N=192, K=160):
    """A layer's forward and backward pass with everything in between: results and the call that makes them."""
    g = rng(11, seed)
    x, w, dy = values(g, M, K, "bf16"), values(g, N, K, "f32"), values(g, M, N, "bf16")
    xd, dyd, wd = matrix(x, "bf16"), matrix(dy, "bf16"), stored(sq, w, 4)
    gamma, beta = torch.ones(K, device=DEV), torch.zeros(K, device=DEV)
    E = lambda *s, dtype=torch.bfloat16: torch.empty(*s, dtype=dtype, device=DEV)      # noqa: E731
    buf = lambda r, k, bits: [b.t for b in coded_buffers(sq, r, k, bits)]              # noqa: E731
    out = dict(h=E(M, K), mean=E(M, dtype=torch.float32), rstd=E(M, dtype=torch.float32), y=E(M, N), a=E(M, N), da=E(M, N), dh=E(M, K),
               dw=E(N, K, dtype=torch.float32), db=E(N, dtype=torch.float32), dx=E(M, K), dgamma=E(K, dtype=torch.float32),
               dbeta=E(K, dtype=torch.float32), y2=E(M, N))
    kx, h4, h8, ky = buf(M, K, 8), buf(M, K, 4), buf(M, K, 8), buf(M, N, 8)
    ws = E(max(sq.sparq_mx_linear_workspace_bytes(M, N, K), sq.sparq_mx_gemm_workspace_bytes(M, N, K), sq.sparq_mx_linear_dx_workspace_bytes(M, N, K),
               sq.sparq_mx_linear_dw_workspace_bytes(M, N, K), sq.sparq_mx_norm_grad_workspace_bytes(M, K)) + 1, dtype=torch.uint8)

    def run():
        sq.sparq_mx_norm(xd, gamma, beta, 1e-5, out["h"], mean=out["mean"], rstd=out["rstd"], codes=kx[0], scales=kx[1])
        sq.sparq_mx_quantize(out["h"], *h4, *h8)
        sq.sparq_mx_gemm(*h4, *wd, K, out["y"], workspace=ws)
        sq.sparq_mx_linear(out["h"], *wd, out["y2"], workspace=ws)
        sq.sparq_mx_act("silu", out["y"], out["a"], gate_codes=ky[0], gate_scales=ky[1])
        sq.sparq_mx_act_grad("silu", dyd, *ky, out["da"])
        sq.sparq_mx_linear_dx(out["da"], *wd, out["dh"], workspace=ws)
        sq.sparq_mx_linear_dw(out["da"], *h8, out["dw"], db=out["db"], workspace=ws)
        sq.sparq_mx_norm_grad(out["dh"], *kx, out["mean"], out["rstd"], gamma, out["dx"], dgamma=out["dgamma"], dbeta=out["dbeta"], workspace=ws)
    return out, run


def test_on_another_stream_and_twice(sq):
    """The same to the bit on a stream of one's own, behind work that the stream still has to do."""
    out, run = _block(sq, 1)
    run()
    torch.cuda.synchronize()
    first = {k: v.clone() for k, v in out.items()}
    s = torch.cuda.Stream()
    for v in out.values():
        v.fill_(3.0)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
    s.synchronize()
    for k, v in out.items():
        assert torch.equal(v, first[k]), k


def test_in_a_graph(sq):
    """Captured once and replayed, with eager work between the replays: every replay is the eager result."""
    out, run = _block(sq, 2)
    run()
    torch.cuda.synchronize()
    first = {k: v.clone() for k, v in out.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(4):
        for v in out.values():
            v.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        for k, v in out.items():
            assert torch.equal(v, first[k]), k
        run()
        torch.cuda.synchronize()


def test_rows_more_than_32_bits_apart(sq):
    """Three rows 2^31 + 8 elements apart: offsets beyond 32 bits, elements and bytes."""
    M, K, N, ld = 3, 200, 72, (1 << 31) + 8
    g = rng(12)
    far = torch.empty(2 * ld + 4096, dtype=torch.bfloat16, device=DEV)
    x, w, dy = values(g, M, K, "bf16"), values(g, N, K, "f32"), values(g, M, N, "bf16")
    view = lambda n, at=0: far.as_strided((M, n), (ld, 1), at)      # noqa: E731
    xd, out = view(K), view(K, 512)
    xd.copy_(torch.from_numpy(x))
    near = matrix(x, "bf16")
    a, b = coded_buffers(sq, M, K, 8), coded_buffers(sq, M, K, 8)
    sq.sparq_mx_quantize(xd, codes8=a[0].t, scales8=a[1].t)
    sq.sparq_mx_quantize(near, codes8=b[0].t, scales8=b[1].t)
    assert np.array_equal(a[0].get(), b[0].get()) and np.array_equal(a[1].get(), b[1].get())
    near_out = torch.empty(M, K, dtype=torch.bfloat16, device=DEV)
    same = lambda: torch.equal(out.contiguous(), near_out)      # noqa: E731
    sq.sparq_mx_dequantize(a[0].t, a[1].t, 8, out)
    sq.sparq_mx_dequantize(a[0].t, a[1].t, 8, near_out)
    assert same()
    sq.sparq_mx_act("gelu", xd, out)
    sq.sparq_mx_act("gelu", near, near_out)
    assert same()
    ones = torch.ones(K, device=DEV)
    sq.sparq_mx_norm(xd, ones, None, 1e-5, out)
    sq.sparq_mx_norm(near, ones, None, 1e-5, near_out)
    assert same()
    wd = stored(sq, w, 4)
    far_y, near_y = view(N, 1024), torch.empty(M, N, dtype=torch.bfloat16, device=DEV)
    ws = workspace(sq.sparq_mx_linear_workspace_bytes(M, N, K) + sq.sparq_mx_linear_dx_workspace_bytes(M, N, K) + sq.sparq_mx_linear_dw_workspace_bytes(M, N, K))[1]
    sq.sparq_mx_linear(xd, *wd, far_y, workspace=ws)
    sq.sparq_mx_linear(near, *wd, near_y, workspace=ws)
    assert torch.equal(far_y.contiguous(), near_y)
    far_y.copy_(torch.from_numpy(dy))
    near_y.copy_(torch.from_numpy(dy))
    sq.sparq_mx_linear_dx(far_y, *wd, out, workspace=ws)
    sq.sparq_mx_linear_dx(near_y, *wd, near_out, workspace=ws)
    assert same()
    dw = [torch.empty(N, K, device=DEV) for _ in range(2)]
    for d, y in zip(dw, (far_y, near_y)):
        sq.sparq_mx_linear_dw(y, a[0].t, a[1].t, d, workspace=ws)
    assert torch.equal(*dw)


def test_a_large_call_is_its_pieces(sq):
    """Calls of more bytes than the caches hold, to the bit what calls for a few rows at a time give."""
    M, K, piece = 17001, 8200, 3001
    g = torch.Generator(DEV).manual_seed(5)
    new = lambda: torch.randn(M, K, generator=g, device=DEV, dtype=torch.float32).to(torch.bfloat16)      # noqa: E731
    x, up, dy = new(), new(), new()
    gamma, beta = torch.rand(K, generator=g, device=DEV) + 0.5, torch.rand(K, generator=g, device=DEV)
    coded = lambda bits: (torch.zeros(M, sq.sparq_mx_code_bytes(K, bits), dtype=torch.uint8, device=DEV),      # noqa: E731
                          torch.zeros(M, sq.sparq_mx_scale_bytes(K), dtype=torch.uint8, device=DEV))
    like = lambda: torch.full_like(x, 7.0)      # noqa: E731
    results = []
    for rows in (M, piece):
        c4, c8, cu, cn = coded(4), coded(8), coded(8), coded(8)
        back4, back8, y, dgate, dup, n, dx = (like() for _ in range(7))
        mean, rstd = torch.zeros(M, device=DEV), torch.zeros(M, device=DEV)
        dg, db = torch.zeros(K, device=DEV), torch.zeros(K, device=DEV)
        ws = torch.empty(sq.sparq_mx_norm_grad_workspace_bytes(rows, K), dtype=torch.uint8, device=DEV)
        for r in range(0, M, rows):
            p = slice(r, min(M, r + rows))
            at = lambda *ts: [t[p] for t in ts]      # noqa: E731
            sq.sparq_mx_quantize(x[p], *at(*c4, *c8))
            sq.sparq_mx_dequantize(*at(*c4), 4, back4[p])
            sq.sparq_mx_dequantize(*at(*c8), 8, back8[p])
            sq.sparq_mx_act("gelu", x[p], y[p], up=up[p], up_codes=cu[0][p], up_scales=cu[1][p])
            sq.sparq_mx_act_grad("gelu", dy[p], *at(*c8), dgate[p], up_codes=cu[0][p], up_scales=cu[1][p], dup=dup[p])
            sq.sparq_mx_norm(x[p], gamma, beta, 1e-5, n[p], mean=mean[p], rstd=rstd[p], codes=cn[0][p], scales=cn[1][p])
            sq.sparq_mx_norm_grad(dy[p], *at(*cn), mean[p], rstd[p], gamma, dx[p], dgamma=dg, dbeta=db, workspace=ws)
        torch.cuda.synchronize()
        results.append([*c4, *c8, *cu, *cn, back4, back8, y, dgate, dup, n, dx, mean, rstd])
        if rows == M:
            h = back8.double().sub_(mean.double()[:, None]).mul_(rstd.double()[:, None])
            wrong = lambda got, terms: float(((got.double() - terms.sum(0)).abs() / terms.abs().sum(0)).max())      # noqa: E731
            assert wrong(dg, dy.double() * h) <= (M + 10) * u and wrong(db, dy.double()) <= (M + 2) * u
            del h
    for i, (a, b) in enumerate(zip(*results)):
        assert torch.equal(a, b), i


def test_binding_refuses_wrong_shapes(sq):
    x, c, s = torch.zeros(4, 64, device=DEV), torch.zeros(4, 64, dtype=torch.uint8, device=DEV), torch.zeros(4, 16, dtype=torch.uint8, device=DEV)
    with pytest.raises(ValueError, match="codes4 must hold 256"):
        sq.sparq_mx_quantize(x, c[1:], s)
    with pytest.raises(ValueError, match="go together"):
        sq.sparq_mx_quantize(x, c)
    with pytest.raises(ValueError, match="next to each other"):
        sq.sparq_mx_quantize(x.t(), c, s)
    with pytest.raises(TypeError, match="dtype"):
        sq.sparq_mx_quantize(x.double(), c, s)
    with pytest.raises(sq.SparqError, match="invalid"):
        sq.sparq_mx_quantize(x)
    with pytest.raises(sq.SparqError, match="invalid"):
        sq.sparq_mx_quantize(x[:1].expand(4, 64), c, s)
    with pytest.raises(ValueError, match="same number of rows"):
        sq.sparq_mx_linear(x, c, s, torch.zeros(3, 4, device=DEV))
    with pytest.raises(TypeError, match="type of the call's first"):
        sq.sparq_mx_act("silu", x, x.half())
