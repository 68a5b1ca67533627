"""The microscaled operators on the GPU over what their types hold and what a launch counts: every 16-bit value through the activations, calls of more
rows or columns than one launch takes.
Against the plain reference in 64 bits (tests/mx_reference.py); tolerances stand at the tests, fixed before any run.
u = 2^-24 is fp32's unit roundoff."""
import ctypes

import numpy as np
import pytest
import torch

import mx_reference as R
from test_gpu_mx import DEV, TYPES, Result, close, coded_buffers, matrix, rng, sq, stored, u, values, workspace  # noqa: F401

pytestmark = pytest.mark.gpu


# ---- activations -------------------------------------------------------------------------------------------------------------
def all_values(t):
    """Every finite value of a 16-bit type, as float64."""
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(TYPES[t]).double()
    return bits[bits.isfinite()].numpy()


def relative(name, v):
    """The relative error of f(v), and of the factor of v in it, before it is rounded to 16 bits.  gelu: 9 u of the fitted function, 3 u v^2 log2(e)/2
    ln 2 = 1.5 v^2 u of the exponent's three roundings, 20 u of the others.  silu: 2 u |v| of the exponent's two, 8 u of the others."""
    return (32 + 2 * v * v) * u if name == "gelu" else (8 + 2 * np.abs(v)) * u


# What fp32 does not hold between: the exponential below 2^-126 (gelu), a quotient below 2^-126 (silu), times |v| < 128 there.
LEAST = 2.0 ** -119


@pytest.mark.parametrize("name", ("silu", "gelu"))
@pytest.mark.parametrize("t", ("f16", "bf16"))
def test_act_of_every_16_bit_value(sq, name, t):  # noqa: F811
    """Relative to the value itself, in the far tail as elsewhere."""
    v = all_values(t)[None]
    y = Result(1, v.shape[1], t)
    sq.sparq_mx_act(name, matrix(v, t), y.view)
    with np.errstate(over="ignore"):
        f = R.function(name, v)
        off = np.where(np.abs(v) < 1e3, relative(name, np.clip(v, -1e3, 1e3)), 8 * u) * np.abs(f)
    close(y.get(), f, off + LEAST, t)


@pytest.mark.parametrize("name", ("silu", "gelu"))
@pytest.mark.parametrize("t", ("f16", "bf16"))
def test_act_gradient_over_the_tail(sq, name, t):  # noqa: F811
    """Checkpoints of blocks of every power of two up to 16: all their codes, so that the tail is met in every binade.  f' = c + v c' with c in
    (0, 1): the two terms' errors, relative each, and the sum's rounding."""
    k = np.arange(-127, 128)
    x = np.concatenate([np.concatenate([np.append(np.sign(k[i]) * 127, k[i:i + 31]) for i in range(0, 255, 31)] + [np.zeros(32)])[: 32 * 9] * 2.0 ** (e - 6)
                        for e in range(-4, 5)])
    x = np.where(np.arange(x.size) % 32 == 0, np.where(x == 0, 127 * 2.0 ** -20, x), x)[None]
    c, s = coded_buffers(sq, 1, x.shape[1], 8)
    sq.sparq_mx_quantize(matrix(x, "f32"), codes8=c.t, scales8=s.t)
    X = R.quantised(x, 8)
    assert X.min() < -15 and X.max() > 15
    dg, du = Result(1, x.shape[1], t), Result(1, x.shape[1], t)
    one = matrix(np.ones_like(x), t)
    sq.sparq_mx_act_grad(name, one, c.t, s.t, dg.view, up_codes=c.t, up_scales=s.t, dup=du.view)
    f, d = R.function(name, X), R.slope(name, X)
    factor = f / np.where(X == 0, 1, X)
    close(du.get(), f, relative(name, X) * np.abs(f) + LEAST, t)
    # dgate = dy up f', here X f'
    off = (relative(name, X) + 4 * u) * (np.abs(factor) + np.abs(d - factor)) * np.abs(X)
    close(dg.get(), X * d, off + LEAST, t)


@pytest.mark.parametrize("name", ("silu", "gelu"))
def test_act_of_fp32_over_the_tail(sq, name):  # noqa: F811
    """fp32 goes through the library's functions, 32 u (16 units of the last place) and a few roundings; the exponent's or erfc's argument, off by
    2 u, adds 2 u |v| or 2 u v^2."""
    v = torch.linspace(-13, 13, 52001, dtype=torch.float64).float().double().numpy()[None]
    y = Result(1, v.shape[1], "f32")
    sq.sparq_mx_act(name, matrix(v, "f32"), y.view)
    f = R.function(name, v)
    close(y.get(), f, (40 + (2 * v * v if name == "gelu" else 2 * np.abs(v))) * u * np.abs(f) + LEAST, "f32")


# ---- what a launch counts ----------------------------------------------------------------------------------------------------
# A launch has fewer than 2^32 threads along an axis; calls within the documented sizes that would need more.  Each is held, to the bit, to
# calls for its pieces.
def coded(sq, rows, K, bits):  # noqa: F811
    return (torch.zeros(rows, sq.sparq_mx_code_bytes(K, bits), dtype=torch.uint8, device=DEV),
            torch.zeros(rows, sq.sparq_mx_scale_bytes(K), dtype=torch.uint8, device=DEV))


@pytest.fixture
def emptied():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def test_codec_of_more_rows_than_a_launch_has_wavefronts(sq, emptied):  # noqa: F811
    rows, K, piece = (1 << 26) + 5, 1, 1 << 25
    x = torch.randn(rows, K, device=DEV, dtype=torch.float16, generator=torch.Generator(DEV).manual_seed(21))
    for bits in (4, 8):
        c, s = coded(sq, rows, K, bits)
        sq.sparq_mx_quantize(x, **{f"codes{bits}": c, f"scales{bits}": s})
        y = torch.full_like(x, 7.0)
        sq.sparq_mx_dequantize(c, s, bits, y)
        for r in range(0, rows, piece):
            p = slice(r, min(rows, r + piece))
            c1, s1 = coded(sq, p.stop - r, K, bits)
            sq.sparq_mx_quantize(x[p], **{f"codes{bits}": c1, f"scales{bits}": s1})
            assert torch.equal(c[p], c1) and torch.equal(s[p], s1), (bits, r)
            y1 = torch.full_like(x[p], 9.0)
            sq.sparq_mx_dequantize(c1, s1, bits, y1)
            assert torch.equal(y[p], y1), (bits, r)


def test_act_of_more_rows_than_a_launch_has_wavefronts(sq, emptied):  # noqa: F811
    rows, K, piece = (1 << 26) + 5, 2, 1 << 25
    g = torch.Generator(DEV).manual_seed(22)
    gate, up, dy = (torch.randn(rows, K, device=DEV, dtype=torch.bfloat16, generator=g) for _ in range(3))
    gc, uc = coded(sq, rows, K, 8), coded(sq, rows, K, 8)
    y, dg, du = (torch.full_like(gate, 7.0) for _ in range(3))
    sq.sparq_mx_act("silu", gate, y, up=up, gate_codes=gc[0], gate_scales=gc[1], up_codes=uc[0], up_scales=uc[1])
    sq.sparq_mx_act_grad("silu", dy, *gc, dg, up_codes=uc[0], up_scales=uc[1], dup=du)
    for r in range(0, rows, piece):
        p = slice(r, min(rows, r + piece))
        g1, u1 = coded(sq, p.stop - r, K, 8), coded(sq, p.stop - r, K, 8)
        y1, dg1, du1 = (torch.full_like(gate[p], 9.0) for _ in range(3))
        sq.sparq_mx_act("silu", gate[p], y1, up=up[p], gate_codes=g1[0], gate_scales=g1[1], up_codes=u1[0], up_scales=u1[1])
        sq.sparq_mx_act_grad("silu", dy[p], *g1, dg1, up_codes=u1[0], up_scales=u1[1], dup=du1)
        for a, b in zip((gc[0][p], gc[1][p], uc[0][p], uc[1][p], y[p], dg[p], du[p]), (*g1, *u1, y1, dg1, du1)):
            assert torch.equal(a, b), r


def test_norm_of_more_short_rows_than_a_launch_has_workgroups(sq, emptied):  # noqa: F811
    rows, K, piece = (1 << 24) + 9, 5, 1 << 23
    g = torch.Generator(DEV).manual_seed(23)
    x = torch.randn(rows, K, device=DEV, dtype=torch.float16, generator=g)
    gamma, beta = torch.rand(K, device=DEV, generator=g) + 0.5, torch.rand(K, device=DEV, generator=g)
    c, y, mean, rstd = coded(sq, rows, K, 8), torch.full_like(x, 7.0), torch.zeros(rows, device=DEV), torch.zeros(rows, device=DEV)
    sq.sparq_mx_norm(x, gamma, beta, 1e-5, y, mean=mean, rstd=rstd, codes=c[0], scales=c[1])
    for r in range(0, rows, piece):
        p = slice(r, min(rows, r + piece))
        c1, y1, m1, r1 = coded(sq, p.stop - r, K, 8), torch.full_like(x[p], 9.0), torch.ones(p.stop - r, device=DEV), torch.ones(p.stop - r, device=DEV)
        sq.sparq_mx_norm(x[p], gamma, beta, 1e-5, y1, mean=m1, rstd=r1, codes=c1[0], scales=c1[1])
        for a, b in zip((c[0][p], c[1][p], y[p], mean[p], rstd[p]), (*c1, y1, m1, r1)):
            assert torch.equal(a, b), r


def test_norm_gradient_of_more_short_rows_than_a_launch_has_wavefronts(sq, emptied):  # noqa: F811
    rows, K, piece = (1 << 26) + 7, 3, 1 << 25
    g = torch.Generator(DEV).manual_seed(24)
    x, dy = (torch.randn(rows, K, device=DEV, dtype=torch.bfloat16, generator=g) for _ in range(2))
    gamma = torch.rand(K, device=DEV, generator=g) + 0.5
    c, dx = coded(sq, rows, K, 8), torch.full_like(x, 7.0)
    mean, rstd = torch.randn(rows, device=DEV, generator=g), torch.rand(rows, device=DEV, generator=g) + 0.5
    for r in range(0, rows, piece):
        p = slice(r, min(rows, r + piece))
        sq.sparq_mx_quantize(x[p], codes8=c[0][p], scales8=c[1][p])
    dgamma, dbeta = torch.zeros(K, device=DEV), torch.zeros(K, device=DEV)
    ws = torch.empty(sq.sparq_mx_norm_grad_workspace_bytes(rows, K), dtype=torch.uint8, device=DEV)
    sq.sparq_mx_norm_grad(dy, *c, mean, rstd, gamma, dx, dgamma=dgamma, dbeta=dbeta, workspace=ws)
    h = torch.empty_like(x, dtype=torch.float32)
    for r in range(0, rows, piece):
        p = slice(r, min(rows, r + piece))
        dx1, one, two = torch.full_like(x[p], 9.0), torch.zeros(K, device=DEV), torch.zeros(K, device=DEV)
        sq.sparq_mx_norm_grad(dy[p], c[0][p], c[1][p], mean[p], rstd[p], gamma, dx1, dgamma=one, dbeta=two, workspace=ws)
        assert torch.equal(dx[p], dx1), r
        sq.sparq_mx_dequantize(c[0][p], c[1][p], 8, h[p])
    # 256 sums of rows / 256 terms, and their sum: (rows / 256 + 256 + 8) u of the terms' magnitudes
    h.sub_(mean[:, None]).mul_(rstd[:, None])
    for got, terms in ((dgamma, h.double() * dy.double()), (dbeta, dy.double())):
        assert bool(((got.double() - terms.sum(0)).abs() <= (rows / 256 + 264) * u * terms.abs().sum(0)).all())


def test_norm_gradient_of_a_row_of_more_columns_than_a_launch_joins(sq, emptied):  # noqa: F811
    """One row: dbeta is dy, dgamma dy h."""
    K = (1 << 26) + 40
    g = torch.Generator(DEV).manual_seed(25)
    x, dy = (torch.randn(1, K, device=DEV, dtype=torch.bfloat16, generator=g) for _ in range(2))
    c, gamma, y, dx = coded(sq, 1, K, 8), torch.ones(K, device=DEV), torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(1, device=DEV), torch.empty(1, device=DEV)
    sq.sparq_mx_norm(x, gamma, None, 1e-5, y, mean=mean, rstd=rstd, codes=c[0], scales=c[1])
    dgamma, dbeta, X = torch.full((K,), 9.0, device=DEV), torch.full((K,), 9.0, device=DEV), torch.empty(1, K, device=DEV)
    ws = torch.empty(sq.sparq_mx_norm_grad_workspace_bytes(1, K), dtype=torch.uint8, device=DEV)
    sq.sparq_mx_norm_grad(dy, *c, mean, rstd, gamma, dx, dgamma=dgamma, dbeta=dbeta, workspace=ws)
    assert torch.equal(dbeta, dy[0].float())
    sq.sparq_mx_dequantize(*c, 8, X)
    ref = (X.double() - mean.double()) * rstd.double() * dy.double()
    off = 4 * u * (X.double().abs() + mean.double().abs()) * rstd.double() * dy.double().abs()
    assert bool(((dgamma.double() - ref[0]).abs() <= off[0]).all())


def test_few_rows_of_a_product_with_more_columns_than_a_launch_counts(sq, emptied):  # noqa: F811
    M, N, K, piece = 1, 1 << 28, 64, 1 << 27
    g = torch.Generator(DEV).manual_seed(26)
    w, ws = torch.empty(N, sq.sparq_mx_code_bytes(K, 4), dtype=torch.uint8, device=DEV), torch.zeros(N, sq.sparq_mx_scale_bytes(K), dtype=torch.uint8, device=DEV)
    w.random_(0, 256, generator=g)
    w[:, K // 2:] = 0
    ws[:, :2] = 127
    bias = torch.randn(N, device=DEV, generator=g)
    x = torch.randn(M, K, device=DEV, dtype=torch.bfloat16, generator=g)
    x4 = coded(sq, M, K, 4)
    sq.sparq_mx_quantize(x, *x4)
    for product, first, rest in ((sq.sparq_mx_gemm, x4, (K,)), (sq.sparq_mx_linear, (x,), ())):
        scratch = torch.empty(max(sq.sparq_mx_gemm_workspace_bytes(M, N, K), sq.sparq_mx_linear_workspace_bytes(M, N, K)) + 1, dtype=torch.uint8, device=DEV)
        y = torch.full((M, N), 7.0, dtype=torch.bfloat16, device=DEV)
        product(*first, w, ws, *rest, y, bias=bias, workspace=scratch)
        for n in range(0, N, piece):
            p = slice(n, n + piece)
            y1 = torch.full((M, piece), 9.0, dtype=torch.bfloat16, device=DEV)
            product(*first, w[p], ws[p], *rest, y1, bias=bias[p], workspace=scratch)
            assert torch.equal(y[:, p], y1), n


def test_gradient_of_the_bias_of_as_many_outputs_as_there_may_be(sq, emptied):  # noqa: F811
    M, N, K = 3, 1 << 28, 1
    g = torch.Generator(DEV).manual_seed(27)
    x, dy = torch.randn(M, K, device=DEV, generator=g), torch.randn(M, N, device=DEV, dtype=torch.bfloat16, generator=g)
    c = coded(sq, M, K, 8)
    sq.sparq_mx_quantize(x, codes8=c[0], scales8=c[1])
    X = torch.empty(M, K, device=DEV)
    sq.sparq_mx_dequantize(*c, 8, X)
    dw, db = torch.full((N, K), 9.0, device=DEV), torch.full((N,), 9.0, device=DEV)
    ws = torch.empty(sq.sparq_mx_linear_dw_workspace_bytes(M, N, K), dtype=torch.uint8, device=DEV)
    sq.sparq_mx_linear_dw(dy, *c, dw, db=db, workspace=ws)
    assert bool(((db.double() - dy.double().sum(0)).abs() <= 4 * u * dy.double().abs().sum(0)).all())
    assert bool(((dw[:, 0].double() - (dy.double() * X.double()).sum(0)).abs() <= 10 * u * (dy.double() * X.double()).abs().sum(0)).all())


def test_product_gradient_of_more_rows_than_a_launch_has_tiles(sq, emptied):  # noqa: F811
    """dx of one output is dy w: one product, rounded once."""
    M = (1 << 31) + 200
    dy = torch.empty(M, 1, dtype=torch.bfloat16, device=DEV).normal_(generator=torch.Generator(DEV).manual_seed(28))
    w4 = coded(sq, 1, 1, 4)
    sq.sparq_mx_quantize(torch.full((1, 1), 0.375, device=DEV), *w4)
    dx = torch.full_like(dy, 7.0)
    ws = torch.empty(sq.sparq_mx_linear_dx_workspace_bytes(M, 1, 1), dtype=torch.uint8, device=DEV)
    sq.sparq_mx_linear_dx(dy, *w4, dx, workspace=ws)
    assert torch.equal(dx, dy.mul_(0.375))


# ---- no rows -----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("N,K", [(8, 64), (5, 33), (300, 1000)])
def test_no_rows_and_no_dy_give_gradients_of_zero(sq, N, K):  # noqa: F811
    """Through the C entry points, dy NULL and its rows 0 apart."""
    n, z, big = None, ctypes.c_int64(0), ctypes.c_size_t(1 << 40)
    pointer = lambda t: ctypes.c_void_p(t.data_ptr())      # noqa: E731
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    for t in (0, 1, 2):
        dw, db = Result(N, K, "f32", 3, 1), torch.full((N,), 9.0, device=DEV)
        ws = torch.empty(sq.sparq_mx_linear_dw_workspace_bytes(0, N, K) + 256, dtype=torch.uint8, device=DEV)
        assert sq.lib.sparq_mx_linear_dw(n, t, z, n, n, pointer(dw.view), 0, ctypes.c_int64(dw.view.stride(0)), pointer(db), z, N, K, pointer(ws), big, stream) == 0
        assert not dw.get().any() and not db.any()
    dgamma, dbeta = torch.full((K,), 9.0, device=DEV), torch.full((K,), 9.0, device=DEV)
    assert sq.lib.sparq_mx_norm_grad(n, z, n, n, n, n, n, n, z, 2, pointer(dgamma), pointer(dbeta), z, K, n, ctypes.c_size_t(0), stream) == 0
    assert not dgamma.any() and not dbeta.any()

# ---- the product's gradients -------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("M,N,K", [(5, 7, 40), (200, 130, 300)])
def test_product_gradients_of_the_largest_values(sq, M, N, K):  # noqa: F811
    """fp32 has values above bf16's largest: they enter whole as well, and weights of zero leave nothing of them."""
    g = rng(30, M, N, K)
    x, w, dy = values(g, M, K, "f32", 2.0 ** -9), values(g, N, K, "f32", 2.0 ** -9), values(g, M, N, "f32", 2.0 ** 100)
    top = float(np.finfo(np.float32).max)
    for i in range(min(M, N)):
        dy[i, i] = (top, -top, float(np.float32(top * (1 - 2.0 ** -9))), 1.5 * 2.0 ** 127)[i % 4]
    w[:, 0], x[:, 0] = 0.0, 0.0
    X, W = R.quantised(x, 8), R.quantised(w, 4)
    dx, dw = Result(M, K, "f32"), Result(N, K, "f32")
    dyd = matrix(dy, "f32")
    sq.sparq_mx_linear_dx(dyd, *stored(sq, w, 4), dx.view, workspace=workspace(sq.sparq_mx_linear_dx_workspace_bytes(M, N, K))[1])
    sq.sparq_mx_linear_dw(dyd, *stored(sq, x, 8), dw.view, workspace=workspace(sq.sparq_mx_linear_dw_workspace_bytes(M, N, K))[1])
    assert not dx.get()[:, 0].any() and not dw.get()[:, 0].any()
    close(dx.get(), dy @ W, 2 * (3 * N + 2) * u * (np.abs(dy) @ np.abs(W)), "f32")
    close(dw.get(), dy.T @ X, 2 * (3 * M + 2) * u * (np.abs(dy).T @ np.abs(X)), "f32")
