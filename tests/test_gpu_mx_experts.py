"""The operators of a block with experts on the GPU against the plain reference in 64 bits (tests/mx_experts_reference.py).

Tolerances, fixed before any run.  u = 2^-24 is fp32's unit roundoff, U the result type's; every result is rounded once (test_gpu_mx.close).
  sort, gather, dropout's mask   to the bit
  combine       a sum of n products, each rounded once and each addition once: (n + 2) u of the terms' magnitudes; dweights: a sum of K
                products, (K + 2) u of theirs
  products      as in test_gpu_mx.py: 2 (K + 2) u sum |a||w|, and the bias's addition 2 u (|z| + |b|)
  epilogue      f's slope is at most 1.13 in magnitude; f itself is off by what test_gpu_mx.test_act allows; the residual's addition u (|f| + |r|)
  kept form     half a step of the block's power of two, a whole one where 127 is the last code, and z's own error
"""
import os
import sys

import numpy as np
import pytest
import torch

import mx_experts_reference as E
import mx_reference as R
from test_gpu_mx import DEV, TYPES, Bytes, Result, close, coded_buffers, guard, matrix, rng, sq, stored, u, values, workspace  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def Block():
    """The example's block, which runs the operators together."""
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import experts
    return experts.Block


class Whole:
    """An int32 buffer with a guard behind it."""

    def __init__(self, *shape):
        n = int(np.prod(shape))
        self.all = torch.full((n + 64,), 0x5A5A5A5A, dtype=torch.int32, device=DEV)
        self.t = self.all[:n].view(*shape)

    def get(self):
        torch.cuda.synchronize()
        assert bool((self.all[self.t.numel():] == 0x5A5A5A5A).all()), "written past the buffer"
        return self.t.cpu().numpy()


def ints(a):
    return torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).to(DEV)


def floats(a):
    return torch.from_numpy(np.ascontiguousarray(a).astype(np.float32)).to(DEV)


# ---- sort ----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("experts", (1, 2, 8, 63, 64, 65, 300, 1024))
@pytest.mark.parametrize("slots", (0, 1, 2, 63, 64, 65, 128, 129, 1000, 5003, 8192, 8193, 20000, 70001))
def test_sort(sq, slots, experts):  # noqa: F811
    g = rng(1, slots, experts)
    choice = g.integers(0, experts, slots)
    choice = np.where(g.random(slots) < 0.3, choice // 3, choice)                # some experts are liked more
    bad = g.random(slots) < 0.1
    choice = np.where(bad, g.choice([-1, experts, -2 ** 31, 2 ** 31 - 1, experts + 1], slots), choice)
    offsets, place, order = Whole(experts + 1), Whole(slots), Whole(slots)
    ws, view = workspace(sq.sparq_mx_sort_workspace_bytes(slots, experts))
    sq.sparq_mx_sort(ints(choice), offsets.t, place.t, order=order.t, workspace=view)
    for got, ref in zip((offsets, place, order), E.sort(choice, experts)):
        assert np.array_equal(got.get(), ref)
    guard(ws, view)
    again, none = Whole(slots), Whole(experts + 1)
    sq.sparq_mx_sort(ints(choice), none.t, again.t, workspace=view)
    assert np.array_equal(again.get(), place.get()) and np.array_equal(none.get(), offsets.get())


@pytest.mark.parametrize("slots", (100, 9000, 1 << 20))
@pytest.mark.parametrize("kind", ("all of one", "all refused", "the last"))
def test_sort_of_one_kind(sq, slots, kind):  # noqa: F811
    experts = 37
    choice = np.full(slots, {"all of one": 5, "all refused": -1, "the last": experts - 1}[kind])
    offsets, place, order = Whole(experts + 1), Whole(slots), Whole(slots)
    ws, view = workspace(sq.sparq_mx_sort_workspace_bytes(slots, experts))
    sq.sparq_mx_sort(ints(choice), offsets.t, place.t, order=order.t, workspace=view)
    for got, ref in zip((offsets, place, order), E.sort(choice, experts)):
        assert np.array_equal(got.get(), ref)


# ---- rows to their experts and back ------------------------------------------------------------------------------------------
ROUTE = [(1, 1, 1), (1, 2, 64), (3, 3, 31), (5, 8, 129), (7, 5, 513), (40, 2, 1000), (9, 6, 2057), (130, 4, 96), (2, 70, 40), (33, 4, 4096)]


def places(g, tokens, per, spare=3, refused=0.2):
    """Places in random order, some slots refused, `spare` rows that nobody has."""
    n = tokens * per
    rows = n + spare
    place = g.permutation(rows)[:n]
    place = np.where(g.random(n) < refused, g.choice([-1, rows, 2 ** 31 - 1, -2 ** 31], n), place)
    return place.reshape(tokens, per), rows


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("tokens,per,K", ROUTE)
@pytest.mark.parametrize("pad,at", [(0, 0), (5, 3)])
def test_gather(sq, t, tokens, per, K, pad, at):  # noqa: F811
    g = rng(2, tokens, per, K)
    x = values(g, tokens, K, t)
    place, rows = places(g, tokens, per)
    ref, has = E.gather(x, place, rows)
    xd, pd = matrix(x, t, pad, at), ints(place)
    alone = Result(rows, K, t, pad, at)
    sq.sparq_mx_gather(xd, pd, y=alone.view)
    y = Result(rows, K, t, at, pad)
    both = coded_buffers(sq, rows, K, 4) + coded_buffers(sq, rows, K, 8)
    sq.sparq_mx_gather(xd, pd, y.view, *[b.t for b in both])
    want = np.where(has[:, None], ref, -55)
    assert np.array_equal(alone.get(), want) and np.array_equal(y.get(), want)
    for bits in (4, 8):
        code, scale = (sq.sparq_mx_code_bytes(K, bits), sq.sparq_mx_scale_bytes(K))
        c, s = R.store(*R.encode(ref, bits), bits, code, scale)
        c, s = np.where(has[:, None], c, 0xA5), np.where(has[:, None], s, 0xA5)
        one = coded_buffers(sq, rows, K, bits)
        sq.sparq_mx_gather(xd, pd, **{f"codes{bits}": one[0].t, f"scales{bits}": one[1].t})
        for got in (one, both[:2] if bits == 4 else both[2:]):
            assert np.array_equal(got[0].get(), c) and np.array_equal(got[1].get(), s)


def test_gather_moves_bits(sq):  # noqa: F811
    """What a row holds arrives as it is, NaN with its bits among it."""
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(64, 1024).to(DEV)
    place = ints(np.arange(64)[::-1].reshape(64, 1))
    for t in (torch.float16, torch.bfloat16):
        y = torch.zeros(64, 1024, dtype=t, device=DEV)
        sq.sparq_mx_gather(bits.view(t), place, y=y)
        assert torch.equal(y.view(torch.int16), bits.flip(0))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("tokens,per,K", ROUTE)
@pytest.mark.parametrize("weighted,residual,pad,at", [(False, False, 0, 0), (True, False, 5, 3), (True, True, 0, 0), (False, True, 1, 0)])
def test_combine(sq, t, tokens, per, K, weighted, residual, pad, at):  # noqa: F811
    g = rng(3, tokens, per, K)
    place, rows = places(g, tokens, per)
    x = values(g, rows, K, t)
    w = np.float32(g.standard_normal((tokens, per))).astype(np.float64)
    there = (place >= 0) & (place < rows)
    w[~there] = np.nan                                                           # nobody looks at a refused slot's weight
    r = values(g, tokens, K, t)
    ref, size = E.combine(x, place, w if weighted else None, r if residual else None)
    xd = matrix(x, t, pad, at)
    spare = np.setdiff1d(np.arange(rows), place[there])
    xd[spare.tolist()] = float("nan")                                            # ... nor at rows that nobody has
    y = Result(tokens, K, t, pad, at)
    sq.sparq_mx_combine(xd, ints(place), y.view, weights=floats(w) if weighted else None, residual=matrix(r, t, at, pad) if residual else None)
    close(y.get(), ref, (per + 2) * u * size, t)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("tokens,per,K", ROUTE)
@pytest.mark.parametrize("pad,at", [(0, 0), (5, 3)])
def test_combine_grad(sq, t, tokens, per, K, pad, at):  # noqa: F811
    g = rng(4, tokens, per, K)
    place, rows = places(g, tokens, per)
    x, dy, w = values(g, rows, K, t), values(g, tokens, K, t, 0.1), np.float32(g.standard_normal((tokens, per))).astype(np.float64)
    dx, has, dw, size = E.combine_grad(dy, place, w, x)
    xd, dyd, pd, wd = matrix(x, t, pad, at), matrix(dy, t, at, pad), ints(place), floats(w)
    a, b, both = Result(rows, K, t, pad, at), Result(rows, K, t), torch.full((tokens, per), 9.0, device=DEV)
    alone = torch.full((tokens, per), 9.0, device=DEV)
    sq.sparq_mx_combine_grad(dyd, pd, wd, dx=a.view, x=xd, dweights=both)
    sq.sparq_mx_combine_grad(dyd, pd, wd, dx=b.view)
    sq.sparq_mx_combine_grad(dyd, pd, x=xd, dweights=alone)
    for got in (a, b):
        got = got.get()
        assert np.all(got[~has] == -55)
        close(got[has], dx[has], 0, t)
    for got in (both, alone):
        assert np.all(np.abs(got.double().cpu().numpy() - dw) <= (K + 2) * u * size)


def test_route_of_nothing(sq):  # noqa: F811
    """All slots refused, no tokens, no rows."""
    place = ints(np.full((3, 2), -1))
    x, rows = torch.ones(3, 40, device=DEV), torch.full((5, 40), float("nan"), device=DEV)
    y = torch.full((3, 40), 7.0, device=DEV)
    sq.sparq_mx_combine(rows, place, y)
    assert torch.equal(y, torch.zeros_like(y))
    sq.sparq_mx_combine(rows, place, y, residual=x)
    assert torch.equal(y, x)
    dw = torch.full((3, 2), 7.0, device=DEV)
    sq.sparq_mx_combine_grad(x, place, x=rows, dweights=dw)
    assert torch.equal(dw, torch.zeros_like(dw))
    out = torch.full((5, 40), 7.0, device=DEV)
    sq.sparq_mx_gather(x, place, y=out)
    assert bool((out == 7).all())
    none, some = torch.empty(0, 40, device=DEV), ints(np.arange(6).reshape(3, 2))
    sq.sparq_mx_gather(x, some, y=none)
    y.fill_(7.0)
    sq.sparq_mx_combine(none, some, y)
    assert torch.equal(y, torch.zeros_like(y))
    dw.fill_(7.0)
    sq.sparq_mx_combine_grad(x, some, torch.ones(3, 2, device=DEV), dx=none, x=none, dweights=dw)
    assert torch.equal(dw, torch.zeros_like(dw))
    sq.sparq_mx_combine_grad(x, some, torch.ones(3, 2, device=DEV), dx=none)
    sq.sparq_mx_gather(none, ints(np.zeros((0, 2))), y=out)
    sq.sparq_mx_combine(out, ints(np.zeros((0, 2))), none)
    assert bool((out == 7).all())


# ---- the experts' product --------------------------------------------------------------------------------------------------------
def offsets_of(counts):
    return np.cumsum([0] + list(counts))


COUNTS = {
    "one row": [0, 1, 0],
    "few": [1, 0, 3, 2, 0, 0, 5, 1],
    "sixteens": [16, 17, 0, 15, 33, 1, 40],
    "one has all": [0, 0, 150, 0],
    "middling": [70, 0, 64, 130, 1, 63],
    "many": [300, 513, 0, 256, 700, 3],
    "of one": [90],
    "nobody": [0, 0, 0],
}
EXPERTS = [("one row", 40, 96), ("one row", 1000, 2100), ("few", 1, 1), ("few", 65, 129), ("few", 257, 1030), ("few", 48, 3), ("sixteens", 130, 700), ("sixteens", 1030, 4200),
           ("one has all", 33, 260), ("one has all", 300, 1000), ("middling", 100, 520), ("middling", 515, 64), ("many", 333, 200), ("many", 130, 1500),
           ("of one", 200, 300), ("nobody", 70, 130)]
EPILOGUES = [("bf16", None, False, False, 0, 0), ("f32", "gelu", True, True, 3, 1), ("f16", "silu", True, False, 0, 0), ("bf16", "gelu", True, True, 8, 5),
             ("f32", "silu", False, False, 0, 0)]


def epilogue(z, z_off, f, residual):
    """y and what it may be off by before it is rounded."""
    v = E.function(f, z)
    off = 1.2 * z_off + (0 if f is None else 16 * u * ((2 + np.abs(z)) * np.abs(v) + (np.abs(z) if f == "gelu" else 0) + 2.0 ** -126))
    if residual is None:
        return v, off
    return v + residual, off + 2 * u * (np.abs(v) + np.abs(residual))


def check_kept(got, z, z_off, has):
    """The kept form stands for z, block by block."""
    v = R.decode(*got, 8)
    rows, N = z.shape
    blocks = -(-N // 32)
    top = np.zeros((rows, blocks * 32))
    top[:, :N] = np.abs(z) + z_off
    step = np.repeat(2.0 ** np.floor(np.log2(np.maximum(top.reshape(rows, blocks, 32).max(2), 2.0 ** -126))) / 64, 32, 1)[:, :N]
    off = np.abs(v - z)
    assert np.all((off <= step + z_off)[has]) and np.all((off <= step / 2 + z_off)[has & (np.abs(z) < 127 * step).all(1)])


def codes_of(c, s, N):
    """Codes and scale bytes as R.decode takes them."""
    return c[:, :N].astype(np.int8).astype(np.int64), s[:, : -(-N // 32)].astype(np.int64)


def run_product(sq, g, M, N, K, offsets, t, f, bias, residual, pad, at, kept=False, x_type="bf16"):  # noqa: F811
    """Both forms of the product against the reference; offsets None: a layer."""
    experts = 1 if offsets is None else len(offsets) - 1
    x, W = values(g, M, K, x_type), values(g, experts * N, K, "f32") / np.sqrt(K)
    b = np.float32(g.standard_normal((experts, N))).astype(np.float64) if bias else None
    r = values(g, M, N, t) if residual else None
    A, V = R.quantised(x, 4), R.quantised(W, 4).reshape(experts, N, K)
    z, size, has = E.product(A, V, [0, M] if offsets is None else offsets, b)
    z_off = 2 * (K + 2) * u * size + 2 * u * np.abs(z)
    ref, off = epilogue(z, z_off, f, r)
    w, a = stored(sq, W, 4), stored(sq, x, 4)
    beside = dict(offsets=None if offsets is None else ints(offsets), bias=None if b is None else floats(b), function=f,
                  residual=None if r is None else matrix(r, t, at, pad))
    for form in ("gemm", "linear"):
        y = Result(M, N, t, pad, at)
        c = coded_buffers(sq, M, N, 8) if kept else None
        if kept:
            beside.update(kept_codes=c[0].t, kept_scales=c[1].t)
        ws, view = workspace(getattr(sq, f"sparq_mx_experts_{form}_workspace_bytes")(M, N, K, experts))
        if form == "gemm":
            sq.sparq_mx_experts_gemm(*a, *w, K, y.view, workspace=view, **beside)
        else:
            sq.sparq_mx_experts_linear(matrix(x, x_type, pad, at), *w, y.view, workspace=view, **beside)
        got = y.get()
        guard(ws, view)
        assert np.all(got[~has] == -55), "rows that nobody has were written"
        close(got[has], ref[has], off[has], t)
        if kept:
            codes, scales = c[0].get(), c[1].get()
            assert np.all(codes[~has] == 0xA5) and np.all(scales[~has] == 0xA5)
            assert not codes[has][:, N:].any() and not scales[has][:, -(-N // 32):].any(), "what lies past the rows' ends is not zero"
            check_kept(codes_of(codes, scales, N), z, z_off, has)


@pytest.mark.parametrize("counts,N,K", EXPERTS)
@pytest.mark.parametrize("t,f,bias,residual,pad,at", EPILOGUES)
def test_experts(sq, counts, N, K, t, f, bias, residual, pad, at):  # noqa: F811
    offsets = offsets_of(COUNTS[counts])
    run_product(sq, rng(5, N, K), int(offsets[-1]) + 2, N, K, offsets, t, f, bias, residual, pad, at)


@pytest.mark.parametrize("counts,N,K", [("few", 65, 129), ("one row", 40, 96), ("middling", 515, 64), ("many", 333, 200), ("many", 600, 140), ("nobody", 70, 130)])
@pytest.mark.parametrize("t,f,bias,residual", [("bf16", "gelu", True, False), ("f32", "silu", False, True), ("f16", None, True, False)])
def test_experts_kept(sq, counts, N, K, t, f, bias, residual):  # noqa: F811
    offsets = offsets_of(COUNTS[counts])
    run_product(sq, rng(6, N, K), int(offsets[-1]) + 2, N, K, offsets, t, f, bias, residual, 0, 0, kept=True)


LAYER = [(1, 40, 300), (1, 515, 4100), (13, 65, 735), (16, 300, 64), (17, 1000, 1030), (60, 130, 2100), (64, 64, 64), (70, 100, 8300), (300, 333, 260), (1000, 1030, 500),
         (600, 3000, 400), (1500, 8200, 150)]


@pytest.mark.parametrize("M,N,K", LAYER)
@pytest.mark.parametrize("t,f,bias,residual,pad,at", EPILOGUES)
def test_layer(sq, M, N, K, t, f, bias, residual, pad, at):  # noqa: F811
    run_product(sq, rng(7, M, N, K), M, N, K, None, t, f, bias, residual, pad, at, x_type=t)


@pytest.mark.parametrize("M,N,K", [(1, 40, 300), (13, 65, 735), (64, 640, 64), (70, 100, 8300), (300, 333, 260), (600, 1030, 400), (1500, 8200, 150)])
@pytest.mark.parametrize("t,f,bias", [("bf16", "gelu", True), ("f32", "silu", False)])
def test_layer_kept(sq, M, N, K, t, f, bias):  # noqa: F811
    run_product(sq, rng(8, M, N, K), M, N, K, None, t, f, bias, True, 3, 2, kept=True)


@pytest.mark.parametrize("counts,M,N,K", [([900, 0, 1500, 800, 200], 3400, 4100, 200), ([1024, 2048, 1024], 4096, 3328, 640), ([37] * 130, 4810, 520, 300), ([1] * 1024, 1030, 70, 64),
                                              ([3000, 1100, 5], 4105, 3400, 2100), ([20, 0, 130] * 30, 4500, 300, 200), ([16] * 64, 1024, 100, 300), ([100] * 65, 6500, 40, 40)])
def test_experts_of_many_tiles(sq, counts, M, N, K):  # noqa: F811
    run_product(sq, rng(9, N, K), M, N, K, offsets_of(counts), "bf16", "silu", True, False, 0, 0)


def test_kept_to_the_bit(sq):  # noqa: F811
    """Whole numbers, whose sums are exact: the kept form to the bit, in every kernel."""
    for M, N, K, counts in ((5, 70, 64, [2, 0, 3]), (200, 200, 96, None), (3000, 2200, 64, [1000, 2000]), (700, 600, 128, [700])):
        g = rng(10, M)
        experts = len(counts) if counts else 1
        x, W = g.integers(-3, 4, (M, K)).astype(np.float64), g.integers(-3, 4, (experts * N, K)).astype(np.float64)
        assert np.array_equal(R.quantised(x, 4), x) and np.array_equal(R.quantised(W, 4), W)
        offsets = offsets_of(counts) if counts else np.array([0, M])
        z = E.product(x, W.reshape(experts, N, K), offsets)[0]
        c, y = coded_buffers(sq, M, N, 8), Result(M, N, "f32")
        ws, view = workspace(sq.sparq_mx_experts_gemm_workspace_bytes(M, N, K, experts))
        sq.sparq_mx_experts_gemm(*stored(sq, x, 4), *stored(sq, W, 4), K, y.view, offsets=ints(offsets) if counts else None, kept_codes=c[0].t, kept_scales=c[1].t,
                                 workspace=view)
        assert np.array_equal(y.get(), z)
        for got, want in zip(c, R.store(*R.encode(z, 8), 8, c[0].t.shape[1], c[1].t.shape[1])):
            assert np.array_equal(got.get(), want)


def test_experts_of_wrong_offsets(sq):  # noqa: F811
    """Offsets that leave the rows or fall are cut off at the borders: nothing outside is touched, and rows that one expert alone has are right."""
    g = rng(11)
    N, K, M = 40, 96, 30
    x, W = values(g, M, K, "bf16"), values(g, 3 * N, K, "f32")
    for offsets in ([-5, 10, 200, 300], [0, 2 ** 31 - 1, 5, 8], [-2 ** 31, 2 ** 31 - 1, -1, 4], [40, 50, 60, 70]):
        y, dx = Result(M, N, "bf16"), Result(M, K, "bf16")
        ws, view = workspace(max(sq.sparq_mx_experts_linear_workspace_bytes(M, N, K, 3), sq.sparq_mx_experts_dx_workspace_bytes(M, N, K, 3)))
        sq.sparq_mx_experts_linear(matrix(x, "bf16"), *stored(sq, W, 4), y.view, offsets=ints(offsets), workspace=view)
        y.get()
        sq.sparq_mx_experts_dx(y.view, ints(offsets), *stored(sq, W, 4), dx.view, workspace=view)
        dx.get()
        dw = Result(3 * N, K, "f32")
        sq.sparq_mx_experts_dw(y.view, ints(offsets), *stored(sq, x, 8), dw.view)
        dw.get()
        guard(ws, view)
    offsets = [-5, 10, 200, 300]
    z, size, has = E.product(R.quantised(x, 4), R.quantised(W, 4).reshape(3, N, K), offsets)
    assert has.all()
    y = Result(M, N, "f32")
    ws, view = workspace(sq.sparq_mx_experts_linear_workspace_bytes(M, N, K, 3))
    sq.sparq_mx_experts_linear(matrix(x, "bf16"), *stored(sq, W, 4), y.view, offsets=ints(offsets), workspace=view)
    close(y.get(), z, 2 * (K + 2) * u * size, "f32")


def test_what_is_not_finite_stays_in_its_rows(sq):  # noqa: F811
    """A NaN or an infinity among a row's values makes that row's results NaN and no other's; the next expert's weights touch its rows alone."""
    g = rng(12)
    N, K = 70, 130
    for counts in ([3, 2, 4], [100, 60, 90]):
        offsets = offsets_of(counts)
        M = int(offsets[-1])
        x, W = values(g, M, K, "bf16"), values(g, 3 * N, K, "f32")
        x[1, 5], x[M - 1, 100], W[N + 7, 3] = np.nan, np.inf, np.nan
        y = Result(M, N, "bf16")
        ws, view = workspace(sq.sparq_mx_experts_linear_workspace_bytes(M, N, K, 3))
        sq.sparq_mx_experts_linear(matrix(x, "bf16"), *stored(sq, W, 4), y.view, offsets=ints(offsets), workspace=view)
        nan = np.zeros((M, N), bool)
        nan[[1, M - 1]] = True
        nan[offsets[1]: offsets[2], 7] = True
        assert np.array_equal(np.isnan(y.get()), nan)


# ---- the gradients -----------------------------------------------------------------------------------------------------------------
GRAD_TYPES = [("bf16", "bf16", 0, 0), ("f16", "f32", 3, 1), ("f32", "f32", 0, 0), ("bf16", "f32", 8, 5), ("f16", "f16", 1, 0)]


def run_gradients(sq, g, counts, behind, N, K, t, o, pad, at):  # noqa: F811
    offsets, experts = offsets_of(counts), len(counts)
    M = int(offsets[-1]) + behind
    x, dy, W = values(g, M, K, "bf16"), values(g, M, N, t, 0.1), values(g, experts * N, K, "f32")
    V, X = R.quantised(W, 4).reshape(experts, N, K), R.quantised(x, 8)
    dyd, od, w = matrix(dy, t, pad, at), ints(offsets), stored(sq, W, 4)
    if behind:
        dyd[-behind:] = float("nan")                                             # rows that nobody has are not read
    dx, dw = Result(M, K, o, pad, at), Result(experts * N, K, o, pad, at)
    db = torch.full((experts, N), 7.0, device=DEV)
    ws, view = workspace(sq.sparq_mx_experts_dx_workspace_bytes(M, N, K, experts))
    sq.sparq_mx_experts_dx(dyd, od, *w, dx.view, workspace=view)
    guard(ws, view)
    ws, view = workspace(sq.sparq_mx_experts_dw_workspace_bytes(M, N, K, experts))
    sq.sparq_mx_experts_dw(dyd, od, *stored(sq, x, 8), dw.view, db=db, workspace=view)
    guard(ws, view)
    got_dx, got_dw, got_db = dx.get(), dw.get().reshape(experts, N, K), db.double().cpu().numpy()
    assert np.all(got_dx[offsets[-1]:] == -55)
    for e in range(experts):
        a, b = offsets[e], offsets[e + 1]
        close(got_dx[a:b], dy[a:b] @ V[e], 2 * (3 * N + 2) * u * (np.abs(dy[a:b]) @ np.abs(V[e])), o)
        close(got_dw[e], dy[a:b].T @ X[a:b], 2 * (3 * (b - a) + 2) * u * (np.abs(dy[a:b]).T @ np.abs(X[a:b])), o)
        assert np.all(np.abs(got_db[e] - dy[a:b].sum(0)) <= (b - a + 2) * u * np.abs(dy[a:b]).sum(0))


@pytest.mark.parametrize("counts,N,K", [("one row", 40, 96), ("few", 1, 1), ("few", 65, 129), ("sixteens", 130, 300), ("one has all", 33, 260), ("middling", 100, 520),
                                        ("middling", 515, 64), ("many", 333, 200), ("many", 64, 128), ("of one", 200, 300), ("nobody", 70, 130), ("middling", 3, 5)])
@pytest.mark.parametrize("t,o,pad,at", GRAD_TYPES)
def test_gradients(sq, counts, N, K, t, o, pad, at):  # noqa: F811
    run_gradients(sq, rng(13, N, K), COUNTS[counts], 3, N, K, t, o, pad, at)


@pytest.mark.parametrize("counts,N,K", [([900, 0, 1500, 800, 200], 1030, 1100), ([130, 1000, 2000, 70], 2056, 1700), ([1024, 512, 64, 2048], 1664, 2048), ([50] * 40, 400, 900),
                                        ([20, 0, 130] * 30, 300, 200), ([16] * 64, 100, 300), ([4096, 5001, 0, 255, 7032], 72, 1000),
                                        ([16100, 290], 40, 1024)])
@pytest.mark.parametrize("t,o", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f32", "f32")])
def test_gradients_in_large_tiles(sq, counts, N, K, t, o):  # noqa: F811
    run_gradients(sq, rng(14, N, K), counts, 0, N, K, t, o, 0, 0)


def test_gradients_of_no_rows(sq):  # noqa: F811
    """No rows at all: dw and db are zeros."""
    N, K, none = 40, 96, torch.empty(0, 40, device=DEV)
    dw, db = Result(3 * N, K, "f32", 5, 2), torch.full((3, N), 7.0, device=DEV)
    empty = torch.empty(0, dtype=torch.uint8, device=DEV)
    sq.sparq_mx_experts_dw(none, ints([0, 0, 0, 0]), empty, empty, dw.view, db=db)
    assert not dw.get().any() and not bool(db.any())
    sq.sparq_mx_experts_dx(none, ints([0, 0, 0, 0]), *stored(sq, np.ones((3 * N, K)), 4), torch.empty(0, K, device=DEV))


def test_gradients_are_the_differences(sq):  # noqa: F811
    """Of the product as it is computed: along a direction in which inputs and weights stay on their grids, so that the quantisers do not move."""
    g = rng(15)
    counts, N, K = [5, 0, 40, 19], 33, 64
    offsets, M = offsets_of(counts), 64
    x, W = g.choice([-6.0, -3, 0, 1.5, 4, 6], (M, K)), g.choice([-6.0, -2, 0.5, 0, 3, 6], (4 * N, K))
    x[:, ::32], W[:, ::32] = 6, 6                                                # (each block's largest: the scales stay)
    dy = g.choice([-1.0, 0.5, 2], (M, N))

    def y(x, W):
        out = Result(M, N, "f32")
        ws, view = workspace(sq.sparq_mx_experts_linear_workspace_bytes(M, N, K, 4))
        sq.sparq_mx_experts_linear(matrix(x, "bf16"), *stored(sq, W, 4), out.view, offsets=ints(offsets), workspace=view)
        return (out.get() * dy).sum()

    dx, dw = Result(M, K, "f32"), Result(4 * N, K, "f32")
    ws, view = workspace(sq.sparq_mx_experts_dx_workspace_bytes(M, N, K, 4))
    sq.sparq_mx_experts_dx(matrix(dy, "f32"), ints(offsets), *stored(sq, W, 4), dx.view, workspace=view)
    sq.sparq_mx_experts_dw(matrix(dy, "f32"), ints(offsets), *stored(sq, x, 8), dw.view)
    dx, dw = dx.get(), dw.get()
    free = np.arange(K) % 32 != 0
    step_x, step_w = np.where(free & (g.random((M, K)) < 0.3), -2 * x, 0), np.where(free & (g.random((4 * N, K)) < 0.3), -2 * W, 0)    # some signs turned
    assert (y(x + step_x, W) - y(x, W)) == (dx * step_x).sum()                   # whole quarters below 2^24: exact
    assert (y(x, W + step_w) - y(x, W)) == (dw * step_w).sum()


# ---- dropout ---------------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows,K", [(1, 1), (3, 7), (2, 8), (5, 513), (3, 1000), (40, 33), (2, 4100)])
@pytest.mark.parametrize("p,residual,pad,at", [(0.1, False, 0, 0), (0.5, True, 5, 3), (0.0, True, 0, 0), (1.0, False, 0, 0), (1.0, True, 1, 0), (0.9, False, 3, 2)])
def test_dropout(sq, t, rows, K, p, residual, pad, at):  # noqa: F811
    """One product and one sum, rounded in fp32: 2 u of either."""
    g = rng(16, rows, K)
    x, r = values(g, rows, K, t), values(g, rows, K, t)
    seed, offset = 0xFEDCBA9876543210, 3 + rows
    keep, q = E.kept(rows, K, p, seed, offset)
    ref = np.where(keep, x / (1 - q) if q < 1 else 0, 0)
    y = Result(rows, K, t, pad, at)
    sq.sparq_mx_dropout(matrix(x, t, pad, at), p, seed, y.view, offset=offset, residual=matrix(r, t, at, pad) if residual else None)
    off = 2 * u * np.abs(ref)
    close(y.get(), ref + r if residual else ref, off + (2 * u * np.abs(ref + r) if residual else 0), t)


def test_dropout_of_what_is_not_finite(sq):  # noqa: F811
    """Dropped is dropped: NaN and infinity among it."""
    x = np.full((4, 100), np.nan)
    x[1::2] = np.inf
    keep, _ = E.kept(4, 100, 0.5, 7, 0)
    y = Result(4, 100, "bf16")
    sq.sparq_mx_dropout(matrix(x, "bf16"), 0.5, 7, y.view)
    got = y.get()
    assert np.all(got[~keep] == 0) and np.isnan(got[::2][keep[::2]]).all() and np.isinf(got[1::2][keep[1::2]]).all()


def test_dropout_step_and_backward(sq):  # noqa: F811
    """The number in device memory moves the counter, beyond 32 and past 64 bits too; dy meets the mask that x met; the mask goes by rows, whatever lies between."""
    x = torch.ones(20, 300, device=DEV)
    masks = []
    for offset, step in ((0, 0), (0, 5), (5, 0), (2 ** 32, 0), (2 ** 64 - 1, 6), (0, -(2 ** 63))):
        y = torch.empty_like(x)
        sq.sparq_mx_dropout(x, 0.25, 99, y, offset=offset, step=torch.tensor([step], device=DEV))
        keep, _ = E.kept(20, 300, 0.25, 99, offset + step)
        assert np.array_equal((y != 0).cpu().numpy(), keep)
        masks.append(keep)
    assert np.array_equal(masks[1], masks[2]) and np.array_equal(masks[1], masks[4])
    assert len({m.tobytes() for m in masks}) == 4
    dy = torch.randn(20, 300, dtype=torch.float64).to(torch.bfloat16).to(DEV)
    dx = torch.empty_like(dy)
    sq.sparq_mx_dropout(dy, 0.25, 99, dx, offset=5)
    assert np.array_equal((dx != 0).cpu().numpy(), masks[1] & (dy != 0).cpu().numpy())


def test_dropout_keeps_its_share(sq):  # noqa: F811
    """Of 2^22 elements the kept ones' number is off by less than six standard deviations, and neighbours are independent."""
    x, y = torch.ones(1024, 4096, device=DEV), torch.empty(1024, 4096, device=DEV)
    for p in (0.1, 0.5, 1 / 65536):
        sq.sparq_mx_dropout(x, p, 12345, y)
        n, m = x.numel(), (y != 0)
        assert abs(int(m.sum()) - n * (1 - p)) <= 6 * (n * p * (1 - p)) ** 0.5 + 1e-9
        both = int((m[:, 1:] & m[:, :-1]).sum())
        assert abs(both - m[:, 1:].numel() * (1 - p) ** 2) <= 9 * (n * p * (1 - p)) ** 0.5 + 1


# ---- far apart, elsewhere, twice -----------------------------------------------------------------------------------------------------------
def test_rows_more_than_32_bits_apart(sq):  # noqa: F811
    """Rows 2^31 + 8 elements apart: offsets beyond 32 bits, of elements and of bytes, give what rows side by side give."""
    g = rng(17)
    T, K, N, ld = 3, 200, 72, (1 << 31) + 8
    far = torch.empty(2 * ld + 8192, dtype=torch.bfloat16, device=DEV)
    view = lambda n, at: far.as_strided((T, n), (ld, 1), at)      # noqa: E731
    place = ints(np.array([[2], [0], [1]]))
    w, offsets = floats(g.standard_normal((T, 1))), ints([0, 1, 3])
    near_x, near_dy = matrix(values(g, T, K, "bf16"), "bf16"), matrix(values(g, T, N, "bf16"), "bf16")
    far_x, far_dy = view(K, 0), view(N, 512)
    far_x.copy_(near_x)
    far_dy.copy_(near_dy)
    wq, x8 = stored(sq, values(g, 2 * N, K, "f32"), 4), coded_buffers(sq, T, K, 8)
    sq.sparq_mx_quantize(near_x, codes8=x8[0].t, scales8=x8[1].t)
    ws = torch.empty(1 << 16, dtype=torch.uint8, device=DEV)

    def run(x, dy, out):
        o = [out(K) for _ in range(5)] + [out(N) for _ in range(3)]
        sq.sparq_mx_gather(x, place, y=o[0])
        c = coded_buffers(sq, T, K, 4)
        sq.sparq_mx_gather(x, place, codes4=c[0].t, scales4=c[1].t)
        sq.sparq_mx_combine(x, place, o[1], weights=w, residual=x)
        dw = torch.empty(T, 1, device=DEV)
        sq.sparq_mx_combine_grad(x, place, w, dx=o[2], x=x, dweights=dw)
        sq.sparq_mx_dropout(x, 0.5, 3, o[3], residual=x)
        sq.sparq_mx_experts_dx(dy, offsets, *wq, o[4], workspace=ws)
        sq.sparq_mx_experts_linear(x, *wq, o[5], offsets=offsets, function="silu", residual=dy, workspace=ws)
        kept = coded_buffers(sq, T, N, 8)
        sq.sparq_mx_experts_linear(x, *wq, o[6], offsets=offsets, function="gelu", residual=dy, kept_codes=kept[0].t, kept_scales=kept[1].t, workspace=ws)
        sq.sparq_mx_experts_linear(x, wq[0][:N], wq[1][:N], o[7], residual=dy, workspace=ws)
        grad, db = torch.empty(2 * N, K, device=DEV), torch.empty(2, N, device=DEV)
        sq.sparq_mx_experts_dw(dy, offsets, x8[0].t, x8[1].t, grad, db=db)
        return [v.contiguous() for v in o] + [c[0].t, c[1].t, dw, kept[0].t, kept[1].t, grad, db]

    places_ = iter(range(1024, 8192, 512))
    got = run(far_x, far_dy, lambda n: view(n, next(places_)))
    want = run(near_x, near_dy, lambda n: torch.empty(T, n, dtype=torch.bfloat16, device=DEV))
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and len(got) == len(want)


def test_on_another_stream_and_twice(sq, Block):  # noqa: F811
    """The same calls on a stream of their own, at work beside the default one, and again: the same bits."""
    tokens, per, experts = 700, 3, 9
    chosen, weights = choices(2, tokens, per, experts)
    x = torch.randn(tokens, 192, device=DEV).bfloat16()
    dy = torch.randn(tokens, 192, device=DEV).bfloat16()
    torch.cuda.synchronize()

    def run():
        block = Block(tokens, per, experts, 192, 136)
        block.forward(x, chosen, weights, 0.3, None)
        block.backward(dy, weights, 0.3, None)
        return block.results()

    first = run()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        second = run()
    third = run()
    torch.cuda.synchronize()
    for k, v in first.items():
        assert torch.equal(v, second[k]) and torch.equal(v, third[k]), k


def test_the_same_rows_in_any_company(sq):  # noqa: F811
    """A row's result does not depend on which rows are beside it as long as the kernel is the same: rows of one expert among others' and alone."""
    g = rng(18)
    N, K = 96, 256
    x, W = values(g, 60, K, "bf16"), values(g, 3 * N, K, "f32")
    w = stored(sq, W, 4)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    a, b = torch.empty(60, N, device=DEV), torch.empty(30, N, device=DEV)
    sq.sparq_mx_experts_linear(matrix(x, "bf16"), *w, a, offsets=ints([0, 10, 40, 60]), workspace=ws)
    sq.sparq_mx_experts_linear(matrix(x[10:40], "bf16"), *w, b, offsets=ints([0, 0, 30, 30]), workspace=ws)
    z, size, _ = E.product(R.quantised(x, 4), R.quantised(W, 4).reshape(3, N, K), [0, 10, 40, 60])
    off = 2 * (K + 2) * u * size
    close(a.double().cpu().numpy(), z, off, "f32")
    close(b.double().cpu().numpy(), z[10:40], off[10:40], "f32")


# ---- together --------------------------------------------------------------------------------------------------------------------------
def choices(seed, tokens, per, experts):
    g = torch.Generator(device=DEV).manual_seed(seed)
    top, chosen = torch.topk(torch.randn(tokens, experts, generator=g, device=DEV), per, dim=1)
    chosen = torch.where(torch.rand(tokens, per, generator=g, device=DEV) < 0.1, -1, chosen).int()
    return chosen.contiguous(), torch.softmax(top, 1).contiguous()


def test_a_block_with_experts(sq, Block):  # noqa: F811
    """Outputs and gradients beside those of the same block in fp32 by autograd, whose operands are not quantised: they point the same way (a cosine of 0.99 a product of
    4-bit operands, up to three of them on the way)."""
    tokens, per, experts, width, hidden, p = 600, 2, 6, 256, 320, 0.1
    block = Block(tokens, per, experts, width, hidden)
    g = torch.Generator(device=DEV).manual_seed(4)
    x = torch.randn(tokens, width, generator=g, device=DEV).bfloat16()
    dy = (torch.randn(tokens, width, generator=g, device=DEV) / tokens).bfloat16()
    chosen, weights = choices(5, tokens, per, experts)
    block.forward(x, chosen, weights, p, None)
    block.backward(dy, weights, p, None)
    leaves = [v.detach().float().clone().requires_grad_() for v in (x, weights, block.w1, block.w2, block.b1)]
    xf, wf, w1, w2, b1 = leaves
    keep, q = E.kept(tokens, width, p, 17, 0)
    c = torch.zeros(tokens, width, device=DEV)
    for e in range(experts):
        for j in range(per):
            t = (chosen[:, j] == e).nonzero()[:, 0]
            h = torch.nn.functional.gelu(xf[t] @ w1[e * hidden:(e + 1) * hidden].t() + b1[e])
            c = c.index_add(0, t, wf[t, j, None] * (h @ w2[e * width:(e + 1) * width].t()))
    y = xf + c * torch.from_numpy(keep).to(DEV) / (1 - q)
    y.backward(dy.float())
    pairs = [("y", block.y.float() - xf, y - xf)] + [(n, getattr(block, n), v.grad) for n, v in zip(("dx", "dweights", "dw1", "dw2", "db1"), leaves)]
    for name, got, ref in pairs:
        if name == "dx":
            got, ref = got.float() - dy.float(), ref - dy.float()
        cosine = float(torch.nn.functional.cosine_similarity(got.detach().float().flatten(), ref.detach().flatten(), 0))
        assert cosine > 0.95, (name, cosine)


def test_a_block_in_a_graph(sq, Block):  # noqa: F811
    """Captured once and replayed on other choices and another step, beside the same calls made one by one, on a stream of its own."""
    tokens, per, experts = 300, 2, 5
    block = Block(tokens, per, experts, 128, 192)
    x = torch.randn(tokens, 128, device=DEV).bfloat16()
    dy = torch.randn(tokens, 128, device=DEV).bfloat16()
    chosen, weights = choices(1, tokens, per, experts)
    step = torch.zeros(1, dtype=torch.int64, device=DEV)

    def run():
        block.forward(x, chosen, weights, 0.2, step)
        block.backward(dy, weights, 0.2, step)

    run()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        run()
    for n in range(5):
        c, w = choices(10 + n, tokens, per, experts)
        chosen.copy_(c if n != 3 else torch.full_like(c, -1))
        weights.copy_(w)
        step.fill_(n)
        run()
        torch.cuda.synchronize()
        want = {k: v.clone() for k, v in block.results().items()}
        for v in block.results().values():
            v.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        for k, v in block.results().items():
            assert torch.equal(v, want[k]), (n, k)


def test_binding_refuses_wrong_shapes(sq):  # noqa: F811
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)      # noqa: E731
    x = torch.zeros(4, 64, device=DEV)
    wq = coded_buffers(sq, 16, 64, 4)
    cases = [
        (ValueError, "one number more", lambda: sq.sparq_mx_sort(i(4), i(1), i(4))),
        (ValueError, "place must hold 4", lambda: sq.sparq_mx_sort(i(4), i(3), i(5))),
        (ValueError, "order must hold 4", lambda: sq.sparq_mx_sort(i(4), i(3), i(4), order=i(3))),
        (TypeError, "torch.int32", lambda: sq.sparq_mx_sort(i(4).long(), i(3), i(4))),
        (ValueError, "place must hold a row", lambda: sq.sparq_mx_gather(x, i(3, 2), y=x)),
        (ValueError, "place must hold a row", lambda: sq.sparq_mx_gather(x, i(4, 0), y=x)),
        (ValueError, "one of y, codes4", lambda: sq.sparq_mx_gather(x, i(4, 2))),
        (ValueError, "same length", lambda: sq.sparq_mx_gather(x, i(4, 2), y=torch.zeros(8, 65, device=DEV))),
        (TypeError, "type", lambda: sq.sparq_mx_gather(x, i(4, 2), y=x.half())),
        (ValueError, "codes4 must hold", lambda: sq.sparq_mx_gather(x, i(4, 2), y=x, codes4=wq[0].t, scales4=wq[1].t)),
        (ValueError, "weights must hold 8", lambda: sq.sparq_mx_combine(x, i(4, 2), x, weights=torch.zeros(4, device=DEV))),
        (ValueError, "residual must hold", lambda: sq.sparq_mx_combine(x, i(4, 2), x, residual=x[:3])),
        (ValueError, "dx without weights", lambda: sq.sparq_mx_combine_grad(x, i(4, 2), dx=x)),
        (ValueError, "one of dx", lambda: sq.sparq_mx_combine_grad(x, i(4, 2), x=x)),
        (ValueError, "go together", lambda: sq.sparq_mx_combine_grad(x, i(4, 2), dweights=torch.zeros(4, 2, device=DEV))),
        (ValueError, "dx must hold", lambda: sq.sparq_mx_combine_grad(x, i(4, 2), torch.zeros(4, 2, device=DEV), dx=x[:3], x=x, dweights=torch.zeros(4, 2, device=DEV))),
        (ValueError, "w_codes must hold", lambda: sq.sparq_mx_experts_linear(x, wq[0].t, wq[1].t, torch.zeros(4, 16, device=DEV), offsets=i(3))),
        (ValueError, "bias must hold 16", lambda: sq.sparq_mx_experts_linear(x, wq[0].t, wq[1].t, torch.zeros(4, 8, device=DEV), offsets=i(3), bias=torch.zeros(8, device=DEV))),
        (ValueError, "silu", lambda: sq.sparq_mx_experts_linear(x, wq[0].t, wq[1].t, torch.zeros(4, 16, device=DEV), function="relu")),
        (ValueError, "residual must hold", lambda: sq.sparq_mx_experts_linear(x, wq[0].t, wq[1].t, torch.zeros(4, 16, device=DEV), residual=x)),
        (TypeError, "residual must have the type", lambda: sq.sparq_mx_experts_linear(x, wq[0].t, wq[1].t, torch.zeros(4, 16, device=DEV), residual=torch.zeros(4, 16, device=DEV).half())),
        (ValueError, "its scales go together", lambda: sq.sparq_mx_experts_linear(x, wq[0].t, wq[1].t, torch.zeros(4, 16, device=DEV), kept_codes=wq[0].t)),
        (ValueError, "dw must have one row", lambda: sq.sparq_mx_experts_dw(x, i(3), wq[0].t, wq[1].t, x)),
        (ValueError, "same number of rows", lambda: sq.sparq_mx_experts_dx(x, i(3), wq[0].t, wq[1].t, x[:3])),
        (sq.SparqError, "invalid", lambda: sq.sparq_mx_sort(i(20000), i(3), i(20000))),
        (sq.SparqError, "invalid", lambda: sq.sparq_mx_dropout(x, 1.5, 0, torch.empty_like(x))),
        (ValueError, "seed must be", lambda: sq.sparq_mx_dropout(x, 0.5, -1, torch.empty_like(x))),
        (TypeError, "seed must be", lambda: sq.sparq_mx_dropout(x, 0.5, 1.0, torch.empty_like(x))),
        (ValueError, "y must hold", lambda: sq.sparq_mx_dropout(x, 0.5, 1, torch.zeros(4, 65, device=DEV))),
        (TypeError, "torch.int64", lambda: sq.sparq_mx_dropout(x, 0.5, 1, torch.empty_like(x), step=i(1))),
    ]
    for error, text, call in cases:
        with pytest.raises(error, match=text):
            call()
