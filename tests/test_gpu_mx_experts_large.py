"""The kernels of a block with experts that large calls get, at the smallest sizes that get them (which: test_mx_experts_plan.py asks the library's rules, without a GPU; of rows on
their way and dropout the sizes stand beside the cases).  Bounds are those of test_gpu_mx_experts.py; what moves or quantises rows is compared to the bit."""
import numpy as np
import pytest
import torch

import mx_experts_reference as E
import mx_reference as R
from test_gpu_mx import DEV, TYPES, UNIT, Result, close, guard, matrix, rng, sq, stored, u, values, workspace  # noqa: F401
from test_gpu_mx_experts import COUNTS, Whole, floats, ints, offsets_of, places, run_gradients, run_product
from test_gpu_mx_range import emptied  # noqa: F401

pytestmark = pytest.mark.gpu


# ---- products ----------------------------------------------------------------------------------------------------------------
# counts (None: a layer of M rows), rows behind them or M, N, K, type, function, bias, residual, kept, pad, at
TILES_OF_256 = [
    (None, 2900, 2900, 2100, "bf16", None, True, False, False, 0, 0),
    (None, 2905, 2901, 2850, "f32", None, False, True, False, 3, 1),
    (None, 2900, 2910, 4500, "f16", "silu", True, True, False, 0, 0),
    (None, 2900, 2900, 7000, "bf16", "gelu", True, True, True, 8, 5),
    (None, 2900, 3000, 3100, "f32", None, False, False, True, 0, 0),
    ([900, 0, 1550, 500], 2, 2900, 2100, "bf16", None, True, False, False, 0, 0),
    ([1025, 700, 1, 1230], 0, 2907, 7001, "f32", "gelu", True, True, True, 1, 0),
    ([2000, 300, 650], 3, 2900, 3601, "f16", "silu", False, False, False, 0, 0),
    ([2500, 1700, 800], 0, 5000, 2000, "bf16", None, True, False, False, 0, 0),          # (more tiles than places)
]
TILES_OF_128 = [(COUNTS["many"], 2, 1000, 200, "bf16", None, True, True, False, 0, 0), (COUNTS["many"], 0, 1030, 333, "f32", "gelu", True, True, True, 3, 1),
                ([100] * 70, 1, 300, 140, "f16", "silu", True, True, False, 0, 0)]
# of up to 48 rows together; of several groups a wavefront, each with offsets
FEW = [(None, 33, 130, 700, "bf16", "gelu", True, True, False, 0, 0), (None, 40, 65, 64, "f32", None, False, False, False, 3, 1), (None, 48, 1003, 2100, "f16", "silu", True, False, False, 0, 0),
       (COUNTS["few"], 2, 65, 4200, "bf16", "silu", True, True, False, 0, 0), (COUNTS["few"], 0, 40, 9000, "f32", None, True, False, False, 0, 0)]


def rows_of(case):
    """M and the number of experts."""
    return (case[1], 1) if case[0] is None else (sum(case[0]) + case[1], len(case[0]))


@pytest.mark.parametrize("case", TILES_OF_256 + TILES_OF_128 + FEW, ids=lambda c: "x".join(map(str, (*rows_of(c), *c[2:6]))))
def test_products(sq, case):  # noqa: F811
    counts, _, N, K, t, f, bias, residual, kept, pad, at = case
    run_product(sq, rng(41, N, K), rows_of(case)[0], N, K, None if counts is None else offsets_of(counts), t, f, bias, residual, pad, at, kept=kept)


# dx in tiles of 256 with several steps: counts, N, K
GRADIENTS_OF_256 = [([4096, 5001, 0, 255, 7032], 330, 1000), ([16100, 290], 392, 1024)]


@pytest.mark.parametrize("counts,N,K", GRADIENTS_OF_256)
@pytest.mark.parametrize("o", ("bf16", "f32"))
def test_gradients(sq, counts, N, K, o):  # noqa: F811
    run_gradients(sq, rng(42, N, K), counts, 0, N, K, "bf16", o, 0, 0)


# An expert's rows among others' and alone, of as many rows in all, so that the kernel is the same: counts, N, K, function
COMPANY = [([10, 30, 20], 96, 256, "gelu"), ([2, 5, 5], 40, 700, "silu"), ([700, 300, 800], 1000, 200, "gelu"), ([900, 1550, 500], 2900, 2100, None)]


@pytest.mark.parametrize("counts,N,K,f", COMPANY)
def test_the_same_rows_in_any_company_of_one_kernel(sq, counts, N, K, f):  # noqa: F811
    g = torch.Generator(DEV).manual_seed(N)
    M, a, b = sum(counts), counts[0], counts[0] + counts[1]
    x = torch.randn(M, K, generator=g, device=DEV).bfloat16()
    w = [torch.zeros(3 * N, p, dtype=torch.uint8, device=DEV) for p in (sq.sparq_mx_code_bytes(K, 4), sq.sparq_mx_scale_bytes(K))]
    sq.sparq_mx_quantize(torch.randn(3 * N, K, generator=g, device=DEV), *w)
    alone = torch.full_like(x, float("nan"))
    alone[: b - a] = x[a:b]
    ws = torch.empty(sq.sparq_mx_experts_linear_workspace_bytes(M, N, K, 3), dtype=torch.uint8, device=DEV)
    y, z = torch.full((M, N), 7.0, device=DEV), torch.full((M, N), 7.0, device=DEV)
    sq.sparq_mx_experts_linear(x, *w, y, offsets=ints(offsets_of(counts)), function=f, workspace=ws)
    sq.sparq_mx_experts_linear(alone, *w, z, offsets=ints([0, 0, b - a, b - a]), function=f, workspace=ws)
    assert torch.equal(y[a:b], z[: b - a]) and bool((z[b - a:] == 7).all())


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("counts,N,K", [([3, 0, 7], 40, 130), ([100, 61, 33], 72, 200), ([700, 0, 813], 1030, 300), ([2000, 300, 657], 1672, 1032)])
def test_what_nobodys_rows_hold(sq, t, counts, N, K):  # noqa: F811
    """Not numbers, or zeros: the same results to the bit, and what lies there in the results stays."""
    g = torch.Generator(DEV).manual_seed(K)
    own, behind, experts = sum(counts), 37, len(counts)
    M, offsets = own + behind, ints(offsets_of(counts))
    coded = lambda rows, n, bits: [torch.zeros(rows, p, dtype=torch.uint8, device=DEV) for p in (sq.sparq_mx_code_bytes(n, bits), sq.sparq_mx_scale_bytes(n))]      # noqa: E731
    x, dy, r = (torch.randn(M, n, generator=g, device=DEV).to(TYPES[t]) for n in (K, N, N))
    w, x4, x8 = coded(experts * N, K, 4), coded(M, K, 4), coded(M, K, 8)
    sq.sparq_mx_quantize(torch.randn(experts * N, K, generator=g, device=DEV), *w)
    sq.sparq_mx_quantize(x, *x4, *x8)
    place = torch.randperm(own, generator=g, device=DEV).int().view(own, 1)
    place[::5] = -1
    place[place == 0] = -1                                   # (refused slots' lanes read row 0, which nobody has here)
    ws = torch.empty(max(f(M, N, K, experts) for f in (sq.sparq_mx_experts_linear_workspace_bytes, sq.sparq_mx_experts_dx_workspace_bytes)), dtype=torch.uint8, device=DEV)
    results = []
    for value, scale, code in ((0.0, 0, 0), (float("nan"), 255, 0x81)):
        for v in (x, dy, r):
            v[own:] = value
        for codes, scales in (x4, x8):
            codes[own:], scales[own:] = code, scale
        there = torch.zeros(own, dtype=torch.bool, device=DEV)
        there[place[place >= 0].long()] = True
        rows = torch.where(there[:, None], dy[:own], torch.full_like(dy[:own], value))
        y, z, dx, kept = (torch.full((M, n), 7.0, dtype=TYPES[t], device=DEV) for n in (N, N, K, N))
        kept8 = [torch.full_like(v, 0xA5) for v in coded(M, N, 8)]
        dw, db, dweights = (torch.full(s, 7.0, device=DEV) for s in ((experts * N, K), (experts, N), (own, 1)))
        back = torch.full((own, N), 7.0, dtype=TYPES[t], device=DEV)
        sq.sparq_mx_experts_linear(x, *w, y, offsets=offsets, function="silu", residual=r, workspace=ws)
        sq.sparq_mx_experts_gemm(*x4, *w, K, z, offsets=offsets, workspace=ws)
        sq.sparq_mx_experts_gemm(*x4, *w, K, kept, offsets=offsets, function="gelu", kept_codes=kept8[0], kept_scales=kept8[1], workspace=ws)
        sq.sparq_mx_experts_dx(dy, offsets, *w, dx, workspace=ws)
        sq.sparq_mx_experts_dw(dy, offsets, *x8, dw, db=db)
        sq.sparq_mx_combine(rows, place, back)
        sq.sparq_mx_combine_grad(dy[:own], place, x=rows, dweights=dweights)
        for v in (y, z, dx, kept):
            assert bool((v[own:] == 7).all())
        assert all(bool((v[own:] == 0xA5).all()) for v in kept8)
        results.append([y, z, dx, kept, *kept8, dw, db, back, dweights])
    for i, (a, b) in enumerate(zip(*results)):
        assert torch.equal(a, b) and (not a.dtype.is_floating_point or bool(a.isfinite().all())), i


# ---- sort --------------------------------------------------------------------------------------------------------------------
# One workgroup whose wavefronts have several ranges' worth; and more slots than 4096 (2048 of more than 512 experts) wavefronts take 128 of.
@pytest.mark.parametrize("slots,experts", [(2049, 8), (3000, 64), (4095, 300), (4096, 1024), (4097, 5), (524289, 8), (600001, 256), (300001, 1024), (2500003, 37)])
def test_sort_of_mixed_choices(sq, slots, experts):  # noqa: F811
    g = rng(43, slots)
    choice = np.where(g.random(slots) < 0.1, g.choice([-1, experts, 2 ** 31 - 1], slots), np.minimum(g.integers(0, experts, slots), g.integers(0, experts, slots)))
    offsets, place, order = Whole(experts + 1), Whole(slots), Whole(slots)
    ws, view = workspace(sq.sparq_mx_sort_workspace_bytes(slots, experts))
    sq.sparq_mx_sort(ints(choice), offsets.t, place.t, order=order.t, workspace=view)
    for got, ref in zip((offsets, place, order), E.sort(choice, experts)):
        assert np.array_equal(got.get(), ref)
    guard(ws, view)


# ---- rows on their way ---------------------------------------------------------------------------------------------------------
# From 8192 pieces of 512 values on a wavefront makes two of them: 10500 with a last one of 9 values, 8200 with one of 491, 8196 whole ones.
@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("tokens,per,K", [(2100, 2, 2057), (4100, 3, 1003), (2049, 5, 2048)])
@pytest.mark.parametrize("weighted,residual,pad,at", [(False, False, 0, 0), (True, True, 5, 3), (True, False, 0, 0)])
def test_combine_of_many(sq, t, tokens, per, K, weighted, residual, pad, at):  # noqa: F811
    g = rng(44, tokens)
    place, rows = places(g, tokens, per)
    there = (place >= 0) & (place < rows)
    x, r = values(g, rows, K, t), values(g, tokens, K, t)
    w = np.where(there, np.float32(g.standard_normal((tokens, per))) if weighted else 1.0, 0.0)
    terms = w[..., None] * x[np.where(there, place, 0)]
    ref, size = terms.sum(1), np.abs(terms).sum(1)
    if residual:
        ref, size = ref + r, size + np.abs(r)
    xd = matrix(x, t, pad, at)
    xd[np.setdiff1d(np.arange(rows), place[there]).tolist()] = float("nan")
    y = Result(tokens, K, t, pad, at)
    sq.sparq_mx_combine(xd, ints(place), y.view, weights=floats(np.where(there, w, np.nan)) if weighted else None, residual=matrix(r, t, at, pad) if residual else None)
    close(y.get(), ref, (per + 2) * u * size, t)


# From 2048 tokens on: one wavefront a token of up to 1024 values, two of up to 2048.
@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("tokens,per,K,pad,at", [(2049, 2, 40, 0, 0), (2050, 5, 1003, 5, 3), (2051, 3, 1024, 0, 0), (2049, 5, 1030, 0, 0), (2050, 2, 2040, 1, 2), (2051, 3, 2048, 0, 0)])
def test_combine_grad_of_many(sq, t, tokens, per, K, pad, at):  # noqa: F811
    g = rng(45, tokens, K)
    place, rows = places(g, tokens, per)
    there = (place >= 0) & (place < rows)
    x, dy, w = values(g, rows, K, t), values(g, tokens, K, t, 0.1), np.float32(g.standard_normal((tokens, per))).astype(np.float64)
    rows_there = np.where(there, place, 0)
    dx, has = np.zeros((rows, K)), np.zeros(rows, bool)
    dx[place[there]], has[place[there]] = (w[..., None] * dy[:, None])[there], True
    dw, size = (np.where(there, np.einsum("tk,tjk->tj", a(dy), a(x)[rows_there]), 0.0) for a in (np.asarray, np.abs))
    xd, dyd, pd, wd = matrix(x, t, pad, at), matrix(dy, t, at, pad), ints(place), floats(w)
    a, b, both, alone = Result(rows, K, t, pad, at), Result(rows, K, t), torch.full((tokens, per), 9.0, device=DEV), torch.full((tokens, per), 9.0, device=DEV)
    sq.sparq_mx_combine_grad(dyd, pd, wd, dx=a.view, x=xd, dweights=both)
    sq.sparq_mx_combine_grad(dyd, pd, wd, dx=b.view)
    sq.sparq_mx_combine_grad(dyd, pd, x=xd, dweights=alone)
    for got in (a, b):
        got = got.get()
        assert np.all(got[~has] == -55)
        close(got[has], dx[has], 0, t)
    for got in (both, alone):
        assert np.all(np.abs(got.double().cpu().numpy() - dw) <= (K + 2) * u * size)


# 16-bit calls: results of at most 16 MB go past the caches, and all of a call that moves 256 MB or more; in between nothing does.
@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("tokens,per,K", [(301, 3, 1003), (8195, 2, 4001), (14001, 2, 4096), (40001, 2, 1500)])
def test_gather_of_every_form(sq, emptied, t, tokens, per, K):  # noqa: F811
    g = rng(46, tokens)
    place, rows = places(g, tokens, per)
    there = torch.from_numpy((place >= 0) & (place < rows)).to(DEV)
    at, token = torch.from_numpy(place).to(DEV)[there], torch.arange(tokens, device=DEV)[:, None].expand(-1, per)[there]
    x = torch.randn(tokens, K, device=DEV, generator=torch.Generator(DEV).manual_seed(tokens)).to(TYPES[t])
    pitch = dict(codes4=sq.sparq_mx_code_bytes(K, 4), scales4=sq.sparq_mx_scale_bytes(K), codes8=sq.sparq_mx_code_bytes(K, 8), scales8=sq.sparq_mx_scale_bytes(K))
    of_tokens = {k: torch.empty(tokens, p, dtype=torch.uint8, device=DEV) for k, p in pitch.items()}
    sq.sparq_mx_quantize(x, *of_tokens.values())
    new = lambda: dict(y=torch.full((rows, K), 7.0, dtype=TYPES[t], device=DEV), **{k: torch.full((rows, p), 0xA5, dtype=torch.uint8, device=DEV) for k, p in pitch.items()})      # noqa: E731
    want = new()
    for k, v in dict(y=x, **of_tokens).items():
        want[k][at] = v[token]
    for forms in (("y",), ("4",), ("8",), ("4", "8"), ("y", "4"), ("y", "8"), ("y", "4", "8")):
        got = {k: v for k, v in new().items() if k[-1] in forms}
        sq.sparq_mx_gather(x, ints(place), **got)
        for k, v in got.items():
            assert torch.equal(v, want[k]), (forms, k)


# ---- dropout -------------------------------------------------------------------------------------------------------------------
def kept(rows, K, p, seed, offset):
    """Which elements dropout keeps, on the device (sums and products of 64 bits wrap), and the rounded p."""
    low, per = 0xFFFFFFFF, -(-K // 8)
    groups = torch.arange(rows * per, device=DEV)
    c = [groups & low, groups >> 32, torch.full_like(groups, offset & low), torch.full_like(groups, offset >> 32)]
    k = [seed & low, seed >> 32]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32 & low) ^ c[1] ^ k[0], b & low, (a >> 32 & low) ^ c[3] ^ k[1], a & low]
        k = [k[0] + 0x9E3779B9 & low, k[1] + 0xBB67AE85 & low]
    limit = int(np.rint(p * 65536))
    keep = torch.empty(rows * per, 8, dtype=torch.bool, device=DEV)
    for i in range(8):
        keep[:, i] = (c[i // 2] >> 16 * (i % 2) & 0xFFFF) >= limit
    return keep.view(rows, per * 8)[:, :K], limit / 65536


def test_the_devices_mask_is_the_references(sq):  # noqa: F811
    for rows, K in ((3, 1000), (40, 33)):
        for seed, offset in ((0xFEDCBA9876543210, 3), (5, 2 ** 40 + 7)):
            assert np.array_equal(kept(rows, K, 0.3, seed, offset)[0].cpu().numpy(), E.kept(rows, K, 0.3, seed, offset)[0])


# As above: kept by the caches, with and without the residual; past them.
@pytest.mark.parametrize("t,rows,K,residual", [("bf16", 6001, 4097, True), ("f16", 12003, 4096, False), ("bf16", 12001, 4101, True), ("f16", 20001, 4096, False), ("f16", 100003, 520, True),
                                               ("f32", 9001, 5000, True)])
def test_dropout_of_many(sq, emptied, t, rows, K, residual):  # noqa: F811
    g = torch.Generator(DEV).manual_seed(rows)
    x, r = (torch.randn(rows, K, generator=g, device=DEV).to(TYPES[t]) for _ in range(2))
    seed, offset, y = 0x123456789ABCDEF0, 2 ** 33 + 1, torch.full((rows, K), 7.0, dtype=TYPES[t], device=DEV)
    sq.sparq_mx_dropout(x, 0.3, seed, y, offset=offset, residual=r if residual else None)
    keep, q = kept(rows, K, 0.3, seed, offset)
    for a in range(0, rows, 4096):                           # (in pieces, or 64 bits take the memory)
        b = slice(a, a + 4096)
        ref = torch.where(keep[b], x[b].double() / (1 - q), 0.0)
        off = 2 * u * ref.abs()
        if residual:
            ref = ref + r[b].double()
            off += 2 * u * ref.abs()
        off += UNIT[t] * ref.abs() * (1 + 2 ** -7) + (2.0 ** -25 if t == "f16" else 0.0)
        assert bool(((y[b].double() - ref).abs() <= off).all()), a
