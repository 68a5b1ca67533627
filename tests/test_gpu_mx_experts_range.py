"""The operators of a block with experts on the GPU at the largest sizes that the header names and where a call takes more than one launch."""
import numpy as np
import pytest
import torch

import mx_reference as R
from test_gpu_mx import DEV, sq, u  # noqa: F401
from test_gpu_mx_experts import ints
from test_gpu_mx_range import emptied  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("offsets", ([0, 7, 2 ** 31 - 1], [0] * 70 + [2 ** 31 - 1]), ids=("by lanes", "by a table"))
def test_product_of_as_many_rows_as_there_may_be(sq, emptied, offsets):  # noqa: F811
    """2^31 - 1 rows, nearly all of one expert; whole numbers, whose sums are exact.  All rows alike but some at the borders of both ends and in the middle."""
    M, N, K, experts = 2 ** 31 - 1, 1, 32, len(offsets) - 1
    pitch, scale_pitch = sq.sparq_mx_code_bytes(K, 4), sq.sparq_mx_scale_bytes(K)
    if torch.cuda.mem_get_info()[0] < M * (pitch + scale_pitch + 6) + (4 << 30):
        pytest.skip("needs 192 GB of device memory")
    g = np.random.default_rng(31)
    some = torch.cat([torch.arange(a, b) for a, b in ((0, 300), (2 ** 30 - 5, 2 ** 30 + 300), (M - 300, M))]).to(DEV)
    x = g.integers(-3, 4, (len(some), K)).astype(np.float64)
    x[:, 0] = 3
    W = g.integers(-3, 4, (experts * N, K)).astype(np.float64)
    W[:, 0] = 3

    def stored(v):
        c, s = R.store(*R.encode(v, 4), 4, pitch, scale_pitch)
        return torch.from_numpy(c).to(DEV), torch.from_numpy(s).to(DEV)

    alike = stored(x[:1])
    codes, scales = (torch.empty(M, p, dtype=torch.uint8, device=DEV) for p in (pitch, scale_pitch))
    codes.copy_(alike[0])
    scales.copy_(alike[1])
    for whole, part in zip((codes, scales), stored(x)):
        whole[some] = part
    expert = np.searchsorted(offsets[1:], some.cpu().numpy(), side="right")
    y = torch.full((M, N), 77.0, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(sq.sparq_mx_experts_gemm_workspace_bytes(M, N, K, experts), dtype=torch.uint8, device=DEV)
    sq.sparq_mx_experts_gemm(codes, scales, *stored(W), K, y, offsets=ints(offsets), workspace=ws)
    assert torch.equal(y[some, 0].double().cpu(), torch.from_numpy((x * W[expert]).sum(1)).to(torch.bfloat16).double())
    y[some] = float((x[0] * W[-1]).sum())
    assert bool((y == y[0]).all()) and float(y[0, 0]) == float(torch.tensor((x[0] * W[-1]).sum()).bfloat16())


# ---- more than one launch: a launch has 2^31 threads, 64 a token of up to 512 values; each held, to the bit, to calls for its pieces ----
def pieces(n):
    return [slice(a, min(n, a + (1 << 24))) for a in range(0, n, 1 << 24)]


def test_rows_on_their_way_of_more_tokens_than_a_launch_has_wavefronts(sq, emptied):  # noqa: F811
    tokens, per, K = (1 << 25) + 5, 1, 3
    g = torch.Generator(DEV).manual_seed(32)
    rows = tokens + 2
    place = torch.randperm(rows, generator=g, device=DEV)[:tokens].int().view(tokens, per)
    place[torch.rand(tokens, generator=g, device=DEV) < 0.01] = -1
    x, dy, r = (torch.randn(n, K, generator=g, device=DEV).bfloat16() for n in (tokens, tokens, rows))
    weights = torch.randn(tokens, per, generator=g, device=DEV)

    def new():
        return (torch.full((rows, K), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((rows, sq.sparq_mx_code_bytes(K, 4)), 0xA5, dtype=torch.uint8, device=DEV),
                torch.full((rows, sq.sparq_mx_scale_bytes(K)), 0xA5, dtype=torch.uint8, device=DEV), torch.full((tokens, K), 7.0, dtype=torch.bfloat16, device=DEV),
                torch.full((rows, K), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((tokens, per), 7.0, device=DEV))

    results = []
    for parts in ([slice(0, tokens)], pieces(tokens)):
        copies, codes, scales, y, dx, dweights = new()
        for p in parts:
            sq.sparq_mx_gather(x[p], place[p], y=copies, codes4=codes, scales4=scales)
            sq.sparq_mx_combine(r, place[p], y[p], weights=weights[p], residual=x[p])
            sq.sparq_mx_combine_grad(dy[p], place[p], weights[p], dx=dx, x=r, dweights=dweights[p])
        results.append((copies, codes, scales, y, dx, dweights))
    for i, (a, b) in enumerate(zip(*results)):
        assert torch.equal(a, b), i
    there = place[:, 0] >= 0
    copies, _, _, y, _, dweights = results[0]
    at = place[there, 0].long()
    assert torch.equal(copies[at], x[there]) and int((copies == 7).all(1).sum()) >= rows - int(there.sum()) and torch.equal(y[~there], x[~there])
    assert torch.equal(dweights[~there], torch.zeros_like(dweights[~there]))


def test_dropout_of_more_rows_than_a_launch_has_wavefronts(sq, emptied):  # noqa: F811
    """p and the residual of zeros leave what is kept; the generator's rows go on behind the first launch's."""
    from test_gpu_mx_experts_large import kept
    rows, K = (1 << 25) + 5, 5
    x, y = torch.ones(rows, K, dtype=torch.bfloat16, device=DEV), torch.full((rows, K), 7.0, dtype=torch.bfloat16, device=DEV)
    sq.sparq_mx_dropout(x, 0.5, 77, y, offset=9)
    keep, _ = kept(rows, K, 0.5, 77, 9)
    assert torch.equal(y, torch.where(keep, 2.0, 0.0).bfloat16())


def test_sums_of_more_columns_than_a_launch_has_workgroups(sq, emptied):  # noqa: F811
    """Experts of one and of two rows: db is the row, or a sum of two, rounded once.  dw is one product, which is exact, or a sum of two by the matrix instruction, whose adder
    may cut terms off where it aligns them, each by less than 2 u of the largest one, and the sum by as much of itself: 2 (n + 2) u of the magnitudes, n = 2, as for all products."""
    M, N, K = 3, (1 << 27) + 72, 1
    g = torch.Generator(DEV).manual_seed(33)
    dy = torch.empty(M, N, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    x = torch.tensor([[0.5], [1.0], [2.0]], device=DEV)
    c, s = (torch.zeros(M, p, dtype=torch.uint8, device=DEV) for p in (sq.sparq_mx_code_bytes(K, 8), sq.sparq_mx_scale_bytes(K)))
    sq.sparq_mx_quantize(x, codes8=c, scales8=s)
    dw, db = torch.full((2 * N, K), 9.0, device=DEV), torch.full((2, N), 9.0, device=DEV)
    ws = torch.empty(sq.sparq_mx_experts_dw_workspace_bytes(M, N, K, 2), dtype=torch.uint8, device=DEV)
    sq.sparq_mx_experts_dw(dy, ints([0, 1, 3]), c, s, dw, db=db, workspace=ws)
    d = dy.float()
    assert torch.equal(db[0], d[0]) and torch.equal(db[1], d[1] + d[2])
    assert torch.equal(dw[:N, 0], d[0] * 0.5)
    ref, size = d[1].double() + 2 * d[2].double(), d[1].double().abs() + 2 * d[2].double().abs()
    assert bool(((dw[N:, 0].double() - ref).abs() <= 8 * u * size).all())
