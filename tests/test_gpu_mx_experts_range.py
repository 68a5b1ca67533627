"""The operators of a block with experts on the GPU at the largest sizes that the header names and where a call takes more than one launch."""
import numpy as np
import pytest
import torch

import mx_reference as R
from test_gpu_mx import DEV, sq  # noqa: F401
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
