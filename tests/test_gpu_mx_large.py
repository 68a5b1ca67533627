"""The main loops behind large calls, at the smallest sizes that enter them: workgroups that take a second tile or row, sums of many rows in parts,
and calls streamed past the caches.  Bounds are those of test_gpu_mx.py; streamed calls are their pieces to the bit."""
import pytest
import torch

from test_gpu_mx import DEV, sq, test_norm, test_product, u  # noqa: F401

pytestmark = pytest.mark.gpu

norm, product = test_norm, test_product
del test_norm, test_product


# More tiles than a GPU has places for: 256 x 256, one a CU (324, 323, 289, 272 of 256), and 128 x 128, two (728, 675 of 512), of one group of four
# steps, of several, and of one that ends inside a step or a group.
@pytest.mark.parametrize("M,N,K", [(4400, 4500, 512), (4860, 4350, 1300), (4352, 4345, 100), (4090, 4352, 2048), (3300, 3500, 200), (3200, 3450, 1111)])
@pytest.mark.parametrize("t,bias", [("bf16", True), ("f32", False)])
def test_product_of_more_tiles_than_places(sq, M, N, K, t, bias):  # noqa: F811
    product(sq, M, N, K, t, bias, 0, 0)


# More rows than places (forward), more than 1024 or 512 (backward: the weights' gradients in parts), for each number of wavefronts and of
# values a lane.
@pytest.mark.parametrize("rows,K", [(8300, 40), (8211, 508), (5200, 1000), (5133, 777), (2100, 2000), (2063, 1531), (1400, 4096), (1290, 4001), (1100, 5000), (1031, 8191)])
@pytest.mark.parametrize("t,pad,at", [("bf16", 0, 0), ("f32", 8, 0), ("f16", 5, 1)])
def test_norm_of_many_rows(sq, rows, K, t, pad, at):  # noqa: F811
    norm(sq, t, rows, K, pad, at)


def coded(sq, rows, K, bits):  # noqa: F811
    return (torch.zeros(rows, sq.sparq_mx_code_bytes(K, bits), dtype=torch.uint8, device=DEV),
            torch.zeros(rows, sq.sparq_mx_scale_bytes(K), dtype=torch.uint8, device=DEV))


@pytest.mark.parametrize("t,M,K", [(torch.bfloat16, 7001, 8192), (torch.float16, 27001, 2048), (torch.bfloat16, 56001, 1024), (torch.float16, 14003, 4096), (torch.bfloat16, 120007, 504)])
def test_a_streamed_norm_is_its_pieces(sq, t, M, K):  # noqa: F811
    g = torch.Generator(DEV).manual_seed(K)
    x, dy = (torch.randn(M, K, generator=g, device=DEV).to(t) for _ in range(2))
    gamma, beta = torch.rand(K, generator=g, device=DEV) + 0.5, torch.rand(K, generator=g, device=DEV)
    results = []
    for rows in (M, M // 5 + 1):
        c, y, dx = coded(sq, M, K, 8), torch.full_like(x, 7.0), torch.full_like(x, 7.0)
        mean, rstd, dg, db = torch.zeros(M, device=DEV), torch.zeros(M, device=DEV), torch.zeros(K, device=DEV), torch.zeros(K, device=DEV)
        ws = torch.empty(sq.sparq_mx_norm_grad_workspace_bytes(rows, K), dtype=torch.uint8, device=DEV)
        for r in range(0, M, rows):
            p = slice(r, min(M, r + rows))
            sq.sparq_mx_norm(x[p], gamma, beta, 1e-5, y[p], mean=mean[p], rstd=rstd[p], codes=c[0][p], scales=c[1][p])
            sq.sparq_mx_norm_grad(dy[p], c[0][p], c[1][p], mean[p], rstd[p], gamma, dx[p], dgamma=dg, dbeta=db, workspace=ws)
        results.append([*c, y, mean, rstd, dx])
        if rows == M:
            h = torch.empty(M, K, device=DEV)
            sq.sparq_mx_dequantize(*c, 8, h)
            h = h.double().sub_(mean.double()[:, None]).mul_(rstd.double()[:, None])
            # h's own roundings: of the difference, 2 u of the larger of its terms, and of the products
            near = h.abs() + (mean.double().abs() * rstd.double())[:, None]
            for got, terms, size in ((dg, dy.double() * h, dy.double().abs() * near), (db, dy.double(), dy.double().abs())):
                assert bool(((got.double() - terms.sum(0)).abs() <= (M + 10) * u * size.sum(0)).all())
            del h, near
    for i, (a, b) in enumerate(zip(*results)):
        assert torch.equal(a, b), i


@pytest.mark.parametrize("t,K", [(torch.bfloat16, 8192), (torch.float16, 4097), (torch.float32, 8192)])
def test_a_streamed_silu_and_fp32_codec_are_their_pieces(sq, t, K):  # noqa: F811
    M = (300 << 20) // (K * 4)
    g = torch.Generator(DEV).manual_seed(K)
    gate, up, dy = (torch.randn(M, K, generator=g, device=DEV).to(t) for _ in range(3))
    results = []
    for rows in (M, M // 4 + 1):
        c4, gc, uc = coded(sq, M, K, 4), coded(sq, M, K, 8), coded(sq, M, K, 8)
        y, dg, du = (torch.full_like(gate, 7.0) for _ in range(3))
        back4, back8 = (torch.full((M, K), 7.0, device=DEV) for _ in range(2))
        for r in range(0, M, rows):
            p = slice(r, min(M, r + rows))
            sq.sparq_mx_act("silu", gate[p], y[p], up=up[p], gate_codes=gc[0][p], gate_scales=gc[1][p], up_codes=uc[0][p], up_scales=uc[1][p])
            sq.sparq_mx_act_grad("silu", dy[p], gc[0][p], gc[1][p], dg[p], up_codes=uc[0][p], up_scales=uc[1][p], dup=du[p])
            sq.sparq_mx_quantize(gate[p], c4[0][p], c4[1][p])
            sq.sparq_mx_dequantize(c4[0][p], c4[1][p], 4, back4[p])
            sq.sparq_mx_dequantize(gc[0][p], gc[1][p], 8, back8[p])
        results.append([*c4, *gc, *uc, y, dg, du, back4, back8])
    for i, (a, b) in enumerate(zip(*results)):
        assert torch.equal(a, b), i
