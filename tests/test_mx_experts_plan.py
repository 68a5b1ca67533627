"""Which kernel the products and gradients of test_gpu_mx_experts_large.py get (CPU only): what those tests are for stays what they run when the rules change."""
import shutil
import subprocess

import pytest

import test_gpu_mx_experts_large as L
from test_mx_experts_reads import CLANG, build

FUNCTION = {None: -1, "silu": 0, "gelu": 1}


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if shutil.which(CLANG) is None:
        pytest.skip("needs the compiler that hipcc calls")
    exe = build(tmp_path_factory.mktemp("plan"), "experts_plan_check")
    return lambda *args: [int(v) for v in subprocess.run([exe, *map(str, args)], capture_output=True, text=True, check=True).stdout.split()]


def product(plan, case):
    M, experts = L.rows_of(case)
    _, _, N, K, _, f, _, residual, kept = case[:9]
    return plan("product", M, N, K, experts, int(case[0] is not None), FUNCTION[f], int(residual), int(kept))


@pytest.mark.parametrize("tile,cases", [(256, L.TILES_OF_256), (128, L.TILES_OF_128)])
def test_tiles(plan, tile, cases):
    for case in cases:
        assert product(plan, case) == [tile, 0, 1], case


def test_few_rows(plan):
    for case in L.FEW:
        assert product(plan, case) == [0, 3 if case[0] is None else 1, 1], case
        assert case[0] is None or case[3] > 4096, case                           # (several groups of 512 a wavefront)


def test_tiles_of_the_inputs_gradient(plan):
    for counts, N, K in L.GRADIENTS_OF_256:
        assert plan("dx", 2, sum(counts), N, K, len(counts)) == [256] and N >= 5 * 64


def test_company_is_of_every_kernel(plan):
    assert [plan("product", sum(c), N, K, 3, 1, FUNCTION[f], 0, 0)[0] for c, N, K, f in L.COMPANY] == [64, 0, 128, 256]
