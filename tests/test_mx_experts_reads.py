"""Where the kernels of a block with experts read (CPU only): the device code compiled for the host (tests/host_gpu), every load by buffer held against its tensor, and the
tensors' ends against pages that may not be read."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CLANG = "/opt/rocm/llvm/bin/clang++"
FLAGS = ["-x", "hip", "--offload-host-only", "-nogpuinc", "-nohipwrapperinc", "-nogpulib", "-std=c++17", "-O1", "-w", "-I", os.path.join(HERE, "host_gpu")]


def build(folder, name):
    exe = str(folder / name)
    subprocess.run([CLANG, *FLAGS, os.path.join(HERE, name + ".cpp"), "-o", exe, "-lpthread"], check=True)
    return exe


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if shutil.which(CLANG) is None:
        pytest.skip("needs the compiler that hipcc calls")
    return build(tmp_path_factory.mktemp("reads"), "experts_reads_check")


def check(exe, *args):
    r = subprocess.run([exe, *map(str, args)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.startswith("ok"), r.stdout + r.stderr


# Last steps of 1 to 64 rows of the last expert, with nothing or something behind them; rows side by side, apart, of odd lengths.
@pytest.mark.parametrize("tile", (64, 128, 256))
@pytest.mark.parametrize("J,K,lddy,before,rows,behind", [(70, 100, 70, 100, 37, 0), (72, 100, 72, 0, 64, 1), (200, 300, 200, 10, 100, 0), (300, 260, 304, 70, 257, 5), (301, 33, 301, 64, 300, 0),
                                                         (5, 3, 9, 64, 131, 0), (1, 1, 1, 64, 131, 0), (64, 513, 64, 700, 1027, 0), (72, 40, 80, 3, 500, 0), (8, 8, 8, 0, 1, 0)])
def test_weights_gradient(program, tile, J, K, lddy, before, rows, behind):
    check(program, "dw", "bf16", tile, J, K, lddy, before, rows, behind)


@pytest.mark.parametrize("t", ("f16", "f32"))
@pytest.mark.parametrize("tile", (64, 128))
@pytest.mark.parametrize("J,K,lddy,before,rows,behind", [(70, 100, 70, 100, 37, 0), (131, 140, 131, 64, 131, 0), (5, 3, 9, 64, 131, 3), (64, 64, 64, 0, 64, 0)])
def test_weights_gradient_of_wider_types(program, t, tile, J, K, lddy, before, rows, behind):
    check(program, "dw", t, tile, J, K, lddy, before, rows, behind)


@pytest.mark.parametrize("t,tile", [("bf16", 64), ("bf16", 128), ("bf16", 256), ("f16", 64), ("f16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("rows,N,K,lddy", [(1, 64, 1, 64), (70, 200, 300, 203), (300, 64, 129, 65), (257, 130, 513, 130), (3, 5, 40, 5)])
def test_inputs_gradient(program, t, tile, rows, N, K, lddy):
    check(program, "dx", t, tile, rows, N, K, lddy)


# Blocks of columns past the last one, groups past a row's last one (wavefronts without any, a row of several groups a wavefront), columns past N.
@pytest.mark.parametrize("N,K,M,blocks", [(40, 600, 5, 2), (40, 600, 5, 1), (17, 64, 16, 1), (65, 2500, 7, 3), (100, 5000, 3, 8), (16, 512, 1, 1), (1, 1, 1, 8), (130, 4096, 2, 4)])
def test_few_rows(program, N, K, M, blocks):
    check(program, "few", N, K, M, blocks)


@pytest.mark.parametrize("tile", (64, 128, 256))
@pytest.mark.parametrize("N,K,first,second", [(40, 100, 3, 70), (300, 520, 257, 1), (1, 1, 1, 1), (130, 2100, 128, 300), (256, 512, 0, 256)])
def test_product(program, tile, N, K, first, second):
    check(program, "gemm", tile, N, K, first, second)
