"""Experts' rows in tiles (CPU only): the device code that counts and finds them, compiled for the host (tests/host_gpu), against plain counting in 64 bits."""
import shutil

import pytest

from test_mx_experts_reads import CLANG, build, check

MOST = 2 ** 31 - 1               # rows


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if shutil.which(CLANG) is None:
        pytest.skip("needs the compiler that hipcc calls")
    return build(tmp_path_factory.mktemp("tiles"), "experts_tiles_check")


@pytest.mark.parametrize("tile", (64, 128, 256))
@pytest.mark.parametrize("rows,offsets", [(1, [0, 1]), (100, [0, 10, 100]), (1000, [0, 10, 10, 700, 1000]), (5000, [0, 0, 64, 192, 193, 4800, 4990]), (4096, list(range(0, 4097, 64))),
                                          (3000, [0] * 70 + list(range(0, 3000, 100))), (1024, list(range(1025)))])
def test_tiles(program, tile, rows, offsets):
    check(program, rows, tile, *offsets)


@pytest.mark.parametrize("tile", (128, 256))
@pytest.mark.parametrize("offsets", ([0, MOST], [0, 7, MOST], [0, MOST, MOST], [0] * 70 + [MOST], [0, 2 ** 30 + 1, MOST]), ids=("one", "two", "first", "last of 70", "halves"))
def test_as_many_rows_as_there_may_be(program, tile, offsets):
    """Rows and a tile's length together do not fit 32 bits."""
    check(program, MOST, tile, *offsets)


@pytest.mark.parametrize("rows,offsets", [(1000, [500, 0, 1000, -5, 300]), (1000, [-2 ** 31, 2 ** 31 - 1, -1, 4]), (1 << 30, ([0, 1 << 30] * 501)[:1001])], ids=("few", "beyond", "many"))
def test_offsets_that_fall(program, rows, offsets):
    """More tiles than the table has places for, or than fit 32 bits: nothing outside of it is written, no tile leaves the rows."""
    check(program, rows, 128, *offsets)
