"""The prefixes' line of tiles at the documented limits: index arithmetic of the attention kernels, compiled for the host."""
import ctypes as C

import pytest

import native_probe

SOURCE = r"""
#include "espo_attn_common.cuh"
extern "C" long long before(int row, int rows_per_block, int tiles) { return espo::tiles_before_row(row, rows_per_block, tiles); }
extern "C" void split(long long at, int tiles, int* block, int* tile) { espo::block_and_tile(at, tiles, *block, *tile); }
"""


@pytest.fixture(scope="module")
def line(tmp_path_factory):
    lib = native_probe.compile_probe(SOURCE, tmp_path_factory.mktemp("probe"))
    lib.before.restype = C.c_longlong
    return lib


# a prefix of 2^22 pages of 128 tokens is 2^22 tiles; 64 queries a key/value head put two rows in a block
@pytest.mark.parametrize("tiles", [1, 5, (1 << 22) - 1, 1 << 22])
@pytest.mark.parametrize("rows_per_block", [2, 18, 128])
@pytest.mark.parametrize("row", [0, 1, 17, 1023, 1024, 5001, 99999])
def test_tiles_of_long_prefixes_and_many_rows(line, tiles, rows_per_block, row):
    block = row // rows_per_block
    assert line.before(row, rows_per_block, tiles) == block * tiles
    for tile in {0, tiles // 2, tiles - 1}:
        b, t = C.c_int(), C.c_int()
        line.split(C.c_longlong(block * tiles + tile), tiles, C.byref(b), C.byref(t))
        assert (b.value, t.value) == (block, tile)
