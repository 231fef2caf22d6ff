"""Where the tiles of each slot begin (csrc/tile_sums.cuh), on the host: the sums are 64 bits wide, a slot has all of its tiles or none."""
import ctypes

import numpy as np
import pytest

from tests import host_code

SOURCE = """
#include "tile_sums.cuh"
extern "C" int tiles_of(int rows, int rows_of_tile, int column_tiles) { return tile_sums::tiles_of(rows, rows_of_tile, column_tiles); }
extern "C" int most() { return tile_sums::kMost; }
// what a warp does, one lane after the other; tiles has S + 1 entries
extern "C" void sums(int* tiles, int S, int most) {
  long long before[33] = {};
  int kept = 0;
  for (int l = 0; l < 32; ++l) before[l + 1] = before[l] + tile_sums::Lane(l, S).sum(tiles);
  for (int l = 0; l < 32; ++l) {
    const int k = tile_sums::Lane(l, S).kept(tiles, before[l], most);
    kept = k > kept ? k : kept;
  }
  for (int l = 0; l < 32; ++l) tile_sums::Lane(l, S).write(tiles, before[l], kept);
  tiles[S] = kept;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return host_code.compiled(tmp_path_factory.mktemp("tile_sums"), SOURCE)


def sums(lib, counts, most):
    tiles = np.array(list(counts) + [-1], dtype=np.int32)
    lib.sums(tiles.ctypes.data_as(ctypes.c_void_p), len(counts), most)
    return tiles.tolist()


def expected(counts, most):
    begin, at = [], 0
    for n in counts:                                    # from the first slot that does not fit on, none
        begin.append(at)
        if at + n > most:
            return begin + [at] * (len(counts) + 1 - len(begin))
        at += n
    return begin + [at]


@pytest.mark.parametrize("S", [1, 2, 31, 32, 33, 63, 100, 1023, 1024])
def test_sums_of_any_number_of_slots(lib, S):
    rng = np.random.default_rng(S)
    counts = rng.choice([0, 0, 1, 2, 7, 1000], S).tolist()
    whole = [0] + np.cumsum(counts).tolist()
    assert sums(lib, counts, lib.most()) == whole
    for most in sorted({0, 1, whole[-1] // 3, whole[-1] // 2, max(0, whole[-1] - 1), whole[-1]}):
        assert sums(lib, counts, most) == expected(counts, most)


@pytest.mark.parametrize("S", [33, 600, 1024])
def test_sums_beyond_32_bits(lib, S):
    """Every other slot is the same 2^22 (2^28, 2^30) tiles: 2^31, 2^32 and more of them in all, as slots that overlap may have."""
    for each in (1 << 22, 1 << 28, 1 << 30, (1 << 30) + 1):
        counts = [each if s % 2 == 0 else 0 for s in range(S)]
        got = sums(lib, counts, lib.most())
        assert got == expected(counts, lib.most())
        assert all(0 <= b - a <= lib.most() and b - a in (0, each) for a, b in zip(got, got[1:]))


def test_a_step_of_a_grid_behind_the_last_tile_fits(lib):
    assert lib.most() + 65535 < 2 ** 31


def test_tiles_of_a_slot(lib):
    for rows in (1, 127, 128, 129, 2 ** 31 - 258, 2 ** 31 - 2, 2 ** 31 - 1):
        for tile in (128, 256):
            for columns in (1, 3, 56, 16384):
                assert lib.tiles_of(rows, tile, columns) == min(-(-rows // tile) * columns, lib.most() + 1)
    assert lib.tiles_of(0, 128, 5) == 0
