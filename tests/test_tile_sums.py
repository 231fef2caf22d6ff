"""Where the tiles of each slot begin (csrc/tile_sums.cuh), on the host: no sum wraps, a slot has all of its tiles or none."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2506_07366_b200 import binding
from tests import host_code

SOURCE = """
#include "tile_sums.cuh"
extern "C" int tiles_of(int rows, int rows_of_tile, int column_tiles) { return tile_sums::tiles_of(rows, rows_of_tile, column_tiles); }
extern "C" int most() { return tile_sums::kMost; }
// what a warp does, one lane after the other; tiles has S + 1 entries
extern "C" void sums(int* tiles, int S, int most) {
  unsigned before[33] = {};
  unsigned kept = 0;
  for (int l = 0; l < 32; ++l) before[l + 1] = tile_sums::add(before[l], tile_sums::Lane(l, S).sum(tiles));
  for (int l = 0; l < 32; ++l) {
    const unsigned k = tile_sums::Lane(l, S).kept(tiles, before[l], most);
    kept = k > kept ? k : kept;
  }
  for (int l = 0; l < 32; ++l) tile_sums::Lane(l, S).write(tiles, before[l], kept);
  tiles[S] = (int)kept;
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


@pytest.mark.gpu
@pytest.mark.parametrize("S", [1, 31, 33, 64, 1000, 1024])
def test_tiles_of_many_slots_on_the_gpu(S):
    """The same sums in the kernel: slots of many lengths, every row as the formula has it; the same slots twice (they overlap, which no
    plan makes, far below the limit) give the same."""
    E, D, F = min(S, 5), 64, 72
    rng = np.random.default_rng(S)
    rows = rng.choice([0, 1, 100, 128, 129, 300], S)
    rows[0] = 5
    T = int(rows.sum())
    shape = binding.Shape(T, D, F, E, 1, S, 0, 1)
    g = torch.Generator(device="cuda").manual_seed(S)
    normal = lambda *n: torch.randn(*n, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    x, w_gate, w_up, w_down = normal(T, D), normal(E, F, D) / 8, normal(E, F, D) / 8, normal(E, D, F) / 8
    off = torch.from_numpy(np.concatenate(([0], np.cumsum(rows)))).int().cuda()
    expert = torch.from_numpy(rng.integers(0, E, S)).int().cuda()
    ctx = binding.Context(shape)
    h, y = torch.empty(T, F, dtype=torch.bfloat16, device="cuda"), torch.zeros_like(x)
    ctx.expert_ffn(x, off, expert, w_gate, w_up, w_down, h, y)
    ctx.check_status()
    e = expert.long().repeat_interleave(torch.from_numpy(rows).cuda())
    for i in range(E):
        a = x[e == i].double()
        gate = a @ w_gate[i].double().T
        want = (gate / (1 + torch.exp(-gate)) * (a @ w_up[i].double().T)) @ w_down[i].double().T
        if want.numel():
            assert (y[e == i].double() - want).abs().max() <= 2e-2 * want.abs().max()
    if S < 512:
        twice = binding.Context(binding.Shape(T, D, F, E, 1, 2 * S + 1, 0, 1))
        # back to row 0 by a slot without an expert, whose extent is empty or skipped
        table = torch.cat((off, off))
        experts = torch.cat((expert, torch.full((1,), -1, dtype=torch.int32, device="cuda"), expert))
        again = torch.zeros_like(x)
        twice.expert_ffn(x, table, experts, w_gate, w_up, w_down, h, again)
        twice.status()                                   # (the extent from the last row back to the first is reported)
        assert torch.equal(again, y)
