// Exclusive sums of the tiles of slots, 32 lanes with some consecutive slots each.  Slots that overlap can have more tiles than an
// int32 holds: sums stop above `kMost`, and the first slot that would end behind it, and all after it, get none.  (No slot gets a
// part of its tiles: decoding divides by their number.)  A lane at a time, so that a host program can do the same.  With sums 64 bits
// wide a layer of 8 slots took 0.1 us a launch more.
#pragma once

#include <stdint.h>

namespace tile_sums {

// Far above what disjoint slots in the memory of a GPU have, and a grid's step on top of it still fits an int32.
constexpr uint32_t kMost = 1u << 30;

// sums up to kMost are exact, above it is kMost + 1
__host__ __device__ inline uint32_t add(uint32_t a, uint32_t b) {
  const uint32_t n = a + b;                            // at most 2^31 + 2
  return n > kMost ? kMost + 1 : n;
}

// tiles of a slot: row tiles x column tiles
__host__ __device__ inline int32_t tiles_of(int32_t rows, int32_t rows_of_tile, int32_t column_tiles) {
  const int64_t n = (int64_t)(rows / rows_of_tile + (rows % rows_of_tile != 0)) * column_tiles;
  return n > kMost ? (int32_t)(kMost + 1) : (int32_t)n;
}

struct Lane {
  int first, last;                  // its slots
  __host__ __device__ Lane(int lane, int S) {
    const int per = (S + 31) / 32;
    first = lane * per < S ? lane * per : S;
    last = first + per < S ? first + per : S;
  }
  __host__ __device__ uint32_t sum(const int32_t* tiles) const {
    uint32_t n = 0;
    for (int s = first; s < last; ++s) n = add(n, tiles[s]);
    return n;
  }
  // before: tiles of the lanes before; the largest of the sums at the ends of its slots that is not above `most` (0: none)
  __host__ __device__ uint32_t kept(const int32_t* tiles, uint32_t before, uint32_t most) const {
    uint32_t at = before, good = 0;
    for (int s = first; s < last && at <= most; ++s) {
      at = add(at, tiles[s]);
      if (at <= most) good = at;
    }
    return good;
  }
  // kept: the largest of all lanes' kept(); tiles[s] becomes the sum before slot s
  __host__ __device__ void write(int32_t* tiles, uint32_t before, uint32_t kept) const {
    uint32_t at = before;
    for (int s = first; s < last; ++s) {
      const int32_t n = tiles[s];
      tiles[s] = (int32_t)(at < kept ? at : kept);
      at = add(at, n);
    }
  }
};

}  // namespace tile_sums
