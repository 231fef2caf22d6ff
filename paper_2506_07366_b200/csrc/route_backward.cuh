// Workspace of the router's gradient: its size (for moegps_route_backward_workspace_bytes) and its parts.
#pragma once

#include <stdint.h>

#include "common.cuh"

namespace route_backward {

constexpr int kTileE = 128, kTileD = 256, kTileT = 64;   // experts, columns (at most) and tokens of a block's products
// That run at the same time, one for each SM.  A constant: the cut decides the workspace's size, which is asked for by shape,
// without a device.
constexpr int kBlocks = 148;

// Most token tiles that one sum runs over: the tensor core truncates at every accumulation.
constexpr int kMostSteps = 16;

// How the products are cut: column tiles of `cols`, tokens into `splits` parts of `per` tiles (none longer than kMostSteps).
// Taken is the cut with the least time, rounds of blocks over the SMs x a block's time: its MMAs (per x cols) and about
// three steps' worth of set-up and storing.  (4096 x 7168, 256 experts: 208 columns and 4 parts, two rounds, 79 us in all;
// 256 columns and 4 parts 82 us.)
struct Cut {
  int cols, splits, per;
};
static inline Cut cut_of(const moegps_shape_t& s) {
  const int64_t steps = ((int64_t)s.T + kTileT - 1) / kTileT, least = (steps + kMostSteps - 1) / kMostSteps;
  Cut best = {kTileD, 1, (int)(steps > 0 ? steps : 1)};
  int64_t best_time = INT64_MAX;
  for (int cols = kTileD; steps > 0 && cols >= kTileD / 2; cols -= 16) {
    const int64_t tiles = (int64_t)((s.E + kTileE - 1) / kTileE) * ((s.D + cols - 1) / cols);
    for (int r = 0; r <= 4; ++r) {
      int64_t n = r * kBlocks / tiles;
      n = n < least ? least : n > steps ? steps : n;
      const int64_t per = (steps + n - 1) / n;
      n = (steps + per - 1) / per;
      const int64_t time = (tiles * n + kBlocks - 1) / kBlocks * (per + 3) * cols;
      if (time < best_time) {
        best_time = time;
        best = {cols, (int)n, (int)per};
      }
    }
  }
  return best;
}

struct Workspace {
  float* part;           // [splits][E][D] partial sums of dw_router
  float* logits;         // [T][E], sigmoid form only
  int32_t* pair_expert;  // [T K], softmax form only
};

static inline size_t part_bytes(const moegps_shape_t& s) { return (size_t)cut_of(s).splits * s.E * s.D * sizeof(float); }
static inline size_t bytes(const moegps_shape_t& s) {
  return 32 + part_bytes(s) + (size_t)s.T * (s.gate_mode == 1 ? s.E : s.K) * 4;
}

static inline Workspace carve(const moegps_shape_t& s, void* base) {
  // partial sums are stored 32 bytes at a time
  char* p = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(base) + 31) & ~(uintptr_t)31);
  char* rest = p + part_bytes(s);
  return {reinterpret_cast<float*>(p), reinterpret_cast<float*>(rest), reinterpret_cast<int32_t*>(rest)};
}

}  // namespace route_backward
