// Workspace of the router's gradient: its size (for moegps_route_backward_workspace_bytes) and its parts.
#pragma once

#include "common.cuh"

namespace route_backward {

constexpr int kTileE = 128, kTileD = 256, kTileT = 64;   // experts, columns and tokens of a block's products
constexpr int kBlocks = 148;                             // that run at the same time: one for each SM

// The tokens are cut into `splits` parts of `per` tiles, so that (expert tiles x column tiles x splits) blocks fill the SMs.
struct Splits {
  int splits, per;
};
static inline Splits splits_of(const moegps_shape_t& s) {
  const int64_t tiles = (int64_t)((s.E + kTileE - 1) / kTileE) * ((s.D + kTileD - 1) / kTileD);
  const int64_t steps = ((int64_t)s.T + kTileT - 1) / kTileT;
  int64_t n = kBlocks / tiles;
  if (n > steps) n = steps;
  if (n < 1) n = 1;
  const int64_t per = (steps + n - 1) / n;
  return {per ? (int)((steps + per - 1) / per) : 1, (int)per};
}

struct Workspace {
  float* part;           // [splits][E][D] partial sums of dw_router
  float* logits;         // [T][E], sigmoid form only
  int32_t* pair_expert;  // [T K], softmax form only
};

static inline size_t part_bytes(const moegps_shape_t& s) { return (size_t)splits_of(s).splits * s.E * s.D * sizeof(float); }
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
