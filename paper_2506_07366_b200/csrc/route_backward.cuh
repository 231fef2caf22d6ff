// Workspace of the router's gradient: its size (for moegps_route_backward_workspace_bytes) and its parts.
#pragma once

#include "common.cuh"

namespace route_backward {

constexpr int kUnitRows = 64;      // rows of one expert that one block sums
constexpr int kSliceCols = 128;    // columns of x and Wr whose products one block adds up

// every expert may end in a partly filled unit
static inline int64_t max_units(const moegps_shape_t& s) { return s.E + moegps_rcap_of(s) / kUnitRows; }

static inline int slices(const moegps_shape_t& s) { return (s.D + kSliceCols - 1) / kSliceCols; }

// floats of the partial sums: of the logits first (sigmoid form), of dw_router after that
static inline size_t part_floats(const moegps_shape_t& s) {
  const size_t dw = (size_t)max_units(s) * s.D, logits = s.gate_mode == 1 ? (size_t)slices(s) * s.T * s.K : 0;
  return ((dw > logits ? dw : logits) + 3) & ~(size_t)3;
}

struct Workspace {
  int32_t* unit_first;   // [E+1] first unit of each expert, and their number
  int4* units;           // [max_units] expert, first row, end row
  float* part;           // [slices][T K] partial logits, then [max_units][D] partial sums of dw_router
  float* part_b;         // [max_units] partial sums of dbias
};

static inline size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

static inline size_t bytes(const moegps_shape_t& s) {
  const size_t n = (size_t)max_units(s);
  return up16((s.E + 1) * sizeof(int32_t)) + n * sizeof(int4) + part_floats(s) * sizeof(float) + up16(n * sizeof(float));
}

static inline Workspace carve(const moegps_shape_t& s, void* base) {
  const size_t n = (size_t)max_units(s);
  char* p = static_cast<char*>(base);
  Workspace w;
  w.unit_first = reinterpret_cast<int32_t*>(p);
  p += up16((s.E + 1) * sizeof(int32_t));
  w.units = reinterpret_cast<int4*>(p);
  p += n * sizeof(int4);
  w.part = reinterpret_cast<float*>(p);
  p += part_floats(s) * sizeof(float);
  w.part_b = reinterpret_cast<float*>(p);
  return w;
}

}  // namespace route_backward
