// Workspace of the router's gradient: its size (for moegps_route_backward_workspace_bytes) and its parts.
#pragma once

#include "common.cuh"

namespace route_backward {

constexpr int kUnitRows = 64;      // rows of one expert that one block sums

// every expert may end in a partly filled unit
static inline int64_t max_units(const moegps_shape_t& s) { return s.E + moegps_rcap_of(s) / kUnitRows; }

static inline size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

struct Workspace {
  int32_t* unit_first;   // [E+1] first unit of each expert, and their number
  int4* units;           // [max_units] expert, first row, end row
  float* part;           // [max_units][D] partial sums of dw_router
  float* part_b;         // [max_units] partial sums of dbias
  float* logits;         // [T][E], sigmoid form only
};

static inline size_t bytes(const moegps_shape_t& s) {
  const size_t n = (size_t)max_units(s);
  return up16((s.E + 1) * sizeof(int32_t)) + n * sizeof(int4) + n * s.D * sizeof(float) + up16(n * sizeof(float)) +
         (s.gate_mode == 1 ? up16((size_t)s.T * s.E * sizeof(float)) : 0);
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
  p += n * s.D * sizeof(float);
  w.part_b = reinterpret_cast<float*>(p);
  p += up16(n * sizeof(float));
  w.logits = reinterpret_cast<float*>(p);
  return w;
}

}  // namespace route_backward
