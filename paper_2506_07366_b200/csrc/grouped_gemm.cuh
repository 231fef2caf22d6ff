// What the grouped GEMM kernels share: the tile and ring geometry, the table of tiles over ragged slots and
// the tensor maps.  (The kernels themselves: expert_ffn.cu, expert_ffn_backward.cu.)
#pragma once

#include "common.cuh"
#include "sm100.cuh"

namespace grouped_gemm {

constexpr int BM = 128;            // rows per tile
constexpr int BNACC = 256;         // accumulator columns per tile
#ifndef MOEGPS_FFN_BK
#define MOEGPS_FFN_BK 64
#endif
// K elements per stage = one swizzle row of BK*2 bytes.  Measured on B200: 64 (128-byte rows, 4
// stages of 48 KiB) beats 32 (64-byte rows, 8 stages of 24 KiB) by about 25 %: TMA moves 128-byte
// rows far more efficiently, which outweighs the deeper ring.
constexpr int BK = MOEGPS_FFN_BK;
constexpr int kRowBytes = BK * 2;
constexpr int kABytes = BM * BK * 2;
constexpr int kBHalfBytes = 128 * BK * 2;
constexpr int kStageBytes = kABytes + 2 * kBHalfBytes;       // 48 KiB
constexpr int kMaxS = 1024;

template <int kStages_, int kAccs_, int kEpiWarps_, int kCtasPerSm_>
struct GemmCfg {
  static constexpr int kStages = kStages_;        // ring depth (48 KiB per stage)
  static constexpr int kAccs = kAccs_;            // 256-column TMEM accumulators
  static constexpr int kEpiWarps = kEpiWarps_;    // 4: one per TMEM lane quarter; 8: two per quarter, half the columns each
  static constexpr int kCtasPerSm = kCtasPerSm_;
  static constexpr int kThreads = 64 + 32 * kEpiWarps_;   // producer warp, MMA warp, epilogue warps
  static constexpr int kTmemCols = 256 * kAccs_;
};
using WideCfg = GemmCfg<256 / BK, 2, 8, 1>;       // 192 KiB of ring

// Per-CTA copy of what decoding a tile needs.  tile_base[s] = first tile index of slot s.
struct __align__(16) Tables {
  int32_t tile_base[kMaxS + 1];
};

constexpr int kStageRowBytes = 80;                 // epilogue staging: 64 payload bytes per row, conflict-free pitch
constexpr int kStagingBytesPerWarp = 32 * kStageRowBytes;

template <class Cfg>
constexpr size_t smem_bytes_of() {
  return 1024 /* alignment slack */ + (size_t)Cfg::kStages * kStageBytes + sizeof(Tables) + 256 +
         (size_t)Cfg::kEpiWarps * kStagingBytesPerWarp;
}
static_assert(smem_bytes_of<WideCfg>() <= 227 * 1024, "one CTA per SM");

struct TileCoord {
  int m0;        // first row of the tile in the permuted buffer
  int row_end;   // one past the last row of the slot's extent
  int n_tile;
  int expert;
};

template <int kRows = BM>
__device__ __forceinline__ TileCoord decode_tile(const Tables& tb, const int32_t* __restrict__ slot_row_off,
                                               const int32_t* __restrict__ slot_expert, int S, int tile, int n_tiles) {
  int lo = 0, hi = S;                 // find s with tile_base[s] <= tile < tile_base[s+1]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (tb.tile_base[mid] <= tile) lo = mid; else hi = mid;
  }
  const int s = lo;
  const int local = tile - tb.tile_base[s];
  const int mt = (tb.tile_base[s + 1] - tb.tile_base[s]) / n_tiles;   // row tiles of this slot
  TileCoord c;
  c.n_tile = local / mt;
  // (the slot tables are a few KiB that every CTA reads: they stay in L1/L2; only slots that passed
  // the checks of the table build own tiles, so these values are in range)
  c.m0 = __ldg(slot_row_off + s) + (local % mt) * kRows;
  c.row_end = __ldg(slot_row_off + s + 1);
  c.expert = __ldg(slot_expert + s);
  return c;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// One 32-column chunk of an epilogue warp's 32 rows (lane = row, 16 packed bf16 pairs) -> global, through the
// warp's staging buffer: four lanes per row, i.e. whole 64-byte segments (see drain_tile in expert_ffn.cu).
__device__ __forceinline__ void store_chunk(const uint32_t (&o)[16], uint8_t* staging, int lane, __nv_bfloat16* out, int row0,
                                            int row_end, int col_begin, int n_dim) {
  uint4* mine = reinterpret_cast<uint4*>(staging + lane * kStageRowBytes);
#pragma unroll
  for (int v = 0; v < 4; ++v) mine[v] = make_uint4(o[4 * v], o[4 * v + 1], o[4 * v + 2], o[4 * v + 3]);
  __syncwarp();
  const int piece = lane & 3;                       // which 16 bytes of the row's 64
  const int col = col_begin + 8 * piece;
#pragma unroll
  for (int it = 0; it < 4; ++it) {
    const int r = it * 8 + (lane >> 2);
    const uint4 val = *reinterpret_cast<const uint4*>(staging + r * kStageRowBytes + piece * 16);
    const int row = row0 + r;
    if (row < row_end && col + 8 <= n_dim) *reinterpret_cast<uint4*>(out + (size_t)row * n_dim + col) = val;
  }
  __syncwarp();
}

// Tiles per slot and their exclusive prefix sum -> tb.tile_base[0..S]; the total is tb.tile_base[S], after the
// caller's next __syncthreads().  All kThreads threads of the block call it.  Only the S entries in use are walked: with
// all 1024 this took over 2 us of a 12 us launch on an 8-slot layer.
// A slot whose extent is not inside [0, rcap] (offsets negative, decreasing or past the buffers) gets no
// tiles: nothing is read or written for it, and the caller is told.
template <int kThreads, int kRows = BM>       // kRows: rows of a tile
__device__ __forceinline__ void build_tables(Tables& tb, const int32_t* __restrict__ slot_row_off,
                                             const int32_t* __restrict__ slot_expert, int S, int E, int n_tiles, int rcap,
                                             int32_t* __restrict__ status) {
  for (int s = threadIdx.x; s < S; s += kThreads) {
    int cnt = 0;
    const int lo = slot_row_off[s], hi = slot_row_off[s + 1];
    const int e = slot_expert[s];
    if (lo < 0 || hi < lo || hi > rcap) {
      if (blockIdx.x == 0) moegps_report(status, MOEGPS_ERR_BAD_INDEX, s);
    } else if (hi > lo && e >= 0 && e < E) {
      cnt = ((hi - lo + kRows - 1) / kRows) * n_tiles;
    } else if (hi > lo && e >= E) {
      if (blockIdx.x == 0) moegps_report(status, MOEGPS_ERR_BAD_INDEX, s);
    }
    tb.tile_base[s] = cnt;
  }
  __syncthreads();
  // exclusive prefix sum of the counts (warp 0: lane l owns `per` consecutive entries)
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x, per = (S + 31) / 32, first = min(lane * per, S), last = min(first + per, S);
    int sum = 0;
    for (int s = first; s < last; ++s) sum += tb.tile_base[s];
    int incl = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += o;
    }
    int run = incl - sum;
    for (int s = first; s < last; ++s) {
      const int v = tb.tile_base[s];
      tb.tile_base[s] = run;
      run += v;
    }
    if (lane == 31) tb.tile_base[S] = incl;
  }
}

}  // namespace grouped_gemm

// bf16 [rows, cols] row-major; box = box_cols (64, 32 or 16) columns x box_rows rows, swizzle span =
// the box's row length, zero fill outside.
bool moegps_make_tmap_2d(CUtensorMap* tm, const void* base, uint64_t rows, uint64_t cols, uint32_t box_rows,
                         uint32_t box_cols);
// bf16 [batch, rows, cols]; box = box_cols columns x box_rows rows x 1 batch entry.
bool moegps_make_tmap_3d(CUtensorMap* tm, const void* base, uint64_t batch, uint64_t rows, uint64_t cols,
                         uint32_t box_rows, uint32_t box_cols);
// the same with the box that an epilogue warp stores: 32 columns x 32 rows
bool moegps_make_tmap_store(CUtensorMap* tm, void* base, uint64_t batch, uint64_t rows, uint64_t cols);
