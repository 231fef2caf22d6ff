// expert_ffn4: the experts' SwiGLU FFN on 4-bit weights (mx4.cuh) over ragged slots, from the few rows of a token being
// generated to long prompts:
//   split      x = two e4m3 terms with a scale for 32 values (exact, see mx4.cuh)
//   gate + up  g = x Wg^T, u = x Wu^T, h = silu(g) u, as two terms
//   down       y = h Wd^T
// The products are block-scaled MMAs (e2m1 x e4m3, fp32 accumulators in tensor memory) with the WEIGHTS as the 128-row
// operand and the slot's rows as the other one, so that a slot of few rows costs few columns.  A weight tile is expanded to 16-byte
// groups by the TMA load that brings it (8 bytes of codes, 8 unused): 8 KB of memory traffic for 16 KB of shared memory,
// and no thread touches a weight.  The scales of the rows lie in the workspace as tensor memory wants them, tile by tile.
//
// Two ways, side by side in a call or one for all (mx4::cut_of): for runs of few rows one launch that is bound by reading
// weights (short_kernel), for long ones three that are bound by products (split_kernel, wide_kernel twice).  Every wait is bounded.
#include <type_traits>

#include "common.cuh"
#include "grouped_gemm.cuh"
#include "mx4.cuh"
#include "sm100.cuh"

namespace {

using namespace sm100;
using grouped_gemm::kMaxS;
using mx4::kChunk;
using mx4::kScaleTile;
using mx4::kTile;

__host__ __device__ constexpr int round_up(int n, int to) { return (n + to - 1) / to * to; }

// Slots that follow one another and hold copies of one expert are one run of rows (a plan puts copies side by side): their weights
// are read once, and tiles are cut from all their rows (48 tokens over 64 experts in 80 slots 55 -> 48 us).  Tiles and rows before
// each slot; a run counts as its first slot.
struct alignas(16) Runs {
  int32_t tiles[kMaxS + 1], rows[kMaxS + 1];
  uint32_t begins[kMaxS / 32];        // a bit for each slot that is not of the run before it
};

// All kThreads threads of the block call it; the sums are there after the next __syncthreads().  A slot whose extent is not inside
// [0, rcap] gets no tiles, and the caller is told.  Runs of fewer than min_rows or more than max_rows rows are left to another
// launch.  Tiles from number max_tiles on (there are so many only where slots overlap) are left out, and the caller is told.
template <int kThreads, int kRows>
__device__ __forceinline__ void build_runs(Runs& runs, const int32_t* __restrict__ slot_row_off, const int32_t* __restrict__ slot_expert,
                                           int S, int E, int rcap, int min_rows, int max_rows, int max_tiles,
                                           int32_t* __restrict__ status) {
  constexpr int kTurns = (kMaxS + kThreads - 1) / kThreads;
  const int lane = threadIdx.x & 31;
  // an expert, or a negative number where there is no copy or none that is in order
  auto key_of = [&](int s, bool report) {
    const int lo = slot_row_off[s], hi = slot_row_off[s + 1], e = slot_expert[s];
    const bool good = lo >= 0 && hi >= lo && hi <= rcap;
    if (report && (!good || (hi > lo && e >= E)) && blockIdx.x == 0) moegps_report(status, MOEGPS_ERR_BAD_INDEX, s);
    return good && e < E ? e : -1;
  };
  int key[kTurns];
#pragma unroll
  for (int i = 0; i < kTurns; ++i) {
    const int s = i * kThreads + threadIdx.x;
    if (s - lane >= S) break;                                    // (a whole warp)
    key[i] = s < S ? key_of(s, true) : -1;
    int before = __shfl_up_sync(0xffffffffu, key[i], 1);
    if (lane == 0 && s > 0) before = key_of(s - 1, false);
    const uint32_t begins = __ballot_sync(0xffffffffu, s < S && (s == 0 || key[i] != before));
    if (lane == 0) runs.begins[s / 32] = begins;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kTurns; ++i) {
    const int s = i * kThreads + threadIdx.x;
    if (s >= S) break;
    int word = s / 32, rows = 0;
    if (key[i] >= 0 && (runs.begins[word] >> lane & 1)) {
      uint32_t next = runs.begins[word] & ~((2u << lane) - 1);
      while (!next && ++word < (S + 31) / 32) next = runs.begins[word];
      rows = slot_row_off[next ? 32 * word + __ffs(next) - 1 : S] - slot_row_off[s];
      if (rows < min_rows || rows > max_rows) rows = 0;
    }
    runs.tiles[s] = rows / kRows + (rows % kRows != 0);
    runs.rows[s] = rows;
  }
  __syncthreads();
  // exclusive sums of both, a warp for each, lane l has `per` consecutive slots
  if (threadIdx.x < 64) {
    int32_t* base = threadIdx.x < 32 ? runs.tiles : runs.rows;
    const int per = (S + 31) / 32, first = min(lane * per, S), last = min(first + per, S);
    int64_t sum = 0;                                             // (slots that overlap can have more rows than an int32 holds)
    for (int s = first; s < last; ++s) sum += base[s];
    int64_t incl = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t o = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += o;
    }
    const int64_t most = threadIdx.x < 32 ? max_tiles : INT32_MAX;
    int64_t run = incl - sum;
    for (int s = first; s < last; ++s) {
      const int v = base[s];
      base[s] = (int)min(run, most);
      run += v;
    }
    if (lane == 31) {
      base[S] = (int)min(incl, most);
      if (incl > most && blockIdx.x == 0) moegps_report(status, MOEGPS_ERR_BAD_INDEX, S);
    }
  }
}

// A tile: rows row0 .. row0 + rows - 1 of one run, times tile m of its expert's outputs.
struct Tile {
  int row0, rows, m, expert, row_tile;
};

// Tiles are ordered by run, in it by groups of up to `group` row tiles, then by outputs, then by rows, so that neighbours share weights
// and the rows of a group stay in L2.
template <int kRows>
__device__ __forceinline__ Tile tile_at(const Runs& runs, const int32_t* __restrict__ slot_row_off,
                                        const int32_t* __restrict__ slot_expert, int S, int64_t t, int m_tiles, int group) {
  int lo = 0, hi = S;                 // the last s with tiles[s] * m_tiles <= t
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if ((int64_t)runs.tiles[mid] * m_tiles <= t) lo = mid; else hi = mid;
  }
  const int base = runs.tiles[lo];
  int n = runs.tiles[lo + 1] - base, local = (int)(t - (int64_t)base * m_tiles), j = 0;       // below n * m_tiles of one run
  if (n > group) {
    j = local / (group * m_tiles) * group;
    local -= j * m_tiles;
    n = min(group, n - j);
  }
  Tile c;
  c.m = local / n;
  j += local - c.m * n;
  c.row0 = __ldg(slot_row_off + lo) + j * kRows;
  c.rows = max(1, min(kRows, runs.rows[lo + 1] - runs.rows[lo] - j * kRows));    // (1: sums of rows that were cut off)
  c.expert = __ldg(slot_expert + lo);
  c.row_tile = base + j;
  return c;
}

__device__ __forceinline__ void linger() {
  for (int i = 0; i < 1000; ++i) __nanosleep(1000);           // let copies in flight land before the block retires
}

// ------------------------------------------------------------------------------------------- split
constexpr int kSplitThreads = 256;

// Sixteen columns of a row from `x` on (zeros behind column D).
struct Cols16 {
  uint4 v[2];
};
__device__ __forceinline__ Cols16 load16(const __nv_bfloat16* __restrict__ x, int col, int D) {
  Cols16 c;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    c.v[i] = make_uint4(0, 0, 0, 0);
    if (col + 8 * i < D) c.v[i] = *reinterpret_cast<const uint4*>(x + col + 8 * i);
  }
  return c;
}
// Sixteen columns for each lane -> its codes of both terms; word: the four scale bytes of the chunk that its 8 lanes hold.
// (Two lanes to a block of 32, and two values in each step behind the scaling: x 2^-k has no more bits than an fp16.  With 8
// columns for each lane and single values this arithmetic took longer than memory.)
__device__ __forceinline__ void split16(const Cols16& c, int lane, uint4 (&code)[2], uint32_t (&word)[2]) {
  const uint32_t w[8] = {c.v[0].x, c.v[0].y, c.v[0].z, c.v[0].w, c.v[1].x, c.v[1].y, c.v[1].z, c.v[1].w};
  uint32_t m2 = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) m2 = __vmaxu2(m2, w[j] & 0x7fff7fffu);
  uint32_t m = max(m2 & 0xffffu, m2 >> 16);           // as integers, NaN and infinity are the largest
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
  const uint32_t b1 = mx4::term_scale(m << 16), b2 = mx4::second_scale(b1);
  const float inv = mx4::inverse_scale(b1);
  const __half2 ratio = __float2half2_rn(mx4::scale_ratio(b1, b2));
  uint32_t out[2][4] = {};
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const __half2 y = __floats2half2_rn(__uint_as_float(w[j] << 16) * inv, __uint_as_float(w[j] & 0xffff0000u) * inv);
    const __nv_fp8x2_storage_t c1 = __nv_cvt_halfraw2_to_fp8x2(y, __NV_SATFINITE, __NV_E4M3);
    const __half2 f = __nv_cvt_fp8x2_to_halfraw2(c1, __NV_E4M3);
    const __nv_fp8x2_storage_t c2 = __nv_cvt_halfraw2_to_fp8x2(__hmul2(__hsub2(y, f), ratio), __NV_SATFINITE, __NV_E4M3);
    out[0][j >> 1] |= (uint32_t)c1 << (16 * (j & 1));
    out[1][j >> 1] |= (uint32_t)c2 << (16 * (j & 1));
  }
  // the scale bytes, from lanes 0, 2, 4, 6 of the eight
  word[0] = b1 << (8 * ((lane >> 1) & 3));
  word[1] = b2 << (8 * ((lane >> 1) & 3));
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    code[t] = make_uint4(out[t][0], out[t][1], out[t][2], out[t][3]);
    word[t] |= __shfl_xor_sync(0xffffffffu, word[t], 2);
    word[t] |= __shfl_xor_sync(0xffffffffu, word[t], 4);
  }
}

// The rows of all runs (kUnits for each count of `before`), and of each its columns in blocks of kCols, dealt to `workers` warps one
// after the other: body(first slot, row of the run, first column), until it says false.  (Without a division for each unit:
// a 64-bit one takes as long as a unit's arithmetic.)
template <int kCols, int kUnits, class Body>
__device__ __forceinline__ void for_rows(const int32_t* before, int S, int D, int worker, int workers, Body&& body) {
  const int rows = before[S] * kUnits, col_blocks = (D + kCols - 1) / kCols;
  const int row_step = workers / col_blocks, col_step = workers - row_step * col_blocks;
  int n = worker / col_blocks, block = worker - n * col_blocks, slot = 0;
  while (n < rows) {
    if (before[slot + 1] * kUnits <= n) {
      int hi = S;                                      // the last slot that begins at or before row n
      while (hi - slot > 1) {
        const int mid = (slot + hi) >> 1;
        if (before[mid] * kUnits <= n) slot = mid; else hi = mid;
      }
    }
    if (!body(slot, n - before[slot] * kUnits, block * kCols)) return;
    n = n > INT32_MAX - row_step - 1 ? INT32_MAX : n + row_step;
    block += col_step;
    if (block >= col_blocks) { block -= col_blocks; ++n; }
  }
}

// For long runs.  A warp does 512 columns of rows b, b + 32, b + 64, b + 96 of 128 rows of a tile, whose scales lie side by
// side: 16 bytes at a time (49152 rows x 2048 77 us under a profiler, 85 with 4 bytes at a time).
__global__ void __launch_bounds__(kSplitThreads)
split_kernel(const __nv_bfloat16* __restrict__ xp, const int32_t* __restrict__ slot_row_off, const int32_t* __restrict__ slot_expert,
             int S, int E, int D, int rcap, int min_rows, int max_tiles, const mx4::Rows out, int32_t* __restrict__ status) {
  constexpr int kRows = mx4::kLongRows, kUnits = 64;  // of a tile: 2 x 128 rows at most
  __shared__ Runs runs;
  launch_dependents();
  wait_for_predecessor();
  build_runs<kSplitThreads, kRows>(runs, slot_row_off, slot_expert, S, E, rcap, min_rows, INT32_MAX, max_tiles, status);
  __syncthreads();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int chunks = mx4::chunks_of(D);
  constexpr int kWarps = kSplitThreads / 32;
  for_rows<512, kUnits>(runs.tiles, S, D, blockIdx.x * kWarps + warp, gridDim.x * kWarps, [&](int slot, int unit, int col0) {
    const int first = __ldg(slot_row_off + slot), j = unit / kUnits, half = unit / 32 % 2, b = unit % 32;
    const int rows = min(kRows, runs.rows[slot + 1] - runs.rows[slot] - j * kRows), in_tile = half * 128 + b;
    if (in_tile >= rows) return true;
    const size_t row = (size_t)first + j * kRows + in_tile;
    const int col = col0 + 16 * lane;
    Cols16 v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = load16(xp + (row + 32 * q) * D, col, in_tile + 32 * q < rows ? D : 0);
    uint32_t words[2][4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      uint4 code[2];
      uint32_t word[2];
      split16(v[q], lane, code, word);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        words[t][q] = word[t];
        if (in_tile + 32 * q < rows && col < chunks * kChunk)
          *reinterpret_cast<uint4*>(out.code[t] + (row + 32 * q) * (size_t)(chunks * kChunk) + col) = code[t];
      }
    }
    if ((lane & 7) == 0 && col < chunks * kChunk) {
      uint8_t* scales =
          out.scale + ((size_t)(runs.tiles[slot] + j) * chunks + col / kChunk) * mx4::kRowScaleBytes<kRows>;
#pragma unroll
      for (int t = 0; t < 2; ++t)
        *reinterpret_cast<uint4*>(scales + mx4::row_scale_at<kRows>(in_tile, t, rows)) =
            make_uint4(words[t][0], words[t][1], words[t][2], words[t][3]);
    }
    return true;
  });
}

// ------------------------------------------------------------------------------------------- epilogues
__device__ __forceinline__ float silu(float g) { return __fdividef(g, 1.0f + __expf(-g)); }

// What a warp holds of 16 rows (a lane has one column of each) goes to memory through 1 KB of shared memory: 16 bytes a lane in
// runs of 32 or 64, where a store of one byte or bf16 by each lane for each row held the epilogue up (gate + up on 49152
// rows x 2048, F 1408, 64 experts: 1030 us, 755 without the stores).
constexpr int kStaging = 1024;

// 16 rows of h = silu(g) u for a warp's 32 outputs (one for each lane; they are one block): codes into `staging`, the first
// term's 16 rows of 32 bytes and then the second's; returns the scale byte of row lane % 16, lanes 0 to 15 of the first term's.
// Step by step over all rows, and two rows in a conversion: row by row it took 150 clocks a row, one latency after the other.
__device__ __forceinline__ uint32_t encode_h(const float (&g)[16], const float (&u)[16], uint8_t* staging, int lane) {
  float v[16];
  uint32_t top[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = silu(g[i]) * u[i];
#pragma unroll
  for (int i = 0; i < 16; ++i) top[i] = __reduce_max_sync(0xffffffffu, __float_as_uint(v[i]) & 0x7fffffffu);
  uint32_t byte = 0;
#pragma unroll
  for (int i = 0; i < 16; i += 2) {
    uint32_t b1[2], b2[2];
    float inv[2], ratio[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      b1[j] = mx4::term_scale(top[i + j]);
      b2[j] = mx4::second_scale(b1[j]);
      inv[j] = mx4::inverse_scale(b1[j]);
      ratio[j] = mx4::scale_ratio(b1[j], b2[j]);
      if ((lane & 15) == i + j) byte = lane < 16 ? b1[j] : b2[j];
    }
    uint32_t c1, c2;
    mx4::split2(v[i], v[i + 1], inv, ratio, c1, c2);
    staging[i * 32 + lane] = (uint8_t)c1;
    staging[(i + 1) * 32 + lane] = (uint8_t)(c1 >> 8);
    staging[512 + i * 32 + lane] = (uint8_t)c2;
    staging[512 + (i + 1) * 32 + lane] = (uint8_t)(c2 >> 8);
  }
  __syncwarp();
  return byte;
}

// They go to rows of `pitch` bytes; row: the first one's place there, in_tile: in its tile of `rows`; col0: the first lane's
// column; scales: of the tile and its chunk; block: which of the chunk's four.
template <int kRows>
__device__ __forceinline__ void store_h(const mx4::Rows& h, const float (&g)[16], const float (&u)[16], uint8_t* staging,
                                        int row, int in_tile, int rows, size_t pitch, int col0, uint8_t* scales, int block, int lane) {
  const uint32_t byte = encode_h(g, u, staging, lane);
  const int r = lane >> 1;                             // two lanes for each row
  if (in_tile + r < rows) {
    const size_t at = (size_t)(row + r) * pitch + col0 + 16 * (lane & 1);
#pragma unroll
    for (int t = 0; t < 2; ++t)
      *reinterpret_cast<uint4*>(h.code[t] + at) = *reinterpret_cast<const uint4*>(staging + 512 * t + 16 * lane);
  }
  if (in_tile + (lane & 15) < rows)
    scales[mx4::row_scale_at<kRows>(in_tile + (lane & 15), lane >> 4, rows) + block] = (uint8_t)byte;
  __syncwarp();
}

// ... or into the image of the tile's chunk.
template <int kRows>
__device__ __forceinline__ void store_h_image(uint8_t* image, const float (&g)[16], const float (&u)[16], uint8_t* staging,
                                              int in_tile, int rows, int block, int lane) {
  const uint32_t byte = encode_h(g, u, staging, lane);
  const int r = in_tile + (lane >> 1);
  if (r < rows) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
      *reinterpret_cast<uint4*>(image + mx4::image_code_at(r, t, rows, 2 * block + (lane & 1))) =
          *reinterpret_cast<const uint4*>(staging + 512 * t + 16 * lane);
  }
  if (in_tile + (lane & 15) < rows)
    image[mx4::row_scale_at<kRows>(in_tile + (lane & 15), lane >> 4, rows) + block] = (uint8_t)byte;
  __syncwarp();
}

// 16 rows of y for a warp's 32 outputs, col0 the first
__device__ __forceinline__ void store_y(__nv_bfloat16* __restrict__ y, const float (&v)[16], uint8_t* staging, int row, int in_tile,
                                        int rows, int D, int col0, int lane) {
#pragma unroll
  for (int i = 0; i < 16; ++i)
    reinterpret_cast<__nv_bfloat16*>(staging)[i * 32 + lane] = __float2bfloat16_rn(v[i]);
  __syncwarp();
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int r = 8 * k + (lane >> 2), col = col0 + 8 * (lane & 3);      // four lanes for each row; D is a multiple of 8
    if (in_tile + r < rows && col < D)
      *reinterpret_cast<uint4*>(y + (size_t)(row + r) * D + col) = *reinterpret_cast<const uint4*>(staging + 512 * k + 16 * lane);
  }
  __syncwarp();
}

// ------------------------------------------------------------------------------------------- short runs
// The whole FFN in one launch, for runs of few rows: what there is to do is to read the weights, and three launches in a row
// cost 35 us beside the 29 that two 4096 x 14336 experts take to read (each has to start, build its tables, fill its ring and join
// its sums).  The blocks are one for each SM, a cooperative launch, and wait for one another: all for all when the rows are split,
// then for the parts of h that they need; the weights of the next product are loaded meanwhile.
//  - A tile is two weight tiles of 128 outputs (gate and up of the same outputs, or two neighbours of down) times the rows of a
//    slot.  The K steps of all tiles are dealt to the blocks (Share).  Sums that several blocks share are added up in the order of
//    the blocks, by the one that begins the tile: it is the last tile of that block and the first of the other (there are mostly
//    two), whose part is there by then.  A tile of down that three or more share is added up by all of them, some of the rows
//    each, at the end.  (Joined by the block that came last, behind a fence and an atomic count, it took 5.5
//    us at the end of each product; down by the first of five blocks 8, and two blocks that add up half of the rows each 6.6.)
//  - Both terms of a row are columns of one MMA (of few columns it takes 40 clocks whatever their number: it waits for its 128
//    weight rows), side by side in the accumulator, and added up in the epilogue.
//  - x and h lie in the workspace as the images that a chunk of a tile has in shared memory (512 bytes of scales, then 128-byte
//    rows, swizzled): one bulk copy for each chunk.
//  - What a step costs beside its bytes: a wait, an expected count and a TMA load take one thread 300 clocks, so a stage is two
//    weight tiles, 16 KB of memory, and the warp that loads rows also states the bytes and brings the second tile's scales (with
//    weights that lie in L2, 4096 rows of an expert 4096 x 4096 in tiles of 32: 451 us, 432 so); the waits around four MMAs take 380 clocks in which the tensor core, which holds few of
//    them, runs dry, so two warps issue, each for its tile of the two (one warp for both: 409 ns for a stage, memory takes 370).
// Warps: 0 loads weights; 1..7 split the rows first (eight rows of 7168 columns 5.1 us after the start, 8.1 with four warps), then 2 loads
//    rows, 1 and 3 issue products, 4..7 drain the accumulators.
template <int kRows_, int kStages_>
struct Short {
  static constexpr int kRows = kRows_;                 // of a tile at most
  static constexpr int kStages = kStages_;
  static constexpr int kFlag = kRows == 48 ? 0 : 1;    // of ffn4_attr_done
  static constexpr int kCols = 2 * kRows;              // accumulator columns of a weight tile: both terms
  static constexpr int kABytes = kTile * kChunk;       // a weight tile in shared memory; half of them are loaded
  static constexpr int kImage = mx4::kImageBytes<kRows>;
  static constexpr int kScalesAt = 2 * kABytes;        // of a stage: the weights' scales, then the image, its rows from a multiple of 1024
  static constexpr int kImageAt = kScalesAt + 3 * kScaleTile;
  static constexpr int kStageBytes = round_up(kImageAt + kImage, 1024);
  static constexpr int kStagingOffset = kStages * kStageBytes;
  static constexpr int kTablesOffset = kStagingOffset + 4 * kStaging;
  static constexpr int kBarsOffset = kTablesOffset + (int)sizeof(Runs);
  static constexpr int kAccCols = 2 * kCols;
  static constexpr int kColsUsed = 2 * kAccCols + 16 * kStages;      // each issuing warp has its own copies of the scales
  static constexpr int kTmemCols = kColsUsed <= 256 ? 256 : 512;
  static constexpr int kThreads = 256;
  static constexpr size_t kSmem = 1024 + kBarsOffset + 256;
  static_assert((kImageAt + kScaleTile) % 1024 == 0, "swizzled rows");
  static_assert(kRows % 16 == 0 && kCols <= 128 && kColsUsed <= 512 && kSmem <= 227 * 1024, "does not fit");
  static_assert(kSmem > 114 * 1024, "one block for each SM: the blocks wait for one another");
};

// What a block does: `left` K steps of the tiles one after the other, from step `chunk` of tile `tile` on.  The steps are dealt
// evenly, but whole tiles where that makes no block's share longer by more than kWorth steps: a step takes some 0.4 us, and parts of
// a tile cost 4 to 6 to join (256 tokens of 8 experts 512 x 1024: 27.0 us in parts, 20.8 whole; one token of two 4096 x 14336
// experts, where whole tiles of gate + up are 16 steps more: 51.3 and 53.7).  (32-bit divisions where they can be: a 64-bit one
// takes half a microsecond.)
struct Share {
  static constexpr int kWorth = 14;
  int64_t each;                     // units of a block, one more in the first `more`
  int more, unit;                   // unit: steps that are dealt together
  int64_t left, tile;
  int chunk;
  __device__ Share(int64_t tiles, int chunks, int grid, int block) {
    each = left = tile = more = chunk = 0;
    unit = 1;
    if (tiles <= 0) return;
    const int64_t rounds = tiles >> 31 ? (tiles + grid - 1) / grid : ((uint32_t)tiles + grid - 1) / (uint32_t)grid;
    // rounds * chunks - steps / grid <= kWorth
    if ((rounds * grid - tiles) * chunks <= (int64_t)kWorth * grid) unit = chunks;
    const int64_t units = unit == 1 ? tiles * chunks : tiles;
    if (units >> 32) {
      each = units / grid;
      more = (int)(units % grid);
    } else {
      each = (uint32_t)units / (uint32_t)grid;
      more = (uint32_t)units % (uint32_t)grid;
    }
    const int64_t begin = begin_of(block);
    left = begin_of(block + 1) - begin;
    tile = begin >> 32 ? begin / chunks : (uint32_t)begin / (uint32_t)chunks;
    chunk = (int)(begin - tile * chunks);
  }
  __device__ int64_t begin_of(int b) const { return (b * each + min(b, more)) * unit; }
  // the blocks that share a tile of block b
  __device__ int first_of(int64_t t, int chunks, int b) const {
    while (begin_of(b) > t * chunks) --b;
    return b;
  }
  __device__ int last_of(int64_t t, int chunks, int b) const {
    while (begin_of(b + 1) < (t + 1) * chunks) ++b;
    return b;
  }
};

__device__ __forceinline__ unsigned long long load_acquire(const unsigned long long* p) {
  unsigned long long v;
  asm volatile("ld.acquire.gpu.global.u64 %0, [%1];" : "=l"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ int load_acquire(const int* p) {
  int v;
  asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void add_release(int* p, int n) {
  asm volatile("red.release.gpu.global.add.s32 [%0], %1;" ::"l"(p), "r"(n) : "memory");
}

// polls until ready() holds, for a limited time
template <class Ready>
__device__ __forceinline__ bool poll(volatile int* abort_flag, Ready&& ready) {
  const long long t0 = clock64();
  while (!ready()) {
    if (*abort_flag) return false;
    if (clock64() - t0 > kWaitLimitCycles) {
      *abort_flag = 1;
      return false;
    }
  }
  return true;
}

// The blocks' barrier, once in a launch: a count in the context's memory that only grows, by the number of blocks each time.
// It serves all launches of a context, on whatever streams: no block of another one arrives before all of a launch's have.  For there
// are as many blocks as SMs, all resident at once (the launch is cooperative), and each takes more than half of an SM's shared
// memory, so a block of the other launch finds room where one has retired; and every block waits here before it retires.  (Fewer blocks
// than SMs, or a block that does not wait, and the counts of two launches mix.  A block that retires because a wait ran out does so
// too, but then MOEGPS_ERR_TIMEOUT is recorded in the same context.)
struct Meeting {
  unsigned long long* count;
  volatile unsigned long long* goal;               // shared memory: what the count is when all have come; 0 = not here yet
  // by one thread, after a barrier behind the others' writes
  __device__ void arrive() const {
    __threadfence();
    const unsigned long long n = gridDim.x, old = atomicAdd(count, 1ull);
    *goal = (old / n + 1) * n;
  }
  __device__ bool wait(volatile int* abort_flag) const {
    return poll(abort_flag, [&]() { const unsigned long long want = *goal; return want && load_acquire(count) >= want; });
  }
};

// this thread's writes to global memory before, and what it reads there after, an exchange with bulk copies
__device__ __forceinline__ void fence_proxy_async_global() { asm volatile("fence.proxy.async.global;" ::: "memory"); }

template <class Cfg>
__global__ void __launch_bounds__(Cfg::kThreads, 1)
short_kernel(const __grid_constant__ CUtensorMap tm_gate, const __grid_constant__ CUtensorMap tm_up,
             const __grid_constant__ CUtensorMap tm_down, const uint8_t* __restrict__ gate_scale, const uint8_t* __restrict__ up_scale,
             const uint8_t* __restrict__ down_scale, const __nv_bfloat16* __restrict__ xp, const int32_t* __restrict__ slot_row_off,
             const int32_t* __restrict__ slot_expert, int S, int E, int D, int F, int rcap, int max_rows, int max_tiles, uint8_t* x_image, uint8_t* h_image,
             __nv_bfloat16* __restrict__ y, int* part_there, int* h_there, float* partial, unsigned long long* meetings,
             int32_t* __restrict__ status) {
  constexpr int kRows = Cfg::kRows, kStages = Cfg::kStages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  Runs& runs = *reinterpret_cast<Runs*>(smem + Cfg::kTablesOffset);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + Cfg::kBarsOffset);     // [kStages]  loads -> MMAs; the one that loads rows says how many bytes
  uint64_t* empty = full + kStages;                  // [kStages]  both issuing warps -> loaders
  uint64_t* acc_full = empty + kStages;              // [2]  both issuing warps -> epilogue
  uint64_t* acc_empty = acc_full + 2;                // [2]
  volatile unsigned long long* goal = reinterpret_cast<volatile unsigned long long*>(acc_empty + 2);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 3);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  static_assert((2 * kStages + 5) * 8 + 8 <= 256, "barriers fit their space");

  const int warp = uniform_warp_index(), lane = threadIdx.x & 31;
  const int d_chunks = mx4::chunks_of(D), f_chunks = mx4::chunks_of(F);      // f_chunks also the tiles of gate + up
  const int d_tiles = (d_chunks + 1) / 2;                                    // of down
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 2); }
    for (int i = 0; i < 2; ++i) { mbar_init(&acc_full[i], 2); mbar_init(&acc_empty[i], 4); }
    *goal = 0;
    *abort_flag = 0;
    fence_mbar_init();
    prefetch_tensormap(&tm_gate);
    prefetch_tensormap(&tm_up);
    prefetch_tensormap(&tm_down);
  }
  if (warp == 1) {
    tmem_alloc(tmem_slot, Cfg::kTmemCols);
    tmem_relinquish();
  }
  build_runs<Cfg::kThreads, kRows>(runs, slot_row_off, slot_expert, S, E, rcap, 1, max_rows, max_tiles, status);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  const int64_t row_tiles = runs.tiles[S];
  const Share up_share(row_tiles * f_chunks, d_chunks, gridDim.x, blockIdx.x);
  const Share down_share(row_tiles * d_tiles, f_chunks, gridDim.x, blockIdx.x);
  const Meeting meeting = {meetings, goal};

  // calls body(tile, its number, k0, k1) for each tile, or part of one, of this block
  auto for_tiles = [&](const Share& share, int m_tiles, int chunks, auto&& body) {
    int64_t t = share.tile, left = share.left;
    for (int k0 = share.chunk; left > 0; k0 = 0, ++t) {
      const int k1 = (int)min((int64_t)chunks, k0 + left);
      if (!body(tile_at<kRows>(runs, slot_row_off, slot_expert, S, t, m_tiles, INT32_MAX), t, k0, k1)) return false;
      left -= k1 - k0;
    }
    return true;
  };
  auto up_tiles = [&](auto&& body) { return for_tiles(up_share, f_chunks, d_chunks, body); };
  auto down_tiles = [&](auto&& body) { return for_tiles(down_share, d_tiles, f_chunks, body); };

  // x in two terms, by all warps but the one that loads weights: a warp does 1024 columns of a row
  constexpr int kSplitters = Cfg::kThreads - 32;
  if (warp > 0) {
    const int worker = warp - 1, thread = worker * 32 + lane;
    // nothing of h or of shared sums is there yet
    if (thread < 3) part_there[thread * mx4::kMaxCtas + blockIdx.x] = 0;
    for (int64_t i = (int64_t)blockIdx.x * kSplitters + thread; i < row_tiles * f_chunks; i += (int64_t)kSplitters * gridDim.x) h_there[i] = 0;
    for_rows<1024, 1>(runs.rows, S, D, worker * gridDim.x + blockIdx.x, kSplitters / 32 * gridDim.x, [&](int slot, int r, int col0) {
      const int in_tile = r % kRows;
      const int rows_in_tile = min(kRows, runs.rows[slot + 1] - runs.rows[slot] - (r - in_tile));
      const int tile = runs.tiles[slot] + r / kRows;
      if (tile >= runs.tiles[slot + 1]) return false;      // left out, like all behind it
      uint8_t* image = x_image + (size_t)tile * d_chunks * Cfg::kImage;
      const __nv_bfloat16* x = xp + (size_t)(__ldg(slot_row_off + slot) + r) * D;
      Cols16 v[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) v[i] = load16(x, col0 + 512 * i + 16 * lane, D);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int col = col0 + 512 * i + 16 * lane;
        uint4 code[2];
        uint32_t word[2];
        split16(v[i], lane, code, word);
        if (col < d_chunks * kChunk) {
          uint8_t* at = image + (size_t)(col / kChunk) * Cfg::kImage;
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            *reinterpret_cast<uint4*>(at + mx4::image_code_at(in_tile, t, rows_in_tile, col % kChunk / 16)) = code[t];
            if ((lane & 7) == 0) *reinterpret_cast<uint32_t*>(at + mx4::row_scale_at<kRows>(in_tile, t, rows_in_tile)) = word[t];
          }
        }
      }
      return true;
    });
    fence_proxy_async_global();
    named_sync(1, kSplitters);
    if (thread == 0) meeting.arrive();
  }

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      // the two weight tiles of chunks k0 .. k1 - 1: rows m0, m1 of either matrix (m1 < 0: there is one), the first's scales at s0
      auto load = [&](const CUtensorMap* tm0, const CUtensorMap* tm1, int expert, int m0, int m1, const uint8_t* s0, int k0, int k1) {
        for (int c = k0; c < k1; ++c, s0 += kScaleTile) {
          if (!mbar_wait(&empty[stage], phase ^ 1u, abort_flag)) return false;
          uint8_t* a = smem + stage * Cfg::kStageBytes;
          tma_load_3d(a, tm0, &full[stage], c * kChunk, m0, expert);
          if (m1 >= 0) tma_load_3d(a + Cfg::kABytes, tm1, &full[stage], c * kChunk, m1, expert);
          bulk_load(a + Cfg::kScalesAt, s0, kScaleTile, &full[stage]);
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
        return true;
      };
      const bool ok = up_tiles([&](const Tile& tc, int64_t, int k0, int k1) {
        const size_t at = (((size_t)tc.expert * f_chunks + tc.m) * d_chunks + k0) * kScaleTile;
        return load(&tm_gate, &tm_up, tc.expert, tc.m * kTile, tc.m * kTile, gate_scale + at, k0, k1);
      }) && down_tiles([&](const Tile& tc, int64_t, int k0, int k1) {
        const uint8_t* s0 = down_scale + (((size_t)tc.expert * d_chunks + 2 * tc.m) * f_chunks + k0) * kScaleTile;
        return load(&tm_down, &tm_down, tc.expert, 2 * tc.m * kTile, 2 * tc.m + 1 < d_chunks ? (2 * tc.m + 1) * kTile : -1, s0, k0, k1);
      });
      if (!ok) linger();
    }
  } else if (warp == 2) {
    int stage = 0;
    uint32_t phase = 0;
    // by one lane: the rows, and the second weight tile's scales at s1 (if there is one)
    auto load = [&](const uint8_t* image, const uint8_t* s1, const Tile& tc, int chunks, int k0, int k1) {
      const uint32_t image_bytes = kScaleTile + 2 * round_up(tc.rows, 16) * kChunk;
      const uint32_t bytes = image_bytes + (s1 ? 2 : 1) * (Cfg::kABytes / 2 + kScaleTile);
      const uint8_t* from = image + ((size_t)tc.row_tile * chunks + k0) * Cfg::kImage;
      for (int c = k0; c < k1; ++c, from += Cfg::kImage) {
        if (!mbar_wait(&empty[stage], phase ^ 1u, abort_flag)) return false;
        uint8_t* a = smem + stage * Cfg::kStageBytes;
        mbar_arrive_expect_tx(&full[stage], bytes);
        bulk_load(a + Cfg::kImageAt, from, image_bytes, &full[stage]);
        if (s1) bulk_load(a + Cfg::kScalesAt + kScaleTile, s1 + (size_t)(c - k0) * kScaleTile, kScaleTile, &full[stage]);
        if (++stage == kStages) { stage = 0; phase ^= 1u; }
      }
      return true;
    };
    bool ok = true;
    if (lane == 0) {
      ok = meeting.wait(abort_flag);
      fence_proxy_async_global();
      ok = ok && up_tiles([&](const Tile& tc, int64_t, int k0, int k1) {
        return load(x_image, up_scale + (((size_t)tc.expert * f_chunks + tc.m) * d_chunks + k0) * kScaleTile, tc, d_chunks, k0, k1);
      });
    }
    ok = __all_sync(0xffffffffu, ok);
    // 32 chunks of h at a time, when the four warps that wrote each have reported
    ok = ok && down_tiles([&](const Tile& tc, int64_t, int k0, int k1) {
      const uint8_t* s1 = down_scale + ((size_t)tc.expert * d_chunks + 2 * tc.m + 1) * f_chunks * kScaleTile;
      for (int c = k0; c < k1; c += 32) {
        const int* there = h_there + (size_t)tc.row_tile * f_chunks + min(c + lane, k1 - 1);
        bool go = poll(abort_flag, [&]() { return load_acquire(there) == 4; });
        go = __all_sync(0xffffffffu, go);
        if (lane == 0 && go) {
          fence_proxy_async_global();
          go = load(h_image, 2 * tc.m + 1 < d_chunks ? s1 + (size_t)c * kScaleTile : nullptr, tc, f_chunks, c, min(c + 32, k1));
        }
        if (!__all_sync(0xffffffffu, go)) return false;
      }
      return true;
    });
    if (!ok && lane == 0) linger();
  } else if (warp == 1 || warp == 3) {
    const int which = warp >> 1;                       // of the two weight tiles
    const uint32_t base = smem_u32(smem);
    const uint32_t scale_cols = tmem_base + 2 * Cfg::kAccCols + 8 * which;
    int stage = 0, acc = 0;
    uint32_t phase = 0, acc_phase = 0;
    auto multiply = [&](bool there, const Tile& tc, int k0, int k1) {
      const uint32_t idesc = idesc_mx_e2m1_e4m3(kTile, 2 * round_up(tc.rows, 16));
      if (!warp_wait(&acc_empty[acc], acc_phase ^ 1u, abort_flag)) return false;
      tc_fence_after_sync();
      const uint32_t d = tmem_base + (uint32_t)acc * Cfg::kAccCols + which * Cfg::kCols;
      for (int c = k0; c < k1; ++c) {
        if (!warp_wait(&full[stage], phase, abort_flag)) return false;
        tc_fence_after_sync();
        const uint32_t at = base + stage * Cfg::kStageBytes;
        const uint64_t da = smem_desc_k_sw128(at + which * Cfg::kABytes), db = smem_desc_k_sw128(at + Cfg::kImageAt + kScaleTile);
        const uint32_t ws = scale_cols + 16 * stage, rs = ws + 4;      // (the ring frees a stage's columns with it)
        if (elect_one()) {
          if (there) {
            copy_scales(rs, smem_desc_scales(at + Cfg::kImageAt));
            copy_scales(ws, smem_desc_scales(at + Cfg::kScalesAt + which * kScaleTile));
#pragma unroll
            for (int j = 0; j < kChunk / mx4::kBlock; ++j)
              mma_mx(d, da + (uint64_t)((j * mx4::kBlock) >> 4), db + (uint64_t)((j * mx4::kBlock) >> 4), idesc | idesc_mx_block(j), ws,
                     rs, (c - k0) | j);
          }
          mma_commit(&empty[stage]);
        }
        if (++stage == kStages) { stage = 0; phase ^= 1u; }
      }
      if (elect_one()) mma_commit(&acc_full[acc]);
      acc ^= 1;
      if (acc == 0) acc_phase ^= 1u;
      return true;
    };
    const bool ok = up_tiles([&](const Tile& tc, int64_t, int k0, int k1) { return multiply(true, tc, k0, k1); }) &&
                    down_tiles([&](const Tile& tc, int64_t, int k0, int k1) { return multiply(2 * tc.m + which < d_chunks, tc, k0, k1); });
    if (!ok) linger();
  } else {
    const int quarter = warp & 3, thread = quarter * 32 + lane;
    uint8_t* staging = smem + Cfg::kStagingOffset + quarter * kStaging;

    int acc = 0;
    uint32_t acc_phase = 0;
    bool ok = true;
    // what a block leaves of a tile that it shares: 0 of gate + up, begun by another, of down 1 begun by another, 2 begun by itself;
    // the four warps count when it is there
    auto there_of = [&](int which, int block) { return part_there + which * mx4::kMaxCtas + block; };
    auto part = [&](int which, int block) { return partial + ((size_t)which * mx4::kMaxCtas + block) * 2 * kRows * kTile + thread; };
    auto drain = [&](auto gate_up, const Share& share, const Tile& tc, int64_t t, int k0, int k1, int chunks) {
      constexpr bool kGateUp = decltype(gate_up)::value;
      const int padded = round_up(tc.rows, 16);
      const int first = share.first_of(t, chunks, blockIdx.x), last = share.last_of(t, chunks, blockIdx.x);
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)acc * Cfg::kAccCols;
      auto read = [&](float (&v)[2][16], int r) {
        uint32_t term[2][2][16];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          tmem_ld16(taddr + m * Cfg::kCols + r, term[m][0]);
          tmem_ld16(taddr + m * Cfg::kCols + padded + r, term[m][1]);
        }
        tmem_ld_wait();
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int i = 0; i < 16; ++i) v[m][i] = __uint_as_float(term[m][0][i]) + __uint_as_float(term[m][1][i]);
      };
      // what the other blocks have of 16 rows
      auto others = [&](float (&v)[2][16], int r) {
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int i = 0; i < 16; ++i) v[m][i] = 0.0f;
        for (int b = first + 1; b <= last; ++b) {
          const float* from = part(kGateUp ? 0 : 1, b);
#pragma unroll
          for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (r + i < tc.rows) v[m][i] += __ldcg(from + (m * kRows + r + i) * kTile);
        }
      };
      if (first == (int)blockIdx.x && (kGateUp || last <= first + 1)) {
        float rest[2][16];
        if (last > first && lane == 0)
          for (int b = first + 1; ok && b <= last; ++b) ok = poll(abort_flag, [&]() { return load_acquire(there_of(kGateUp ? 0 : 1, b)) == 4; });
        ok = __all_sync(0xffffffffu, ok);
        if (ok) others(rest, 0);                       // under way while its own part is still being added up
        ok = ok && __all_sync(0xffffffffu, mbar_wait(&acc_full[acc], acc_phase, abort_flag, 64));
        tc_fence_after_sync();
        for (int r = 0; ok && r < tc.rows; r += 16) {
          float v[2][16];
          if (r > 0) others(rest, r);
          read(v, r);
#pragma unroll
          for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) v[m][i] += rest[m][i];
          if constexpr (kGateUp) {
            store_h_image<kRows>(h_image + ((size_t)tc.row_tile * f_chunks + tc.m) * Cfg::kImage, v[0], v[1], staging, r, tc.rows,
                                 quarter, lane);
          } else {
#pragma unroll
            for (int m = 0; m < 2; ++m) store_y(y, v[m], staging, tc.row0 + r, r, tc.rows, D, (2 * tc.m + m) * kTile + quarter * 32, lane);
          }
        }
        if (kGateUp) {
          fence_proxy_async_global();
          __syncwarp();
          if (lane == 0 && ok) add_release(h_there + (size_t)tc.row_tile * f_chunks + tc.m, 1);
        }
      } else {
        ok = ok && __all_sync(0xffffffffu, mbar_wait(&acc_full[acc], acc_phase, abort_flag, 64));
        tc_fence_after_sync();
        const int which = kGateUp ? 0 : 1 + (first == (int)blockIdx.x);
        float* to = part(which, blockIdx.x);
        for (int r = 0; ok && r < tc.rows; r += 16) {
          float v[2][16];
          read(v, r);
#pragma unroll
          for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (r + i < tc.rows) __stcg(to + (m * kRows + r + i) * kTile, v[m][i]);
        }
        __syncwarp();
        if (lane == 0 && ok) add_release(there_of(which, blockIdx.x), 1);
      }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&acc_empty[acc]);
      acc ^= 1;
      if (acc == 0) acc_phase ^= 1u;
      return ok;
    };
    if (lane == 0) ok = meeting.wait(abort_flag);      // the counts that are added to below have been set to zero
    ok = __all_sync(0xffffffffu, ok);
    ok = ok && up_tiles([&](const Tile& tc, int64_t t, int k0, int k1) {
      return drain(std::true_type(), up_share, tc, t, k0, k1, d_chunks);
    });
    ok = ok && down_tiles([&](const Tile& tc, int64_t t, int k0, int k1) {
      return drain(std::false_type(), down_share, tc, t, k0, k1, f_chunks);
    });
    ok = ok && down_tiles([&](const Tile& tc, int64_t t, int k0, int k1) {
      const int first = down_share.first_of(t, f_chunks, blockIdx.x), last = down_share.last_of(t, f_chunks, blockIdx.x);
      const int n = last - first + 1, i = (int)blockIdx.x - first, end = tc.rows * (i + 1) / n;
      if (n <= 2) return true;
      for (int b = first + lane; ok && b <= last; b += 32)
        ok = poll(abort_flag, [&]() { return load_acquire(there_of(1 + (b == first), b)) == 4; });
      ok = __all_sync(0xffffffffu, ok);
      for (int r = tc.rows * i / n; ok && r < end; r += 4) {
        float v[2][4] = {};
#pragma unroll 4
        for (int b = first; b <= last; ++b) {
          const float* from = part(1 + (b == first), b);
#pragma unroll
          for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (r + j < end) v[m][j] += __ldcg(from + (m * kRows + r + j) * kTile);
        }
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          const int col = (2 * tc.m + m) * kTile + thread;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (r + j < end && col < D) y[(size_t)(tc.row0 + r + j) * D + col] = __float2bfloat16_rn(v[m][j]);
        }
      }
      return ok;
    });
  }

  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) moegps_report(status, MOEGPS_ERR_TIMEOUT, (int)blockIdx.x);
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem_base, Cfg::kTmemCols);
  }
}

struct Weights {
  const uint8_t* scale[2];          // gate, up; or down
};

// ------------------------------------------------------------------------------------------- wide
// A pair of CTAs works 256 weight rows x up to 224 rows of a run; each CTA loads its 128 weight rows and half of those
// rows.  Gate + up: a CTA's 128 weight rows are 64 gate rows and the 64 up rows of the same outputs, so that a tile needs
// 224 accumulator columns and not twice that, and two tiles fit tensor memory; in the epilogue the warps of the gate's
// lanes and of the up's exchange half of their values through shared memory.
// Shared memory is what feeds the MMAs: one of 224 columns takes 112 clocks and reads 128 + 112 rows of 32 bytes, 60 clocks
// of shared memory's 128 bytes; the loads write 44 KB for eight of them, 352 clocks of 896.  (One CTA by itself reads all 224 rows, and
// at 112 columns for each of two accumulators it was 60 clocks of reads for 56 of products: 0.99 PFLOP/s for gate + up, 0.65
// for down, on 16384 tokens x 4096, F 14336, 8 experts.)
template <bool kGateUp_>
struct Wide {
  static constexpr bool kGateUp = kGateUp_;
  static constexpr int kFlag = kGateUp ? 2 : 3;        // of ffn4_attr_done
  static constexpr int kRows = mx4::kLongRows, kStages = 4;
  static constexpr int kABytes = kTile * kChunk;       // half of them are loaded
  static constexpr int kBBytes = kRows / 2 * kChunk;   // of a term
  static constexpr int kRowScales = mx4::kRowScaleBytes<kRows>;
  static constexpr int kScaleOffset = kABytes + 2 * kBBytes;             // rows' scales, (down) weights' scales
  static constexpr int kStageBytes = round_up(kScaleOffset + kRowScales + (kGateUp ? 0 : kScaleTile), 1024);
  // (gate + up) the weights' scales have a ring of their own, kGroup chunks at a time
  static constexpr int kGroup = 4, kGroups = kGateUp ? 4 : 0;
  static constexpr int kGroupBytes = kGroup * kScaleTile;
  static constexpr int kScaleCols = 4 + 4 * kRowScales / kScaleTile;
  static constexpr int kScaleBufs = 3;                 // tensor memory has no room for four
  static constexpr int kOutputs = kGateUp ? 128 : 256; // of a pair's tile
  // Bytes of both terms of the rows of a group, which are read once for each tile of outputs: runs of 14400 rows x 4096, 118 MB, in
  // one group pushed each other out of L2 (16384 tokens 8.8 ms, 10.3 so).  4 to 48 MB take the same.
  static constexpr int kGroupL2 = 24 << 20;
  static constexpr int kEpilogueWarps = 8;
  static constexpr int kExchange = kGateUp ? kEpilogueWarps * 16 * 32 * 4 : 0;      // 16 x 32 fp32 for each epilogue warp
  static constexpr int kThreads = 128 + 32 * kEpilogueWarps;
  static constexpr size_t kSmem =
      1024 + (size_t)kStages * kStageBytes + kGroups * kGroupBytes + kExchange + sizeof(Runs) + 256 + kEpilogueWarps * kStaging;
  // Rows come in one TMA box of 112 or in boxes of 32: a box takes its warp some 60 clocks, and 14 boxes of 16 for a chunk,
  // with the weights' two, held the products up (down on 16384 tokens 3.5 ms, 2.8 with one box).
  static constexpr int kBigBox = kRows / 2, kSmallBox = 32;
  __device__ static constexpr int loaded_rows(int half) { return half > kBigBox / 2 ? kBigBox : round_up(half, kSmallBox); }
  static_assert(2 * kRows + kScaleBufs * kScaleCols <= 512 && kSmem <= 227 * 1024, "does not fit");
};

template <class Cfg>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(Cfg::kThreads, 1)
wide_kernel(const __grid_constant__ CUtensorMap tm_w0, const __grid_constant__ CUtensorMap tm_w1,
            const __grid_constant__ CUtensorMap tm_r0, const __grid_constant__ CUtensorMap tm_r1,
            const __grid_constant__ CUtensorMap tm_big0, const __grid_constant__ CUtensorMap tm_big1,
            const __grid_constant__ CUtensorMap tm_ws, const __grid_constant__ CUtensorMap tm_rs, const Weights w,
            const int32_t* __restrict__ slot_row_off, const int32_t* __restrict__ slot_expert, int S, int E, int n_dim, int k_dim,
            int rcap, int min_rows, int max_tiles, const mx4::Rows h, __nv_bfloat16* __restrict__ y, int32_t* __restrict__ status) {
  constexpr int kStages = Cfg::kStages, kRows = Cfg::kRows;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* w_scales = smem + (size_t)kStages * Cfg::kStageBytes;
  float* exchange = reinterpret_cast<float*>(w_scales + Cfg::kGroups * Cfg::kGroupBytes);
  Runs& runs = *reinterpret_cast<Runs*>(reinterpret_cast<uint8_t*>(exchange) + Cfg::kExchange);
  uint64_t* bars = reinterpret_cast<uint64_t*>(reinterpret_cast<uint8_t*>(&runs) + sizeof(Runs));
  uint64_t* full = bars;                     // [kStages]  both CTAs' loads -> MMA, on the leader
  uint64_t* empty = bars + kStages;          // [kStages]  MMA -> loads, in both
  uint64_t* acc_full = bars + 2 * kStages;   // [2]  MMA -> epilogue, in both
  uint64_t* acc_empty = acc_full + 2;        // [2]  both epilogues -> MMA, on the leader
  uint64_t* scales_full = acc_empty + 2;               // [kGroups]  both CTAs' copies -> MMA, on the leader
  uint64_t* scales_empty = scales_full + Cfg::kGroups; // [kGroups]  MMA -> copies, in both
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(scales_empty + Cfg::kGroups);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  static_assert((2 * kStages + 4 + 2 * Cfg::kGroups) * 8 + 8 <= 256, "barriers fit their space");

  const int warp = uniform_warp_index(), lane = threadIdx.x & 31;
  const int rank = (int)cluster_ctarank(), pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const int m_tiles = (n_dim + Cfg::kOutputs - 1) / Cfg::kOutputs, chunks = mx4::chunks_of(k_dim);

  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
    for (int i = 0; i < Cfg::kGroups; ++i) { mbar_init(&scales_full[i], 2); mbar_init(&scales_empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&acc_full[i], 1); mbar_init(&acc_empty[i], 2 * Cfg::kEpilogueWarps); }
    *abort_flag = 0;
    fence_mbar_init();
    prefetch_tensormap(&tm_w0);
    prefetch_tensormap(&tm_w1);
    prefetch_tensormap(&tm_r0);
    prefetch_tensormap(&tm_r1);
    prefetch_tensormap(&tm_ws);
    prefetch_tensormap(&tm_rs);
  }
  launch_dependents();
  wait_for_predecessor();
  if (warp == 1) {
    tmem_alloc_pair(tmem_slot, 512);
    tmem_relinquish_pair();
  }
  build_runs<Cfg::kThreads, kRows>(runs, slot_row_off, slot_expert, S, E, rcap, min_rows, INT32_MAX, max_tiles, status);
  __syncwarp();
  tc_fence_before_sync();
  cluster_sync_all();
  tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  const int64_t total = (int64_t)runs.tiles[S] * m_tiles;
  const int rows_together = max(1, Cfg::kGroupL2 / (2 * kRows * kChunk * chunks));

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      const uint32_t leader_full = map_to_cta(smem_u32(full), 0);
      for (int64_t t = pair; ok && t < total; t += pairs) {
        const Tile tc = tile_at<kRows>(runs, slot_row_off, slot_expert, S, t, m_tiles, rows_together);
        const uint32_t bytes =
            2 * (Cfg::kABytes / 2 + 2 * Cfg::loaded_rows(round_up(tc.rows, 32) / 2) * kChunk + Cfg::kRowScales +
                 (Cfg::kGateUp ? 0 : kScaleTile));
        const int out0 = tc.m * Cfg::kOutputs + rank * (Cfg::kOutputs / 2);
        // (down) rows of 128 bytes of the weights' scales; outputs behind the last tile meet zero weights, whatever their scales
        const int ws0 = ((tc.expert * mx4::tiles_of(n_dim) + out0 / kTile) * chunks) * (kScaleTile / 128);
        for (int c = 0; c < chunks; ++c) {
          if (!mbar_wait(&empty[stage], phase ^ 1u, abort_flag)) { ok = false; break; }
          uint8_t* a = smem + (size_t)stage * Cfg::kStageBytes;
          if (rank == 0) mbar_arrive_expect_tx(&full[stage], bytes);
          const uint32_t to = leader_full + stage * 8;
          tma_load_3d_pair(a, &tm_w0, to, c * kChunk, out0, tc.expert);
          if constexpr (Cfg::kGateUp)
            tma_load_3d_pair(a + Cfg::kABytes / 2, &tm_w1, to, c * kChunk, out0, tc.expert);
          else
            tma_load_2d_pair(a + Cfg::kScaleOffset + Cfg::kRowScales, &tm_ws, to, 0, ws0 + c * (kScaleTile / 128));
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
      }
      if (!ok) linger();
    }
  } else if (warp == 3) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      const uint32_t leader_full = map_to_cta(smem_u32(full), 0);
      for (int64_t t = pair; ok && t < total; t += pairs) {
        const Tile tc = tile_at<kRows>(runs, slot_row_off, slot_expert, S, t, m_tiles, rows_together);
        const int half = round_up(tc.rows, 32) / 2, row0 = tc.row0 + rank * half;
        const int rs0 = tc.row_tile * chunks * (Cfg::kRowScales / 128);
        for (int c = 0; c < chunks; ++c) {
          if (!mbar_wait(&empty[stage], phase ^ 1u, abort_flag)) { ok = false; break; }
          uint8_t* b = smem + (size_t)stage * Cfg::kStageBytes + Cfg::kABytes;
          const uint32_t to = leader_full + stage * 8;
          tma_load_2d_pair(b + 2 * Cfg::kBBytes, &tm_rs, to, 0, rs0 + c * (Cfg::kRowScales / 128));
          if (half > Cfg::kBigBox / 2) {
            tma_load_2d_pair(b, &tm_big0, to, c * kChunk, row0);
            tma_load_2d_pair(b + Cfg::kBBytes, &tm_big1, to, c * kChunk, row0);
          } else {
            for (int r = 0; r < half; r += Cfg::kSmallBox) {
              tma_load_2d_pair(b + r * kChunk, &tm_r0, to, c * kChunk, row0 + r);
              tma_load_2d_pair(b + Cfg::kBBytes + r * kChunk, &tm_r1, to, c * kChunk, row0 + r);
            }
          }
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
      }
      if (!ok) linger();
    }
  } else if (Cfg::kGateUp && warp == 2) {
    // scales of 64 gate rows and 64 up rows: 8 of the 16 bytes of each lane, of either matrix.  Some twelve chunks ahead of the
    // products and four at a time: what a step costs here (a wait, a proxy fence, an arrival) would hold up each of theirs (gate
    // + up on 16384 tokens 9.1 ms with these copies as part of a stage, 6.2 without them).
    constexpr int kAhead = Cfg::kGroups - 2;           // groups under way when one is handed over
    int group = 0, pending = 0, done = 0;
    uint32_t phase = 0;
    bool ok = true;
    const uint32_t leader_full = map_to_cta(smem_u32(scales_full), 0);
    auto hand_over = [&]() {
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive_remote(leader_full + done * 8);
      if (++done == Cfg::kGroups) done = 0;
      --pending;
    };
    for (int64_t t = pair; ok && t < total; t += pairs) {
      const Tile tc = tile_at<kRows>(runs, slot_row_off, slot_expert, S, t, m_tiles, rows_together);
      const size_t at = ((size_t)tc.expert * m_tiles + tc.m) * chunks * kScaleTile + 16 * lane + 8 * rank;
      for (int c = 0; c < chunks; c += Cfg::kGroup) {
        if (!__all_sync(0xffffffffu, mbar_wait(&scales_empty[group], phase ^ 1u, abort_flag))) { ok = false; break; }
        const uint32_t to = smem_u32(w_scales + group * Cfg::kGroupBytes) + 16 * lane;
#pragma unroll
        for (int i = 0; i < Cfg::kGroup; ++i) {
          if (c + i < chunks) {
            copy_async8(to + i * kScaleTile, w.scale[0] + at + (size_t)(c + i) * kScaleTile);
            copy_async8(to + i * kScaleTile + 8, w.scale[1] + at + (size_t)(c + i) * kScaleTile);
          }
        }
        copy_async_commit();
        if (++pending > kAhead) {
          copy_async_wait<kAhead>();
          hand_over();
        }
        if (++group == Cfg::kGroups) { group = 0; phase ^= 1u; }
      }
    }
    copy_async_wait<0>();
    while (pending > 0) hand_over();
  } else if (warp == 1) {
    if (rank == 0) {
      const uint32_t ring = smem_u32(smem);
      const uint32_t scale_cols = tmem_base + 2 * kRows;
      int stage = 0, acc = 0, buf = 0, group = 0;
      uint32_t phase = 0, acc_phase = 0, group_phase = 0;
      int64_t step = 0;
      bool ok = true;
      for (int64_t t = pair; ok && t < total; t += pairs) {
        const Tile tc = tile_at<kRows>(runs, slot_row_off, slot_expert, S, t, m_tiles, rows_together);
        const uint32_t idesc = idesc_mx_e2m1_e4m3(2 * kTile, round_up(tc.rows, 32));
        if (!warp_wait_cluster(&acc_empty[acc], acc_phase ^ 1u, abort_flag)) { ok = false; break; }
        tc_fence_after_sync();
        const uint32_t d = tmem_base + (uint32_t)acc * kRows;
        for (int c = 0; c < chunks; ++c, ++step) {
          // the scale columns of three steps ago are free when that step's MMAs are done
          if (step >= Cfg::kScaleBufs) {
            const int64_t old = step - Cfg::kScaleBufs;
            if (!warp_wait(&empty[old % kStages], (uint32_t)(old / kStages) & 1u, abort_flag)) { ok = false; break; }
          }
          if (Cfg::kGateUp && c % Cfg::kGroup == 0 && !warp_wait_cluster(&scales_full[group], group_phase, abort_flag)) {
            ok = false;
            break;
          }
          if (!warp_wait(&full[stage], phase, abort_flag)) { ok = false; break; }
          tc_fence_after_sync();
          const uint32_t a = ring + (uint32_t)stage * Cfg::kStageBytes;
          const uint32_t sc = a + Cfg::kScaleOffset;
          const uint32_t wsc =
              Cfg::kGateUp ? smem_u32(w_scales) + group * Cfg::kGroupBytes + (c % Cfg::kGroup) * kScaleTile : sc + Cfg::kRowScales;
          const uint64_t da = smem_desc_k_sw128(a), db = smem_desc_k_sw128(a + Cfg::kABytes);
          const uint32_t ts = scale_cols + (uint32_t)buf * Cfg::kScaleCols;
          const bool group_end = Cfg::kGateUp && (c % Cfg::kGroup == Cfg::kGroup - 1 || c == chunks - 1);
          if (elect_one()) {
            copy_scales_pair(ts, smem_desc_scales(wsc));
#pragma unroll
            for (int i = 0; i < Cfg::kRowScales / kScaleTile; ++i)
              copy_scales_pair(ts + 4 + 4 * i, smem_desc_scales(sc + i * kScaleTile));
#pragma unroll
            for (int j = 0; j < kChunk / mx4::kBlock; ++j) {
#pragma unroll
              for (int term = 0; term < 2; ++term)
                mma_mx_pair(d, da + (uint64_t)((j * mx4::kBlock) >> 4), db + (uint64_t)((term * Cfg::kBBytes + j * mx4::kBlock) >> 4),
                            idesc | idesc_mx_block(j), ts, ts + 4 + 8 * term, (c | j | term) != 0);
            }
            mma_commit_pair(&empty[stage]);
            if (group_end) mma_commit_pair(&scales_empty[group]);
          }
          if (group_end && ++group == Cfg::kGroups) { group = 0; group_phase ^= 1u; }
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
          if (++buf == Cfg::kScaleBufs) buf = 0;
        }
        if (!ok) break;
        if (elect_one()) mma_commit_pair(&acc_full[acc]);
        acc ^= 1;
        if (acc == 0) acc_phase ^= 1u;
      }
      if (!ok) linger();
    }
  } else if (warp >= 4) {
    // two warps for each quarter of the lanes: with one, the epilogue of a gate + up tile took 14000 clocks, as long as the products
    // of 2048 columns
    const int quarter = warp & 3, turn = (warp - 4) >> 2;
    uint8_t* staging = reinterpret_cast<uint8_t*>(bars) + 256 + (warp - 4) * kStaging;
    const uint32_t leader_empty = map_to_cta(smem_u32(acc_empty), 0);
    int acc = 0;
    uint32_t acc_phase = 0;
    bool ok = true;                  // a warp whose wait ran out still meets its partner at every barrier below
    for (int64_t t = pair; t < total; t += pairs) {
      const Tile tc = tile_at<kRows>(runs, slot_row_off, slot_expert, S, t, m_tiles, rows_together);
      const int padded = round_up(tc.rows, 32);
      ok = ok && __all_sync(0xffffffffu, mbar_wait(&acc_full[acc], acc_phase, abort_flag, 64));
      tc_fence_after_sync();
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)acc * kRows;
      if constexpr (Cfg::kGateUp) {
        const bool up = quarter >= 2;
        const int block = rank * 2 + (quarter & 1);    // which 32 of the tile's 128 outputs
        const int col0 = tc.m * kChunk + block * 32;
        uint8_t* scales = h.scale + ((size_t)tc.row_tile * m_tiles + tc.m) * Cfg::kRowScales;
        const int half = padded / 2;
        float* own_buffer = exchange + (warp - 4) * 16 * 32 + lane;
        const float* partners = exchange + ((warp - 4) ^ 2) * 16 * 32 + lane;
        for (int i = 16 * turn; i < half; i += 32) {
          // the gate's warps finish the first half of the rows, the up's the second
          const int mine = up ? half + i : i, other = up ? i : half + i;
          uint32_t give[16], keep[16];
          if (ok) {
            tmem_ld16(taddr + other, give);
            tmem_ld16(taddr + mine, keep);
            tmem_ld_wait();
          }
#pragma unroll
          for (int j = 0; j < 16; ++j) own_buffer[j * 32] = __uint_as_float(give[j]);
          named_sync(1 + 2 * turn + (quarter & 1), 64);
          float gate[16], value[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const float get = partners[j * 32], kept = __uint_as_float(keep[j]);
            gate[j] = up ? get : kept;
            value[j] = up ? kept : get;
          }
          named_sync(1 + 2 * turn + (quarter & 1), 64);                // the buffers have been read
          if (ok)
            store_h<kRows>(h, gate, value, staging, tc.row0 + mine, mine, tc.rows, (size_t)m_tiles * kChunk, col0, scales, block, lane);
        }
      } else {
        const int col0 = tc.m * Cfg::kOutputs + rank * kTile + quarter * 32;
        for (int r = 16 * turn; ok && r < tc.rows; r += 32) {
          uint32_t bits[16];
          float v[16];
          tmem_ld16(taddr + r, bits);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(bits[i]);
          store_y(y, v, staging, tc.row0 + r, r, tc.rows, n_dim, col0, lane);
        }
      }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive_remote(leader_empty + acc * 8);
      acc ^= 1;
      if (acc == 0) acc_phase ^= 1u;
    }
  }

  __syncwarp();
  tc_fence_before_sync();
  cluster_sync_all();                                  // nobody touches the other CTA's memory after this
  if (threadIdx.x == 0 && *abort_flag) moegps_report(status, MOEGPS_ERR_TIMEOUT, (int)blockIdx.x);
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc_pair(tmem_base, 512);
  }
}

// ------------------------------------------------------------------------------------------- host
using Short48 = Short<48, 4>;
using Short32 = Short<32, 5>;
constexpr int kFlags[] = {Short48::kFlag, Short32::kFlag, Wide<true>::kFlag, Wide<false>::kFlag};
static_assert(kFlags[0] == 0 && kFlags[1] == 1 && kFlags[2] == 2 && kFlags[3] == 3 &&
                  sizeof(moegps_ctx::ffn4_attr_done) / sizeof(bool) == 4,
              "each kernel has a flag of its own for its raised shared-memory limit");

struct Call {
  const void* xp;
  const int32_t *slot_row_off, *slot_expert;
  const void *gate4, *up4, *down4;
  Weights up_scale, down_scale;
  __nv_bfloat16* yp;
  uint8_t* workspace;
  mx4::Layout l;
  mx4::Rows x, h;
};

int tmap_failed(moegps_ctx* ctx) {
  ctx->last_cuda_error = (int)cudaErrorInvalidValue;
  return MOEGPS_ERR_CUDA;
}

int launch_split(moegps_ctx* ctx, const Call& c, cudaStream_t st) {
  const moegps_shape_t& s = ctx->shape;
  const int64_t units = c.l.long_tiles * 64 * ((s.D + 511) / 512) / (kSplitThreads / 32);
  const int64_t resident = 4 * (int64_t)ctx->sm_count;         // what runs at once by registers (8 for each SM take the same)
  split_kernel<<<(unsigned)(units < resident ? units : resident), kSplitThreads, 0, st>>>(
      static_cast<const __nv_bfloat16*>(c.xp), c.slot_row_off, c.slot_expert, s.S, s.E, s.D, (int)c.l.rows,
      c.l.cut.short_rows + 1, (int)c.l.long_tiles, c.x, ctx->d_status);
  MOEGPS_AFTER_LAUNCH(ctx);
  return MOEGPS_OK;
}

template <class Cfg>
int launch_short(moegps_ctx* ctx, const Call& c, cudaStream_t st) {
  const moegps_shape_t& s = ctx->shape;
  const int dc = mx4::chunks_of(s.D) * kChunk, fc = mx4::chunks_of(s.F) * kChunk;
  CUtensorMap gate, up, down;
  if (!moegps_make_tmap_codes4(&gate, c.gate4, s.E, s.F, dc, kTile) || !moegps_make_tmap_codes4(&up, c.up4, s.E, s.F, dc, kTile) ||
      !moegps_make_tmap_codes4(&down, c.down4, s.E, s.D, fc, kTile))
    return tmap_failed(ctx);
  bool& attr_done = ctx->ffn4_attr_done[Cfg::kFlag];
  if (!attr_done) {
    MOEGPS_CUDA_TRY(ctx, cudaFuncSetAttribute(short_kernel<Cfg>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg::kSmem));
    attr_done = true;
  }
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeCooperative;            // all blocks run at once: they wait for one another
  attr.val.cooperative = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(mx4::short_blocks(ctx->sm_count));
  cfg.blockDim = dim3(Cfg::kThreads);
  cfg.dynamicSmemBytes = Cfg::kSmem;
  cfg.stream = st;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  uint8_t* ws = c.workspace;
  MOEGPS_CUDA_TRY(ctx, cudaLaunchKernelEx(&cfg, short_kernel<Cfg>, gate, up, down, c.up_scale.scale[0], c.up_scale.scale[1],
                                          c.down_scale.scale[0], static_cast<const __nv_bfloat16*>(c.xp), c.slot_row_off, c.slot_expert,
                                          s.S, s.E, s.D, s.F, (int)c.l.rows, c.l.cut.short_rows, (int)c.l.short_tiles, ws + c.l.x_image, ws + c.l.h_image, c.yp,
                                          reinterpret_cast<int*>(ws + c.l.part_there), reinterpret_cast<int*>(ws + c.l.h_there),
                                          reinterpret_cast<float*>(ws + c.l.partial),
                                          ctx->d_meetings, ctx->d_status));
  MOEGPS_AFTER_LAUNCH(ctx, "rows=%d", Cfg::kRows);
  return MOEGPS_OK;
}

template <class Cfg>
int launch_wide(moegps_ctx* ctx, const Call& c, cudaStream_t st) {
  const moegps_shape_t& s = ctx->shape;
  const int n_dim = Cfg::kGateUp ? s.F : s.D, k_dim = Cfg::kGateUp ? s.D : s.F;
  const int chunks = mx4::chunks_of(k_dim), cols = chunks * kChunk;
  const mx4::Rows& in = Cfg::kGateUp ? c.x : c.h;
  const Weights& ws = Cfg::kGateUp ? c.up_scale : c.down_scale;
  CUtensorMap w0, w1, r0, r1, big0, big1, wsm, rsm;
  const int box = Cfg::kGateUp ? 64 : kTile;
  if (!moegps_make_tmap_codes4(&w0, Cfg::kGateUp ? c.gate4 : c.down4, s.E, n_dim, cols, box) ||
      !moegps_make_tmap_codes4(&w1, Cfg::kGateUp ? c.up4 : c.down4, s.E, n_dim, cols, box) ||
      !moegps_make_tmap_bytes(&r0, in.code[0], c.l.rows, cols, Cfg::kSmallBox, true) ||
      !moegps_make_tmap_bytes(&r1, in.code[1], c.l.rows, cols, Cfg::kSmallBox, true) ||
      !moegps_make_tmap_bytes(&big0, in.code[0], c.l.rows, cols, Cfg::kBigBox, true) ||
      !moegps_make_tmap_bytes(&big1, in.code[1], c.l.rows, cols, Cfg::kBigBox, true) ||
      !moegps_make_tmap_bytes(&wsm, ws.scale[0], (uint64_t)s.E * mx4::tiles_of(n_dim) * chunks * (kScaleTile / 128), 128,
                              kScaleTile / 128, false) ||
      !moegps_make_tmap_bytes(&rsm, in.scale, (uint64_t)c.l.long_tiles * chunks * (Cfg::kRowScales / 128), 128,
                              Cfg::kRowScales / 128, false))
    return tmap_failed(ctx);
  bool& attr_done = ctx->ffn4_attr_done[Cfg::kFlag];
  if (!attr_done) {
    MOEGPS_CUDA_TRY(ctx, cudaFuncSetAttribute(wide_kernel<Cfg>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg::kSmem));
    attr_done = true;
  }
  MOEGPS_CUDA_TRY(ctx, launch_after(wide_kernel<Cfg>, dim3(ctx->sm_count / 2 * 2), Cfg::kThreads, Cfg::kSmem, st, w0, w1, r0, r1,
                                    big0, big1, wsm, rsm, ws, c.slot_row_off, c.slot_expert, s.S, s.E, n_dim, k_dim, (int)c.l.rows, c.l.cut.short_rows + 1, (int)c.l.long_tiles, c.h,
                                    c.yp,
                                    ctx->d_status));
  MOEGPS_AFTER_LAUNCH(ctx, "rows=%d", Cfg::kRows);
  return MOEGPS_OK;
}

}  // namespace

int moegps_launch_expert_ffn4(moegps_ctx* ctx, const void* xp, const int32_t* slot_row_off, const int32_t* slot_expert,
                              const void* gate4, const void* up4, const void* down4, const void* gate4_scale, const void* up4_scale,
                              const void* down4_scale, void* yp, void* workspace, cudaStream_t st) {
  Call c = {xp, slot_row_off, slot_expert, gate4, up4, down4,
            {{static_cast<const uint8_t*>(gate4_scale), static_cast<const uint8_t*>(up4_scale)}},
            {{static_cast<const uint8_t*>(down4_scale), nullptr}},
            static_cast<__nv_bfloat16*>(yp), static_cast<uint8_t*>(workspace), mx4::layout_of(ctx->shape), {}, {}};
  uint8_t* ws = c.workspace;
  c.x = {{ws + c.l.x_code, ws + c.l.x_code + c.l.x_code_bytes}, ws + c.l.x_scale};
  c.h = {{ws + c.l.h_code, ws + c.l.h_code + c.l.h_code_bytes}, ws + c.l.h_scale};
  if (mx4::short_blocks(ctx->sm_count) == 0) return MOEGPS_ERR_UNIMPLEMENTED;
  int rc = MOEGPS_OK;
  if (!c.l.cut.all_short()) {
    rc = launch_split(ctx, c, st);
    if (rc == MOEGPS_OK) rc = launch_wide<Wide<true>>(ctx, c, st);
    if (rc == MOEGPS_OK) rc = launch_wide<Wide<false>>(ctx, c, st);
  }
  if (rc == MOEGPS_OK && c.l.cut.short_rows > 0)
    rc = c.l.cut.tile_rows == 32 ? launch_short<Short32>(ctx, c, st) : launch_short<Short48>(ctx, c, st);
  return rc;
}
