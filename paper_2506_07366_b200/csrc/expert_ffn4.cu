// expert_ffn4: the experts' SwiGLU FFN on 4-bit weights (mx4.cuh) over ragged slots, from the few rows of a token being
// generated to long prompts.  Three launches:
//   split      x = two e4m3 terms with a scale for 32 values (exact, see mx4.cuh)
//   gate + up  g = x Wg^T, u = x Wu^T, h = silu(g) u, written as two terms
//   down       y = h Wd^T
// The products are block-scaled MMAs (e2m1 x e4m3, fp32 accumulators in tensor memory) with the WEIGHTS as the 128-row
// operand and the slot's rows as the other one, so that a slot of few rows costs few columns.  A weight tile is expanded to 16-byte
// groups by the TMA load that brings it (8 bytes of codes, 8 unused): 8 KB of memory traffic for 16 KB of shared memory,
// and no thread touches a weight.
//
// Warps: 0 loads weights, their scales and the rows' codes (TMA), 2 the rows' scales (the words of a tile's rows go to
// the places where tensor memory wants them, 4-byte asynchronous copies), 1 issues scale copies and MMAs, 4..7 drain the
// accumulators (two, so that a tile's epilogue overlaps the next one's products).  Every wait is bounded.
#include "common.cuh"
#include "grouped_gemm.cuh"
#include "mx4.cuh"
#include "sm100.cuh"

namespace {

using namespace sm100;
using grouped_gemm::build_tables;
using grouped_gemm::decode_tile;
using grouped_gemm::Tables;
using grouped_gemm::TileCoord;

// ------------------------------------------------------------------------------------------- split
constexpr int kSplitRows = 8;      // rows of a block: one for each warp
constexpr int kSplitCols = 1024;   // columns of a block

__global__ void __launch_bounds__(256) split_kernel(const __nv_bfloat16* __restrict__ xp, const int32_t* __restrict__ slot_row_off,
                                                    int S, int D, int rcap, int pitch, const mx4::Rows out) {
  __shared__ int last_row;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  launch_dependents();
  wait_for_predecessor();
  if (threadIdx.x == 0) last_row = 0;
  __syncthreads();
  // one past the last row of any slot (slots with an extent outside the buffers have no rows)
  int last = 0;
  for (int s = threadIdx.x; s < S; s += blockDim.x) {
    const int lo = slot_row_off[s], hi = slot_row_off[s + 1];
    if (lo >= 0 && hi > lo && hi <= rcap) last = max(last, hi);
  }
  if (last) atomicMax(&last_row, last);
  __syncthreads();
  const int rows = last_row, chunks = mx4::chunks_of(D);
  const int col_blocks = (chunks * mx4::kChunk + kSplitCols - 1) / kSplitCols;
  const int64_t work = (int64_t)((rows + kSplitRows - 1) / kSplitRows) * col_blocks;
  for (int64_t b = blockIdx.x; b < work; b += gridDim.x) {
    const int row = (int)(b / col_blocks) * kSplitRows + warp, col0 = (int)(b % col_blocks) * kSplitCols;
    if (row >= rows) continue;
    uint4 v[kSplitCols / 256];
#pragma unroll
    for (int i = 0; i < kSplitCols / 256; ++i) {
      const int col = col0 + 256 * i + 8 * lane;
      v[i] = make_uint4(0, 0, 0, 0);
      if (col < D) v[i] = *reinterpret_cast<const uint4*>(xp + (size_t)row * D + col);
    }
#pragma unroll
    for (int i = 0; i < kSplitCols / 256; ++i) {
      const int col = col0 + 256 * i + 8 * lane;      // a warp's 256 columns are two chunks: whole half-warps are inside or not
      const uint32_t words[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
      const uint32_t m2 = __vmaxu2(__vmaxu2(words[0] & 0x7fff7fffu, words[1] & 0x7fff7fffu),
                                   __vmaxu2(words[2] & 0x7fff7fffu, words[3] & 0x7fff7fffu));
      uint32_t m = max(m2 & 0xffffu, m2 >> 16);
      m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
      m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
      const uint32_t b1 = mx4::term_scale(m << 16), b2 = mx4::second_scale(b1);
      const float inv = mx4::inverse_scale(b1), ratio = mx4::scale_ratio(b1, b2);
      uint32_t c1[4], c2[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        mx4::split2(__uint_as_float(words[j] << 16), __uint_as_float(words[j] & 0xffff0000u), inv, ratio, c1[j], c2[j]);
      // the four scale bytes of a chunk, from lanes 0, 4, 8, 12 of its half-warp
      uint32_t w1 = b1 << (8 * ((lane >> 2) & 3)), w2 = b2 << (8 * ((lane >> 2) & 3));
      w1 |= __shfl_xor_sync(0xffffffffu, w1, 4);
      w2 |= __shfl_xor_sync(0xffffffffu, w2, 4);
      w1 |= __shfl_xor_sync(0xffffffffu, w1, 8);
      w2 |= __shfl_xor_sync(0xffffffffu, w2, 8);
      if (col < chunks * mx4::kChunk) {
        const size_t at = (size_t)row * (chunks * mx4::kChunk) + col;
        *reinterpret_cast<uint2*>(out.code[0] + at) = make_uint2(c1[0] | c1[1] << 16, c1[2] | c1[3] << 16);
        *reinterpret_cast<uint2*>(out.code[1] + at) = make_uint2(c2[0] | c2[1] << 16, c2[2] | c2[3] << 16);
        if ((lane & 15) == 0) {
          const size_t word = (size_t)(col / mx4::kChunk) * pitch + row;
          out.scale[0][word] = w1;
          out.scale[1][word] = w2;
        }
      }
    }
  }
}

// ------------------------------------------------------------------------------------------- products
__host__ __device__ constexpr int round_up(int n, int to) { return (n + to - 1) / to * to; }

template <int kN_, bool kGateUp_, int kStages_>
struct Cfg {
  static constexpr int kN = kN_;                       // rows of a tile at most
  static constexpr bool kGateUp = kGateUp_;
  static constexpr int kStages = kStages_;
  static constexpr int kMats = kGateUp ? 2 : 1;        // weight matrices that share the rows
  static constexpr int kBoxRows = 16;                  // rows of one TMA box
  static constexpr int kABytes = mx4::kTile * mx4::kChunk;      // of shared memory; half of them are loaded
  static constexpr int kALoaded = kABytes / 2;
  static constexpr int kBBytes = kN * mx4::kChunk;
  static constexpr int kScaleTiles = (kN + 127) / 128;          // 512-byte groups of a term's scales
  static constexpr int kTermScaleBytes = kScaleTiles * mx4::kScaleTile;
  static constexpr int kScaleOffset = kMats * kABytes + 2 * kBBytes;
  static constexpr int kStageBytes = round_up(kScaleOffset + kMats * mx4::kScaleTile + 2 * kTermScaleBytes, 1024);
  static constexpr int kScaleCols = 4 * kMats + 8 * kScaleTiles;
  static constexpr int kAccCols = kMats * kN;
  static constexpr int kColsUsed = 2 * kAccCols + kStages * kScaleCols;
  static constexpr int kTmemCols = kColsUsed <= 128 ? 128 : kColsUsed <= 256 ? 256 : 512;
  static constexpr int kThreads = 256;
  // the loader of the rows' scales runs this many stages ahead of what it hands over
  static constexpr int kScaleLag = kStages - 1 < 3 ? kStages - 1 : 3;
  static constexpr size_t kSmem = 1024 + (size_t)kStages * kStageBytes + sizeof(Tables) + 256;
  static_assert(kN % 16 == 0 && kN <= 256 && kColsUsed <= 512 && kSmem <= 227 * 1024 && kStages >= 2, "does not fit");
};

struct Operands {
  const uint8_t* w_scale[2];        // gate, up; or down
  const uint32_t* row_scale[2];     // the two terms
  int pitch;                        // words of a chunk of row_scale
};

__device__ __forceinline__ float silu(float g) { return __fdividef(g, 1.0f + __expf(-g)); }

// kGateUp: h = silu(g) u as two terms into `h`; otherwise y = accumulator into `y` [rcap, n_dim].
template <class Cfg>
__global__ void __launch_bounds__(Cfg::kThreads, 1)
product4_kernel(const __grid_constant__ CUtensorMap tm_w0, const __grid_constant__ CUtensorMap tm_w1,
                const __grid_constant__ CUtensorMap tm_r0, const __grid_constant__ CUtensorMap tm_r1, const Operands op,
                const int32_t* __restrict__ slot_row_off, const int32_t* __restrict__ slot_expert, int S, int E, int n_dim, int k_dim,
                int rcap, const mx4::Rows h, __nv_bfloat16* __restrict__ y, int32_t* __restrict__ status) {
  constexpr int kStages = Cfg::kStages, kN = Cfg::kN, kMats = Cfg::kMats;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  Tables& tb = *reinterpret_cast<Tables*>(smem + (size_t)kStages * Cfg::kStageBytes);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + (size_t)kStages * Cfg::kStageBytes + sizeof(Tables));
  uint64_t* full = bars;                     // [kStages]  loaders -> MMA
  uint64_t* empty = bars + kStages;          // [kStages]  MMA -> loaders
  uint64_t* acc_full = bars + 2 * kStages;   // [2]  MMA -> epilogue
  uint64_t* acc_empty = acc_full + 2;        // [2]  epilogue -> MMA
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = uniform_warp_index(), lane = threadIdx.x & 31;
  const int m_tiles = mx4::tiles_of(n_dim), chunks = mx4::chunks_of(k_dim);

  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) { mbar_init(&full[i], 2); mbar_init(&empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&acc_full[i], 1); mbar_init(&acc_empty[i], 4); }
    *abort_flag = 0;
    fence_mbar_init();
    prefetch_tensormap(&tm_w0);
    prefetch_tensormap(&tm_w1);
    prefetch_tensormap(&tm_r0);
    prefetch_tensormap(&tm_r1);
  }
  launch_dependents();
  wait_for_predecessor();
  if (warp == 1) {
    tmem_alloc(tmem_slot, Cfg::kTmemCols);
    tmem_relinquish();
  }
  build_tables<Cfg::kThreads, kN>(tb, slot_row_off, slot_expert, S, E, m_tiles, rcap, status);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  const int total_tiles = tb.tile_base[S];

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int tile = blockIdx.x; ok && tile < total_tiles; tile += gridDim.x) {
        const TileCoord tc = decode_tile<kN>(tb, slot_row_off, slot_expert, S, tile, m_tiles);
        const int boxes = (min(kN, tc.row_end - tc.m0) + Cfg::kBoxRows - 1) / Cfg::kBoxRows;
        const uint32_t bytes = kMats * (Cfg::kALoaded + mx4::kScaleTile) + 2 * boxes * Cfg::kBoxRows * mx4::kChunk;
        const size_t scale_at = ((size_t)tc.expert * m_tiles + tc.n_tile) * chunks * mx4::kScaleTile;
        for (int c = 0; c < chunks; ++c) {
          if (!mbar_wait(&empty[stage], phase ^ 1u, abort_flag)) { ok = false; break; }
          uint8_t* a = smem + (size_t)stage * Cfg::kStageBytes;
          uint8_t* b = a + kMats * Cfg::kABytes;
          uint8_t* sc = a + Cfg::kScaleOffset;
          mbar_arrive_expect_tx(&full[stage], bytes);
#pragma unroll
          for (int m = 0; m < kMats; ++m) {
            tma_load_3d(a + m * Cfg::kABytes, m ? &tm_w1 : &tm_w0, &full[stage], c * mx4::kChunk, tc.n_tile * mx4::kTile,
                        tc.expert);
            bulk_load(sc + m * mx4::kScaleTile, op.w_scale[m] + scale_at + (size_t)c * mx4::kScaleTile, mx4::kScaleTile,
                      &full[stage]);
          }
          for (int i = 0; i < boxes; ++i) {
            const int r = i * Cfg::kBoxRows;
            tma_load_2d(b + r * mx4::kChunk, &tm_r0, &full[stage], c * mx4::kChunk, tc.m0 + r);
            tma_load_2d(b + Cfg::kBBytes + r * mx4::kChunk, &tm_r1, &full[stage], c * mx4::kChunk, tc.m0 + r);
          }
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
      }
      if (!ok) {
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);      // let copies in flight land before the block retires
      }
    }
  } else if (warp == 2) {
    constexpr int kLag = Cfg::kScaleLag;
    int stage = 0, pending = 0, done = 0;      // copies issued and not handed over; stage of the next one to hand over
    uint32_t phase = 0;
    bool ok = true;
    auto hand_over = [&]() {                   // the copies of stage `done` have landed in this thread's view
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(&full[done]);
      done = done + 1 == kStages ? 0 : done + 1;
      --pending;
    };
    for (int tile = blockIdx.x; ok && tile < total_tiles; tile += gridDim.x) {
      const TileCoord tc = decode_tile<kN>(tb, slot_row_off, slot_expert, S, tile, m_tiles);
      const int rows = min(kN, tc.row_end - tc.m0);
      for (int c = 0; c < chunks; ++c) {
        if (!__all_sync(0xffffffffu, mbar_wait(&empty[stage], phase ^ 1u, abort_flag))) { ok = false; break; }
        const uint32_t dst = smem_u32(smem + (size_t)stage * Cfg::kStageBytes + Cfg::kScaleOffset + kMats * mx4::kScaleTile);
        const size_t src = (size_t)c * op.pitch + tc.m0;
        for (int r = lane; r < round_up(rows, 32); r += 32) {
          const uint32_t at = dst + (r / 128) * mx4::kScaleTile + mx4::scale_byte_at(r % 128);
          const size_t from = src + (r < rows ? r : 0);
          copy_async4(at, op.row_scale[0] + from, r < rows ? 4 : 0);
          copy_async4(at + Cfg::kTermScaleBytes, op.row_scale[1] + from, r < rows ? 4 : 0);
        }
        copy_async_commit();
        ++pending;
        if (pending > kLag) {
          copy_async_wait<kLag>();
          hand_over();
        }
        if (++stage == kStages) { stage = 0; phase ^= 1u; }
      }
    }
    copy_async_wait<0>();
    while (pending > 0) hand_over();
  } else if (warp == 1) {
    const uint32_t ring = smem_u32(smem);
    const uint32_t scale_cols = tmem_base + 2 * Cfg::kAccCols;
    int stage = 0, acc = 0;
    uint32_t phase = 0, acc_phase = 0;
    bool ok = true;
    for (int tile = blockIdx.x; ok && tile < total_tiles; tile += gridDim.x) {
      const TileCoord tc = decode_tile<kN>(tb, slot_row_off, slot_expert, S, tile, m_tiles);
      const uint32_t idesc = idesc_mx_e2m1_e4m3(mx4::kTile, round_up(min(kN, tc.row_end - tc.m0), 16));
      if (!warp_wait(&acc_empty[acc], acc_phase ^ 1u, abort_flag)) { ok = false; break; }
      tc_fence_after_sync();
      const uint32_t d = tmem_base + (uint32_t)acc * Cfg::kAccCols;
      for (int c = 0; c < chunks; ++c) {
        if (!warp_wait(&full[stage], phase, abort_flag)) { ok = false; break; }
        tc_fence_after_sync();
        const uint32_t a = ring + (uint32_t)stage * Cfg::kStageBytes;
        const uint32_t sc = a + Cfg::kScaleOffset;
        const uint64_t da = smem_desc_k_sw128(a);
        const uint64_t db = smem_desc_k_sw128(a + kMats * Cfg::kABytes);
        const uint32_t ts = scale_cols + (uint32_t)stage * Cfg::kScaleCols;
        if (elect_one()) {
#pragma unroll
          for (int i = 0; i < kMats + 2 * Cfg::kScaleTiles; ++i)
            copy_scales(ts + 4 * i, smem_desc_scales(sc + i * mx4::kScaleTile));
#pragma unroll
          for (int j = 0; j < mx4::kChunk / mx4::kBlock; ++j) {
#pragma unroll
            for (int m = 0; m < kMats; ++m) {
#pragma unroll
              for (int t = 0; t < 2; ++t)
                mma_mx(d + m * kN, da + (uint64_t)((m * Cfg::kABytes + j * mx4::kBlock) >> 4),
                       db + (uint64_t)((t * Cfg::kBBytes + j * mx4::kBlock) >> 4), idesc | idesc_mx_block(j), ts + 4 * m,
                       ts + 4 * kMats + 4 * Cfg::kScaleTiles * t, (c | j | t) != 0);
            }
          }
          mma_commit(&empty[stage]);
        }
        if (++stage == kStages) { stage = 0; phase ^= 1u; }
      }
      if (!ok) break;
      if (elect_one()) mma_commit(&acc_full[acc]);
      acc ^= 1;
      if (acc == 0) acc_phase ^= 1u;
    }
    if (!ok) {
      for (int i = 0; i < 1000; ++i) __nanosleep(1000);
    }
  } else if (warp >= 4) {
    const int quarter = warp & 3;
    const int k_pitch = m_tiles * mx4::kChunk;         // bytes of a row of h
    int acc = 0;
    uint32_t acc_phase = 0;
    for (int tile = blockIdx.x; tile < total_tiles; tile += gridDim.x) {
      const TileCoord tc = decode_tile<kN>(tb, slot_row_off, slot_expert, S, tile, m_tiles);
      const int rows = min(kN, tc.row_end - tc.m0);
      if (!mbar_wait(&acc_full[acc], acc_phase, abort_flag, 64)) break;
      tc_fence_after_sync();
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)acc * Cfg::kAccCols;
      const int out = tc.n_tile * mx4::kTile + quarter * 32 + lane;        // this thread's output
      for (int c0 = 0; c0 < rows; c0 += 16) {
        uint32_t g[16];
        tmem_ld16(taddr + c0, g);
        if constexpr (Cfg::kGateUp) {
          uint32_t u[16];
          tmem_ld16(taddr + kN + c0, u);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            if (c0 + i < rows) {                       // the same for the whole warp
              const float v = silu(__uint_as_float(g[i])) * __uint_as_float(u[i]);
              const uint32_t b1 = mx4::term_scale(__reduce_max_sync(0xffffffffu, __float_as_uint(v) & 0x7fffffffu));
              const uint32_t b2 = mx4::second_scale(b1);
              uint32_t c1, c2;
              mx4::split2(v, 0.0f, mx4::inverse_scale(b1), mx4::scale_ratio(b1, b2), c1, c2);
              const size_t row = tc.m0 + c0 + i;
              h.code[0][row * k_pitch + out] = (uint8_t)c1;
              h.code[1][row * k_pitch + out] = (uint8_t)c2;
              if (lane < 2)
                reinterpret_cast<uint8_t*>(h.scale[lane] + (size_t)tc.n_tile * op.pitch + row)[quarter] = (uint8_t)(lane ? b2 : b1);
            }
          }
        } else {
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (c0 + i < rows && out < n_dim)
              y[(size_t)(tc.m0 + c0 + i) * n_dim + out] = __float2bfloat16_rn(__uint_as_float(g[i]));
        }
      }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&acc_empty[acc]);
      acc ^= 1;
      if (acc == 0) acc_phase ^= 1u;
    }
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

template <class Cfg>
int launch_product(moegps_ctx* ctx, const CUtensorMap& w0, const CUtensorMap& w1, const CUtensorMap& r0, const CUtensorMap& r1,
                   const Operands& op, const int32_t* slot_row_off, const int32_t* slot_expert, int n_dim, int k_dim,
                   const mx4::Rows& h, void* y, cudaStream_t st) {
  const moegps_shape_t& s = ctx->shape;
  MOEGPS_CUDA_TRY(ctx, cudaFuncSetAttribute(product4_kernel<Cfg>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg::kSmem));
  MOEGPS_CUDA_TRY(ctx, launch_after(product4_kernel<Cfg>, dim3(ctx->sm_count), Cfg::kThreads, Cfg::kSmem, st, w0, w1, r0, r1, op,
                                    slot_row_off, slot_expert, s.S, s.E, n_dim, k_dim, (int)moegps_rcap_of(s), h,
                                    static_cast<__nv_bfloat16*>(y), ctx->d_status));
  MOEGPS_AFTER_LAUNCH(ctx, "rows=%d", Cfg::kN);
  return MOEGPS_OK;
}

mx4::Rows rows_at(void* workspace, size_t code, size_t code_bytes, size_t scale, size_t scale_bytes) {
  uint8_t* w = static_cast<uint8_t*>(workspace);
  return {{w + code, w + code + code_bytes},
          {reinterpret_cast<uint32_t*>(w + scale), reinterpret_cast<uint32_t*>(w + scale + scale_bytes)}};
}

}  // namespace

int moegps_launch_expert_ffn4(moegps_ctx* ctx, const void* xp, const int32_t* slot_row_off, const int32_t* slot_expert,
                              const void* gate4, const void* up4, const void* down4, const void* gate4_scale, const void* up4_scale,
                              const void* down4_scale, void* yp, void* workspace, cudaStream_t st) {
  const moegps_shape_t& s = ctx->shape;
  const mx4::Layout l = mx4::layout_of(s);
  const mx4::Rows x = rows_at(workspace, l.x_code, l.x_code_bytes, l.x_scale, l.x_scale_bytes);
  const mx4::Rows h = rows_at(workspace, l.h_code, l.h_code_bytes, l.h_scale, l.h_scale_bytes);
  const int dc = mx4::chunks_of(s.D) * mx4::kChunk, fc = mx4::chunks_of(s.F) * mx4::kChunk;
  CUtensorMap tg, tu, td, tx[2], th[2];
  bool ok = moegps_make_tmap_codes4(&tg, gate4, s.E, s.F, dc, mx4::kTile) && moegps_make_tmap_codes4(&tu, up4, s.E, s.F, dc, mx4::kTile) &&
            moegps_make_tmap_codes4(&td, down4, s.E, s.D, fc, mx4::kTile);
  for (int t = 0; t < 2; ++t)
    ok = ok && moegps_make_tmap_bytes(&tx[t], x.code[t], l.rows, dc, 16) && moegps_make_tmap_bytes(&th[t], h.code[t], l.rows, fc, 16);
  if (!ok) {
    ctx->last_cuda_error = (int)cudaErrorInvalidValue;
    return MOEGPS_ERR_CUDA;
  }
  const int64_t split_blocks = (l.rows + kSplitRows - 1) / kSplitRows * ((dc + kSplitCols - 1) / kSplitCols);
  const int64_t resident = 8 * (int64_t)ctx->sm_count;
  split_kernel<<<(unsigned)(split_blocks < resident ? split_blocks : resident), 256, 0, st>>>(
      static_cast<const __nv_bfloat16*>(xp), slot_row_off, s.S, s.D, (int)l.rows, (int)l.pitch, x);
  MOEGPS_AFTER_LAUNCH(ctx);
  const Operands up_op = {{static_cast<const uint8_t*>(gate4_scale), static_cast<const uint8_t*>(up4_scale)},
                          {x.scale[0], x.scale[1]}, (int)l.pitch};
  const Operands down_op = {{static_cast<const uint8_t*>(down4_scale), nullptr}, {h.scale[0], h.scale[1]}, (int)l.pitch};
  const int64_t R = (int64_t)s.T * s.K;
  const int64_t per_slot = (R + s.S - 1) / s.S;
  const mx4::Rows none = {};
  int rc;
  if (per_slot <= 16)
    rc = launch_product<Cfg<16, true, 5>>(ctx, tg, tu, tx[0], tx[1], up_op, slot_row_off, slot_expert, s.F, s.D, h, nullptr, st);
  else if (per_slot <= 64)
    rc = launch_product<Cfg<64, true, 4>>(ctx, tg, tu, tx[0], tx[1], up_op, slot_row_off, slot_expert, s.F, s.D, h, nullptr, st);
  else
    rc = launch_product<Cfg<112, true, 3>>(ctx, tg, tu, tx[0], tx[1], up_op, slot_row_off, slot_expert, s.F, s.D, h, nullptr, st);
  if (rc != MOEGPS_OK) return rc;
  if (per_slot <= 16)
    return launch_product<Cfg<16, false, 9>>(ctx, td, td, th[0], th[1], down_op, slot_row_off, slot_expert, s.D, s.F, none, yp, st);
  if (per_slot <= 64)
    return launch_product<Cfg<64, false, 6>>(ctx, td, td, th[0], th[1], down_op, slot_row_off, slot_expert, s.D, s.F, none, yp, st);
  return launch_product<Cfg<208, false, 3>>(ctx, td, td, th[0], th[1], down_op, slot_row_off, slot_expert, s.D, s.F, none, yp, st);
}
