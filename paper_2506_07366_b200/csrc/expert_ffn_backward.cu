// Gradient of the expert-parallel SwiGLU FFN over ragged slots.  With g = xp W1^T, u = xp W3^T kept in 8 bits by
// moegps_expert_ffn_gate_up_save (act8.cuh), s = sigmoid(g), h = g s u and yp = h W2^T:
//   1. act     : dh = dyp W2;  dgate = dh u s (1 + g (1 - s)),  dup = dh g s,  and h again      [rows x F, over D]
//   2. input   : dxp = dgate W1 + dup W3                                                        [rows x D, over 2 F]
//   3. weights : dW1[e] = dgate^T xp, dW3[e] = dup^T xp, dW2[e] = dyp^T h                       [F x D and D x F, over rows]
// Three persistent kernels on the tensor cores, with the ring, the TMEM accumulators and the warp roles of the
// forward GEMMs (expert_ffn.cu).  What differs is the operands' orientation: the weights are stored for the forward
// product, so in (1) and (2) the contraction runs along their row index, and in (3) along the row index of both
// operands.  Nothing is transposed in memory: TMA brings boxes of 64 contiguous elements x 64 rows, and the MMA reads
// them as MN-major operands.
// dgate, dup and h are rounded to bf16 between the kernels (they are operands of bf16 MMAs); dh never leaves the
// accumulator.  All sums are fp32 in tensor memory, rounded to bf16 once at the store.
//
// Measured (tensor pipe busy / SM clock): on 8192 rows x 4096 x 7168, 8 experts, (1) 0.40 ms, 86 % at 1.34 GHz, (2) 0.75 ms,
// 93 % at 1.31, (3) 1.15 ms, 70 % at 1.48; on 49152 rows x 2048 x 1408, 64 experts, 0.36 / 0.49 / 0.86 ms, 60 / 88 / 53 %.
// The long launches run at the chip's power limit (1.9 GHz is the most): there the clock gives what the pipe does not wait.
// (3) on many small experts is short of work for each tile: a tile of few rows ends before the one before it is stored.
#include "act8.cuh"
#include "grouped_gemm.cuh"

namespace {

using namespace sm100;
using namespace grouped_gemm;

constexpr int kBoxBytes = 64 * BK * 2;             // a box of an MN-major operand: 64 elements x BK rows
static_assert(BK == 64, "boxes are one 128-byte swizzle span wide and BK rows high");
static_assert(kABytes == 2 * kBoxBytes && 2 * kBHalfBytes == 4 * kBoxBytes, "a stage holds 2 + 4 boxes");

// Launch shape of (1) and (2): BM x BN tiles, a ring of 192 KiB whatever the stage's size.  256 columns feed the tensor
// core best (a stage's bytes against its products); 128 or 64 are for layers with fewer tiles than SMs, where one CTA
// would otherwise stream a whole column of the weights by itself while others idle.
template <int BN_>
struct DataCfg {
  static constexpr int BN = BN_, kStageBytes = kABytes + BN * kRowBytes, kStages = 192 * 1024 / kStageBytes;
  static constexpr int kAccs = 2, kEpiWarps = 8, kThreads = 64 + 32 * kEpiWarps, kTmemCols = kAccs * BN;
  static constexpr size_t kSmem = 1024 + 192 * 1024 + sizeof(Tables) + 256 + (size_t)kEpiWarps * kStagingBytesPerWarp;
};
static_assert(DataCfg<256>::kStages == 4 && DataCfg<128>::kStages == 6 && DataCfg<64>::kStages == 8, "whole stages");
static_assert(DataCfg<256>::kSmem <= 227 * 1024, "one CTA per SM");

// The 8-bit activations that (1) reads: codes [rcap][pitch], scales [blocks][rcap].
struct KeptActs {
  const uint8_t *gate8, *up8, *gate_scale, *up_scale;
};
struct ActOutputs {
  __nv_bfloat16 *dgate, *dup, *h;
};

// A lane's 32 + 32 codes of one block, with their scales; zero where there is no such row or block.
struct KeptBlock {
  uint4 g[2], u[2];
  uint32_t gs, us;
};
__device__ __forceinline__ void load_block(KeptBlock& b, const KeptActs& kept, int row, int row_end, int col, int n_dim,
                                           int rcap) {
  if (row < row_end && col < n_dim) {
    const size_t at = (size_t)row * act8::pitch_of(n_dim) + col;
    const uint4* g = reinterpret_cast<const uint4*>(kept.gate8 + at);
    const uint4* u = reinterpret_cast<const uint4*>(kept.up8 + at);
    b.g[0] = __ldg(g);
    b.g[1] = __ldg(g + 1);
    b.u[0] = __ldg(u);
    b.u[1] = __ldg(u + 1);
    const size_t sc = (size_t)(col / act8::kBlock) * rcap + row;
    b.gs = __ldg(kept.gate_scale + sc);
    b.us = __ldg(kept.up_scale + sc);
  } else {
    b.g[0] = b.g[1] = b.u[0] = b.u[1] = make_uint4(0, 0, 0, 0);
    b.gs = b.us = 0;
  }
}

// 1 / (1 + exp(-x)) by the hardware's exp2 and reciprocal (relative error a few 2^-22; the results are rounded to bf16,
// 2^-8).  The forms that flush subnormals: exp(-x) is 0 or infinite far out, where the sigmoid is 1 or 0 to fp32 anyway,
// and without the flush each costs several instructions more in the longest epilogue here.
__device__ __forceinline__ float sigmoid_fast(float x) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(-1.4426950408889634f * x));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
  return r;
}

// The four values of one code word each, with their part of dh -> packed dgate, dup, h.
__device__ __forceinline__ void act_gradient(uint32_t gw, uint32_t uw, float gs, float us, const uint32_t* dh, uint32_t* dgate,
                                             uint32_t* dup, uint32_t* h) {
  float g[4], u[4];
  act8::decode4(gw, gs, g);
  act8::decode4(uw, us, u);
  float dg[4], du[4], hh[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float d = __uint_as_float(dh[i]);
    const float s = sigmoid_fast(g[i]);
    const float a = g[i] * s;                       // silu
    dg[i] = d * u[i] * fmaf(a, 1.f - s, s);         // s (1 + g (1 - s)) = s + a (1 - s)
    du[i] = d * a;
    hh[i] = a * u[i];
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    dgate[i] = pack_bf16(dg[2 * i], dg[2 * i + 1]);
    dup[i] = pack_bf16(du[2 * i], du[2 * i + 1]);
    h[i] = pack_bf16(hh[2 * i], hh[2 * i + 1]);
  }
}

// 16 consecutive bf16 of one row; the first and the second eight may lie beyond the row's end.
__device__ __forceinline__ void store16(__nv_bfloat16* at, const uint32_t (&o)[8], bool first, bool second, bool whole_sectors) {
  if (whole_sectors && second) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(at), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]),
                 "r"(o[4]), "r"(o[5]), "r"(o[6]), "r"(o[7])
                 : "memory");
  } else {
    if (first) *reinterpret_cast<uint4*>(at) = make_uint4(o[0], o[1], o[2], o[3]);
    if (second) *reinterpret_cast<uint4*>(at + 8) = make_uint4(o[4], o[5], o[6], o[7]);
  }
}

// whether 16 columns that start at a multiple of 16 are a whole 32-byte sector in all three results
__device__ __forceinline__ bool act_whole_sectors(const ActOutputs& out, int n_dim) {
  return ((reinterpret_cast<uintptr_t>(out.dgate) | reinterpret_cast<uintptr_t>(out.dup) | reinterpret_cast<uintptr_t>(out.h) |
           (uintptr_t)n_dim * 2) & 31) == 0;
}

// Epilogue of (1) for one warp: 32 rows x [c_begin, c_end) columns of dh, one row for each lane.  The codes of a chunk are
// loaded while the chunk before it is worked on (the first one before the accumulator is complete).  A lane stores 16
// columns of its row at a time, a whole 32-byte sector, straight from its registers: with three results to store, keeping
// a chunk of each for the staging buffer that the other epilogues use costs more registers than there are.
__device__ __forceinline__ void drain_act(uint32_t taddr, int lane, const KeptActs& kept, KeptBlock& next, const ActOutputs& out,
                                          int row0, int row_end, int col0, int n_dim, int c_begin, int c_end, int rcap,
                                          bool whole_sectors) {
  const int row = row0 + lane;
#pragma unroll 1
  for (int c0 = c_begin; c0 < c_end; c0 += 32) {
    const KeptBlock cur = next;
    if (c0 + 32 < c_end) load_block(next, kept, row, row_end, col0 + c0 + 32, n_dim, rcap);
    uint32_t acc[32];
    tmem_ld32(taddr + c0, acc);
    tmem_ld_wait();
    const float gs = act8::scale_of(cur.gs), us = act8::scale_of(cur.us);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const uint32_t gw[4] = {cur.g[half].x, cur.g[half].y, cur.g[half].z, cur.g[half].w};
      const uint32_t uw[4] = {cur.u[half].x, cur.u[half].y, cur.u[half].z, cur.u[half].w};
      uint32_t dgate[8], dup[8], h[8];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        act_gradient(gw[i], uw[i], gs, us, acc + 16 * half + 4 * i, dgate + 2 * i, dup + 2 * i, h + 2 * i);
      const int col = col0 + c0 + 16 * half;
      const bool first = row < row_end && col + 8 <= n_dim, second = row < row_end && col + 16 <= n_dim;
      const size_t at = (size_t)row * n_dim + col;
      store16(out.dgate + at, dgate, first, second, whole_sectors);
      store16(out.dup + at, dup, first, second, whole_sectors);
      store16(out.h + at, h, first, second, whole_sectors);
    }
  }
}

// Epilogue of (2): accumulator -> bf16 -> global.
__device__ __forceinline__ void drain_plain(uint32_t taddr, uint8_t* staging, int lane, __nv_bfloat16* out, int row0,
                                            int row_end, int col0, int n_dim, int c_begin, int c_end) {
#pragma unroll 1
  for (int c0 = c_begin; c0 < c_end; c0 += 32) {
    uint32_t o[16], a[32];
    tmem_ld32(taddr + c0, a);
    tmem_ld_wait();
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] = pack_bf16(__uint_as_float(a[2 * i]), __uint_as_float(a[2 * i + 1]));
    store_chunk(o, staging, lane, out, row0, row_end, col0 + c0, n_dim);
  }
}

// The barriers behind the ring, and what else the roles share.
template <class Cfg>
struct Bars {
  uint64_t *full, *empty, *acc_full, *acc_empty;
  uint32_t* tmem_slot;
  volatile int* abort_flag;
  __device__ explicit Bars(uint8_t* at) {
    full = reinterpret_cast<uint64_t*>(at);         // [kStages] TMA -> MMA
    empty = full + Cfg::kStages;                    // [kStages] MMA -> TMA
    acc_full = empty + Cfg::kStages;                // [kAccs]   MMA -> epilogue
    acc_empty = acc_full + Cfg::kAccs;              // [kAccs]   epilogue -> MMA
    tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + Cfg::kAccs);
    abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  }
  __device__ void init() const {
    for (int i = 0; i < Cfg::kStages; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
    for (int i = 0; i < Cfg::kAccs; ++i) { mbar_init(&acc_full[i], 1); mbar_init(&acc_empty[i], Cfg::kEpiWarps); }
    *abort_flag = 0;
    fence_mbar_init();
  }
};

// let copies and MMAs that are still in flight end before the CTA retires
__device__ __forceinline__ void linger() {
  for (int i = 0; i < 1000; ++i) __nanosleep(1000);
}

// ------------------------------------------------------------------------------------------------ (1) and (2)
// C[rows, n_dim] = sum over `pairs` of A_p[rows, k_dim] B_p[e][k_dim, n_dim]; A K-major, B MN-major.
// kAct: one pair (dyp, W2) and the activation's gradient as epilogue; else two pairs (dgate, W1), (dup, W3).
template <bool kAct, class Cfg>
__global__ void __launch_bounds__(Cfg::kThreads, 1)
data_gradient_kernel(const __grid_constant__ CUtensorMap tm_a0, const __grid_constant__ CUtensorMap tm_b0,
                     const __grid_constant__ CUtensorMap tm_a1, const __grid_constant__ CUtensorMap tm_b1,
                     const int32_t* __restrict__ slot_row_off, const int32_t* __restrict__ slot_expert, int S, int E, int n_dim,
                     int k_dim, int rcap, const KeptActs kept, const ActOutputs act_out, __nv_bfloat16* __restrict__ out,
                     int32_t* __restrict__ status) {
  constexpr int kStages = Cfg::kStages, kAccs = Cfg::kAccs, kThreads = Cfg::kThreads, BN = Cfg::BN;
  constexpr int kStageBytes = Cfg::kStageBytes;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* stage_mem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  Tables& tb = *reinterpret_cast<Tables*>(stage_mem + (size_t)kStages * kStageBytes);
  const Bars<Cfg> bar(stage_mem + (size_t)kStages * kStageBytes + sizeof(Tables));

  const int warp = uniform_warp_index(), lane = threadIdx.x & 31;
  const int n_tiles = (n_dim + BN - 1) / BN;
  const int kb_per_pair = (k_dim + BK - 1) / BK;
  const int num_kb = kAct ? kb_per_pair : 2 * kb_per_pair;

  if (threadIdx.x == 0) {
    bar.init();
    prefetch_tensormap(&tm_a0);
    prefetch_tensormap(&tm_b0);
    if (!kAct) { prefetch_tensormap(&tm_a1); prefetch_tensormap(&tm_b1); }
  }
  launch_dependents();
  wait_for_predecessor();
  if (warp == 1) {
    tmem_alloc(bar.tmem_slot, Cfg::kTmemCols);
    tmem_relinquish();
  }
  build_tables<kThreads>(tb, slot_row_off, slot_expert, S, E, n_tiles, rcap, status);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = *bar.tmem_slot;
  const int total_tiles = tb.tile_base[S];

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int tile = blockIdx.x; ok && tile < total_tiles; tile += gridDim.x) {
        const TileCoord tc = decode_tile(tb, slot_row_off, slot_expert, S, tile, n_tiles);
        const int nb0 = tc.n_tile * BN;
        for (int kb = 0; kb < num_kb; ++kb) {
          if (!mbar_wait(&bar.empty[stage], phase ^ 1u, bar.abort_flag)) { ok = false; break; }
          uint8_t* sa = stage_mem + (size_t)stage * kStageBytes;
          mbar_arrive_expect_tx(&bar.full[stage], kStageBytes);
          const bool second = !kAct && kb >= kb_per_pair;
          const int k0 = (second ? kb - kb_per_pair : kb) * BK;
          const CUtensorMap* ta = second ? &tm_a1 : &tm_a0;
          const CUtensorMap* tbm = second ? &tm_b1 : &tm_b0;
          tma_load_2d(sa, ta, &bar.full[stage], k0, tc.m0);
#pragma unroll
          for (int i = 0; i < BN / 64; ++i)
            tma_load_3d(sa + kABytes + i * kBoxBytes, tbm, &bar.full[stage], nb0 + 64 * i, k0, tc.expert);
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
      }
      if (!ok) linger();
    }
  } else if (warp == 1) {
    constexpr uint32_t idesc = idesc_bf16_f32(BM, BN, false, true);
    const uint32_t ring = smem_u32(stage_mem);
    int stage = 0, acc = 0;
    uint32_t phase = 0, acc_phase = 0;
    bool ok = true;
    for (int tile = blockIdx.x; ok && tile < total_tiles; tile += gridDim.x) {
      if (!warp_wait(&bar.acc_empty[acc], acc_phase ^ 1u, bar.abort_flag)) { ok = false; break; }
      tc_fence_after_sync();
      const uint32_t d_tmem = tmem_base + (uint32_t)acc * BN;
      for (int kb = 0; kb < num_kb; ++kb) {
        if (!warp_wait(&bar.full[stage], phase, bar.abort_flag)) { ok = false; break; }
        tc_fence_after_sync();
        const uint32_t sa = ring + (uint32_t)stage * kStageBytes;
        const uint64_t da = smem_desc_k<kRowBytes>(sa);
        const uint64_t db = smem_desc_mn(sa + kABytes, kBoxBytes);
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < BK / 16; ++k)      // A advances 32 bytes along its rows, B 16 rows of 128 bytes
            mma_bf16(d_tmem, da + (uint64_t)(k * 2), db + (uint64_t)(k * 128), idesc, (kb | k) != 0);
          mma_commit(&bar.empty[stage]);
        }
        if (++stage == kStages) { stage = 0; phase ^= 1u; }
      }
      if (!ok) break;
      if (elect_one()) mma_commit(&bar.acc_full[acc]);
      if (++acc == kAccs) { acc = 0; acc_phase ^= 1u; }
    }
    if (!ok) linger();
  } else {
    const int quarter = warp & 3;                 // TMEM lanes this warp may read
    constexpr int kShare = BN / (Cfg::kEpiWarps / 4);
    const int c_begin = ((warp - 2) >> 2) * kShare;
    uint8_t* staging = stage_mem + (size_t)kStages * kStageBytes + sizeof(Tables) + 256 + (warp - 2) * kStagingBytesPerWarp;
    [[maybe_unused]] const bool whole_sectors = act_whole_sectors(act_out, n_dim);
    int acc = 0;
    uint32_t acc_phase = 0;
    bool ok = true;
    for (int tile = blockIdx.x; ok && tile < total_tiles; tile += gridDim.x) {
      const TileCoord tc = decode_tile(tb, slot_row_off, slot_expert, S, tile, n_tiles);
      const int row0 = tc.m0 + quarter * 32, col0 = tc.n_tile * BN;
      [[maybe_unused]] KeptBlock block;
      if constexpr (kAct) load_block(block, kept, row0 + lane, tc.row_end, col0 + c_begin, n_dim, rcap);
      if (!mbar_wait(&bar.acc_full[acc], acc_phase, bar.abort_flag, 256)) { ok = false; break; }
      tc_fence_after_sync();
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)acc * BN;
      if constexpr (kAct)
        drain_act(taddr, lane, kept, block, act_out, row0, tc.row_end, col0, n_dim, c_begin, c_begin + kShare, rcap, whole_sectors);
      else
        drain_plain(taddr, staging, lane, out, row0, tc.row_end, col0, n_dim, c_begin, c_begin + kShare);
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bar.acc_empty[acc]);
      if (++acc == kAccs) { acc = 0; acc_phase ^= 1u; }
    }
  }

  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();
  if (threadIdx.x == 0 && *bar.abort_flag) moegps_report(status, MOEGPS_ERR_TIMEOUT, (int)blockIdx.x);
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem_base, Cfg::kTmemCols);
  }
}

// The barriers of a kernel whose tiles are worked by pairs of CTAs.  full counts both CTAs' bytes on the leader; empty and
// acc_full are signalled in both CTAs by the leader's commits; acc_empty collects both CTAs' epilogue warps on the leader.
// tail_full, tail_ready (weight_gradient_kernel only): at a slot's end, where rows have to be blanked before the MMA, each
// CTA's bytes go to its own tail_full, and the warps that blank report to the leader's tail_ready.
struct PairCfg {
  static constexpr int kStages = 6, kAccs = 2, kEpiWarps = 8, kTmemCols = kAccs * BNACC;
  static constexpr int kAHalf = 2 * kBoxBytes, kStageBytes = 4 * kBoxBytes;        // per CTA: 128 rows of A, 128 columns of B
};
struct PairBars {
  uint64_t *full, *empty, *tail_full, *tail_ready, *acc_full, *acc_empty;
  uint32_t* tmem_slot;
  volatile int* abort_flag;
  __device__ explicit PairBars(uint8_t* at) {
    constexpr int n = PairCfg::kStages;
    full = reinterpret_cast<uint64_t*>(at);
    empty = full + n;
    tail_full = empty + n;
    tail_ready = tail_full + n;
    acc_full = tail_ready + n;
    acc_empty = acc_full + PairCfg::kAccs;
    tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + PairCfg::kAccs);
    abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  }
  __device__ void init() const {
    for (int i = 0; i < PairCfg::kStages; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
      mbar_init(&tail_full[i], 1);
      mbar_init(&tail_ready[i], 2);
    }
    for (int i = 0; i < PairCfg::kAccs; ++i) {
      mbar_init(&acc_full[i], 1);
      mbar_init(&acc_empty[i], 2 * PairCfg::kEpiWarps);
    }
    *abort_flag = 0;
    fence_mbar_init();
  }
};
static_assert((4 * PairCfg::kStages + 2 * PairCfg::kAccs) * 8 + 8 <= 256, "barriers fit their space");

// ------------------------------------------------------------------------------------------------ (1) and (2), by pairs
// The same products on 256 x 256 tiles of a slot: each CTA of a pair has 128 of the rows, loads them and half the columns
// of the weights, 32 KiB for a K block instead of 48.  For long slots (choose_tiles): the last tile of a slot leaves the
// second CTA idle when it has at most 128 rows.  Measured, whole gradient: 2048 rows a slot (16384 tokens, 16
// slots) 20.4 -> 19.8 ms, 614 rows a slot (64 experts, 80 slots) 1.96 -> 1.94 ms, 137 rows a slot not faster.
struct PairDataCfg : PairCfg {
  static constexpr int kThreads = 64 + 32 * kEpiWarps;
  static constexpr size_t kSmem =
      1024 + (size_t)kStages * kStageBytes + sizeof(Tables) + 256 + (size_t)kEpiWarps * kStagingBytesPerWarp;
};
static_assert(PairDataCfg::kSmem <= 227 * 1024, "one CTA per SM");

template <bool kAct>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(PairDataCfg::kThreads, 1)
data_gradient_pair_kernel(const __grid_constant__ CUtensorMap tm_a0, const __grid_constant__ CUtensorMap tm_b0,
                          const __grid_constant__ CUtensorMap tm_a1, const __grid_constant__ CUtensorMap tm_b1,
                          const int32_t* __restrict__ slot_row_off, const int32_t* __restrict__ slot_expert, int S, int E,
                          int n_dim, int k_dim, int rcap, const KeptActs kept, const ActOutputs act_out,
                          __nv_bfloat16* __restrict__ out, int32_t* __restrict__ status) {
  using Cfg = PairDataCfg;
  constexpr int kStages = Cfg::kStages, kAccs = Cfg::kAccs, kStageBytes = Cfg::kStageBytes;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* stage_mem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  Tables& tb = *reinterpret_cast<Tables*>(stage_mem + (size_t)kStages * kStageBytes);
  const PairBars bar(stage_mem + (size_t)kStages * kStageBytes + sizeof(Tables));

  const int warp = uniform_warp_index(), lane = threadIdx.x & 31;
  const int rank = (int)cluster_ctarank(), pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const int n_tiles = (n_dim + BNACC - 1) / BNACC;
  const int kb_per_pair = (k_dim + BK - 1) / BK;
  const int num_kb = kAct ? kb_per_pair : 2 * kb_per_pair;

  if (threadIdx.x == 0) {
    bar.init();
    prefetch_tensormap(&tm_a0);
    prefetch_tensormap(&tm_b0);
    if (!kAct) { prefetch_tensormap(&tm_a1); prefetch_tensormap(&tm_b1); }
  }
  launch_dependents();
  wait_for_predecessor();
  if (warp == 1) {
    tmem_alloc_pair(bar.tmem_slot, Cfg::kTmemCols);
    tmem_relinquish_pair();
  }
  build_tables<Cfg::kThreads, 2 * BM>(tb, slot_row_off, slot_expert, S, E, n_tiles, rcap, status);
  __syncwarp();
  tc_fence_before_sync();
  cluster_sync_all();
  tc_fence_after_sync();
  const uint32_t tmem_base = *bar.tmem_slot;
  const int total_tiles = tb.tile_base[S];

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      const uint32_t leader_full = map_to_cta(smem_u32(bar.full), 0);
      for (int tile = pair; ok && tile < total_tiles; tile += pairs) {
        const TileCoord tc = decode_tile<2 * BM>(tb, slot_row_off, slot_expert, S, tile, n_tiles);
        const int m0 = tc.m0 + rank * BM, n0 = tc.n_tile * BNACC + rank * (BNACC / 2);
        for (int kb = 0; kb < num_kb; ++kb) {
          if (!mbar_wait(&bar.empty[stage], phase ^ 1u, bar.abort_flag)) { ok = false; break; }
          uint8_t* sa = stage_mem + (size_t)stage * kStageBytes;
          if (rank == 0) mbar_arrive_expect_tx(&bar.full[stage], 2 * kStageBytes);
          const bool second = !kAct && kb >= kb_per_pair;
          const int k0 = (second ? kb - kb_per_pair : kb) * BK;
          const CUtensorMap* ta = second ? &tm_a1 : &tm_a0;
          const CUtensorMap* tbm = second ? &tm_b1 : &tm_b0;
          const uint32_t to = leader_full + stage * 8;
          tma_load_2d_pair(sa, ta, to, k0, m0);
#pragma unroll
          for (int i = 0; i < 2; ++i) tma_load_3d_pair(sa + Cfg::kAHalf + i * kBoxBytes, tbm, to, n0 + 64 * i, k0, tc.expert);
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
      }
      if (!ok) linger();
    }
  } else if (warp == 1) {
    if (rank == 0) {
      constexpr uint32_t idesc = idesc_bf16_f32(2 * BM, BNACC, false, true);
      const uint32_t ring = smem_u32(stage_mem);
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      bool ok = true;
      for (int tile = pair; ok && tile < total_tiles; tile += pairs) {
        if (!warp_wait_cluster(&bar.acc_empty[acc], acc_phase ^ 1u, bar.abort_flag)) { ok = false; break; }
        tc_fence_after_sync();
        const uint32_t d_tmem = tmem_base + (uint32_t)acc * BNACC;
        for (int kb = 0; kb < num_kb; ++kb) {
          if (!warp_wait(&bar.full[stage], phase, bar.abort_flag)) { ok = false; break; }
          tc_fence_after_sync();
          const uint32_t sa = ring + (uint32_t)stage * kStageBytes;
          const uint64_t da = smem_desc_k<kRowBytes>(sa);
          const uint64_t db = smem_desc_mn(sa + Cfg::kAHalf, kBoxBytes);
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < BK / 16; ++k)
              mma_bf16_pair(d_tmem, da + (uint64_t)(k * 2), db + (uint64_t)(k * 128), idesc, (kb | k) != 0);
            mma_commit_pair(&bar.empty[stage]);
          }
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
        if (!ok) break;
        if (elect_one()) mma_commit_pair(&bar.acc_full[acc]);
        if (++acc == kAccs) { acc = 0; acc_phase ^= 1u; }
      }
      if (!ok) linger();
    }
  } else {
    const int quarter = warp & 3;
    constexpr int kShare = BNACC / (Cfg::kEpiWarps / 4);
    const int c_begin = ((warp - 2) >> 2) * kShare;
    uint8_t* staging = stage_mem + (size_t)kStages * kStageBytes + sizeof(Tables) + 256 + (warp - 2) * kStagingBytesPerWarp;
    const uint32_t leader_empty = map_to_cta(smem_u32(bar.acc_empty), 0);
    [[maybe_unused]] const bool whole_sectors = act_whole_sectors(act_out, n_dim);
    int acc = 0;
    uint32_t acc_phase = 0;
    for (int tile = pair; tile < total_tiles; tile += pairs) {
      const TileCoord tc = decode_tile<2 * BM>(tb, slot_row_off, slot_expert, S, tile, n_tiles);
      const int row0 = tc.m0 + rank * BM + quarter * 32, col0 = tc.n_tile * BNACC;
      [[maybe_unused]] KeptBlock block;
      if constexpr (kAct) load_block(block, kept, row0 + lane, tc.row_end, col0 + c_begin, n_dim, rcap);
      if (!mbar_wait(&bar.acc_full[acc], acc_phase, bar.abort_flag, 256)) break;
      tc_fence_after_sync();
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)acc * BNACC;
      if (row0 < tc.row_end) {                       // (a warp without rows of the slot has nothing to store)
        if constexpr (kAct)
          drain_act(taddr, lane, kept, block, act_out, row0, tc.row_end, col0, n_dim, c_begin, c_begin + kShare, rcap,
                    whole_sectors);
        else
          drain_plain(taddr, staging, lane, out, row0, tc.row_end, col0, n_dim, c_begin, c_begin + kShare);
      }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive_remote(leader_empty + acc * 8);
      if (++acc == kAccs) { acc = 0; acc_phase ^= 1u; }
    }
  }

  __syncwarp();
  tc_fence_before_sync();
  cluster_sync_all();                                // nobody touches the other CTA's memory after this
  if (threadIdx.x == 0 && *bar.abort_flag) moegps_report(status, MOEGPS_ERR_TIMEOUT, (int)blockIdx.x);
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc_pair(tmem_base, Cfg::kTmemCols);
  }
}

// ------------------------------------------------------------------------------------------------ (3)
// Occupied rows of every slot: first row and count.  The padding that dispatch leaves at a slot's end (row_pair < 0)
// holds no token and must not enter the sums, whatever its memory holds.
struct SlotRows {
  int2 ext[kMaxS];
};

// A tile is 256 x 256, worked by a pair of CTAs: each has 128 of the rows, loads them and half the columns of the right
// operand (32 KiB for a K block, where a CTA by itself needs 48 KiB for a 128 x 256 tile), and keeps its part of the sum in
// its own TMEM.  Neither dimension is ragged here, unlike the rows of the other GEMMs.
// Per expert there are two problems: dgate and dup above one another, times xp (dW1 and dW3; an even number of 128-row
// granules, whichever gradient each belongs to, so no pair has an idle half), and dyp times h (dW2).  A last column tile with
// at most 128 columns is worked as 256 x 128.  Inside a problem the order runs over bands of kBand tiles in M, column by
// column: tiles in flight at the same time form a near-square patch, so the operand columns they read are shared in L2
// (1 % on 64 experts against whole columns).
struct WeightCfg : PairCfg {
  static constexpr int kBlankWarp = 2 + kEpiWarps, kThreads = 32 * (3 + kEpiWarps);          // producer, MMA, epilogue, blank
  static constexpr int kOutBytes = 32 * 64;                                  // of an epilogue warp: 32 rows x 32 columns, bf16
  static constexpr int kAhead = 8;                                           // > tiles that the producer can be ahead: kStages
  static constexpr size_t kSmem = 1024 + (size_t)kStages * kStageBytes + kEpiWarps * kOutBytes + 8 * kMaxS + 256;
};
static_assert(WeightCfg::kSmem + 2 * 257 * 4 <= 227 * 1024, "one CTA per SM");
constexpr int kBand = 8;

// Limit of a wait that lasts as long as the sums over `rows` rows.  A K block of 64 rows takes 600 to 1700 cycles; 64 cycles are
// allowed for each row.  The plain limit, about a second, is passed by a sum over 2 10^8 rows (8 columns: 600 cycles a block).
__device__ __forceinline__ long long wait_limit(long long rows) { return kWaitLimitCycles + 64 * rows; }

struct WTile {
  int expert, problem, m, n0;       // m: tile in M; n0: first column
};
struct WGeom {
  int F, D, granules_f, mt[2], nt[2], per[2];     // tiles in M and N of the two problems, and in all
  __device__ WGeom(int F_, int D_) : F(F_), D(D_) {
    granules_f = (F + BM - 1) / BM;
    mt[0] = granules_f;
    mt[1] = ((D + BM - 1) / BM + 1) / 2;
    nt[0] = (D + BNACC - 1) / BNACC;
    nt[1] = (F + BNACC - 1) / BNACC;
    per[0] = mt[0] * nt[0];
    per[1] = mt[1] * nt[1];
  }
  __device__ WTile decode(int tile) const {
    WTile t;
    const int all = per[0] + per[1];
    t.expert = tile / all;
    int q = tile - t.expert * all;
    t.problem = q >= per[0];
    const int p_mt = t.problem ? mt[1] : mt[0], p_nt = t.problem ? nt[1] : nt[0];
    if (t.problem) q -= per[0];
    const int band = q / (kBand * p_nt);
    q -= band * kBand * p_nt;
    const int high = min(kBand, p_mt - band * kBand), col = q / high;
    t.n0 = col * BNACC;
    t.m = band * kBand + q - col * high;
    return t;
  }
  // columns that a tile works
  __device__ int width(const WTile& t) const { return (t.problem ? F : D) - t.n0 > BNACC / 2 ? BNACC : BNACC / 2; }
  // which gradient (0 dW1, 1 dW3, 2 dW2) and first row of it a CTA of the pair has
  __device__ void rows(const WTile& t, int rank, int& which, int& m0) const {
    int g = 2 * t.m + rank;
    which = 2;
    if (t.problem == 0) {
      which = g >= granules_f;
      g -= which * granules_f;
    }
    m0 = g * BM;
  }
};

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(WeightCfg::kThreads, 1)
weight_gradient_kernel(const __grid_constant__ CUtensorMap tm_dgate, const __grid_constant__ CUtensorMap tm_dup,
                       const __grid_constant__ CUtensorMap tm_dyp, const __grid_constant__ CUtensorMap tm_xp,
                       const __grid_constant__ CUtensorMap tm_h, const __grid_constant__ CUtensorMap tm_dw_gate,
                       const __grid_constant__ CUtensorMap tm_dw_up, const __grid_constant__ CUtensorMap tm_dw_down,
                       const int32_t* __restrict__ slot_row_off, const int32_t* __restrict__ slot_off,
                       const int32_t* __restrict__ row_pair, int S, int E, int F, int D, int row_align, int rcap,
                       int32_t* __restrict__ status) {
  using Cfg = WeightCfg;
  constexpr int kStages = Cfg::kStages, kAccs = Cfg::kAccs, kThreads = Cfg::kThreads, kStageBytes = Cfg::kStageBytes;
  extern __shared__ uint8_t smem_raw[];
  __shared__ int32_t s_slot_off[256 + 1], s_rows[256];       // first slot and occupied rows of every expert
  __shared__ int s_width[WeightCfg::kAhead];                 // of the tiles that the producer is ahead
  uint8_t* stage_mem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* out_mem = stage_mem + (size_t)kStages * kStageBytes;
  SlotRows& sr = *reinterpret_cast<SlotRows*>(out_mem + Cfg::kEpiWarps * Cfg::kOutBytes);
  const PairBars bar(reinterpret_cast<uint8_t*>(&sr) + sizeof(SlotRows));

  const int warp = uniform_warp_index(), lane = threadIdx.x & 31;
  const int rank = (int)cluster_ctarank();           // 0: leader
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const WGeom geom(F, D);
  const int total_tiles = E * (geom.per[0] + geom.per[1]);

  if (threadIdx.x == 0) {
    bar.init();
    for (const CUtensorMap* m : {&tm_dgate, &tm_dup, &tm_dyp, &tm_xp, &tm_h, &tm_dw_gate, &tm_dw_up, &tm_dw_down})
      prefetch_tensormap(m);
  }
  launch_dependents();
  wait_for_predecessor();
  if (warp == 1) {
    tmem_alloc_pair(bar.tmem_slot, Cfg::kTmemCols);
    tmem_relinquish_pair();
  }
  for (int s = threadIdx.x; s < S; s += kThreads) {
    const int lo = slot_row_off[s], hi = slot_row_off[s + 1];
    int n = 0;
    if (lo < 0 || hi < lo || hi > rcap) {
      if (blockIdx.x == 0) moegps_report(status, MOEGPS_ERR_BAD_INDEX, s);
    } else {
      // padding is at the slot's end, fewer than row_align rows: looked at 16 rows at a time (loads that do not wait for
      // one another; a binary search is a chain of memory round trips)
      n = hi - lo;
      const int least = max(0, n - (row_align - 1));
      bool more = n > least;
      while (more) {
        int tail = 0;
        bool pad = true;
#pragma unroll
        for (int i = 1; i <= 16; ++i) {
          const int p = n - i >= least ? row_pair[lo + n - i] : 0;
          pad = pad && p < 0;
          tail += pad ? 1 : 0;
        }
        n -= tail;
        more = tail == 16 && n > least;
      }
    }
    sr.ext[s] = make_int2(lo, n);
  }
  for (int e = threadIdx.x; e <= E; e += kThreads) {
    int v = slot_off[e];
    if (v < 0 || v > S) {
      if (blockIdx.x == 0) moegps_report(status, MOEGPS_ERR_BAD_INDEX, e);
      v = 0;
    }
    s_slot_off[e] = v;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += kThreads) {
    int n = 0;
    for (int s = s_slot_off[e]; s < s_slot_off[e + 1]; ++s) n += sr.ext[s].y;
    s_rows[e] = n;
  }
  __syncwarp();
  tc_fence_before_sync();
  cluster_sync_all();                                // both CTAs' barriers and tables exist
  tc_fence_after_sync();
  const uint32_t tmem_base = *bar.tmem_slot;

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0, ahead = 0;
      uint32_t phase = 0;
      bool ok = true;
      const uint32_t leader_full = map_to_cta(smem_u32(bar.full), 0);
      const uint32_t own_tail = map_to_cta(smem_u32(bar.tail_full), rank);
      for (int tile = pair; ok && tile < total_tiles; tile += pairs) {
        const WTile t = geom.decode(tile);
        if (s_rows[t.expert] == 0) continue;
        int which, m0;
        geom.rows(t, rank, which, m0);
        const CUtensorMap* ta = which == 0 ? &tm_dgate : which == 1 ? &tm_dup : &tm_dyp;
        const CUtensorMap* tbm = t.problem ? &tm_h : &tm_xp;
        const int width = geom.width(t), n0 = t.n0 + rank * (width / 2);
        const uint32_t bytes = Cfg::kAHalf + (width / 128) * kBoxBytes;
        const int last = s_slot_off[t.expert + 1];
        // (the entry is free: the tile that had it last has given back all its stages, or this one would have to wait)
        bool first = true;
        for (int s = s_slot_off[t.expert]; ok && s < last; ++s) {
          const int2 ext = sr.ext[s];
          for (int r = 0; r < ext.y; r += BK) {
            if (!mbar_wait(&bar.empty[stage], phase ^ 1u, bar.abort_flag)) { ok = false; break; }
            if (first) s_width[ahead++ % Cfg::kAhead] = width;         // published by the arrival on full below
            first = false;
            uint8_t* sa = stage_mem + (size_t)stage * kStageBytes;
            const bool blank = ext.y - r < BK && ((ext.y - r) & 15) != 0;
            const uint32_t to = (blank ? own_tail : leader_full) + stage * 8;
            if (blank) {
              mbar_arrive_expect_tx(&bar.tail_full[stage], bytes);
              if (rank == 0) mbar_arrive(&bar.full[stage]);            // its phase passes; nobody waits for it
            } else if (rank == 0) {
              mbar_arrive_expect_tx(&bar.full[stage], 2 * bytes);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) tma_load_2d_pair(sa + i * kBoxBytes, ta, to, m0 + 64 * i, ext.x + r);
            tma_load_2d_pair(sa + Cfg::kAHalf, tbm, to, n0, ext.x + r);
            if (width == BNACC) tma_load_2d_pair(sa + Cfg::kAHalf + kBoxBytes, tbm, to, n0 + 64, ext.x + r);
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
          }
        }
      }
      if (!ok) linger();
    }
  } else if (warp == 1) {
    if (rank == 0) {
      const uint32_t ring = smem_u32(stage_mem);
      int stage = 0, acc = 0, expert = 0, ahead = 0;
      uint32_t phase = 0, acc_phase = 0, tail_phase = 0;       // tail_phase: a bit for each stage
      bool ok = true;
      // The tensor core holds a few MMAs at most, so what this warp does between two tiles is time lost: it takes a
      // tile's expert by counting and its width from the producer instead of decoding the tile (600 cycles).
      const int all = geom.per[0] + geom.per[1];
      int q = pair;
      for (int tile = pair; tile < total_tiles; tile += pairs, q += pairs) {
        for (; q >= all; q -= all) ++expert;
        if (s_rows[expert] == 0) continue;
        if (!warp_wait(&bar.full[stage], phase, bar.abort_flag)) { ok = false; break; }
        const uint32_t idesc = s_width[ahead++ % Cfg::kAhead] == BNACC ? idesc_bf16_f32(2 * BM, BNACC, true, true)
                                                                       : idesc_bf16_f32(2 * BM, BNACC / 2, true, true);
        if (!warp_wait_cluster(&bar.acc_empty[acc], acc_phase ^ 1u, bar.abort_flag)) { ok = false; break; }
        tc_fence_after_sync();
        const uint32_t d_tmem = tmem_base + (uint32_t)acc * BNACC;
        const int last = s_slot_off[expert + 1];
        uint32_t more = 0;                                     // 0: the tile's first block, whose first MMA starts the sum
        for (int s = s_slot_off[expert]; ok && s < last; ++s) {
          for (int left = sr.ext[s].y; left > 0; left -= BK) {
            if (left < BK && (left & 15)) {
              ok = warp_wait_cluster(&bar.tail_ready[stage], (tail_phase >> stage) & 1u, bar.abort_flag);
              tail_phase ^= 1u << stage;
            } else {
              ok = warp_wait(&bar.full[stage], phase, bar.abort_flag);
            }
            if (!ok) break;
            tc_fence_after_sync();
            const uint64_t da = smem_desc_mn(ring + (uint32_t)stage * kStageBytes, kBoxBytes);
            const uint64_t db = smem_desc_mn(ring + (uint32_t)stage * kStageBytes + Cfg::kAHalf, kBoxBytes);
            if (elect_one()) {
#pragma unroll
              for (int k = 0; k < BK / 16; ++k)
                if (16 * k < left)
                  mma_bf16_pair(d_tmem, da + (uint64_t)(k * 128), db + (uint64_t)(k * 128), idesc, k > 0 ? 1u : more);
              mma_commit_pair(&bar.empty[stage]);
            }
            more = 1;
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
          }
        }
        if (!ok) break;
        if (elect_one()) mma_commit_pair(&bar.acc_full[acc]);
        if (++acc == kAccs) { acc = 0; acc_phase ^= 1u; }
      }
      if (!ok) linger();
    }
  } else if (warp == Cfg::kBlankWarp) {
    // Blanks, in this CTA's part of a slot's last K block, the rows behind the slot's end that the last MMA reads (at most
    // 15, of both operands, since 0 * NaN is NaN): as soon as they have landed, while earlier blocks are being multiplied.
    const uint32_t ready = map_to_cta(smem_u32(bar.tail_ready), 0);
    int stage = 0;
    uint32_t tail_phase = 0;
    long long rows = 0;                                // that are multiplied before the next rows to blank are loaded, at most
    bool ok = true;
    for (int tile = pair; ok && tile < total_tiles; tile += pairs) {
      const int expert = tile / (geom.per[0] + geom.per[1]), last = s_slot_off[expert + 1];
      for (int s = s_slot_off[expert]; ok && s < last; ++s) {
        const int n = sr.ext[s].y, tail = n % BK;
        rows += n;
        stage = (stage + n / BK) % kStages;
        if (tail & 15) {
          const bool here =
              mbar_wait(&bar.tail_full[stage], (tail_phase >> stage) & 1u, bar.abort_flag, 100, wait_limit(rows));
          ok = __all_sync(0xffffffffu, here);
          if (!ok) break;
          uint8_t* sa = stage_mem + (size_t)stage * kStageBytes;
          for (int row = tail + (lane >> 3); row < (tail + 15) / 16 * 16; row += 4)       // eight lanes a row
#pragma unroll
            for (int box = 0; box < 4; ++box)
              *reinterpret_cast<uint4*>(sa + box * kBoxBytes + row * kRowBytes + (lane & 7) * 16) = make_uint4(0, 0, 0, 0);
          fence_proxy_async();
          __syncwarp();
          if (lane == 0) mbar_arrive_remote(ready + stage * 8);
          tail_phase ^= 1u << stage;
        }
        if (tail) stage = (stage + 1) % kStages;
      }
    }
  } else {
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    uint8_t* staging = out_mem + (warp - 2) * Cfg::kOutBytes;
    const uint32_t leader_empty = map_to_cta(smem_u32(bar.acc_empty), 0);
    int acc = 0;
    uint32_t acc_phase = 0;
    for (int tile = pair; tile < total_tiles; tile += pairs) {
      const WTile t = geom.decode(tile);
      int which, m0;
      geom.rows(t, rank, which, m0);
      const CUtensorMap* to = which == 0 ? &tm_dw_gate : which == 1 ? &tm_dw_up : &tm_dw_down;
      const int row0 = m0 + quarter * 32, m_dim = t.problem ? D : F, n_dim = t.problem ? F : D, share = geom.width(t) / 2;
      uint32_t o[4][16];                               // 128 columns of this lane's row, packed
      const int rows = s_rows[t.expert];
      if (rows != 0) {
        // (a short sum is awaited closely; through a long one the warps sleep, polling costs power that the MMAs need)
        if (!mbar_wait(&bar.acc_full[acc], acc_phase, bar.abort_flag, rows > 1024 ? 256 : 32, wait_limit(rows))) break;
        tc_fence_after_sync();
        // the accumulator is emptied into registers at one go and handed back, then the columns are stored: for an
        // expert with few rows the next sums are ready before the stores are out
        const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)acc * BNACC + half * share;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          if (32 * c < share) {
            uint32_t a[32];
            tmem_ld32(taddr + 32 * c, a);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) o[c][i] = pack_bf16(__uint_as_float(a[2 * i]), __uint_as_float(a[2 * i + 1]));
          }
        }
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive_remote(leader_empty + acc * 8);
        if (++acc == kAccs) { acc = 0; acc_phase ^= 1u; }
      } else {                                         // no token chose this expert
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[c][i] = 0;
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int col = t.n0 + half * share + 32 * c;
        if (32 * c >= share || col >= n_dim || row0 >= m_dim) break;
        // 32 rows of 64 bytes in the store's 64-byte swizzle (16-byte word w of row r at w ^ (r / 2 % 4)), which also
        // keeps the lanes' writes free of bank conflicts; the TMA unit writes the box
        if (lane == 0) bulk_wait_read<0>();
        __syncwarp();
#pragma unroll
        for (int w = 0; w < 4; ++w)
          *reinterpret_cast<uint4*>(staging + lane * 64 + ((w ^ ((lane >> 1) & 3)) << 4)) =
              make_uint4(o[c][4 * w], o[c][4 * w + 1], o[c][4 * w + 2], o[c][4 * w + 3]);
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
          tma_store_3d(to, staging, col, row0, t.expert);
          bulk_commit();
        }
      }
    }
    if (lane == 0) bulk_wait_all();
  }

  __syncwarp();
  tc_fence_before_sync();
  cluster_sync_all();                                // nobody touches the other CTA's memory after this
  if (threadIdx.x == 0 && *bar.abort_flag) moegps_report(status, MOEGPS_ERR_TIMEOUT, (int)blockIdx.x);
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc_pair(tmem_base, Cfg::kTmemCols);
  }
}

int tmap_failed(moegps_ctx* ctx) {
  ctx->last_cuda_error = (int)cudaErrorInvalidValue;
  return MOEGPS_ERR_CUDA;
}

template <bool kAct, int BN>
int launch_data_gradient(moegps_ctx* ctx, const CUtensorMap& a0, const CUtensorMap& b0, const CUtensorMap& a1,
                         const CUtensorMap& b1, const int32_t* slot_row_off, const int32_t* slot_expert, int n_dim, int k_dim,
                         const KeptActs& kept, const ActOutputs& act_out, void* out, cudaStream_t st) {
  using Cfg = DataCfg<BN>;
  const moegps_shape_t& s = ctx->shape;
  bool& done = ctx->data_gradient_attr_done[kAct ? 0 : 1][BN == 256 ? 2 : BN == 128 ? 1 : 0];
  if (!done) {
    MOEGPS_CUDA_TRY(ctx, cudaFuncSetAttribute(data_gradient_kernel<kAct, Cfg>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                              (int)Cfg::kSmem));
    done = true;
  }
  MOEGPS_CUDA_TRY(ctx, launch_after(data_gradient_kernel<kAct, Cfg>, dim3(ctx->sm_count), Cfg::kThreads, Cfg::kSmem, st, a0, b0,
                                    a1, b1, slot_row_off, slot_expert, s.S, s.E, n_dim, k_dim, (int)moegps_rcap_of(s), kept,
                                    act_out, static_cast<__nv_bfloat16*>(out), ctx->d_status));
  MOEGPS_AFTER_LAUNCH(ctx, "%s tile=%dx%d", kAct ? "act" : "input", BM, BN);
  return MOEGPS_OK;
}

template <bool kAct>
int launch_data_gradient_pair(moegps_ctx* ctx, const CUtensorMap& a0, const CUtensorMap& b0, const CUtensorMap& a1,
                              const CUtensorMap& b1, const int32_t* slot_row_off, const int32_t* slot_expert, int n_dim,
                              int k_dim, const KeptActs& kept, const ActOutputs& act_out, void* out, cudaStream_t st) {
  using Cfg = PairDataCfg;
  const moegps_shape_t& s = ctx->shape;
  bool& done = ctx->data_gradient_attr_done[kAct ? 0 : 1][3];
  if (!done) {
    MOEGPS_CUDA_TRY(ctx, cudaFuncSetAttribute(data_gradient_pair_kernel<kAct>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                              (int)Cfg::kSmem));
    done = true;
  }
  MOEGPS_CUDA_TRY(ctx, launch_after(data_gradient_pair_kernel<kAct>, dim3(ctx->sm_count / 2 * 2), Cfg::kThreads, Cfg::kSmem, st,
                                    a0, b0, a1, b1, slot_row_off, slot_expert, s.S, s.E, n_dim, k_dim, (int)moegps_rcap_of(s),
                                    kept, act_out, static_cast<__nv_bfloat16*>(out), ctx->d_status));
  MOEGPS_AFTER_LAUNCH(ctx, "%s tile=%dx%d", kAct ? "act" : "input", 2 * BM, BNACC);
  return MOEGPS_OK;
}

enum class Tiles { kPair, k256, k128, k64 };

// The tiles for n_dim output columns: what needs the fewest rounds of tiles over the SMs, weighted with a round's time
// (relative to 128 x 256; measured cycles for a K block 690-860, 400, 330 and 600).  The slots' loads are on the device:
// the estimate is that of evenly loaded slots, whose last tile is half full, and which have one tile at least.  Measured,
// all four forced on 16 layers of 3 to 307 rows a slot, even and skewed loads: the choice is the fastest to 1 % in 55 of 64 launches and
// within 14 % of it in the others, the worst the act kernel on 777 x 1000, F 1416, 17 slots (42.5 us by pairs, 37.4 by 128).
Tiles choose_tiles(const moegps_ctx* ctx, int n_dim) {
  const moegps_shape_t& s = ctx->shape;
  const double R = (double)s.T * s.K, slots = s.S < R ? s.S : R;
  Tiles best = Tiles::k256;
  double least = 1e300;
  const struct { Tiles tiles; int rows, cols, sms; double time; } all[] = {
      {Tiles::k256, BM, 256, 1, 1.0}, {Tiles::k128, BM, 128, 1, 0.6}, {Tiles::k64, BM, 64, 1, 0.5}, {Tiles::kPair, 2 * BM, 256, 2, 0.85}};
  for (const auto& t : all) {
    const double of_a_slot = R / slots / t.rows + 0.5, row_tiles = slots * (of_a_slot > 1.0 ? of_a_slot : 1.0);
    const double rounds = row_tiles * ((n_dim + t.cols - 1) / t.cols) / (ctx->sm_count / t.sms);
    // (many rounds even out, a few do not)
    const double time = (rounds < 8 ? (double)(int64_t)(rounds + 0.999) : rounds) * t.time;
    if (time < least) {
      least = time;
      best = t.tiles;
    }
  }
  return best;
}

template <bool kAct, typename... Args>
int launch_data_gradient_any(moegps_ctx* ctx, int n_dim, Args... args) {
  switch (choose_tiles(ctx, n_dim)) {
    case Tiles::kPair: return launch_data_gradient_pair<kAct>(ctx, args...);
    case Tiles::k256: return launch_data_gradient<kAct, 256>(ctx, args...);
    case Tiles::k128: return launch_data_gradient<kAct, 128>(ctx, args...);
    default: return launch_data_gradient<kAct, 64>(ctx, args...);
  }
}

}  // namespace

int moegps_launch_ffn_backward_act(moegps_ctx* ctx, const void* dyp, const int32_t* slot_row_off, const int32_t* slot_expert,
                                   const void* w_down, const void* gate8, const void* up8, const void* gate_scale,
                                   const void* up_scale, void* dgate, void* dup, void* h_ws, cudaStream_t st) {
  const moegps_shape_t& s = ctx->shape;
  CUtensorMap a, b;
  if (!(moegps_make_tmap_2d(&a, dyp, (uint64_t)moegps_rcap_of(s), s.D, BM, BK) &&
        moegps_make_tmap_3d(&b, w_down, s.E, s.D, s.F, BK, 64)))
    return tmap_failed(ctx);
  const KeptActs kept = {static_cast<const uint8_t*>(gate8), static_cast<const uint8_t*>(up8),
                         static_cast<const uint8_t*>(gate_scale), static_cast<const uint8_t*>(up_scale)};
  const ActOutputs out = {static_cast<__nv_bfloat16*>(dgate), static_cast<__nv_bfloat16*>(dup),
                          static_cast<__nv_bfloat16*>(h_ws)};
  return launch_data_gradient_any<true>(ctx, s.F, a, b, a, b, slot_row_off, slot_expert, s.F, s.D, kept, out, nullptr, st);
}

int moegps_launch_ffn_backward_input(moegps_ctx* ctx, const void* dgate, const void* dup, const int32_t* slot_row_off,
                                     const int32_t* slot_expert, const void* w_gate, const void* w_up, void* dxp,
                                     cudaStream_t st) {
  const moegps_shape_t& s = ctx->shape;
  const uint64_t rcap = (uint64_t)moegps_rcap_of(s);
  CUtensorMap a0, b0, a1, b1;
  if (!(moegps_make_tmap_2d(&a0, dgate, rcap, s.F, BM, BK) && moegps_make_tmap_2d(&a1, dup, rcap, s.F, BM, BK) &&
        moegps_make_tmap_3d(&b0, w_gate, s.E, s.F, s.D, BK, 64) && moegps_make_tmap_3d(&b1, w_up, s.E, s.F, s.D, BK, 64)))
    return tmap_failed(ctx);
  return launch_data_gradient_any<false>(ctx, s.D, a0, b0, a1, b1, slot_row_off, slot_expert, s.D, s.F, KeptActs{},
                                         ActOutputs{}, dxp, st);
}

int moegps_launch_ffn_backward_weights(moegps_ctx* ctx, const void* dyp, const void* xp, const void* dgate, const void* dup,
                                       const void* h_ws, const int32_t* slot_row_off, const int32_t* slot_off,
                                       const int32_t* row_pair, void* dw_gate, void* dw_up, void* dw_down, cudaStream_t st) {
  const moegps_shape_t& s = ctx->shape;
  const uint64_t rcap = (uint64_t)moegps_rcap_of(s);
  CUtensorMap t_dgate, t_dup, t_dyp, t_xp, t_h, o_gate, o_up, o_down;
  if (!(moegps_make_tmap_2d(&t_dgate, dgate, rcap, s.F, BK, 64) && moegps_make_tmap_2d(&t_dup, dup, rcap, s.F, BK, 64) &&
        moegps_make_tmap_2d(&t_dyp, dyp, rcap, s.D, BK, 64) && moegps_make_tmap_2d(&t_xp, xp, rcap, s.D, BK, 64) &&
        moegps_make_tmap_2d(&t_h, h_ws, rcap, s.F, BK, 64) && moegps_make_tmap_store(&o_gate, dw_gate, s.E, s.F, s.D) &&
        moegps_make_tmap_store(&o_up, dw_up, s.E, s.F, s.D) && moegps_make_tmap_store(&o_down, dw_down, s.E, s.D, s.F)))
    return tmap_failed(ctx);
  constexpr size_t smem = WeightCfg::kSmem;
  if (!ctx->weight_gradient_attr_done) {
    MOEGPS_CUDA_TRY(ctx, cudaFuncSetAttribute(weight_gradient_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    ctx->weight_gradient_attr_done = true;
  }
  MOEGPS_CUDA_TRY(ctx, launch_after(weight_gradient_kernel, dim3(ctx->sm_count / 2 * 2), WeightCfg::kThreads, smem, st, t_dgate,
                                    t_dup, t_dyp, t_xp, t_h, o_gate, o_up, o_down, slot_row_off, slot_off, row_pair, s.S, s.E, s.F,
                                    s.D, s.row_align, (int)rcap, ctx->d_status));
  MOEGPS_AFTER_LAUNCH(ctx);
  return MOEGPS_OK;
}
