// Gradient of the router.  With m[t] = sum_i w[t,i] dw[t,i] over the K selected experts,
//   softmax over the selection:       dl[t,j] = w[t,j] (dw[t,j] - m[t])
//   sigmoid, then renormalised:       dl[t,j] = w[t,j] (1 - s[t,j]) (dw[t,j] - m[t]),  s = sigmoid(<x[t], Wr[e]> + b[e])
// (the logits that were not selected get no gradient), and
//   dWr[e] = sum over the pairs of e of dl x[t],   db[e] = sum over the pairs of e of dl.
//
// Kernels:
//   1. logits  : (sigmoid form only) the forward pass keeps the weights, not the scores, so the router's own GEMM gives the
//                logits again (route.cu), bit for bit those that the selection was made on.  Its tensor-core sums cost
//                26 us on 4096 tokens x 7168 and 256 experts; 8 dot products for each token on the CUDA cores took 83 us
//                with Wr from L2, and 40 + 6 us with slices of it in shared memory.
//   2. dlogit  : one thread per pair.
//   3. weights : dWr = dl^T x on the tensor cores, dl as a dense [tokens x experts] matrix that exists only in shared
//                memory, tile by tile.  A dl is split into three bf16 (8 + 8 + 8 bits: all of its 24), so the products are
//                exact and the sums are fp32: three MMAs for one, but x is read once for each 128 experts.  An accumulation
//                on the tensor core truncates, so its error grows with their number: the small second and third parts have
//                a sum of their own, and no sum runs over more than 1024 tokens.  Measured against 64 bits, of the norm:
//                8.1e-7 on 8192 tokens and 64 experts, 9.1e-7 on 4096 tokens and 256, 7.8e-7 on 16384 tokens and 8 (a
//                32-bit library product of the same dl: 4.6e-7, 1.2e-6, 4.5e-7); with sums over 2048 tokens 1.4e-6 to 1.8e-6.
//                Summing each expert's rows of x instead, gathered K times from L2, ran at L2's rate (10 TB/s) and took
//                21 us + 8 us for joining the parts on 8192 tokens x 2048, 6 of 64 experts, and 41 + 12 us on 4096 x 7168,
//                8 of 256.
//   4. reduce  : adds the parts of the tokens.  In the dense product a token that did not choose an expert adds 0 x, which
//                is NaN where x is not finite: a sum that is not finite is therefore computed again from the expert's own
//                pairs alone (they are consecutive in the permuted order), and is what the definition gives.
// No atomics: the sums have a fixed order.  Each kernel is launched while the one before it drains (launch_after).
#include "common.cuh"
#include "grouped_gemm.cuh"
#include "route_backward.cuh"

namespace {

using namespace sm100;
using route_backward::kTileD;
using route_backward::kTileE;
using route_backward::kTileT;

constexpr int kThreads = 256;
static_assert(kTileE >= 128, "at most 256 experts are one or two tiles");

template <bool kSigmoid>
__global__ void __launch_bounds__(kThreads)
dlogit_kernel(const float* __restrict__ logits, const int32_t* __restrict__ topk_idx, const float* __restrict__ topk_w,
              const float* __restrict__ dtopk_w, int64_t R, int K, int E, float* __restrict__ dlogit,
              int32_t* __restrict__ status) {
  launch_dependents();
  wait_for_predecessor();
  const int64_t p = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (p >= R) return;
  const int64_t p0 = p / K * K;
  const int e = kSigmoid || topk_idx ? topk_idx[p] : 0;
  const bool valid = e >= 0 && e < E;
  const float logit = kSigmoid && valid ? logits[p / K * E + e] : 0.f;
  float m = 0.f;
  for (int j = 0; j < K; ++j) m = fmaf(topk_w[p0 + j], dtopk_w[p0 + j], m);
  float d = topk_w[p] * (dtopk_w[p] - m);
  if constexpr (kSigmoid) d *= 1.f / (1.f + expf(logit));            // 1 - sigmoid
  if (!valid) {
    moegps_report(status, MOEGPS_ERR_BAD_INDEX, (int)(p / K));
    d = 0.f;
  }
  dlogit[p] = d;
}

// ------------------------------------------------------------------------------------------------ dWr
struct RouterCfg {
  static constexpr int kBoxBytes = 64 * kTileT * 2;                  // 64 contiguous elements x 64 tokens
  static constexpr int kSplitBytes = kTileE * kTileT * 2;            // one of the three parts of a dl tile
  static constexpr int kABytes = 3 * kSplitBytes, kAStages = 2;      // built in shared memory
  static constexpr int kBBytes = kTileD / 64 * kBoxBytes, kBStages = 3;
  static constexpr int kBuilders = 4, kThreads = 32 * (2 + kBuilders), kPairs = kTileT * 8 / (32 * kBuilders);
  static constexpr size_t kSmem = 1024 + kAStages * kABytes + kBStages * kBBytes + 256;
};
static_assert(RouterCfg::kSmem <= 227 * 1024, "fits an SM");

// Byte offset of (token k, expert m) in an MN-major tile with the 128-byte swizzle: see smem_desc_mn.
__device__ __forceinline__ uint32_t dl_offset(int k, int m) {
  return (uint32_t)((m >> 6) * RouterCfg::kBoxBytes + k * 128 + ((((m >> 3) & 7) ^ (k & 7)) << 4) + (m & 7) * 2);
}

// Block = split x tiles + tile, tile = column tile x expert tiles + expert tile: one grid dimension, since there may be more
// than 65535 splits.  Warp 0 loads x, warp 1 multiplies, warps 2..5 build the dl tiles and, at the end, store the sums.
__global__ void __launch_bounds__(RouterCfg::kThreads, 1)
router_weight_kernel(const __grid_constant__ CUtensorMap tm_x, const int32_t* __restrict__ pair_expert,
                     const float* __restrict__ dlogit, int T, int K, int E, int D, int cols, int tiles, int per,
                     float* __restrict__ part, int32_t* __restrict__ status) {
  using Cfg = RouterCfg;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* a_mem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* b_mem = a_mem + Cfg::kAStages * Cfg::kABytes;
  uint64_t* a_full = reinterpret_cast<uint64_t*>(b_mem + Cfg::kBStages * Cfg::kBBytes);
  uint64_t* a_empty = a_full + Cfg::kAStages;
  uint64_t* b_full = a_empty + Cfg::kAStages;
  uint64_t* b_empty = b_full + Cfg::kBStages;
  uint64_t* done = b_empty + Cfg::kBStages;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = uniform_warp_index(), lane = threadIdx.x & 31;
  const int split = blockIdx.x / tiles, tile = blockIdx.x - split * tiles;
  const int e_shift = E > kTileE, e0 = (tile & e_shift) * kTileE, d0 = (tile >> e_shift) * cols;      // (one expert tile or two)
  const int first = split * per, steps = min(per, (T + kTileT - 1) / kTileT - first);

  if (threadIdx.x == 0) {
    for (int i = 0; i < Cfg::kAStages; ++i) { mbar_init(&a_full[i], Cfg::kBuilders); mbar_init(&a_empty[i], 1); }
    for (int i = 0; i < Cfg::kBStages; ++i) { mbar_init(&b_full[i], 1); mbar_init(&b_empty[i], 1); }
    mbar_init(done, 1);
    *abort_flag = 0;
    fence_mbar_init();
    prefetch_tensormap(&tm_x);
  }
  if (warp == 1) {
    tmem_alloc(tmem_slot, 2 * kTileD);
    tmem_relinquish();
  }
  // the dl tiles are zero but for the entries of the present tokens
  for (int i = threadIdx.x; i < Cfg::kAStages * Cfg::kABytes / 16; i += Cfg::kThreads)
    reinterpret_cast<uint4*>(a_mem)[i] = make_uint4(0, 0, 0, 0);
  fence_proxy_async();
  launch_dependents();
  wait_for_predecessor();
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int i = 0; i < steps; ++i) {
        if (!mbar_wait(&b_empty[stage], phase ^ 1u, abort_flag)) { ok = false; break; }
        uint8_t* sb = b_mem + stage * Cfg::kBBytes;
        mbar_arrive_expect_tx(&b_full[stage], Cfg::kBBytes);
#pragma unroll
        for (int c = 0; c < kTileD / 64; ++c)
          tma_load_2d(sb + c * Cfg::kBoxBytes, &tm_x, &b_full[stage], d0 + 64 * c, (first + i) * kTileT);
        if (++stage == Cfg::kBStages) { stage = 0; phase ^= 1u; }
      }
      if (!ok)
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
    }
  } else if (warp == 1) {
    const uint32_t idesc = idesc_bf16_f32(kTileE, cols, true, true);
    const uint32_t a_ring = smem_u32(a_mem), b_ring = smem_u32(b_mem);
    int as = 0, bs = 0;
    uint32_t a_phase = 0, b_phase = 0;
    bool ok = true;
    for (int i = 0; i < steps; ++i) {
      if (!warp_wait(&b_full[bs], b_phase, abort_flag) || !warp_wait(&a_full[as], a_phase, abort_flag)) { ok = false; break; }
      tc_fence_after_sync();
      const uint64_t db = smem_desc_mn(b_ring + bs * Cfg::kBBytes, Cfg::kBoxBytes);
      const uint64_t da = smem_desc_mn(a_ring + as * Cfg::kABytes, Cfg::kBoxBytes);
      if (elect_one()) {
#pragma unroll
        for (int dl_part = 0; dl_part < 3; ++dl_part)
#pragma unroll
          for (int k = 0; k < kTileT / 16; ++k)            // the first part's sum, and the other two's
            mma_bf16(tmem_base + (dl_part ? kTileD : 0), da + (uint64_t)(dl_part * (Cfg::kSplitBytes >> 4) + k * 128),
                     db + (uint64_t)(k * 128), idesc, i != 0 || k != 0 || dl_part == 2);
        mma_commit(&a_empty[as]);
        mma_commit(&b_empty[bs]);
      }
      if (++as == Cfg::kAStages) { as = 0; a_phase ^= 1u; }
      if (++bs == Cfg::kBStages) { bs = 0; b_phase ^= 1u; }
    }
    if (ok && elect_one()) mma_commit(done);
    if (!ok)
      for (int i = 0; i < 1000; ++i) __nanosleep(1000);
  } else {
    const int builder = threadIdx.x - 64;
    // the entries that this thread has set in each stage; -1: none
    int set[Cfg::kAStages][Cfg::kPairs];
#pragma unroll
    for (int s = 0; s < Cfg::kAStages; ++s)
#pragma unroll
      for (int i = 0; i < Cfg::kPairs; ++i) set[s][i] = -1;
    // this thread's pairs of a step: q = builder + 128 n, of token q / K; the next step's are loaded while this one's wait
    // for their stage (all at once: one after the other, each behind the other's branch, they took longer than the MMAs)
    int token[Cfg::kPairs], next_e[Cfg::kPairs];
    float next_dl[Cfg::kPairs];
#pragma unroll
    for (int n = 0; n < Cfg::kPairs; ++n) token[n] = (builder + 32 * Cfg::kBuilders * n) / K;
    auto fetch = [&](int i) {
      const int64_t p0 = (int64_t)(first + i) * kTileT * K;
#pragma unroll
      for (int n = 0; n < Cfg::kPairs; ++n) {
        const int64_t p = p0 + builder + 32 * Cfg::kBuilders * n;
        const bool in = i < steps && token[n] < kTileT && p < (int64_t)T * K;
        next_e[n] = in ? pair_expert[p] : -1;
        next_dl[n] = in ? dlogit[p] : 0.f;
      }
    };
    fetch(0);
    uint32_t phase = 0;
    bool ok = true;
    for (int i0 = 0; i0 < steps; i0 += Cfg::kAStages, phase ^= 1u) {
#pragma unroll
      for (int as = 0; as < Cfg::kAStages; ++as) {
        const int i = i0 + as;
        if (i < steps) {
          int at[Cfg::kPairs];
          float dl[Cfg::kPairs];
#pragma unroll
          for (int n = 0; n < Cfg::kPairs; ++n) {
            const int m = next_e[n] - e0;
            at[n] = next_e[n] >= 0 && m >= 0 && m < kTileE ? (int)dl_offset(token[n], m) : -1;
            dl[n] = next_dl[n];
          }
          fetch(i + 1);
          ok = ok && warp_wait(&a_empty[as], phase ^ 1u, abort_flag);
          uint8_t* sa = a_mem + as * Cfg::kABytes;
#pragma unroll
          for (int n = 0; n < Cfg::kPairs; ++n)
            if (ok && set[as][n] >= 0)
#pragma unroll
              for (int dl_part = 0; dl_part < 3; ++dl_part)
                *reinterpret_cast<__nv_bfloat16*>(sa + dl_part * Cfg::kSplitBytes + set[as][n]) = __float2bfloat16(0.f);
          // no entry is set before all old ones are gone (a warp whose wait failed comes here too: the count stays right)
          asm volatile("bar.sync 1, %0;" ::"n"(32 * Cfg::kBuilders) : "memory");
#pragma unroll
          for (int n = 0; n < Cfg::kPairs; ++n) {
            set[as][n] = at[n];
            if (ok && at[n] >= 0) {
              float rest = dl[n];
#pragma unroll
              for (int dl_part = 0; dl_part < 3; ++dl_part) {
                const __nv_bfloat16 v = __float2bfloat16(rest);       // nearest; what is left is exact in fp32
                *reinterpret_cast<__nv_bfloat16*>(sa + dl_part * Cfg::kSplitBytes + at[n]) = v;
                rest -= __bfloat162float(v);
              }
            }
          }
          fence_proxy_async();
          __syncwarp();
          if (lane == 0) mbar_arrive(&a_full[as]);
        }
      }
    }
    // ---- the sums: a lane's row is an expert ----
    if (ok && mbar_wait(done, 0, abort_flag, 64)) {
      tc_fence_after_sync();
      const int quarter = warp & 3, e = e0 + quarter * 32 + lane;
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16);
      float* row = part + ((int64_t)split * E + e) * D + d0;
#pragma unroll 1
      for (int c = 0; c < cols; c += 32) {
        uint32_t v[32], w[32];
        tmem_ld32(taddr + c, v);
        tmem_ld32(taddr + kTileD + c, w);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) + __uint_as_float(w[i]));
        if (e < E) {
#pragma unroll
          for (int i = 0; i < 32; i += 8)
            if (c + i < cols && d0 + c + i < D)          // (both multiples of 8)
              asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(row + c + i), "r"(v[i]), "r"(v[i + 1]),
                           "r"(v[i + 2]), "r"(v[i + 3]), "r"(v[i + 4]), "r"(v[i + 5]), "r"(v[i + 6]), "r"(v[i + 7])
                           : "memory");
        }
      }
    }
  }

  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) moegps_report(status, MOEGPS_ERR_TIMEOUT, (int)blockIdx.x);
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem_base, 2 * kTileD);
  }
}

// Without topk_idx (the softmax form does not need it otherwise): the expert of every pair from the tables of the permutation.
__global__ void __launch_bounds__(kThreads)
pair_expert_kernel(const int32_t* __restrict__ slot_row_off, const int32_t* __restrict__ slot_off,
                   const int32_t* __restrict__ row_pair, int64_t R, int64_t Rcap, int S, int32_t* __restrict__ pair_expert,
                   int32_t* __restrict__ status) {
  const int e = blockIdx.x;
  const int a = slot_off[e], b = slot_off[e + 1];
  if (a < 0 || b < a || b > S) {
    if (threadIdx.x == 0) moegps_report(status, MOEGPS_ERR_BAD_INDEX, e);
    return;
  }
  const int lo = slot_row_off[a], hi = slot_row_off[b];
  if (lo < 0 || hi < lo || hi > Rcap) {
    if (threadIdx.x == 0) moegps_report(status, MOEGPS_ERR_BAD_INDEX, e);
    return;
  }
  for (int r = lo + threadIdx.x; r < hi; r += kThreads) {
    const int p = row_pair[r];
    if (p >= 0 && p < R) pair_expert[p] = e;
  }
}

// block (e, c): columns [1024 c, 1024 c + 1024) of expert e, four for each thread; the blocks behind the last columns add
// dbias, a thread's pairs 16 at a time (their indices, then their values, in two round trips to memory)
__global__ void __launch_bounds__(kThreads)
reduce_kernel(const float* __restrict__ part, int splits, const __nv_bfloat16* __restrict__ x, const float* __restrict__ dlogit,
              const int32_t* __restrict__ slot_row_off, const int32_t* __restrict__ slot_off,
              const int32_t* __restrict__ row_pair, int64_t R, int64_t Rcap, int K, int E, int S, int D,
              float* __restrict__ dw_router, float* __restrict__ dbias, int32_t* __restrict__ status) {
  __shared__ float s_sum[kThreads / 32];
  launch_dependents();
  wait_for_predecessor();
  const int e = blockIdx.x, tid = threadIdx.x, col = blockIdx.y * 1024 + 4 * tid;
  // the rows of the expert's pairs
  int lo = 0, hi = 0;
  {
    const int a = slot_off[e], b = slot_off[e + 1];
    bool valid = a >= 0 && b >= a && b <= S;
    if (valid) {
      lo = slot_row_off[a];
      hi = slot_row_off[b];
      valid = lo >= 0 && hi >= lo && hi <= Rcap;
    }
    if (!valid) {
      if (tid == 0) moegps_report(status, MOEGPS_ERR_BAD_INDEX, e);
      lo = hi = 0;
    }
  }
  if (col < D) {
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int s = 0; s < splits; ++s) {
      const float4 v = *reinterpret_cast<const float4*>(part + ((int64_t)s * E + e) * D + col);
      a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w;
    }
    if (!(isfinite(a.x) && isfinite(a.y) && isfinite(a.z) && isfinite(a.w))) {
      a = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int r = lo; r < hi; ++r) {
        const int p = row_pair[r];
        if (p < 0 || p >= R) continue;
        const uint2 v = *reinterpret_cast<const uint2*>(x + (int64_t)(p / K) * D + col);
        const float dl = dlogit[p];
        a.x = fmaf(dl, __uint_as_float(v.x << 16), a.x);
        a.y = fmaf(dl, __uint_as_float(v.x & 0xffff0000u), a.y);
        a.z = fmaf(dl, __uint_as_float(v.y << 16), a.z);
        a.w = fmaf(dl, __uint_as_float(v.y & 0xffff0000u), a.w);
      }
    }
    *reinterpret_cast<float4*>(dw_router + (int64_t)e * D + col) = a;
  }
  if (blockIdx.y == gridDim.y - 1) {
    float b = 0.f;
    bool bad = false;
    for (int r0 = lo + tid; r0 < hi; r0 += 16 * kThreads) {
      int p[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] = r0 + i * kThreads < hi ? row_pair[r0 + i * kThreads] : -1;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        bad |= p[i] >= R;
        b += p[i] >= 0 && p[i] < R ? dlogit[p[i]] : 0.f;
      }
    }
    if (bad) moegps_report(status, MOEGPS_ERR_BAD_INDEX, e);      // (inside the loop it would part the loads)
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) b += __shfl_xor_sync(0xffffffffu, b, s);
    if ((tid & 31) == 0) s_sum[tid >> 5] = b;
    __syncthreads();
    if (tid == 0) {
#pragma unroll
      for (int v = 1; v < kThreads / 32; ++v) b += s_sum[v];
      dbias[e] = b;
    }
  }
}

}  // namespace

int moegps_launch_route_backward(moegps_ctx* ctx, const void* x, const void* w_router, const float* bias,
                                 const int32_t* topk_idx, const float* topk_w, const float* dtopk_w,
                                 const int32_t* slot_row_off, const int32_t* slot_off, const int32_t* row_pair,
                                 float* dlogit, float* dw_router, float* dbias, void* workspace, cudaStream_t st) {
  using Cfg = RouterCfg;
  const moegps_shape_t& s = ctx->shape;
  const int64_t Rcap = moegps_rcap_of(s), R = (int64_t)s.T * s.K;
  const route_backward::Workspace ws = route_backward::carve(s, workspace);
  const route_backward::Cut cut = route_backward::cut_of(s);
  CUtensorMap tm_x;
  if (!moegps_make_tmap_2d(&tm_x, x, (uint64_t)s.T, (uint64_t)s.D, kTileT, 64)) {
    ctx->last_cuda_error = (int)cudaErrorInvalidValue;
    return MOEGPS_ERR_CUDA;
  }
  if (!ctx->router_weight_attr_done) {
    MOEGPS_CUDA_TRY(ctx, cudaFuncSetAttribute(router_weight_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg::kSmem));
    ctx->router_weight_attr_done = true;
  }
  const int32_t* pair_expert = topk_idx;
  if (!pair_expert) {                                   // the softmax form without topk_idx
    MOEGPS_CUDA_TRY(ctx, cudaMemsetAsync(ws.pair_expert, 0xff, (size_t)R * sizeof(int32_t), st));
    pair_expert_kernel<<<s.E, kThreads, 0, st>>>(slot_row_off, slot_off, row_pair, R, Rcap, s.S, ws.pair_expert, ctx->d_status);
    MOEGPS_AFTER_LAUNCH(ctx);
    pair_expert = ws.pair_expert;
  }
  if (s.gate_mode == 1)
    if (int rc = moegps_launch_route(ctx, x, w_router, bias, nullptr, nullptr, ws.logits, nullptr, nullptr, st)) return rc;
  MOEGPS_CUDA_TRY(ctx, launch_after(s.gate_mode == 1 ? dlogit_kernel<true> : dlogit_kernel<false>,
                                    dim3((unsigned)((R + kThreads - 1) / kThreads)), kThreads, 0, st, ws.logits, topk_idx, topk_w,
                                    dtopk_w, R, s.K, s.E, dlogit, ctx->d_status));
  MOEGPS_AFTER_LAUNCH(ctx);
  const int tiles = (s.E + kTileE - 1) / kTileE * ((s.D + cut.cols - 1) / cut.cols);
  MOEGPS_CUDA_TRY(ctx, launch_after(router_weight_kernel, dim3((unsigned)tiles * (unsigned)cut.splits),
                                    Cfg::kThreads, Cfg::kSmem, st, tm_x, pair_expert, dlogit, s.T, s.K, s.E, s.D, cut.cols, tiles, cut.per, ws.part, ctx->d_status));
  MOEGPS_AFTER_LAUNCH(ctx, "cols=%d parts=%d steps=%d", cut.cols, cut.splits, cut.per);
  MOEGPS_CUDA_TRY(ctx, launch_after(reduce_kernel, dim3(s.E, (s.D + 1023) / 1024 + 1), kThreads, 0, st, ws.part, cut.splits,
                                    static_cast<const __nv_bfloat16*>(x), dlogit, slot_row_off, slot_off, row_pair, R, Rcap,
                                    s.K, s.E, s.S, s.D, dw_router, dbias, ctx->d_status));
  MOEGPS_AFTER_LAUNCH(ctx);
  return MOEGPS_OK;
}
