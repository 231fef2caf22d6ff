// Gradients of the two row shuffles.
//
// combine:  out[t] = sum_j w[t,j] yp[row(t,j)]      =>  dyp[row(t,j)] = w[t,j] dout[t]
//                                                       dw[t,j] = <dout[t], yp[row(t,j)]>
// dispatch: xp[row(t,j)] = x[t]                     =>  dx[t] = sum_j dxp[row(t,j)]
//           and, where the router is trained, logit[t,e] = <x[t], Wr[e]> + b[e] adds sum_j dl[t,j] Wr[e(t,j)].
//
// Every row of the permuted buffers belongs to one token, so both are gathers by token: no atomics, sums
// in a fixed order, fp32 throughout with one rounding to bf16 at the store.  A team of W warps takes one
// token: its row of dout (or dx) is touched once and its K rows of the permuted buffers once each, which
// is the least that the formulas allow.
#include "bf16x8.cuh"
#include "common.cuh"

namespace {

constexpr int kWarpsPerBlock = 4;
constexpr int kThreads = kWarpsPerBlock * 32;
// Whether a token is spread over the block's four warps: for wide rows, and for few tokens, whose blocks all run at once
// and only the length of one counts.  Measured, us a call in a graph, four warps / one:
//                                   combine        dispatch       dispatch with the router's part
//     256 tokens x  512, K 2      1.7 /   1.9    1.4 /   1.7      1.8 /   2.1
//    1200        x 1024, K 4      4.2 /   5.4    2.5 /   2.6      4.2 /   4.5
//    4096        x 1024, K 4     16.5 /  15.6    5.8 /   6.1     11.4 /  10.5
//    8192        x 1024, K 2     16.1 /  15.7    9.6 /   7.8     13.5 /  11.2
//    8192        x 1024, K 4     30.7 /  27.0   14.2 /  15.8     31.5 /  22.6
//    4096        x 1536, K 2     12.6 /  11.9    4.9 /   6.5      7.2 /   7.0
//    8192        x 1536, K 8     75.2 /  68.1   42.6 /  37.4     75.1 /  50.3
//    8192        x 2048, K 6     67.1 /  68.4   37.8 /  38.2     55.8 /  48.7
//    4096        x 3584, K 4     41.8 /  45.9   23.7 /  24.8     36.1 /  41.0
//    4096        x 7168, K 8    152.8 / 159.8   81.4 /  91.7    117.1 / 131.0    (floors 153, 81, 82)
bool is_wide(const moegps_ctx* ctx, int least_width) {
  return ctx->shape.D >= least_width || ctx->shape.T <= 8 * ctx->sm_count;
}
constexpr int kCombineWidth = 2048, kRouterWidth = 2056;      // (widths are multiples of 8: wider than 2048)
int dispatch_width(int K) { return K > 4 ? 2048 : K > 2 ? 1024 : 1536; }

// The rows of token t's pairs; one outside the buffer is reported and becomes -1.
template <int KT>
__device__ __forceinline__ void load_rows(int (&row)[KT], const int32_t* __restrict__ pair_row, int64_t t, int64_t Rcap,
                                          bool reporter, int32_t* status) {
#pragma unroll
  for (int j = 0; j < KT; ++j) row[j] = pair_row[t * KT + j];
#pragma unroll
  for (int j = 0; j < KT; ++j)
    if (row[j] < 0 || row[j] >= Rcap) {
      if (reporter) moegps_report(status, MOEGPS_ERR_BAD_INDEX, (int)t);
      row[j] = -1;
    }
}

template <int KT, int W>
__global__ void __launch_bounds__(kThreads)
combine_backward_kernel(const uint4* __restrict__ dout, const uint4* __restrict__ yp, const int32_t* __restrict__ pair_row,
                        const float* __restrict__ topk_w, int T, int chunks, int64_t Rcap, uint4* __restrict__ dyp,
                        float* __restrict__ dtopk_w, int32_t* __restrict__ status) {
  constexpr int kTeam = 32 * W;
  __shared__ float part[kWarpsPerBlock][KT];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = threadIdx.x % kTeam;
  const int64_t t = (int64_t)blockIdx.x * (kWarpsPerBlock / W) + warp / W;
  const bool active = t < T;
  launch_dependents();
  wait_for_predecessor();
  float dot[KT];
#pragma unroll
  for (int j = 0; j < KT; ++j) dot[j] = 0.f;
  if (active) {
    int row[KT];
    float w[KT];
    load_rows<KT>(row, pair_row, t, Rcap, l == 0, status);
#pragma unroll
    for (int j = 0; j < KT; ++j) w[j] = topk_w[t * KT + j];
    const uint4* d = dout + t * chunks;
#pragma unroll 2
    for (int c = l; c < chunks; c += kTeam) {
      const uint4 dv = d[c];
      uint4 y[KT];
#pragma unroll
      for (int j = 0; j < KT; ++j) y[j] = row[j] >= 0 ? yp[(int64_t)row[j] * chunks + c] : make_uint4(0, 0, 0, 0);
      float df[8];
      unpack8(df, dv);
#pragma unroll
      for (int j = 0; j < KT; ++j) {
        float yf[8], o[8];
        unpack8(yf, y[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          dot[j] = fmaf(df[i], yf[i], dot[j]);
          o[i] = w[j] * df[i];
        }
        if (row[j] >= 0) dyp[(int64_t)row[j] * chunks + c] = pack8(o);
      }
    }
#pragma unroll
    for (int j = 0; j < KT; ++j)
      if (row[j] < 0) dot[j] = 0.f;                    // (the sum of 0 dout is not 0 where dout is not finite)
  }
#pragma unroll
  for (int j = 0; j < KT; ++j) {
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) dot[j] += __shfl_xor_sync(0xffffffffu, dot[j], s);
  }
  if constexpr (W == 1) {
    if (active && lane == 0)
#pragma unroll
      for (int j = 0; j < KT; ++j) dtopk_w[t * KT + j] = dot[j];
  } else {
    if (lane == 0)
#pragma unroll
      for (int j = 0; j < KT; ++j) part[warp][j] = dot[j];
    __syncthreads();
    if (active && l < KT) {
      float s = 0.f;
#pragma unroll
      for (int v = 0; v < W; ++v) s += part[warp / W * W + v][l];
      dtopk_w[t * KT + l] = s;
    }
  }
}

template <int KT, int W, bool kRouter>
__global__ void __launch_bounds__(kThreads)
dispatch_backward_kernel(const uint4* __restrict__ dxp, const int32_t* __restrict__ pair_row,
                         const int32_t* __restrict__ topk_idx, const float* __restrict__ dlogit,
                         const uint4* __restrict__ w_router, int T, int E, int chunks, int64_t Rcap,
                         uint4* __restrict__ dx, int32_t* __restrict__ status) {
  constexpr int kTeam = 32 * W;
  const int warp = threadIdx.x >> 5, l = threadIdx.x % kTeam;
  const int64_t t = (int64_t)blockIdx.x * (kWarpsPerBlock / W) + warp / W;
  if (t >= T) return;
  launch_dependents();
  wait_for_predecessor();
  int row[KT], expert[KT];
  float dl[KT];
  load_rows<KT>(row, pair_row, t, Rcap, l == 0, status);
  if constexpr (kRouter) {
#pragma unroll
    for (int j = 0; j < KT; ++j) {
      expert[j] = topk_idx[t * KT + j];
      dl[j] = dlogit[t * KT + j];
    }
#pragma unroll
    for (int j = 0; j < KT; ++j)
      if (expert[j] < 0 || expert[j] >= E) {
        if (l == 0) moegps_report(status, MOEGPS_ERR_BAD_INDEX, (int)t);
        expert[j] = -1;
      }
  }
#pragma unroll 2
  for (int c = l; c < chunks; c += kTeam) {
    uint4 v[KT], r[KT];
#pragma unroll
    for (int j = 0; j < KT; ++j) {
      v[j] = row[j] >= 0 ? dxp[(int64_t)row[j] * chunks + c] : make_uint4(0, 0, 0, 0);
      if constexpr (kRouter) r[j] = expert[j] >= 0 ? w_router[(int64_t)expert[j] * chunks + c] : make_uint4(0, 0, 0, 0);
    }
    float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < KT; ++j) {
      fma8(acc, 1.f, v[j]);
      if constexpr (kRouter)
        if (expert[j] >= 0) fma8(acc, dl[j], r[j]);    // (not the product with a row read as zero: dl may be infinite)
    }
    dx[t * chunks + c] = pack8(acc);
  }
}

}  // namespace

#define MOEGPS_FOR_K(K, CASE) \
  switch (K) {                \
    CASE(1) CASE(2) CASE(3) CASE(4) CASE(5) CASE(6) CASE(7) CASE(8) default : return MOEGPS_ERR_UNSUPPORTED_SHAPE; \
  }

int moegps_launch_combine_backward(moegps_ctx* ctx, const void* dout, const void* yp, const int32_t* pair_row,
                                   const float* topk_w, void* dyp, float* dtopk_w, cudaStream_t st) {
  const moegps_shape_t& s = ctx->shape;
  const int chunks = s.D / 8;
  const int64_t Rcap = moegps_rcap_of(s);
  const uint4 *d = static_cast<const uint4*>(dout), *y = static_cast<const uint4*>(yp);
  uint4* o = static_cast<uint4*>(dyp);
  const bool wide = is_wide(ctx, kCombineWidth);
  const int per = wide ? 1 : kWarpsPerBlock;
  const int blocks = (s.T + per - 1) / per;
#define MOEGPS_LAUNCH(KT, W)                                                                                               \
  MOEGPS_CUDA_TRY(ctx, launch_after(combine_backward_kernel<KT, W>, dim3(blocks), kThreads, 0, st, d, y, pair_row, topk_w, s.T, \
                                    chunks, Rcap, o, dtopk_w, ctx->d_status))
#define MOEGPS_CASE(KT)                                                        \
  case KT:                                                                     \
    if (wide) MOEGPS_LAUNCH(KT, kWarpsPerBlock); else MOEGPS_LAUNCH(KT, 1);    \
    break;
  MOEGPS_FOR_K(s.K, MOEGPS_CASE)
#undef MOEGPS_LAUNCH
#undef MOEGPS_CASE
  MOEGPS_AFTER_LAUNCH(ctx, "warps=%d", wide ? kWarpsPerBlock : 1);
  return MOEGPS_OK;
}

int moegps_launch_dispatch_backward(moegps_ctx* ctx, const void* dxp, const int32_t* pair_row, const int32_t* topk_idx,
                                    const float* dlogit, const void* w_router, void* dx, cudaStream_t st) {
  const moegps_shape_t& s = ctx->shape;
  const int chunks = s.D / 8;
  const int64_t Rcap = moegps_rcap_of(s);
  const uint4 *v = static_cast<const uint4*>(dxp), *r = static_cast<const uint4*>(w_router);
  uint4* o = static_cast<uint4*>(dx);
  const bool wide = is_wide(ctx, dlogit ? kRouterWidth : dispatch_width(s.K));
  const int per = wide ? 1 : kWarpsPerBlock;
  const int blocks = (s.T + per - 1) / per;
#define MOEGPS_LAUNCH(KT, W, R)                                                                                          \
  MOEGPS_CUDA_TRY(ctx, launch_after(dispatch_backward_kernel<KT, W, R>, dim3(blocks), kThreads, 0, st, v, pair_row, topk_idx, \
                                    dlogit, r, s.T, s.E, chunks, Rcap, o, ctx->d_status))
#define MOEGPS_CASE(KT)                                                                                  \
  case KT:                                                                                               \
    if (dlogit) {                                                                                        \
      if (wide) MOEGPS_LAUNCH(KT, kWarpsPerBlock, true); else MOEGPS_LAUNCH(KT, 1, true);                \
    } else {                                                                                             \
      if (wide) MOEGPS_LAUNCH(KT, kWarpsPerBlock, false); else MOEGPS_LAUNCH(KT, 1, false);              \
    }                                                                                                    \
    break;
  MOEGPS_FOR_K(s.K, MOEGPS_CASE)
#undef MOEGPS_CASE
#undef MOEGPS_LAUNCH
  MOEGPS_AFTER_LAUNCH(ctx, "warps=%d", wide ? kWarpsPerBlock : 1);
  return MOEGPS_OK;
}
