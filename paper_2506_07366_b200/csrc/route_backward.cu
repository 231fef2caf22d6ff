// Gradient of the router.  With m[t] = sum_i w[t,i] dw[t,i] over the K selected experts,
//   softmax over the selection:       dl[t,j] = w[t,j] (dw[t,j] - m[t])
//   sigmoid, then renormalised:       dl[t,j] = w[t,j] (1 - s[t,j]) (dw[t,j] - m[t]),  s = sigmoid(<x[t], Wr[e]> + b[e])
// (the logits that were not selected get no gradient), and
//   dWr[e] = sum over the pairs of e of dl x[t],   db[e] = sum over the pairs of e of dl.
//
// Three kernels:
//   1. dlogit  : one warp per token.  The forward pass keeps the weights, not the scores, so the sigmoid
//                form recomputes the K selected logits (Wr stays in L2); softmax needs only w and dw.
//                One more block lists the units of the next step.
//   2. partial : dlogit is sparse (K of E), so dWr is a weighted sum of rows rather than a matrix
//                product: the pairs of one expert are consecutive in the permuted order, and a unit is
//                up to kUnitRows of them.  Its rows of x are gathered through row_pair (x is read K
//                times, but from L2: it is the unpermuted tensor) and summed in fp32.
//   3. reduce  : the units of an expert are added in order.
// No atomics: the sums have a fixed order.
#include "bf16x8.cuh"
#include "common.cuh"
#include "route_backward.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kUnitRows = route_backward::kUnitRows;
constexpr int kMaxE = 256;

// Lists the units: expert e owns rows slot_row_off[slot_off[e]] .. slot_row_off[slot_off[e+1]], cut into
// pieces of kUnitRows.  One block; thread e takes expert e (E <= 256).
__device__ void list_units(int E, int S, int64_t Rcap, int max_units, const int32_t* __restrict__ slot_row_off,
                           const int32_t* __restrict__ slot_off, int32_t* __restrict__ unit_first,
                           int4* __restrict__ units, int32_t* status) {
  __shared__ int32_t warp_tot[kWarps];
  const int e = threadIdx.x, lane = e & 31, warp = e >> 5;
  int lo = 0, hi = 0;
  if (e < E) {
    const int a = slot_off[e], b = slot_off[e + 1];
    if (a < 0 || b < a || b > S) {
      moegps_report(status, MOEGPS_ERR_BAD_INDEX, e);
    } else {
      lo = slot_row_off[a];
      hi = slot_row_off[b];
      if (lo < 0 || hi < lo || hi > Rcap) {
        moegps_report(status, MOEGPS_ERR_BAD_INDEX, e);
        lo = hi = 0;
      }
    }
  }
  const int n = (hi - lo + kUnitRows - 1) / kUnitRows;
  int incl = n;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int o = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += o;
  }
  if (lane == 31) warp_tot[warp] = incl;
  __syncthreads();
  int first = incl - n;
  for (int v = 0; v < warp; ++v) first += warp_tot[v];
  if (e < E) unit_first[e] = min(first, max_units);
  if (e == E - 1) unit_first[E] = min(first + n, max_units);
  // extents that overlap (a table no plan makes) could ask for more units than there is room for
  if (first + n > max_units) moegps_report(status, MOEGPS_ERR_BAD_INDEX, e);
  for (int i = 0; i < n && first + i < max_units; ++i)
    units[first + i] = make_int4(e, lo + i * kUnitRows, min(hi, lo + (i + 1) * kUnitRows), 0);
}

template <int KT, bool kSigmoid>
__global__ void __launch_bounds__(kThreads)
dlogit_kernel(const uint4* __restrict__ x, const uint4* __restrict__ w_router, const float* __restrict__ bias,
              const int32_t* __restrict__ topk_idx, const float* __restrict__ topk_w, const float* __restrict__ dtopk_w,
              int T, int E, int S, int chunks, int64_t Rcap, int max_units, const int32_t* __restrict__ slot_row_off,
              const int32_t* __restrict__ slot_off, float* __restrict__ dlogit, int32_t* __restrict__ unit_first,
              int4* __restrict__ units, int32_t* __restrict__ status) {
  if (blockIdx.x == 0) {
    list_units(E, S, Rcap, max_units, slot_row_off, slot_off, unit_first, units, status);
    return;
  }
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t t = ((int64_t)blockIdx.x - 1) * kWarps + warp;
  if (t >= T) return;
  float w[KT], dw[KT], m = 0.f;
#pragma unroll
  for (int j = 0; j < KT; ++j) {
    w[j] = topk_w[t * KT + j];
    dw[j] = dtopk_w[t * KT + j];
  }
#pragma unroll
  for (int j = 0; j < KT; ++j) m = fmaf(w[j], dw[j], m);
  float logit[KT];
#pragma unroll
  for (int j = 0; j < KT; ++j) logit[j] = 0.f;
  if constexpr (kSigmoid) {
    int expert[KT];
#pragma unroll
    for (int j = 0; j < KT; ++j) {
      expert[j] = topk_idx[t * KT + j];
      if (expert[j] < 0 || expert[j] >= E) {
        if (lane == 0) moegps_report(status, MOEGPS_ERR_BAD_INDEX, (int)t);
        expert[j] = 0;
        w[j] = 0.f;
      }
    }
    for (int c = lane; c < chunks; c += 32) {
      float xf[8];
      unpack8(xf, x[t * chunks + c]);
#pragma unroll
      for (int j = 0; j < KT; ++j) {
        float rf[8];
        unpack8(rf, w_router[(int64_t)expert[j] * chunks + c]);
#pragma unroll
        for (int i = 0; i < 8; ++i) logit[j] = fmaf(xf[i], rf[i], logit[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < KT; ++j) {
#pragma unroll
      for (int s = 16; s > 0; s >>= 1) logit[j] += __shfl_xor_sync(0xffffffffu, logit[j], s);
      if (bias) logit[j] += bias[expert[j]];
    }
  }
  if (lane == 0) {
#pragma unroll
    for (int j = 0; j < KT; ++j) {
      float d = w[j] * (dw[j] - m);
      if constexpr (kSigmoid) d *= 1.f / (1.f + expf(logit[j]));      // 1 - sigmoid
      dlogit[t * KT + j] = d;
    }
  }
}

// block (u, c): columns [2048 c, 2048 c + 2048) of unit u; a thread sums eight columns over the unit's rows
__global__ void __launch_bounds__(kThreads)
partial_kernel(const uint4* __restrict__ x, const int32_t* __restrict__ row_pair, const float* __restrict__ dlogit, int64_t R,
               int K, int E, int D, const int32_t* __restrict__ unit_first, const int4* __restrict__ units,
               float* __restrict__ part, float* __restrict__ part_b, int32_t* __restrict__ status) {
  __shared__ float s_dl[kUnitRows];
  __shared__ int s_t[kUnitRows];
  const int u = blockIdx.x;
  if (u >= unit_first[E]) return;
  const int4 unit = units[u];
  const int rows = unit.z - unit.y;
  const int tid = threadIdx.x;
  if (tid < kUnitRows) {
    float dl = 0.f;
    int t = -1;
    if (tid < rows) {
      const int p = row_pair[unit.y + tid];
      if (p >= 0 && p < R) {
        dl = dlogit[p];
        t = p / K;
      } else if (p >= R) {
        moegps_report(status, MOEGPS_ERR_BAD_INDEX, unit.y + tid);
      }
    }
    s_dl[tid] = dl;
    s_t[tid] = t;
  }
  __syncthreads();
  const int chunks = D / 8, c = blockIdx.y * kThreads + tid;
  if (blockIdx.y == 0 && tid == 0) {
    float b = 0.f;
    for (int r = 0; r < rows; ++r) b += s_dl[r];
    part_b[u] = b;
  }
  if (c >= chunks) return;
  float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll 8
  for (int r = 0; r < rows; ++r) {
    const int t = s_t[r];
    if (t >= 0) fma8(acc, s_dl[r], x[(int64_t)t * chunks + c]);
  }
  float4* o = reinterpret_cast<float4*>(part + (int64_t)u * D + 8 * c);
  o[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
  o[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
}

// block (e, c): columns [128 c, 128 c + 128) of expert e; warp v adds units v, v + 8, ..., then the warps are added
__global__ void __launch_bounds__(kThreads)
reduce_kernel(const float* __restrict__ part, const float* __restrict__ part_b, int D,
              const int32_t* __restrict__ unit_first, float* __restrict__ dw_router, float* __restrict__ dbias) {
  __shared__ float4 s_acc[kWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int e = blockIdx.x, col = (blockIdx.y * 32 + lane) * 4;
  const int first = unit_first[e], last = unit_first[e + 1];
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  if (col < D) {
#pragma unroll 4
    for (int u = first + warp; u < last; u += kWarps) {
      const float4 v = *reinterpret_cast<const float4*>(part + (int64_t)u * D + col);
      a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w;
    }
  }
  s_acc[warp][lane] = a;
  __syncthreads();
  if (warp == 0 && col < D) {
#pragma unroll
    for (int v = 1; v < kWarps; ++v) {
      const float4 b = s_acc[v][lane];
      a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w;
    }
    *reinterpret_cast<float4*>(dw_router + (int64_t)e * D + col) = a;
  }
  if (warp == 1 && blockIdx.y == 0) {
    float b = 0.f;
    for (int u = first + lane; u < last; u += 32) b += part_b[u];
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) b += __shfl_xor_sync(0xffffffffu, b, s);
    if (lane == 0) dbias[e] = b;
  }
}

}  // namespace

int moegps_launch_route_backward(moegps_ctx* ctx, const void* x, const void* w_router, const float* bias,
                                 const int32_t* topk_idx, const float* topk_w, const float* dtopk_w,
                                 const int32_t* slot_row_off, const int32_t* slot_off, const int32_t* row_pair,
                                 float* dlogit, float* dw_router, float* dbias, void* workspace, cudaStream_t st) {
  const moegps_shape_t& s = ctx->shape;
  const int chunks = s.D / 8;
  const int64_t Rcap = moegps_rcap_of(s), R = (int64_t)s.T * s.K;
  const int max_units = (int)route_backward::max_units(s);
  const route_backward::Workspace ws = route_backward::carve(s, workspace);
  const uint4 *xv = static_cast<const uint4*>(x), *rv = static_cast<const uint4*>(w_router);
  const int blocks = 1 + (s.T + kWarps - 1) / kWarps;
#define MOEGPS_LAUNCH(KT, G)                                                                                             \
  dlogit_kernel<KT, G><<<blocks, kThreads, 0, st>>>(xv, rv, bias, topk_idx, topk_w, dtopk_w, s.T, s.E, s.S, chunks, Rcap, \
                                                    max_units, slot_row_off, slot_off, dlogit, ws.unit_first, ws.units,  \
                                                    ctx->d_status)
#define MOEGPS_CASE(KT)                                                     \
  case KT:                                                                  \
    if (s.gate_mode == 1) MOEGPS_LAUNCH(KT, true); else MOEGPS_LAUNCH(KT, false); \
    break;
  switch (s.K) {
    MOEGPS_CASE(1) MOEGPS_CASE(2) MOEGPS_CASE(3) MOEGPS_CASE(4)
    MOEGPS_CASE(5) MOEGPS_CASE(6) MOEGPS_CASE(7) MOEGPS_CASE(8)
    default: return MOEGPS_ERR_UNSUPPORTED_SHAPE;
  }
#undef MOEGPS_CASE
#undef MOEGPS_LAUNCH
  MOEGPS_AFTER_LAUNCH(ctx);
  partial_kernel<<<dim3(max_units, (chunks + kThreads - 1) / kThreads), kThreads, 0, st>>>(
      xv, row_pair, dlogit, R, s.K, s.E, s.D, ws.unit_first, ws.units, ws.part, ws.part_b, ctx->d_status);
  MOEGPS_AFTER_LAUNCH(ctx);
  reduce_kernel<<<dim3(s.E, (s.D + 127) / 128), kThreads, 0, st>>>(ws.part, ws.part_b, s.D, ws.unit_first, dw_router, dbias);
  MOEGPS_AFTER_LAUNCH(ctx);
  return MOEGPS_OK;
}
