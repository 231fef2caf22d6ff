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
//   2. dlogit  : one thread per pair.  One more block lists the units of the next step.
//   3. partial : dlogit is sparse (K of E), so dWr is a weighted sum of rows rather than a matrix
//                product: the pairs of one expert are consecutive in the permuted order, and a unit is
//                up to kUnitRows of them.  Its rows of x are gathered through row_pair (x is read K
//                times, but from L2: it is the unpermuted tensor) and summed in fp32.
//   4. reduce  : the units of an expert are added in order.
// No atomics: the sums have a fixed order.  Each kernel is launched while the one before it drains (launch_after).
#include "bf16x8.cuh"
#include "common.cuh"
#include "route_backward.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kUnitRows = route_backward::kUnitRows;

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

template <bool kSigmoid>
__global__ void __launch_bounds__(kThreads)
dlogit_kernel(const float* __restrict__ logits, const int32_t* __restrict__ topk_idx, const float* __restrict__ topk_w, const float* __restrict__ dtopk_w,
              int64_t R, int K, int E, int S, int64_t Rcap, int max_units, const int32_t* __restrict__ slot_row_off,
              const int32_t* __restrict__ slot_off, float* __restrict__ dlogit, int32_t* __restrict__ unit_first,
              int4* __restrict__ units, int32_t* __restrict__ status) {
  launch_dependents();
  wait_for_predecessor();
  if (blockIdx.x == 0) {
    list_units(E, S, Rcap, max_units, slot_row_off, slot_off, unit_first, units, status);
    return;
  }
  const int64_t p = ((int64_t)blockIdx.x - 1) * kThreads + threadIdx.x;
  if (p >= R) return;
  const int64_t p0 = p / K * K;
  float m = 0.f;
  for (int j = 0; j < K; ++j) m = fmaf(topk_w[p0 + j], dtopk_w[p0 + j], m);
  float d = topk_w[p] * (dtopk_w[p] - m);
  if constexpr (kSigmoid) {
    const int e = topk_idx[p];
    const bool valid = e >= 0 && e < E;
    if (!valid) moegps_report(status, MOEGPS_ERR_BAD_INDEX, (int)(p / K));
    const float logit = valid ? logits[p / K * E + e] : 0.f;
    if (!valid) d = 0.f;
    d *= 1.f / (1.f + expf(logit));                   // 1 - sigmoid
  }
  dlogit[p] = d;
}

// block (u, c): columns [1024 c, 1024 c + 1024) of unit u; a thread sums eight columns over the unit's rows, eight rows
// in flight at a time.  An expert with one unit needs no second pass: its sums are the result.
constexpr int kPartThreads = 128;

__global__ void __launch_bounds__(kPartThreads)
partial_kernel(const uint4* __restrict__ x, const int32_t* __restrict__ row_pair, const float* __restrict__ dlogit, int64_t R,
               int K, int E, int D, const int32_t* __restrict__ unit_first, const int4* __restrict__ units,
               float* __restrict__ part, float* __restrict__ part_b, float* __restrict__ dw_router,
               int32_t* __restrict__ status) {
  static_assert(kUnitRows == 64, "two warps list the unit's rows");
  __shared__ float s_dl[kUnitRows];
  __shared__ int s_t[kUnitRows];
  __shared__ int s_n[2];
  launch_dependents();
  wait_for_predecessor();
  const int u = blockIdx.x;
  if (u >= unit_first[E]) return;
  const int4 unit = units[u];
  const int tid = threadIdx.x, lane = tid & 31;
  // the unit's tokens in order, without its padding rows
  int p = -1;
  unsigned have = 0;
  if (tid < kUnitRows) {
    if (unit.y + tid < unit.z) p = row_pair[unit.y + tid];
    if (p >= R) {
      moegps_report(status, MOEGPS_ERR_BAD_INDEX, unit.y + tid);
      p = -1;
    }
    have = __ballot_sync(0xffffffffu, p >= 0);
    if (lane == 0) s_n[tid >> 5] = __popc(have);
  }
  __syncthreads();
  const int n = s_n[0] + s_n[1];
  if (p >= 0) {
    const int at = (tid >= 32 ? s_n[0] : 0) + __popc(have & ((1u << lane) - 1));
    s_dl[at] = dlogit[p];
    s_t[at] = p / K;
  }
  __syncthreads();
  const int chunks = D / 8, c = blockIdx.y * kPartThreads + tid;
  if (blockIdx.y == 0 && tid == 0) {
    float b = 0.f;
    for (int r = 0; r < n; ++r) b += s_dl[r];
    part_b[u] = b;
  }
  if (c >= chunks) return;
  float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  const uint4* xc = x + c;
  int r = 0;
  for (; r + 8 <= n; r += 8) {
    uint4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = xc[(int64_t)s_t[r + i] * chunks];
#pragma unroll
    for (int i = 0; i < 8; ++i) fma8(acc, s_dl[r + i], v[i]);
  }
  for (; r < n; ++r) fma8(acc, s_dl[r], xc[(int64_t)s_t[r] * chunks]);
  const bool only = unit_first[unit.x + 1] - unit_first[unit.x] == 1;
  float4* o = reinterpret_cast<float4*>((only ? dw_router + (int64_t)unit.x * D : part + (int64_t)u * D) + 8 * c);
  o[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
  o[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
}

// The units of expert e are shared by W warps (each takes every W-th one, their sums are added in order), W growing with
// their number, and a block's other warps take further groups of 128 columns: block (e, y) adds columns
// [128 G y, 128 G y + 128 G), G = 8 / W.  The grid has room for G = 1; blocks beyond an expert's columns end at once.
__global__ void __launch_bounds__(kThreads)
reduce_kernel(const float* __restrict__ part, const float* __restrict__ part_b, int D,
              const int32_t* __restrict__ unit_first, float* __restrict__ dw_router, float* __restrict__ dbias) {
  __shared__ float4 s_acc[kWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  launch_dependents();
  wait_for_predecessor();
  const int e = blockIdx.x;
  const int first = unit_first[e], last = unit_first[e + 1], n = last - first;
  const int W = n <= 4 ? 1 : n <= 8 ? 2 : n <= 16 ? 4 : 8;
  const int group = blockIdx.y * (kWarps / W) + warp / W, col = 128 * group + 4 * lane;
  if (blockIdx.y * (kWarps / W) * 128 >= D || (n == 1 && blockIdx.y > 0)) return;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  if (col < D && n != 1) {
#pragma unroll 8
    for (int u = first + warp % W; u < last; u += W) {
      const float4 v = *reinterpret_cast<const float4*>(part + (int64_t)u * D + col);
      a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w;
    }
  }
  s_acc[warp][lane] = a;
  __syncthreads();
  if (warp % W == 0 && col < D && n != 1) {        // (one unit: partial_kernel has stored the result)
    for (int v = 1; v < W; ++v) {
      const float4 b = s_acc[warp + v][lane];
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
  const int64_t Rcap = moegps_rcap_of(s), R = (int64_t)s.T * s.K;
  const int max_units = (int)route_backward::max_units(s);
  const route_backward::Workspace ws = route_backward::carve(s, workspace);
  if (s.gate_mode == 1)
    if (int rc = moegps_launch_route(ctx, x, w_router, bias, nullptr, nullptr, ws.logits, nullptr, nullptr, st)) return rc;
  MOEGPS_CUDA_TRY(ctx, launch_after(s.gate_mode == 1 ? dlogit_kernel<true> : dlogit_kernel<false>,
                                    dim3(1 + (unsigned)((R + kThreads - 1) / kThreads)), kThreads, 0, st, ws.logits, topk_idx,
                                    topk_w, dtopk_w, R, s.K, s.E, s.S, Rcap, max_units, slot_row_off, slot_off, dlogit,
                                    ws.unit_first, ws.units, ctx->d_status));
  MOEGPS_AFTER_LAUNCH(ctx);
  MOEGPS_CUDA_TRY(ctx, launch_after(partial_kernel, dim3(max_units, (s.D / 8 + kPartThreads - 1) / kPartThreads), kPartThreads, 0,
                                    st, static_cast<const uint4*>(x), row_pair, dlogit, R, s.K, s.E, s.D, ws.unit_first,
                                    ws.units, ws.part, ws.part_b, dw_router, ctx->d_status));
  MOEGPS_AFTER_LAUNCH(ctx);
  MOEGPS_CUDA_TRY(ctx, launch_after(reduce_kernel, dim3(s.E, (s.D + 127) / 128), kThreads, 0, st, ws.part, ws.part_b, s.D,
                                    ws.unit_first, dw_router, dbias));
  MOEGPS_AFTER_LAUNCH(ctx);
  return MOEGPS_OK;
}
