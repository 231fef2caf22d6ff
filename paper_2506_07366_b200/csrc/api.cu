// C entry points of libmoegps: context management and host-side argument validation.
// Every step validates its arguments here and launches nothing when they are wrong.
#include <new>

#include <stdlib.h>

#include "common.cuh"
#include "mx4.cuh"
#include "route_backward.cuh"

namespace {

int check_shape(const moegps_shape_t* s) {
  if (!s) return MOEGPS_ERR_INVALID_ARG;
  if (s->T < 0 || s->D <= 0 || s->F <= 0 || s->E <= 0 || s->K <= 0 || s->S <= 0) return MOEGPS_ERR_UNSUPPORTED_SHAPE;
  if (s->K > s->E || s->K > 8 || s->E > 256 || s->S < s->E || s->S > 1024) return MOEGPS_ERR_UNSUPPORTED_SHAPE;
  if ((s->D % 8) != 0 || (s->F % 8) != 0) return MOEGPS_ERR_UNSUPPORTED_SHAPE;
  const int a = s->row_align;
  if (a < 1 || a > 256 || (a & (a - 1)) != 0) return MOEGPS_ERR_UNSUPPORTED_SHAPE;
  if (s->gate_mode != 0 && s->gate_mode != 1) return MOEGPS_ERR_INVALID_ARG;
  if (s->c_max < 0) return MOEGPS_ERR_INVALID_ARG;
  if (moegps_rcap_of(*s) > (int64_t)INT32_MAX - 255) return MOEGPS_ERR_UNSUPPORTED_SHAPE;   // a tile of 256 rows from the last row on
  return MOEGPS_OK;
}

template <typename... P>
bool all_ok(P... ptrs) {
  const void* a[] = {static_cast<const void*>(ptrs)...};
  for (const void* p : a)
    if (p == nullptr || !moegps_aligned16(p)) return false;
  return true;
}

bool aligned32(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 31u) == 0; }

// 4-bit weights: a launch has one block for each tile of a matrix's chunk
bool tiles4_fit(const moegps_shape_t& s) {
  return (int64_t)s.E * mx4::tiles_of(s.F) * mx4::chunks_of(s.D) <= INT32_MAX &&
         (int64_t)s.E * mx4::tiles_of(s.D) * mx4::chunks_of(s.F) <= INT32_MAX;
}

}  // namespace

extern "C" {

int moegps_create(moegps_ctx_t** out, const moegps_shape_t* shape, int device) {
  if (!out) return MOEGPS_ERR_INVALID_ARG;
  *out = nullptr;
  int rc = check_shape(shape);
  if (rc != MOEGPS_OK) return rc;
  int n_dev = 0;
  if (cudaGetDeviceCount(&n_dev) != cudaSuccess || device < 0 || device >= n_dev) return MOEGPS_ERR_CUDA;
  moegps_ctx* ctx = new (std::nothrow) moegps_ctx();
  if (!ctx) return MOEGPS_ERR_CUDA;
  ctx->shape = *shape;
  ctx->device = device;
  ctx->launches = 0;
  ctx->last_cuda_error = 0;
  ctx->tm1_valid = false;
  ctx->tm2_valid = false;
  for (bool& b : ctx->ffn_attr_done) b = false;
  for (auto& v : ctx->data_gradient_attr_done)
    for (bool& b : v) b = false;
  for (bool& b : ctx->ffn4_attr_done) b = false;
  ctx->weight_gradient_attr_done = ctx->router_weight_attr_done = false;
  ctx->rt_valid = false;
  ctx->route_attr_done = false;
  ctx->dispatch_attr_done = false;
  ctx->pack_attr_done = false;
  const char* trace = getenv("MOEGPS_TRACE");
  ctx->trace = trace && trace[0] && trace[0] != '0';
  ctx->d_status = nullptr;
  ctx->d_route_acc = nullptr;
  int prev = 0;
  cudaGetDevice(&prev);
  cudaError_t e = cudaSetDevice(device);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&ctx->sm_count, cudaDevAttrMultiProcessorCount, device);
  constexpr size_t kCtxWords = 4 + 2 * 256 + 2;  // status word, router accumulators (64-bit), a count (64-bit)
  if (e == cudaSuccess) e = cudaMalloc(&ctx->d_status, kCtxWords * sizeof(int32_t));
  if (e == cudaSuccess) e = cudaMemset(ctx->d_status, 0, kCtxWords * sizeof(int32_t));
  ctx->d_route_acc = ctx->d_status ? reinterpret_cast<unsigned long long*>(ctx->d_status + 4) : nullptr;
  ctx->d_meetings = ctx->d_status ? ctx->d_route_acc + 256 : nullptr;
  cudaSetDevice(prev);
  if (e != cudaSuccess) {
    if (ctx->d_status) cudaFree(ctx->d_status);
    delete ctx;
    return MOEGPS_ERR_CUDA;
  }
  *out = ctx;
  return MOEGPS_OK;
}

int moegps_destroy(moegps_ctx_t* ctx) {
  if (!ctx) return MOEGPS_ERR_INVALID_ARG;
  if (ctx->d_status) cudaFree(ctx->d_status);
  delete ctx;
  return MOEGPS_OK;
}

int64_t moegps_rcap(const moegps_shape_t* shape) {
  if (check_shape(shape) != MOEGPS_OK) return -1;
  return moegps_rcap_of(*shape);
}

size_t moegps_workspace_bytes(const moegps_shape_t* shape) {
  if (check_shape(shape) != MOEGPS_OK) return 0;
  const int64_t R = (int64_t)shape->T * shape->K;
  const int64_t nseg = (R + kSegPairs - 1) / kSegPairs;
  // the per-(segment, expert) count matrix + one word for the scan path's ticket counter; or, for
  // the fused form (moegps_route_prepare), one column per router CTA: the router runs one CTA per
  // 128-token tile, or splits the tiles over up to 8 CTAs while the grid stays within about 1.25x
  // the SM count (bounded here by 320 CTAs)
  const int64_t tiles = ((int64_t)shape->T + 127) / 128;
  const int64_t cols = nseg > (tiles > 320 ? tiles : 320) ? nseg : (tiles > 320 ? tiles : 320);
  size_t bytes = ((size_t)cols * shape->E + 1) * sizeof(int32_t);
  return (bytes + 255) & ~(size_t)255;
}

int moegps_route(moegps_ctx_t* ctx, const void* x, const void* w_router, const float* bias,
                 int32_t* topk_idx, float* topk_w, void* stream) {
  if (!ctx) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  if (ctx->shape.T == 0) return MOEGPS_OK;          // nothing to route (empty tensors have no address)
  if (!all_ok(x, w_router, topk_idx, topk_w)) return MOEGPS_ERR_INVALID_ARG;
  if (bias && (reinterpret_cast<uintptr_t>(bias) & 3u)) return MOEGPS_ERR_INVALID_ARG;
  return moegps_launch_route(ctx, x, w_router, bias, topk_idx, topk_w, nullptr, nullptr, nullptr, (cudaStream_t)stream);
}

int moegps_route_histogram(moegps_ctx_t* ctx, const void* x, const void* w_router, const float* bias,
                           int32_t* topk_idx, float* topk_w, int32_t* hist, void* stream) {
  if (!ctx || !all_ok(hist)) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  if (ctx->shape.T == 0)                            // no tokens: the histogram is all zero
    return cudaMemsetAsync(hist, 0, sizeof(int32_t) * ctx->shape.E, (cudaStream_t)stream) == cudaSuccess
               ? MOEGPS_OK : MOEGPS_ERR_CUDA;
  if (!all_ok(x, w_router, topk_idx, topk_w)) return MOEGPS_ERR_INVALID_ARG;
  if (bias && (reinterpret_cast<uintptr_t>(bias) & 3u)) return MOEGPS_ERR_INVALID_ARG;
  return moegps_launch_route(ctx, x, w_router, bias, topk_idx, topk_w, nullptr, hist, nullptr, (cudaStream_t)stream);
}

int moegps_route_prepare(moegps_ctx_t* ctx, const void* x, const void* w_router, const float* bias,
                         int32_t* topk_idx, float* topk_w, int32_t* hist, void* workspace, void* stream) {
  if (!ctx || !all_ok(hist, workspace)) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  if (ctx->shape.T == 0) {                          // no tokens: the histogram is all zero
    MOEGPS_CUDA_TRY(ctx, cudaMemsetAsync(hist, 0, sizeof(int32_t) * ctx->shape.E, st));
    return MOEGPS_OK;
  }
  if (!all_ok(x, w_router, topk_idx, topk_w)) return MOEGPS_ERR_INVALID_ARG;
  if (bias && (reinterpret_cast<uintptr_t>(bias) & 3u)) return MOEGPS_ERR_INVALID_ARG;
  return moegps_launch_route(ctx, x, w_router, bias, topk_idx, topk_w, nullptr, hist, static_cast<int32_t*>(workspace),
                             st);
}

int moegps_dispatch_prepared(moegps_ctx_t* ctx, const void* x, const int32_t* topk_idx, const int32_t* hist,
                             const int32_t* replicas, const int32_t* slot_off, int32_t* slot_row_off,
                             int32_t* row_pair, int32_t* pair_row, void* xp, const void* workspace, void* stream) {
  if (!ctx || !all_ok(hist, replicas, slot_off, slot_row_off, workspace)) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  if (ctx->shape.T == 0) {                          // nothing routed: every slot is empty, no padding exists
    MOEGPS_CUDA_TRY(ctx, cudaMemsetAsync(slot_row_off, 0, sizeof(int32_t) * (ctx->shape.S + 1), (cudaStream_t)stream));
    return MOEGPS_OK;
  }
  if (!all_ok(x, topk_idx, pair_row, xp, row_pair)) return MOEGPS_ERR_INVALID_ARG;
  return moegps_launch_dispatch_prepared(ctx, x, topk_idx, hist, replicas, slot_off, slot_row_off, row_pair, pair_row,
                                         xp, workspace, (cudaStream_t)stream);
}

int moegps_route_logits(moegps_ctx_t* ctx, const void* x, const void* w_router, const float* bias,
                        float* logits, void* stream) {
  if (!ctx) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  if (ctx->shape.T == 0) return MOEGPS_OK;
  if (!all_ok(x, w_router, logits)) return MOEGPS_ERR_INVALID_ARG;
  if (bias && (reinterpret_cast<uintptr_t>(bias) & 3u)) return MOEGPS_ERR_INVALID_ARG;
  return moegps_launch_route(ctx, x, w_router, bias, nullptr, nullptr, logits, nullptr, nullptr, (cudaStream_t)stream);
}

int moegps_histogram(moegps_ctx_t* ctx, const int32_t* topk_idx, int32_t* hist, void* stream) {
  if (!ctx || !all_ok(hist)) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  if (ctx->shape.T > 0 && !all_ok(topk_idx)) return MOEGPS_ERR_INVALID_ARG;
  return moegps_launch_histogram(ctx, topk_idx, hist, (cudaStream_t)stream);
}

int moegps_plan(moegps_ctx_t* ctx, const int32_t* predicted_hist, int32_t n_slots, int32_t* replicas,
                int32_t* slot_off, int32_t* slot_expert, int32_t* bound, void* stream) {
  if (!ctx || !all_ok(predicted_hist, replicas, slot_off, slot_expert) || !bound) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  if (reinterpret_cast<uintptr_t>(bound) & 3u) return MOEGPS_ERR_INVALID_ARG;
  if (n_slots != ctx->shape.S) return MOEGPS_ERR_INVALID_ARG;
  return moegps_launch_plan(ctx, predicted_hist, replicas, slot_off, slot_expert, bound, (cudaStream_t)stream);
}

int moegps_dispatch(moegps_ctx_t* ctx, const void* x, const int32_t* topk_idx, const int32_t* hist,
                    const int32_t* replicas, const int32_t* slot_off, int32_t* slot_row_off,
                    int32_t* row_pair, int32_t* pair_row, void* xp, void* workspace, void* stream) {
  if (!ctx || !all_ok(hist, replicas, slot_off, slot_row_off, workspace)) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  if (ctx->shape.T > 0 && !all_ok(x, topk_idx, pair_row, xp)) return MOEGPS_ERR_INVALID_ARG;
  if (moegps_rcap_of(ctx->shape) > 0 && !all_ok(row_pair)) return MOEGPS_ERR_INVALID_ARG;
  return moegps_launch_dispatch(ctx, x, topk_idx, hist, replicas, slot_off, nullptr, slot_row_off, row_pair, pair_row,
                                xp, workspace, (cudaStream_t)stream);
}

int moegps_dispatch_shares(moegps_ctx_t* ctx, const void* x, const int32_t* topk_idx, const int32_t* hist,
                           const int32_t* replicas, const int32_t* slot_off, const int32_t* slot_share,
                           int32_t* slot_row_off, int32_t* row_pair, int32_t* pair_row, void* xp, void* workspace,
                           void* stream) {
  if (!ctx || !all_ok(hist, replicas, slot_off, slot_share, slot_row_off, workspace)) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  if (ctx->shape.T > 0 && !all_ok(x, topk_idx, pair_row, xp)) return MOEGPS_ERR_INVALID_ARG;
  if (moegps_rcap_of(ctx->shape) > 0 && !all_ok(row_pair)) return MOEGPS_ERR_INVALID_ARG;
  return moegps_launch_dispatch(ctx, x, topk_idx, hist, replicas, slot_off, slot_share, slot_row_off, row_pair,
                                pair_row, xp, workspace, (cudaStream_t)stream);
}

int moegps_expert_ffn(moegps_ctx_t* ctx, const void* xp, const int32_t* slot_row_off,
                      const int32_t* slot_expert, const void* w_gate, const void* w_up, const void* w_down,
                      void* h_ws, void* yp, void* stream) {
  if (!ctx) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  if (ctx->shape.T == 0) return MOEGPS_OK;
  if (!all_ok(xp, slot_row_off, slot_expert, w_gate, w_up, w_down, h_ws, yp)) return MOEGPS_ERR_INVALID_ARG;
  int rc = moegps_launch_ffn_gate_up(ctx, xp, slot_row_off, slot_expert, w_gate, w_up, h_ws, (cudaStream_t)stream);
  if (rc != MOEGPS_OK) return rc;
  return moegps_launch_ffn_down(ctx, h_ws, slot_row_off, slot_expert, w_down, yp, (cudaStream_t)stream);
}

int moegps_expert_ffn_gate_up(moegps_ctx_t* ctx, const void* xp, const int32_t* slot_row_off,
                              const int32_t* slot_expert, const void* w_gate, const void* w_up, void* h_ws,
                              void* stream) {
  if (!ctx) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  if (ctx->shape.T == 0) return MOEGPS_OK;
  if (!all_ok(xp, slot_row_off, slot_expert, w_gate, w_up, h_ws)) return MOEGPS_ERR_INVALID_ARG;
  return moegps_launch_ffn_gate_up(ctx, xp, slot_row_off, slot_expert, w_gate, w_up, h_ws, (cudaStream_t)stream);
}

int moegps_expert_ffn_down(moegps_ctx_t* ctx, const void* h_ws, const int32_t* slot_row_off,
                           const int32_t* slot_expert, const void* w_down, void* yp, void* stream) {
  if (!ctx) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  if (ctx->shape.T == 0) return MOEGPS_OK;
  if (!all_ok(h_ws, slot_row_off, slot_expert, w_down, yp)) return MOEGPS_ERR_INVALID_ARG;
  return moegps_launch_ffn_down(ctx, h_ws, slot_row_off, slot_expert, w_down, yp, (cudaStream_t)stream);
}

int moegps_combine(moegps_ctx_t* ctx, const void* yp, const int32_t* pair_row, const float* topk_w,
                   void* out, void* stream) {
  if (!ctx) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  if (ctx->shape.T == 0) return MOEGPS_OK;
  if (!all_ok(yp, pair_row, topk_w, out)) return MOEGPS_ERR_INVALID_ARG;
  return moegps_launch_combine(ctx, yp, pair_row, topk_w, out, (cudaStream_t)stream);
}

int moegps_expert_ffn_gate_up_save(moegps_ctx_t* ctx, const void* xp, const int32_t* slot_row_off,
                                   const int32_t* slot_expert, const void* w_gate, const void* w_up, void* h_ws,
                                   void* gate8, void* up8, void* gate_scale, void* up_scale, void* stream) {
  if (!ctx) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  if (ctx->shape.T == 0) return MOEGPS_OK;
  if (!all_ok(xp, slot_row_off, slot_expert, w_gate, w_up, h_ws, gate8, up8, gate_scale, up_scale)) return MOEGPS_ERR_INVALID_ARG;
  return moegps_launch_ffn_gate_up_save(ctx, xp, slot_row_off, slot_expert, w_gate, w_up, h_ws, gate8, up8, gate_scale,
                                        up_scale, (cudaStream_t)stream);
}

int moegps_expert_ffn_backward_act(moegps_ctx_t* ctx, const void* dyp, const int32_t* slot_row_off,
                                   const int32_t* slot_expert, const void* w_down, const void* gate8, const void* up8,
                                   const void* gate_scale, const void* up_scale, void* dgate, void* dup, void* h_ws,
                                   void* stream) {
  if (!ctx) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  if (ctx->shape.T == 0) return MOEGPS_OK;
  if (!all_ok(dyp, slot_row_off, slot_expert, w_down, gate8, up8, gate_scale, up_scale, dgate, dup, h_ws))
    return MOEGPS_ERR_INVALID_ARG;
  return moegps_launch_ffn_backward_act(ctx, dyp, slot_row_off, slot_expert, w_down, gate8, up8, gate_scale, up_scale, dgate,
                                        dup, h_ws, (cudaStream_t)stream);
}

int moegps_expert_ffn_backward_input(moegps_ctx_t* ctx, const void* dgate, const void* dup, const int32_t* slot_row_off,
                                     const int32_t* slot_expert, const void* w_gate, const void* w_up, void* dxp,
                                     void* stream) {
  if (!ctx) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  if (ctx->shape.T == 0) return MOEGPS_OK;
  if (!all_ok(dgate, dup, slot_row_off, slot_expert, w_gate, w_up, dxp)) return MOEGPS_ERR_INVALID_ARG;
  return moegps_launch_ffn_backward_input(ctx, dgate, dup, slot_row_off, slot_expert, w_gate, w_up, dxp,
                                          (cudaStream_t)stream);
}

int moegps_expert_ffn_backward_weights(moegps_ctx_t* ctx, const void* dyp, const void* xp, const void* dgate, const void* dup,
                                       const void* h_ws, const int32_t* slot_row_off, const int32_t* slot_off,
                                       const int32_t* row_pair, void* dw_gate, void* dw_up, void* dw_down, void* stream) {
  if (!ctx || !all_ok(dw_gate, dw_up, dw_down)) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  if (ctx->shape.T == 0) {                          // no tokens: every gradient is zero
    const size_t bytes = (size_t)ctx->shape.E * ctx->shape.F * ctx->shape.D * 2;
    for (void* p : {dw_gate, dw_up, dw_down}) MOEGPS_CUDA_TRY(ctx, cudaMemsetAsync(p, 0, bytes, st));
    return MOEGPS_OK;
  }
  if (!all_ok(dyp, xp, dgate, dup, h_ws, slot_row_off, slot_off, row_pair)) return MOEGPS_ERR_INVALID_ARG;
  return moegps_launch_ffn_backward_weights(ctx, dyp, xp, dgate, dup, h_ws, slot_row_off, slot_off, row_pair, dw_gate, dw_up,
                                            dw_down, st);
}

int moegps_expert_ffn_backward(moegps_ctx_t* ctx, const void* dyp, const void* xp, const int32_t* slot_row_off,
                               const int32_t* slot_off, const int32_t* slot_expert, const int32_t* row_pair,
                               const void* w_gate, const void* w_up, const void* w_down, const void* gate8, const void* up8,
                               const void* gate_scale, const void* up_scale, void* dgate, void* dup, void* h_ws, void* dxp,
                               void* dw_gate, void* dw_up, void* dw_down, void* stream) {
  if (!ctx || !all_ok(dw_gate, dw_up, dw_down)) return MOEGPS_ERR_INVALID_ARG;
  // everything is checked before the first launch
  if (ctx->shape.T > 0 && !all_ok(dyp, xp, slot_row_off, slot_off, slot_expert, row_pair, w_gate, w_up, w_down, gate8, up8,
                                  gate_scale, up_scale, dgate, dup, h_ws, dxp))
    return MOEGPS_ERR_INVALID_ARG;
  int rc = moegps_expert_ffn_backward_act(ctx, dyp, slot_row_off, slot_expert, w_down, gate8, up8, gate_scale, up_scale, dgate,
                                          dup, h_ws, stream);
  if (rc != MOEGPS_OK) return rc;
  rc = moegps_expert_ffn_backward_input(ctx, dgate, dup, slot_row_off, slot_expert, w_gate, w_up, dxp, stream);
  if (rc != MOEGPS_OK) return rc;
  return moegps_expert_ffn_backward_weights(ctx, dyp, xp, dgate, dup, h_ws, slot_row_off, slot_off, row_pair, dw_gate, dw_up,
                                            dw_down, stream);
}

int moegps_combine_backward(moegps_ctx_t* ctx, const void* dout, const void* yp, const int32_t* pair_row,
                            const float* topk_w, void* dyp, float* dtopk_w, void* stream) {
  if (!ctx) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  if (ctx->shape.T == 0) return MOEGPS_OK;
  if (!all_ok(dout, yp, pair_row, topk_w, dyp, dtopk_w)) return MOEGPS_ERR_INVALID_ARG;
  return moegps_launch_combine_backward(ctx, dout, yp, pair_row, topk_w, dyp, dtopk_w, (cudaStream_t)stream);
}

int moegps_dispatch_backward(moegps_ctx_t* ctx, const void* dxp, const int32_t* pair_row, const int32_t* topk_idx,
                             const float* dlogit, const void* w_router, void* dx, void* stream) {
  if (!ctx) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  if (ctx->shape.T == 0) return MOEGPS_OK;
  if (!all_ok(dxp, pair_row, dx)) return MOEGPS_ERR_INVALID_ARG;
  if (dlogit && !all_ok(topk_idx, dlogit, w_router)) return MOEGPS_ERR_INVALID_ARG;
  return moegps_launch_dispatch_backward(ctx, dxp, pair_row, topk_idx, dlogit, w_router, dx, (cudaStream_t)stream);
}

size_t moegps_route_backward_workspace_bytes(const moegps_shape_t* shape) {
  return check_shape(shape) == MOEGPS_OK ? route_backward::bytes(*shape) : 0;
}

int moegps_route_backward(moegps_ctx_t* ctx, const void* x, const void* w_router, const float* bias,
                          const int32_t* topk_idx, const float* topk_w, const float* dtopk_w, const int32_t* slot_row_off,
                          const int32_t* slot_off, const int32_t* row_pair, float* dlogit, float* dw_router, float* dbias,
                          void* workspace, void* stream) {
  if (!ctx || !all_ok(dw_router, dbias)) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  const moegps_shape_t& s = ctx->shape;
  cudaStream_t st = (cudaStream_t)stream;
  if (s.T == 0) {                                   // no tokens: every gradient is zero
    MOEGPS_CUDA_TRY(ctx, cudaMemsetAsync(dw_router, 0, sizeof(float) * s.E * s.D, st));
    MOEGPS_CUDA_TRY(ctx, cudaMemsetAsync(dbias, 0, sizeof(float) * s.E, st));
    return MOEGPS_OK;
  }
  if (!all_ok(x, topk_w, dtopk_w, slot_row_off, slot_off, row_pair, dlogit, workspace)) return MOEGPS_ERR_INVALID_ARG;
  if (s.gate_mode == 1 && !all_ok(w_router, topk_idx)) return MOEGPS_ERR_INVALID_ARG;
  if (topk_idx && !all_ok(topk_idx)) return MOEGPS_ERR_INVALID_ARG;
  if (bias && (reinterpret_cast<uintptr_t>(bias) & 3u)) return MOEGPS_ERR_INVALID_ARG;
  return moegps_launch_route_backward(ctx, x, w_router, bias, topk_idx, topk_w, dtopk_w, slot_row_off, slot_off, row_pair,
                                      dlogit, dw_router, dbias, workspace, st);
}

size_t moegps_weights4_bytes(const moegps_shape_t* shape, int32_t down) {
  if (check_shape(shape) != MOEGPS_OK) return 0;
  const size_t rows = down ? shape->D : shape->F;
  return (size_t)shape->E * rows * mx4::chunks_of(down ? shape->F : shape->D) * (mx4::kChunk / 2);
}

size_t moegps_weights4_scale_bytes(const moegps_shape_t* shape, int32_t down) {
  if (check_shape(shape) != MOEGPS_OK) return 0;
  return (size_t)shape->E * mx4::tiles_of(down ? shape->D : shape->F) * mx4::chunks_of(down ? shape->F : shape->D) *
         mx4::kScaleTile;
}

int moegps_weights_quantize4(moegps_ctx_t* ctx, const void* w, int32_t down, void* w4, void* w4_scale, void* stream) {
  if (!ctx || !all_ok(w, w4, w4_scale) || !aligned32(w4)) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  if (!tiles4_fit(ctx->shape)) return MOEGPS_ERR_UNSUPPORTED_SHAPE;
  return moegps_launch_weights_quantize4(ctx, w, down != 0, w4, w4_scale, (cudaStream_t)stream);
}

int moegps_weights_dequantize4(moegps_ctx_t* ctx, const void* w4, const void* w4_scale, int32_t down, void* w, void* stream) {
  if (!ctx || !all_ok(w, w4, w4_scale) || !aligned32(w4)) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  if (!tiles4_fit(ctx->shape)) return MOEGPS_ERR_UNSUPPORTED_SHAPE;
  return moegps_launch_weights_dequantize4(ctx, w4, w4_scale, down != 0, w, (cudaStream_t)stream);
}

size_t moegps_expert_ffn4_workspace_bytes(const moegps_shape_t* shape) {
  return check_shape(shape) == MOEGPS_OK ? mx4::layout_of(*shape).total : 0;
}

int moegps_expert_ffn4(moegps_ctx_t* ctx, const void* xp, const int32_t* slot_row_off, const int32_t* slot_expert,
                       const void* gate4, const void* up4, const void* down4, const void* gate4_scale, const void* up4_scale,
                       const void* down4_scale, void* yp, void* workspace, void* stream) {
  if (!ctx) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  if (ctx->shape.T == 0) return MOEGPS_OK;
  if (!all_ok(xp, slot_row_off, slot_expert, gate4, up4, down4, gate4_scale, up4_scale, down4_scale, yp, workspace) ||
      !aligned32(gate4) || !aligned32(up4) || !aligned32(down4))
    return MOEGPS_ERR_INVALID_ARG;
  if (!tiles4_fit(ctx->shape)) return MOEGPS_ERR_UNSUPPORTED_SHAPE;
  return moegps_launch_expert_ffn4(ctx, xp, slot_row_off, slot_expert, gate4, up4, down4, gate4_scale, up4_scale, down4_scale, yp,
                                   workspace, (cudaStream_t)stream);
}

int moegps_status(moegps_ctx_t* ctx, void* stream, int32_t* host_status) {
  if (!ctx || !host_status) return MOEGPS_ERR_INVALID_ARG;
  if (int rc = moegps_check_device(ctx)) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  int32_t h[2] = {0, 0};      // error code and its detail
  MOEGPS_CUDA_TRY(ctx, cudaMemcpyAsync(h, ctx->d_status, sizeof(h), cudaMemcpyDeviceToHost, st));
  MOEGPS_CUDA_TRY(ctx, cudaMemsetAsync(ctx->d_status, 0, sizeof(h), st));
  MOEGPS_CUDA_TRY(ctx, cudaStreamSynchronize(st));
  host_status[0] = h[0];
  return MOEGPS_OK;
}

int64_t moegps_launch_count(const moegps_ctx_t* ctx) { return ctx ? ctx->launches : -1; }

int moegps_last_cuda_error(const moegps_ctx_t* ctx) { return ctx ? ctx->last_cuda_error : 0; }

const char* moegps_error_string(int code) {
  switch (code) {
    case MOEGPS_OK: return "ok";
    case MOEGPS_ERR_INVALID_ARG: return "invalid argument (null/misaligned pointer, n_slots != S, bad mode)";
    case MOEGPS_ERR_UNSUPPORTED_SHAPE: return "unsupported shape";
    case MOEGPS_ERR_WORKSPACE_TOO_SMALL: return "workspace too small";
    case MOEGPS_ERR_CUDA: return "CUDA call failed";
    case MOEGPS_ERR_UNIMPLEMENTED: return "not implemented";
    case MOEGPS_ERR_BAD_INDEX: return "device saw an index out of range (access skipped)";
    case MOEGPS_ERR_TIMEOUT: return "a bounded wait inside a kernel ran out";
    case MOEGPS_ERR_HIST_MISMATCH: return "hist passed to dispatch disagrees with topk_idx";
    case MOEGPS_ERR_STATIC_SCRATCH_EXCEEDED:
      return "problem too large for the built-in scratch of moegps_dispatch_static (ceil(T*K/256)*E > 262144): "
             "use moegps_dispatch with a caller-provided workspace";
    default: return "unknown moegps error";
  }
}

}  // extern "C"
