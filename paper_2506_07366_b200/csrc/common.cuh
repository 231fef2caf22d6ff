// Shared host/device declarations of the moegps library (context, status word, launch helpers).
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>

#include "moegps.h"

// Layout of the device status word: [0] first error code, [1] detail (index / location), [2..3] unused.
struct moegps_ctx {
  moegps_shape_t shape;
  int device;
  int sm_count;
  int32_t* d_status;        // 4 x int32 on the device
  unsigned long long* d_route_acc;   // behind it: 256 64-bit histogram accumulators of the router (all zero between calls)
  unsigned long long* d_meetings;    // behind them: arrivals of the blocks of expert_ffn4, ever growing
  int64_t launches;         // kernels launched through this context
  int last_cuda_error;
  // cached TMA descriptors of the expert FFN, keyed by the base pointers they were built for
  const void* tm_key1[3];   // xp, w_gate, w_up
  CUtensorMap tm_xp, tm_w1, tm_w3;
  bool tm1_valid;
  const void* tm_key2[2];   // h_ws, w_down
  CUtensorMap tm_h, tm_w2;
  bool tm2_valid;
  bool ffn_attr_done[3]; // dynamic shared-memory limit raised: gate+up, down, gate+up with kept activations
  bool data_gradient_attr_done[2][4];   // the same for the gradient's kernels: (act, input) x tile shapes
  bool ffn4_attr_done[4];   // on 4-bit weights: short runs of slots in tiles of up to 48, 32 rows; gate+up of long ones, their down
  bool weight_gradient_attr_done, router_weight_attr_done;
  // cached TMA descriptors of the router
  const void* rt_key[2];
  CUtensorMap tm_rx, tm_rw;
  bool rt_valid;
  bool route_attr_done;
  bool dispatch_attr_done;
  bool pack_attr_done;
  bool trace;               // MOEGPS_TRACE was set when the context was created: log every launch to stderr
};

// Host-side launch log (off unless the environment asked for it): ordinal, launcher, shape, and what was chosen for the launch
// (printf form) where there is a choice.
__attribute__((format(printf, 3, 4))) inline void moegps_trace_launch(const moegps_ctx* ctx, const char* where,
                                                                      const char* choice = nullptr, ...) {
  if (!ctx->trace) return;
  const moegps_shape_t& s = ctx->shape;
  char more[128] = "";
  if (choice) {
    va_list args;
    va_start(args, choice);
    vsnprintf(more, sizeof(more), choice, args);
    va_end(args);
  }
  fprintf(stderr, "[moegps] launch %lld %s T=%d D=%d F=%d E=%d K=%d S=%d A=%d%s%s\n", (long long)ctx->launches, where, s.T, s.D,
          s.F, s.E, s.K, s.S, s.row_align, choice ? " " : "", more);
}

#define MOEGPS_CUDA_TRY(ctx, expr)                                   \
  do {                                                               \
    cudaError_t _e = (expr);                                         \
    if (_e != cudaSuccess) {                                         \
      (ctx)->last_cuda_error = (int)_e;                              \
      return MOEGPS_ERR_CUDA;                                        \
    }                                                                \
  } while (0)

// Records a launch (and its launch error, if any); further arguments: what was chosen for it, see moegps_trace_launch.
#define MOEGPS_AFTER_LAUNCH(ctx, ...)                                \
  do {                                                               \
    (ctx)->launches += 1;                                            \
    moegps_trace_launch((ctx), __func__, ##__VA_ARGS__);             \
    cudaError_t _e = cudaGetLastError();                             \
    if (_e != cudaSuccess) {                                         \
      (ctx)->last_cuda_error = (int)_e;                              \
      return MOEGPS_ERR_CUDA;                                        \
    }                                                                \
  } while (0)

// Launches a kernel that may start while the stream's previous kernel still runs, as far as its own
// wait_for_predecessor(): the launch and the set-up in front of that call overlap the predecessor's end.
// early = false: an ordinary launch.
template <typename... KArgs, typename... Args>
static inline cudaError_t launch_after_if(bool early, void (*kernel)(KArgs...), dim3 grid, unsigned threads, size_t smem,
                                          cudaStream_t st, Args... args) {
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = &attr;
  cfg.numAttrs = early ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}
template <typename... KArgs, typename... Args>
static inline cudaError_t launch_after(void (*kernel)(KArgs...), dim3 grid, unsigned threads, size_t smem, cudaStream_t st,
                                       Args... args) {
  return launch_after_if(true, kernel, grid, threads, smem, st, args...);
}

static inline bool moegps_aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

static inline int64_t moegps_rcap_of(const moegps_shape_t& s) {
  return (int64_t)s.T * s.K + (int64_t)s.S * (s.row_align - 1);
}

// The status word, the cached tensor maps and the kernel attributes of a context belong to its
// device, so that device must be the calling thread's current one; otherwise nothing is launched.
static inline int moegps_check_device(const moegps_ctx* ctx) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) return MOEGPS_ERR_CUDA;
  return dev == ctx->device ? MOEGPS_OK : MOEGPS_ERR_INVALID_ARG;
}

// Device side of launch_after.  The wait returns when the predecessor grid has ended and its writes are visible (at once
// for a kernel that was launched without one); nothing that an earlier kernel of the stream may write, or still reads,
// is touched before it.
__device__ __forceinline__ void wait_for_predecessor() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// First error wins; later ones are dropped.
__device__ __forceinline__ void moegps_report(int32_t* status, int code, int detail) {
  if (atomicCAS(&status[0], 0, code) == 0) status[1] = detail;
}

// dispatch: pairs per warp segment of the stable ranking (see dispatch.cu)
constexpr int kSegPairs = 256;

// Per-step launchers (each validates nothing: the C entry points in api.cu do that).
// seg_cnt != nullptr: the router also stores its per-CTA expert counts, [E][CTAs] expert-major.
int moegps_launch_route(moegps_ctx* ctx, const void* x, const void* wr, const float* bias,
                        int32_t* topk_idx, float* topk_w, float* logits_out, int32_t* hist,
                        int32_t* seg_cnt, cudaStream_t st);
// rows of a token tile that one router CTA owns (= 128 / its split of the model dimension)
int moegps_route_rows_per_cta(const moegps_ctx* ctx);
int moegps_launch_dispatch_prepared(moegps_ctx* ctx, const void* x, const int32_t* topk_idx, const int32_t* hist,
                                    const int32_t* replicas, const int32_t* slot_off,
                                    int32_t* slot_row_off, int32_t* row_pair, int32_t* pair_row, void* xp,
                                    const void* workspace, cudaStream_t st);
int moegps_launch_histogram(moegps_ctx* ctx, const int32_t* topk_idx, int32_t* hist, cudaStream_t st);
int moegps_launch_plan(moegps_ctx* ctx, const int32_t* pred, int32_t* replicas, int32_t* slot_off,
                       int32_t* slot_expert, int32_t* bound, cudaStream_t st);
int moegps_launch_dispatch(moegps_ctx* ctx, const void* x, const int32_t* topk_idx, const int32_t* hist,
                           const int32_t* replicas, const int32_t* slot_off, const int32_t* slot_share,
                           int32_t* slot_row_off, int32_t* row_pair, int32_t* pair_row, void* xp, void* workspace,
                           cudaStream_t st);
int moegps_launch_ffn_gate_up(moegps_ctx* ctx, const void* xp, const int32_t* slot_row_off,
                              const int32_t* slot_expert, const void* w_gate, const void* w_up, void* h_ws,
                              cudaStream_t st);
int moegps_launch_ffn_down(moegps_ctx* ctx, const void* h_ws, const int32_t* slot_row_off,
                           const int32_t* slot_expert, const void* w_down, void* yp, cudaStream_t st);
int moegps_launch_combine(moegps_ctx* ctx, const void* yp, const int32_t* pair_row, const float* topk_w,
                          void* out, cudaStream_t st);
int moegps_launch_ffn_gate_up_save(moegps_ctx* ctx, const void* xp, const int32_t* slot_row_off,
                                   const int32_t* slot_expert, const void* w_gate, const void* w_up, void* h_ws,
                                   void* gate8, void* up8, void* gate_scale, void* up_scale, cudaStream_t st);
int moegps_launch_ffn_backward_act(moegps_ctx* ctx, const void* dyp, const int32_t* slot_row_off, const int32_t* slot_expert,
                                   const void* w_down, const void* gate8, const void* up8, const void* gate_scale,
                                   const void* up_scale, void* dgate, void* dup, void* h_ws, cudaStream_t st);
int moegps_launch_ffn_backward_input(moegps_ctx* ctx, const void* dgate, const void* dup, const int32_t* slot_row_off,
                                     const int32_t* slot_expert, const void* w_gate, const void* w_up, void* dxp,
                                     cudaStream_t st);
int moegps_launch_ffn_backward_weights(moegps_ctx* ctx, const void* dyp, const void* xp, const void* dgate, const void* dup,
                                       const void* h_ws, const int32_t* slot_row_off, const int32_t* slot_off,
                                       const int32_t* row_pair, void* dw_gate, void* dw_up, void* dw_down, cudaStream_t st);
int moegps_launch_combine_backward(moegps_ctx* ctx, const void* dout, const void* yp, const int32_t* pair_row,
                                   const float* topk_w, void* dyp, float* dtopk_w, cudaStream_t st);
int moegps_launch_dispatch_backward(moegps_ctx* ctx, const void* dxp, const int32_t* pair_row, const int32_t* topk_idx,
                                    const float* dlogit, const void* w_router, void* dx, cudaStream_t st);
int moegps_launch_route_backward(moegps_ctx* ctx, const void* x, const void* w_router, const float* bias,
                                 const int32_t* topk_idx, const float* topk_w, const float* dtopk_w,
                                 const int32_t* slot_row_off, const int32_t* slot_off, const int32_t* row_pair,
                                 float* dlogit, float* dw_router, float* dbias, void* workspace, cudaStream_t st);
int moegps_launch_weights_quantize4(moegps_ctx* ctx, const void* w, bool down, void* w4, void* w4_scale, cudaStream_t st);
int moegps_launch_weights_dequantize4(moegps_ctx* ctx, const void* w4, const void* w4_scale, bool down, void* w, cudaStream_t st);
int moegps_launch_expert_ffn4(moegps_ctx* ctx, const void* xp, const int32_t* slot_row_off, const int32_t* slot_expert,
                              const void* gate4, const void* up4, const void* down4, const void* gate4_scale, const void* up4_scale,
                              const void* down4_scale, void* yp, void* workspace, cudaStream_t st);
