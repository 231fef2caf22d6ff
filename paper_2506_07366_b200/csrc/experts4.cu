// weights_quantize4 / weights_dequantize4: expert matrices to 4 bits and back (format and layout: mx4.cuh).
//
// Both are bound by memory: 2 + 17/32 bytes a weight.  A block of 256 threads owns one tile of 128 outputs and one chunk of
// 128 inputs, so the tile's 512 scale bytes are one run of memory; eight threads share an output's 128 inputs (two to a block of
// 32: with one 16-byte load each and four to a block, the maximum and the scale took as long as memory), four outputs per thread
// are in flight at once.  One matrix quantized and read back, inputs in turn: 8 x 14336 x 4096 403 us (2.13 GB, 5.3 TB/s),
// 13 x 1000 x 1416 20.4 us (3.5 more without the early launch of the second).
#include "bf16x8.cuh"
#include "common.cuh"
#include "mx4.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kPieces = 8;                           // of an output's chunk: 16 inputs each
constexpr int kRowsAtOnce = kThreads / kPieces;
constexpr int kSteps = mx4::kTile / kRowsAtOnce;      // outputs of a thread

__global__ void __launch_bounds__(kThreads) quantize4_kernel(const __nv_bfloat16* __restrict__ w, uint8_t* __restrict__ w4,
                                                             uint8_t* __restrict__ w4_scale, int N, int C) {
  __shared__ __align__(16) uint8_t scales[mx4::kScaleTile];
  const int chunks = mx4::chunks_of(C), tiles = mx4::tiles_of(N);
  const int chunk = blockIdx.x % chunks, tile = blockIdx.x / chunks % tiles, e = blockIdx.x / chunks / tiles;
  const int piece = threadIdx.x % kPieces, row = threadIdx.x / kPieces;
  const int col = chunk * mx4::kChunk + 16 * piece;
  const size_t row0 = (size_t)e * N;
  launch_dependents();
  wait_for_predecessor();
  uint4 v[kSteps][2];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int n = tile * mx4::kTile + i * kRowsAtOnce + row;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      v[i][j] = make_uint4(0, 0, 0, 0);
      if (n < N && col + 8 * j < C) v[i][j] = *reinterpret_cast<const uint4*>(w + (row0 + n) * C + col + 8 * j);
    }
  }
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int r = i * kRowsAtOnce + row, n = tile * mx4::kTile + r;
    const uint32_t words[8] = {v[i][0].x, v[i][0].y, v[i][0].z, v[i][0].w, v[i][1].x, v[i][1].y, v[i][1].z, v[i][1].w};
    uint32_t m2 = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m2 = __vmaxu2(m2, words[j] & 0x7fff7fffu);
    uint32_t m = max(m2 & 0xffffu, m2 >> 16);         // as integers, NaN and infinity are the largest
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));   // over the two threads of a block
    const uint32_t byte = mx4::weight_scale(m << 16);
    const float inv = mx4::inverse_scale(byte);
    uint32_t codes[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j)
      codes[j >> 2] |= (uint32_t)__nv_cvt_float2_to_fp4x2(
                           make_float2(__uint_as_float(words[j] << 16) * inv, __uint_as_float(words[j] & 0xffff0000u) * inv),
                           __NV_E2M1, cudaRoundNearest)
                       << (8 * (j & 3));
    if (byte == 255u) codes[0] = codes[1] = 0;
    if (n < N)
      *reinterpret_cast<uint2*>(w4 + ((row0 + n) * (size_t)chunks + chunk) * (mx4::kChunk / 2) + 8 * piece) =
          make_uint2(codes[0], codes[1]);
    if ((piece & 1) == 0) scales[mx4::scale_byte_at(r, piece >> 1)] = (uint8_t)byte;
  }
  __syncthreads();
  if (threadIdx.x < mx4::kScaleTile / 16)
    reinterpret_cast<uint4*>(w4_scale + (size_t)blockIdx.x * mx4::kScaleTile)[threadIdx.x] =
        reinterpret_cast<const uint4*>(scales)[threadIdx.x];
}

__global__ void __launch_bounds__(kThreads) dequantize4_kernel(const uint8_t* __restrict__ w4, const uint8_t* __restrict__ w4_scale,
                                                               __nv_bfloat16* __restrict__ w, int N, int C) {
  __shared__ __align__(16) uint8_t scales[mx4::kScaleTile];
  const int chunks = mx4::chunks_of(C), tiles = mx4::tiles_of(N);
  const int chunk = blockIdx.x % chunks, tile = blockIdx.x / chunks % tiles, e = blockIdx.x / chunks / tiles;
  // 8 inputs for each thread here: with 16, its two 16-byte stores leave half of every 32-byte sector to each other (273 us
  // instead of 188 on 8 x 14336 x 4096)
  constexpr int kAtOnce = kThreads / 16, kTurns = mx4::kTile / kAtOnce;
  const int piece = threadIdx.x % 16, row = threadIdx.x / 16;
  const int col = chunk * mx4::kChunk + 8 * piece;
  const size_t row0 = (size_t)e * N;
  launch_dependents();
  wait_for_predecessor();
  if (threadIdx.x < mx4::kScaleTile / 16)
    reinterpret_cast<uint4*>(scales)[threadIdx.x] =
        __ldcs(reinterpret_cast<const uint4*>(w4_scale + (size_t)blockIdx.x * mx4::kScaleTile) + threadIdx.x);
  uint32_t codes[kTurns];
#pragma unroll
  for (int i = 0; i < kTurns; ++i) {
    const int n = tile * mx4::kTile + i * kAtOnce + row;
    codes[i] = 0;
    if (n < N)
      codes[i] = __ldcs(reinterpret_cast<const uint32_t*>(w4 + ((row0 + n) * (size_t)chunks + chunk) * (mx4::kChunk / 2) + 4 * piece));
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kTurns; ++i) {
    const int r = i * kAtOnce + row, n = tile * mx4::kTile + r;
    const uint32_t byte = scales[mx4::scale_byte_at(r, piece >> 2)];
    const float scale = __uint_as_float(byte == 0 ? 0x00400000u : byte == 255u ? 0x7fffffffu : byte << 23);   // 2^-127 is subnormal
    float f[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const __half2_raw h = __nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)(codes[i] >> (8 * k)), __NV_E2M1);
      const float2 value = __half22float2(*reinterpret_cast<const __half2*>(&h));
      f[2 * k] = value.x * scale;                     // exact, and so is the rounding to bf16
      f[2 * k + 1] = value.y * scale;
    }
    if (n < N && col < C) *reinterpret_cast<uint4*>(w + (row0 + n) * C + col) = pack8(f);
  }
}

// the matrices are [E, F, D] (gate, up) or [E, D, F] (down)
void dims(const moegps_shape_t& s, bool down, int& N, int& C, unsigned& blocks) {
  N = down ? s.D : s.F;
  C = down ? s.F : s.D;
  blocks = (unsigned)((int64_t)s.E * mx4::tiles_of(N) * mx4::chunks_of(C));
}

}  // namespace

int moegps_launch_weights_quantize4(moegps_ctx* ctx, const void* w, bool down, void* w4, void* w4_scale, cudaStream_t st) {
  int N, C;
  unsigned blocks;
  dims(ctx->shape, down, N, C, blocks);
  MOEGPS_CUDA_TRY(ctx, launch_after(quantize4_kernel, dim3(blocks), kThreads, 0, st, static_cast<const __nv_bfloat16*>(w),
                                    static_cast<uint8_t*>(w4), static_cast<uint8_t*>(w4_scale), N, C));
  MOEGPS_AFTER_LAUNCH(ctx);
  return MOEGPS_OK;
}

int moegps_launch_weights_dequantize4(moegps_ctx* ctx, const void* w4, const void* w4_scale, bool down, void* w, cudaStream_t st) {
  int N, C;
  unsigned blocks;
  dims(ctx->shape, down, N, C, blocks);
  MOEGPS_CUDA_TRY(ctx, launch_after(dequantize4_kernel, dim3(blocks), kThreads, 0, st, static_cast<const uint8_t*>(w4),
                                    static_cast<const uint8_t*>(w4_scale), static_cast<__nv_bfloat16*>(w), N, C));
  MOEGPS_AFTER_LAUNCH(ctx);
  return MOEGPS_OK;
}
