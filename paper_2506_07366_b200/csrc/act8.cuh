// Activations kept in 8 bits: 32 consecutive columns of a row share one power-of-two scale.
//
//   scale 2^k : k is the smallest integer with max|v| <= 448 * 2^k (448 = the largest e4m3 value), so no value
//               saturates and the largest one uses the top binade; dividing by it is exact.
//   code      : v * 2^-k rounded to e4m3, nearest even: relative error at most 2^-4 down to 2^-6 * 2^k, below
//               that an absolute error of at most 2^-10 * 2^k.
//   scale byte: k + 127, and 255 for a block with an infinity or a NaN in it, whose 32 values then all decode
//               to NaN (a gradient that met one should show it).  A block of zeros has byte 0.
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <stdint.h>

namespace act8 {

constexpr int kBlock = 32;

// columns of a row of codes: every row is whole blocks
__host__ __device__ constexpr int pitch_of(int cols) { return (cols + kBlock - 1) / kBlock * kBlock; }

// v: 32 fp32 values (bits) -> 32 codes, returns the scale byte
__device__ __forceinline__ uint32_t encode(const uint32_t (&v)[32], uint32_t (&codes)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) m = max(m, v[i] & 0x7fffffffu);   // as integers, NaN and infinity are the largest
  // exponent field of the maximum, plus one if its mantissa exceeds 1.75 (448 = 1.75 * 2^8)
  const int field = (int)((m + 0x1fffffu) >> 23) - 8;
  const uint32_t byte = m >= 0x7f800000u ? 255u : (uint32_t)max(field, 0);
  const float inv = __uint_as_float(byte == 255u ? 0x7fffffffu : (254u - byte) << 23);   // 2^-k
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 lo = make_float2(__uint_as_float(v[4 * i]) * inv, __uint_as_float(v[4 * i + 1]) * inv);
    const float2 hi = make_float2(__uint_as_float(v[4 * i + 2]) * inv, __uint_as_float(v[4 * i + 3]) * inv);
    codes[i] = (uint32_t)__nv_cvt_float2_to_fp8x2(lo, __NV_SATFINITE, __NV_E4M3) |
               (uint32_t)__nv_cvt_float2_to_fp8x2(hi, __NV_SATFINITE, __NV_E4M3) << 16;
  }
  return byte;
}

// 2^k of a scale byte (2^-127 is subnormal), NaN for 255
__device__ __forceinline__ float scale_of(uint32_t byte) {
  return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255u ? 0x7fffffffu : byte << 23);
}

// four codes of a word -> four values
__device__ __forceinline__ void decode4(uint32_t codes, float scale, float (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(codes >> (16 * i)), __NV_E4M3);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    v[2 * i] = f.x * scale;
    v[2 * i + 1] = f.y * scale;
  }
}

}  // namespace act8
