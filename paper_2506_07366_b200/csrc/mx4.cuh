// 4-bit expert weights and the block-scaled products on them.
//
// Weights (E matrices of N outputs x C inputs, bf16) in 4 bits: 32 consecutive inputs of an output form a block with one
// power-of-two scale.
//   scale 2^k : k is the smallest integer with max|w| <= 6 * 2^k (6 = the largest e2m1 value), -127 <= k <= 125, so
//               dividing is exact and nothing saturates (but weights above 1.5 * 2^127, which become that).
//   code      : w * 2^-k rounded to e2m1 {0, .5, 1, 1.5, 2, 3, 4, 6}, nearest, ties to the even code; bit 3 is the sign.
//   scale byte: k + 127; 255 for a block with an infinity or a NaN in it, whose 32 weights then decode to NaN.  A block
//               of zeros has byte 0.
// Layout: codes uint8 [E][N][chunks * 64], two to a byte, the even input in the low half; chunks = C / 128 rounded up, the
// last chunk filled up with zeros.  Scale bytes uint8 [E][tiles][chunks][512], tiles = N / 128 rounded up: what one tile of
// 128 outputs needs for one chunk of 128 inputs lies together, in the order in which tensor memory takes it: output r of the
// tile and block j of the chunk at byte (r % 32) * 16 + r / 32 * 4 + j.
//
// Activations for these products.  The tensor core multiplies e2m1 by e4m3 at twice its bf16 rate (kind::mxf8f6f4, a scale
// 2^k for 32 values of a row on either side, fp32 accumulation).  A bf16 has 8 significant bits and an e4m3 has 4, so x is
// written as two e4m3 terms: x = 2^k (c1 + 2^-4 c2) with c1 = x 2^-k rounded to nearest and c2 the rest.  k is the smallest
// integer with max|x| <= 448 * 2^k over 32 values.  The rest is at most half a step of c1, i.e. at most 8 steps of bf16, so
// it fits c2 exactly: nothing is lost above 2^-6 * 2^k, and below that the error is at most 2^-14 * 2^k, which is 2^-21 of the
// block's maximum.  Two products at twice the rate cost what one bf16 product costs, and the weights go to the tensor core as
// they are in memory.
// For values with more bits than bf16 (the hidden activations, straight from the accumulator) the same two terms are off by
// at most 2^-9 relative, half of what a rounding to bf16 is.
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp4.h>
#include <cuda_fp8.h>
#include <stdint.h>

#include "moegps.h"

namespace mx4 {

constexpr int kBlock = 32;         // values that share a scale
constexpr int kChunk = 128;        // inputs of a chunk: four blocks, one 128-byte row of shared memory
constexpr int kTile = 128;         // outputs of a tile
constexpr int kScaleTile = 512;    // bytes of scales of a tile's chunk

__host__ __device__ constexpr int chunks_of(int cols) { return (cols + kChunk - 1) / kChunk; }
__host__ __device__ constexpr int tiles_of(int rows) { return (rows + kTile - 1) / kTile; }
// byte of (row r of a tile, block j of a chunk) in its 512 scale bytes; without j: of the word of the row's four blocks
__host__ __device__ constexpr int scale_byte_at(int r, int j = 0) { return (r % 32) * 16 + (r / 32) * 4 + j; }

// scale byte of a block of 4-bit weights whose largest magnitude has these fp32 bits
__device__ __forceinline__ uint32_t weight_scale(uint32_t m) {
  if (m >= 0x7f800000u) return 255u;
  const int field = (int)((m + 0x3fffffu) >> 23) - 2;        // exponent, plus one if the mantissa exceeds 1.5; 6 = 1.5 * 2^2
  return (uint32_t)min(max(field, 0), 252);
}
// scale byte of a block of the first term (e4m3: 448 = 1.75 * 2^8)
__device__ __forceinline__ uint32_t term_scale(uint32_t m) {
  if (m >= 0x7f800000u) return 255u;
  return (uint32_t)max((int)((m + 0x1fffffu) >> 23) - 8, 0);
}
// ... and of the second
__device__ __forceinline__ uint32_t second_scale(uint32_t byte) { return byte == 255u ? 255u : byte < 4u ? 0u : byte - 4u; }
// 2^-k of a scale byte below 255; 0 for 255, whose codes do not matter
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __uint_as_float(byte == 255u ? 0u : (254u - byte) << 23); }
// 2^(k1 - k2), at most 2^4
__device__ __forceinline__ float scale_ratio(uint32_t first, uint32_t second) {
  return __uint_as_float((127u + first - second) << 23);
}

// two values -> the codes of their two terms; inv = 2^-k, ratio = 2^(k1 - k2)
__device__ __forceinline__ void split2(float a, float b, float inv, float ratio, uint32_t& first, uint32_t& second) {
  const float2 y = make_float2(a * inv, b * inv);
  const __nv_fp8x2_storage_t c = __nv_cvt_float2_to_fp8x2(y, __NV_SATFINITE, __NV_E4M3);
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(c, __NV_E4M3);
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
  first = c;
  second = __nv_cvt_float2_to_fp8x2(make_float2((y.x - f.x) * ratio, (y.y - f.y) * ratio), __NV_SATFINITE, __NV_E4M3);
}

// ------------------------------------------------------------------------------------------- workspace of expert_ffn4
// How the rows of a slot are cut into tiles (chosen by shape alone, it decides the layout of the workspace).
enum class Cut { k16, k48, k224 };
inline Cut cut_of(const moegps_shape_t& s) {
  const int64_t R = (int64_t)s.T * s.K, slots = R < s.S ? R : s.S;
  const int64_t per_slot = slots > 0 ? (R + slots - 1) / slots : 0;
  return per_slot <= 16 ? Cut::k16 : per_slot <= 48 ? Cut::k48 : Cut::k224;
}
inline int rows_of(Cut c) { return c == Cut::k16 ? 16 : c == Cut::k48 ? 48 : 224; }

// Scale bytes of a tile's rows for one chunk, in the order of tensor memory (scale_byte_at).
// Tiles of 16 or 48 rows: both terms stacked in one group of 512 bytes, the second term's rows behind the first's, which are
// rounded up to 16.  Tiles of 224 rows: two groups for each term.
template <int kRows>
constexpr int kRowScaleBytes = kRows > 48 ? 4 * kScaleTile : kScaleTile;
template <int kRows>
__host__ __device__ constexpr int row_scale_at(int row, int term, int rows_in_tile) {
  if (kRows > 48) return (2 * term + row / 128) * kScaleTile + scale_byte_at(row % 128);
  return scale_byte_at(row + term * ((rows_in_tile + 15) / 16 * 16));
}

// Tiles of 224 rows.  Rows of activations in two terms: codes [rows][chunks * 128] for each, scales [row tile][chunk]
// [kRowScaleBytes].
struct Rows {
  uint8_t* code[2];
  uint8_t* scale;
};

// Tiles of 16 or 48 rows: for each tile and chunk the image that the products want in shared memory, the scales and behind them
// 128 bytes for each row, the first term's and then (from a multiple of 16 rows) the second's; the 16-byte pieces of a row are
// swizzled by the row's number.
template <int kRows>
constexpr int kImageBytes = kScaleTile + 2 * kRows * kChunk;
__host__ __device__ constexpr int image_code_at(int row, int term, int rows_in_tile, int piece) {
  return kScaleTile + (row + term * ((rows_in_tile + 15) / 16 * 16)) * kChunk + ((piece ^ (row % 8)) * 16);
}

inline size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

constexpr int kMaxCtas = 148;      // blocks of a launch that joins partial sums; what they leave for each other is sized by it

struct Layout {
  Cut cut;
  int64_t rows, row_tiles;         // Rcap; tiles of rows at most
  // offsets: images, or codes (the second term's follow the first's) and scales; what of h and of shared sums is there, their parts
  size_t x_code, x_scale, h_code, h_scale, part_there, h_there, partial, total;
  size_t x_code_bytes, h_code_bytes;
};

inline Layout layout_of(const moegps_shape_t& s) {
  Layout l;
  l.cut = cut_of(s);
  const int n = rows_of(l.cut);
  l.rows = (int64_t)s.T * s.K + (int64_t)s.S * (s.row_align - 1);
  l.row_tiles = l.rows / n + s.S;
  const size_t dc = chunks_of(s.D), fc = chunks_of(s.F);
  l.x_code = 0;
  if (l.cut == Cut::k224) {
    const size_t scales = (size_t)l.row_tiles * kRowScaleBytes<224>;
    l.x_code_bytes = align256((size_t)l.rows * dc * kChunk);
    l.h_code_bytes = align256((size_t)l.rows * fc * kChunk);
    l.x_scale = 2 * l.x_code_bytes;
    l.h_code = l.x_scale + align256(scales * dc);
    l.h_scale = l.h_code + 2 * l.h_code_bytes;
    l.part_there = l.h_there = l.partial = l.total = l.h_scale + align256(scales * fc);
    return l;
  }
  const size_t image = l.cut == Cut::k16 ? kImageBytes<16> : kImageBytes<48>;
  l.x_code_bytes = align256(l.row_tiles * dc * image);
  l.h_code_bytes = align256(l.row_tiles * fc * image);
  l.h_code = l.x_code_bytes;
  l.x_scale = l.h_scale = l.part_there = l.h_code + l.h_code_bytes;
  l.h_there = l.part_there + align256(3 * kMaxCtas * sizeof(int32_t));
  l.partial = l.h_there + align256(l.row_tiles * fc * sizeof(int32_t));
  // a block leaves at most one unfinished tile of gate + up behind and two of down
  l.total = l.partial + (size_t)kMaxCtas * 3 * 2 * n * kTile * sizeof(float);
  return l;
}

}  // namespace mx4
