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
// it fits c2 exactly: nothing is lost above 2^-6 * 2^k, and below that the error is at most 2^-14 * 2^k.  The block's maximum is above
// 224 * 2^k: what may be off is below 2^-13 of it, by at most 2^-21 of it.  Two products at twice the rate cost what one bf16
// product costs, and the weights go to the tensor core as they are in memory.
// For values with more bits than bf16 (the hidden activations, straight from the accumulator) the same two terms are off by at
// most 2^-9 relative, half of what a rounding to bf16 is, or by the 2^-14 * 2^k of the second term's last step where that is more
// (below 2^-12 of the block's maximum; 2^-137 for k < -123).
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

// two values -> the codes of their two terms; inv = 2^-k, ratio = 2^(k1 - k2) of each
__device__ __forceinline__ void split2(float a, float b, const float (&inv)[2], const float (&ratio)[2], uint32_t& first,
                                       uint32_t& second) {
  const float2 y = make_float2(a * inv[0], b * inv[1]);
  const __nv_fp8x2_storage_t c = __nv_cvt_float2_to_fp8x2(y, __NV_SATFINITE, __NV_E4M3);
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(c, __NV_E4M3);
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
  first = c;
  second = __nv_cvt_float2_to_fp8x2(make_float2((y.x - f.x) * ratio[0], (y.y - f.y) * ratio[1]), __NV_SATFINITE, __NV_E4M3);
}

// ------------------------------------------------------------------------------------------- workspace of expert_ffn4
// How the rows are worked (chosen by shape alone, it decides the layout of the workspace).  Copies of an expert side by side are
// one run of rows.  Runs of up to short_rows rows are worked in tiles of tile_rows by the launch for short runs, longer ones in
// tiles of 224 by those for long runs; either may be all.
struct Cut {
  int tile_rows, short_rows;
  bool all_short() const { return short_rows == INT32_MAX; }
};
// By the rows that an expert has on average (the actual loads are only known on the device), the experts, and the time that reading
// all weights once takes, 2.5 ns for 16 KB.  Padding is worked like other rows: where slots are aligned to more rows than a tile of
// 32 has, a run has that many at least (256 experts 7168 x 2048, 8 tokens aligned to 128: 1235 us all short, 536 all long; 8 experts
// 4096 x 14336 363 / 296, 64 experts 2048 x 1408 and 48 tokens 146 / 123).
// Short runs in one launch and long ones in the others cost 20 to 60 us for the launches and save passes over the weights of popular
// experts: the more rows an expert has, the more weights there are, and, where loads differ like 1 / rank, the more experts.  Measured
// (us, all short / both; experts x time of weights in 1000 us beside the layer, rows an expert behind it):
//   256 experts 7168 x 2048 (220)   2: 319 / 337, 4: 486 / 476, 8: 709 / 652, 32: 1650 / 1262
//   64 of 4096 x 14336 (55)         8: 687 / 755, 12: 808 / 814, 16: 985 / 933, 64: 2717 / 2170
//   160 of 4096 x 2048 (49)         8: 283 / 295, 12: 328 / 331, 24: 540 / 465, 96: 1535 / 1046
//   160 of 4096 x 1536 (37)         8: 200 / 215, 12: 273 / 284, 16: 344 / 333, 64: 866 / 636
//   128 of 4096 x 1280 (20)         16: 261 / 266, 24: 312 / 307, 32: 378 / 345, 96: 787 / 555
//   48 of 4096 x 5632 (12)          16: 363 / 396, 32: 538 / 535, 64: 834 / 694
//   32 of 4096 x 8192 (8)           32: 490 / 532, 48: 618 / 609, 64: 750 / 692
//   16 of 4096 x 10752 (3), 64 of 2048 x 1408 (3)     64: 474 / 492 and 139 / 169, 96: 624 / 620 and 189 / 193
// so they part at 480 by rows x experts x time.  (Where all experts are about as popular, rank^-0.3, later: 64 of 4096 x 4096 (16) 32:
// 476 / 509, 64: 770 / 819, 96: 1122 / 1016.)
// Few experts or light weights, which do not come to that before, turn from all short to all long at 96 rows (8 of 4096 x 14336 64:
// 321 / 345, 96: 398 / 421; 64 of 2048 x 1408 64: 139 / 169, 96: 189 / 202), the lightest later, at 3000 by rows x us (32 of 2048 x 1408,
// 21 us, 128: 120 / 129, 192: 160 / 152; 64 of 1024 x 1024, 15 us, 128: 114 / 119, 192: 156 / 148), but at 256 (8 of 1024 x 2048, 4 us,
// 128: 35 / 47, 256: 53 / 56, 512: 84 / 80).  Beyond, both take 3 to 6 % less than all long on 64 of 2048 x 1408, as much on 16 of
// 4096 x 10752, 2 to 12 % more on the others.
// Tiles of 32 or 48 rows, by rows an expert: 64 of 2048 x 1408 4: 47 / 51, 24: 92 / 91, 64: 156 / 139; 8 of 4096 x 14336 16: 146 / 160, 32:
// 219 / 215, 96: 423 / 398; 32 of 4096 x 8192 24: 413 / 465, 32: 490 / 535, 96: 1082 / 954; 16 of 4096 x 10752 16: 227 / 235, 32: 306 / 300.
inline Cut cut_of(const moegps_shape_t& s) {
  const int64_t R = (int64_t)s.T * s.K, experts = R < s.E ? R : s.E;
  const int64_t per = experts > 0 ? (R + experts - 1) / experts : 0;
  const bool padded = s.row_align > 32;
  const double rows = (double)(padded && per < s.row_align ? s.row_align : per);
  const int64_t d = chunks_of(s.D), f = chunks_of(s.F);
  const double weights_us = 0.0025 * s.E * (double)(f * d + (d + 1) / 2 * f);
  const double by_weights = 3e3 / weights_us, part = 480e3 / (s.E * weights_us);
  const double most = by_weights < 96.0 ? 96.0 : by_weights < 256.0 ? by_weights : 256.0;
  if (rows <= (part < most ? part : most)) return {rows <= 24.0 ? 32 : 48, INT32_MAX};
  return {32, part < most && !padded ? 32 : 0};        // (padded: no run is short)
}
constexpr int kLongRows = 224;

// Scale bytes of a tile's rows for one chunk, in the order of tensor memory (scale_byte_at).
// Tiles of up to 48 rows: both terms stacked in one group of 512 bytes, the second term's rows behind the first's, which are
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

// Tiles of up to 48 rows: for each tile and chunk the image that the products want in shared memory, the scales and behind them
// 128 bytes for each row, the first term's and then (from a multiple of 16 rows) the second's; the 16-byte pieces of a row are
// swizzled by the row's number.
template <int kRows>
constexpr int kImageBytes = kScaleTile + 2 * kRows * kChunk;
__host__ __device__ constexpr int image_code_at(int row, int term, int rows_in_tile, int piece) {
  return kScaleTile + (row + term * ((rows_in_tile + 15) / 16 * 16)) * kChunk + ((piece ^ (row % 8)) * 16);
}

inline size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

// Blocks of the launch for short runs: one for each SM, and not fewer (see Meeting in expert_ffn4.cu).  What they leave for each other
// in the workspace is sized by the most that are known, before a device is; more are refused (0).
constexpr int kMaxCtas = 160;
inline int short_blocks(int sm_count) { return sm_count <= kMaxCtas ? sm_count : 0; }

struct Layout {
  Cut cut;
  int64_t rows, short_tiles, long_tiles;       // Rcap; tiles of rows at most
  // offsets: images of x and h; what of h and of shared sums is there, their parts; codes (the second term's follow the first's) and
  // scales of x and h
  size_t x_image, h_image, part_there, h_there, partial, x_code, x_scale, h_code, h_scale, total;
  size_t x_code_bytes, h_code_bytes;
};

inline Layout layout_of(const moegps_shape_t& s) {
  Layout l;
  l.cut = cut_of(s);
  const int n = l.cut.tile_rows;
  l.rows = (int64_t)s.T * s.K + (int64_t)s.S * (s.row_align - 1);
  l.short_tiles = l.cut.all_short() ? l.rows / n + s.S : s.S * ((l.cut.short_rows + n - 1) / n);
  l.long_tiles = l.cut.all_short() ? 0 : l.rows / kLongRows + s.S;
  const size_t dc = chunks_of(s.D), fc = chunks_of(s.F), image = n == 32 ? kImageBytes<32> : kImageBytes<48>;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += align256(bytes);
    return here;
  };
  l.x_image = take(l.short_tiles * dc * image);
  l.h_image = take(l.short_tiles * fc * image);
  l.part_there = take(3 * kMaxCtas * sizeof(int32_t));
  l.h_there = take(l.short_tiles * fc * sizeof(int32_t));
  // a block leaves at most one unfinished tile of gate + up behind and two of down
  l.partial = take((size_t)kMaxCtas * 3 * 2 * n * kTile * sizeof(float));
  const size_t long_rows = l.cut.all_short() ? 0 : l.rows;
  l.x_code_bytes = align256(long_rows * dc * kChunk);
  l.h_code_bytes = align256(long_rows * fc * kChunk);
  l.x_code = take(2 * l.x_code_bytes);
  l.x_scale = take(l.long_tiles * dc * kRowScaleBytes<kLongRows>);
  l.h_code = take(2 * l.h_code_bytes);
  l.h_scale = take(l.long_tiles * fc * kRowScaleBytes<kLongRows>);
  l.total = at;
  return l;
}

}  // namespace mx4
