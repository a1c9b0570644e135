// Microscaled 4-bit floats (MXFP4): e2m1 codes, two to a byte, and one power of two (e8m0) for every 32 of them.
//   codes  [rows][K / 2]           element 2i in the low half of byte i
//   scales [rows][mx4_pitch(K)]    byte b: 2^(b - 127), 255: NaN; K / 32 of them, the rest of the row zero
#pragma once
#include "common.h"

namespace btx {

constexpr int kMxBlock = 32;
constexpr int kMx4MaxExperts = 256;
constexpr int kMx4MostRows = (1 << 28) - 256;         // T k: 32-bit offsets of 16 bytes a row, grids of every tile's height
constexpr int64_t kMx4MostScales = 1 << 30;           // bytes of x's scales; the layer takes fewer
constexpr int kMx4MostColumns = 65535 * 32;           // d and f: rows of the grid of few rows, and 32-bit offsets in a row tile
// bytes from a row of scales to the next: whole 16-byte pieces, which the products copy (one holds the scales of 512 elements)
inline __host__ __device__ int64_t mx4_pitch(int64_t K) { return (K / kMxBlock + 15) / 16 * 16; }

// The scale byte of a block whose largest magnitude has these bits: floor(log2(amax)) - 2, so that amax lies in [4, 8) units and what
// is above 6 of them saturates; at least 2^-127 (byte 0); a block with an infinity or a NaN has a NaN for a scale.
__device__ __forceinline__ uint32_t mx4_scale_byte(uint32_t amax_bits) {
  const uint32_t exponent = amax_bits >> 23;            // (the sign is not in it)
  return exponent == 255u ? 255u : (uint32_t)max((int)exponent - 2, 0);
}
__device__ __forceinline__ float mx4_scale(uint32_t byte) { return byte ? __uint_as_float(byte << 23) : 5.877471754111438e-39f; }
// magnitude of a float as the integer that orders it; NaN above infinity
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Eight floats -> eight codes (value / scale rounded to nearest even, saturating at 6; the hardware's conversion)
__device__ __forceinline__ uint32_t mx4_codes8(const float* v, float scale) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
}

int launch_mx4_quantize(const void* x, int dtype, int64_t batch, int64_t rows, int64_t cols, int axis, uint8_t* codes, uint8_t* scales,
                        hipStream_t s);
int launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, int dtype, int64_t batch, int64_t rows, int64_t cols, int axis, void* out,
                          hipStream_t s);

// The layer of 4-bit experts (mx4_gemm.hip)
int mx4_prepare();                     // one-time set-up on the current device (not capturable)
struct Mx4Shapes { int T, d, f, E, k; };
struct Mx4Matrix { const uint8_t* codes; const uint8_t* scales; };
struct TileInfo { int e, row0, row_end, unused; };      // of an expert's rows the tile has those from row0 on, row_end is the expert's end
inline int mx4_most_tiles(int R, int E, int tile_rows) { return (int)std::min<int64_t>((int64_t)R / tile_rows + std::min(E, R), R); }
// Rows of a row tile: 256 (the products take tiles of them; x and act have their scales in another order then, mx4_scale_at()), 64 or 32
int mx4_tile_rows(const Mx4Shapes& sh);
// Where the scale of block b of a row is in that order: 16 bytes of every row for 16 blocks (two k tiles), in them those of blocks 2g, 2g + 1,
// 8 + 2g and 9 + 2g together, which lane group g takes.
inline __device__ int64_t mx4_scale_at(int64_t rows, int64_t row, int b) {
  return ((int64_t)(b >> 4) * rows + row) * 16 + (((b >> 1) & 3) << 2) + (((b >> 3) & 1) << 1) + (b & 1);
}
// What the layer's first kernel writes: x quantised, the token of every grouped row, and the row tiles (in entry 0, row0: their number)
struct Mx4Layer { Mx4Matrix x; const int32_t* tokens; const TileInfo* tiles; uint8_t* act_codes; uint8_t* act_scales; void* y; };
int launch_mx4_begin(const void* x, const int32_t* perm, const int32_t* offsets, const Mx4Shapes& sh, uint8_t* x_codes, uint8_t* x_scales,
                     int32_t* tokens, TileInfo* tiles, hipStream_t s);
// act = silu(xq W1) * (xq W3), quantised along f: rows in grouped order
int launch_mx4_up(const Mx4Layer& l, const Mx4Matrix& W1, const Mx4Matrix& W3, const Mx4Shapes& sh, hipStream_t s);
// y = act W2, [T*k, d] bf16; or *slices > 1 of its sums in fp32 instead, [slice][T*k, d], for launch_combine() to add and weigh without
// rounding them.  l.y: mx4_y_bytes(R, d)
constexpr int64_t kMx4SumBytes = (int64_t)256 * 256 * 256 * 4;       // of 256 tiles
inline size_t mx4_y_bytes(int64_t R, int d) { return (size_t)std::max(R * d * 2, std::min(R * d * 4 * 8, kMx4SumBytes)); }
int launch_mx4_down(const Mx4Layer& l, const Mx4Matrix& W2, const Mx4Shapes& sh, int* slices, hipStream_t s);

}  // namespace btx
