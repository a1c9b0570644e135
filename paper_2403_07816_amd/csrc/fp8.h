// Block-scaled 8-bit floats: e4m3 codes (largest 448), and one power of two (e8m0) for every 128 of them along the axis that products sum over.
//   codes  [rows][f8_pitch(K)]         zeros behind K: products take whole blocks
//   scales [rows][f8_scale_pitch(K)]   byte b: 2^(b - 127), 255: NaN; ceil(K / 128) of them, the rest of the row zero
#pragma once
#include "common.h"

namespace btx {

constexpr int kF8Block = 128;
constexpr int kF8MaxExperts = 256;
constexpr int kF8MostRows = (1 << 28) - 256;          // T k, M: the grid of a product of few columns
constexpr int kF8MostColumns = 65535 * 32;            // N, d, f and K: 32-bit offsets in a tile of 256 rows
inline __host__ __device__ int64_t f8_pitch(int64_t K) { return (K + kF8Block - 1) / kF8Block * kF8Block; }
// whole 16-byte pieces, which the products copy
inline __host__ __device__ int64_t f8_scale_pitch(int64_t K) { return ((K + kF8Block - 1) / kF8Block + 15) / 16 * 16; }

// The scale byte of a block whose largest magnitude has these bits: the smallest power of two of which it is at most 448 = 1.75 * 2^8 times, so
// that nothing saturates; at least 2^-127 (byte 0); a block with an infinity or a NaN has a NaN for a scale.  (Adding 0x1fffff carries
// into the exponent where the significand is above 1.75.)
__device__ __forceinline__ uint32_t f8_scale_byte(uint32_t amax_bits) {
  return amax_bits >= 0x7f800000u ? 255u : (uint32_t)max((int)((amax_bits + 0x1fffffu) >> 23) - 8, 0);
}
__device__ __forceinline__ float f8_scale(uint32_t byte) { return byte ? __uint_as_float(byte << 23) : 5.877471754111438e-39f; }
// magnitude of a float as the integer that orders it; NaN above infinity
__device__ __forceinline__ uint32_t f8_magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Four floats -> four codes (value / scale, exact, rounded to nearest even; the hardware's conversion)
__device__ __forceinline__ uint32_t f8_codes4(float a, float b, float c, float d, float scale) {
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  s16x2 w = {0, 0};
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, a, b, scale, false);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, scale, true);
  return __builtin_bit_cast(uint32_t, w);
}
// The codes of a block with this scale byte: none of a block that is NaN
__device__ __forceinline__ uint32_t f8_codes4(const float* v, uint32_t byte) {
  return byte == 255u ? 0u : f8_codes4(v[0], v[1], v[2], v[3], f8_scale(byte));
}
// the largest of the 16 lanes of a DPP row
__device__ __forceinline__ uint32_t f8_row_max(uint32_t v) {
  v = max(v, (uint32_t)dpp_i32<kDppXor1>((int)v));
  v = max(v, (uint32_t)dpp_i32<kDppXor2>((int)v));
  v = max(v, (uint32_t)dpp_i32<kDppRor4>((int)v));
  return max(v, (uint32_t)dpp_i32<kDppRor8>((int)v));
}
// the largest of the four lanes that are 16 apart (the halves, then the odd and even rows of 16 change places: no trip through LDS)
__device__ __forceinline__ uint32_t f8_across_max(uint32_t v) {
  const auto a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  v = max(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return max(b[0], b[1]);
}

struct F8Matrix { const uint8_t* codes; const uint8_t* scales; };

int launch_f8_quantize(const void* x, int dtype, int64_t batch, int64_t rows, int64_t cols, int axis, int block_rows, uint8_t* codes,
                       uint8_t* scales, hipStream_t s);
int launch_f8_dequantize(const uint8_t* codes, const uint8_t* scales, int dtype, int64_t batch, int64_t rows, int64_t cols, int axis, void* out,
                         hipStream_t s);
// sum = h + residual (may be NULL: h), rstd, xn = gain * sum * rstd, codes and scales of xn; sum, xn, codes with scales may be NULL
struct F8NormArgs {
  const void* h; const void* residual; int dtype; const float* gain; float eps; int T, d;
  void* sum; void* xn; float* rstd; uint8_t* codes; uint8_t* scales;
};
constexpr int kF8NormMostColumns = 16384;
int launch_f8_norm(const F8NormArgs& a, hipStream_t s);

// out [M, N] = a b^T (+ residual)
struct F8Matmul { F8Matrix a, b; int M, N, K; const void* residual; void* out; int dtype; void* workspace; };
size_t f8_matmul_workspace_bytes(int M, int N, int K);
int launch_f8_matmul(const F8Matmul& m, hipStream_t s);

// The layer of 8-bit experts.  Rows of x are found with 32-bit offsets in tiles of 256: the last one's, 112 bytes of a chunk and the copies' bias
constexpr int64_t kF8MostTokenBytes = ((int64_t)1 << 32) - 2048;
struct F8Layer {
  F8Matrix x, W1, W3, W2; int T, d, f, E, k; const int32_t* offsets; const int32_t* perm;
  uint8_t* act_codes; uint8_t* act_scales; void* y;
};
int launch_f8_up(const F8Layer& l, hipStream_t s);
// y = act W2, [T*k, d] bf16; or *slices > 0 sums of it in fp32 instead, [slice][T*k, d], for launch_combine() to add and weigh without rounding them
size_t f8_y_bytes(int64_t R, int d, int f, int E);
int launch_f8_down(const F8Layer& l, int* slices, hipStream_t s);
int f8_prepare();                      // one-time set-up on the current device (not capturable)

}  // namespace btx
