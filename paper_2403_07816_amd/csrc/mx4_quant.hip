// Tensors to microscaled 4-bit floats and back (layout: mx4.h).  Both directions are bound by the bytes they move: 2 (bf16) or 4 (fp32)
// of an element on one side, 17/32 on the other.
//   axis 1: blocks lie along the rows.  A thread has 8 consecutive elements, four threads a block: its largest magnitude by two DPP steps.
//   axis 0: blocks run down the columns, as the expert weights [K, N] are quantised, whose products sum over K; rows of the result
//           are the columns of the tensor.  A thread has 8 rows of 8 neighbouring columns (16 bytes a load or store of bf16), the four
//           threads of a quad a block of 32 rows in each of them; 64 columns x 256 rows go through LDS, so that 128 consecutive bytes of a
//           row of codes are moved at once.  Workgroups of neighbouring columns follow each other.  Four matrices [4096, 11008] of bf16
//           (361 MB, 96 MB of codes and scales): 87 us to 4 bits, 5.2 TB/s, and 68 us back, 6.7 TB/s.  With two columns a thread and
//           4 bytes a row of them it took 184 and 109 us, the latter also with 16 bytes a row as long as the values were put together
//           from the codes' bits and not by the conversion.
#include "mx4.h"

namespace btx {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kMostBlocks = 1 << 22;                // (a launch has fewer than 2^32 threads)

// ---- axis 1: [rows, K] --------------------------------------------------------------------------------------
// TILES: scales in mx4_scale_at()'s order
template <typename XT, bool TILES>
__device__ __forceinline__ void quantize_rows(int64_t block, const XT* __restrict__ x, int64_t rows, int64_t K, uint32_t* __restrict__ codes,
                                              uint8_t* __restrict__ scales, int64_t pitch) {
  // a row is cut into pieces of 8 elements, and rows are as long as their scales' pitch (whole 512 elements): what lies behind K
  // only writes the zeros behind the scales
  const int64_t per_row = pitch * 4, i = block * kThreads + threadIdx.x;
  const int64_t r = i / per_row;
  if (r >= rows) return;                               // whole blocks of four threads
  const int64_t p = i - r * per_row;
  float v[8];
  uint32_t amax = 0;
  const bool inside = p * 8 < K;
  if (inside) {
    RowVec<XT, 8>::ld_stream(x + r * K + p * 8, v);
#pragma unroll
    for (int q = 0; q < 8; ++q) amax = max(amax, magnitude(v[q]));
  }
  amax = max(amax, (uint32_t)dpp_i32<kDppXor1>((int)amax));
  amax = max(amax, (uint32_t)dpp_i32<kDppXor2>((int)amax));
  const uint32_t byte = mx4_scale_byte(amax);
  if (inside) codes[r * (K / 8) + p] = byte == 255u ? 0u : mx4_codes8(v, mx4_scale(byte));
  if ((threadIdx.x & 3) == 0) scales[TILES ? mx4_scale_at(rows, r, (int)(p / 4)) : r * pitch + p / 4] = inside ? (uint8_t)byte : 0;
}
template <typename XT>
__global__ __launch_bounds__(kThreads) void quantize_rows_kernel(const XT* __restrict__ x, int64_t rows, int64_t K, uint32_t* __restrict__ codes,
                                                                 uint8_t* __restrict__ scales, int64_t pitch) {
  for (int64_t b = blockIdx.x; b * kThreads < rows * pitch * 4; b += gridDim.x) quantize_rows<XT, false>(b, x, rows, K, codes, scales, pitch);
}

// The layer's first launch: its rows quantised, and beside them (the first blocks) the token of every grouped row and the row tiles
template <bool TILES>
__global__ __launch_bounds__(kThreads) void layer_begin_kernel(const bf16_t* __restrict__ x, int64_t T, int64_t d, uint32_t* __restrict__ codes,
                                                               uint8_t* __restrict__ scales, int64_t pitch, const int32_t* __restrict__ perm,
                                                               int R, int k, int token_blocks, int32_t* __restrict__ tokens,
                                                               const int32_t* __restrict__ offsets, int E, int tile_rows, TileInfo* __restrict__ tiles) {
  const int n_first = token_blocks + 1;
  if ((int)blockIdx.x >= n_first) {
    for (int64_t b = (int64_t)blockIdx.x - n_first; b * kThreads < T * pitch * 4; b += gridDim.x - n_first)
      quantize_rows<bf16_t, TILES>(b, x, T, d, codes, scales, pitch);
    return;
  }
  if ((int)blockIdx.x < token_blocks) {
    const int r = blockIdx.x * kThreads + threadIdx.x;
    if (r < R) tokens[r] = perm[r] / k;
    return;
  }
  __shared__ int s_wave[kThreads / kWave];              // thread e: expert e (E <= 256)
  const int e = threadIdx.x, lane = e & (kWave - 1);
  const int o0 = e < E ? offsets[e] : 0, o1 = e < E ? offsets[e + 1] : 0, n = (o1 - o0 + tile_rows - 1) / tile_rows;
  const int incl = wave_incl_scan_i32(n, lane);
  if (lane == kWave - 1) s_wave[e / kWave] = incl;
  __syncthreads();
  int at = 1 + incl - n;
  for (int w = 0; w < e / kWave; ++w) at += s_wave[w];
  for (int i = 0; i < n; ++i) tiles[at + i] = TileInfo{e, o0 + i * tile_rows, o1, 0};
  if (e == kThreads - 1) tiles[0] = TileInfo{0, at + n - 1, 0, 0};
}

__device__ __forceinline__ float scale_value(uint32_t byte) { return byte == 255u ? __uint_as_float(0x7fc00000u) : mx4_scale(byte); }
// The eight values of a word of codes; bf16: past its range (6 * 2^127 ...) or precision (below 2^-126) rounded once.  The hardware's
// conversion: exact for every code and every scale, 2^-127 and NaN among them (a test goes through all of them).
__device__ __forceinline__ void decode8(uint32_t w, float scale, float* v) {
  typedef __attribute__((ext_vector_type(2))) float f32x2;
  const f32x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1),
                      __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3)};
#pragma unroll
  for (int q = 0; q < 8; ++q) v[q] = p[q / 2][q % 2];
}

template <typename XT>
__global__ __launch_bounds__(kThreads) void dequantize_rows_kernel(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t rows,
                                                                   int64_t K, int64_t pitch, XT* __restrict__ out) {
  const int64_t per_row = K / 8;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < rows * per_row; i += (int64_t)gridDim.x * kThreads) {
    const int64_t r = i / per_row, p = i - r * per_row;
    float v[8];
    decode8(codes[i], scale_value(scales[r * pitch + p / 4]), v);
    RowVec<XT, 8>::st_stream(out + r * K + p * 8, v);
  }
}

// ---- axis 0: [batch, K, N] -> rows [batch, N] of K ------------------------------------------------------------
constexpr int kCols = 64, kBlocks = 8;                  // columns, blocks of 32 rows of a workgroup: 32 threads x 8
// Column c's codes of block b, in LDS: the threads that write or read at once, of eight columns' distance or of the same column, are
// on different banks
__device__ __forceinline__ int col_piece(int c, int b) { return b ^ (c >> 3 & 7); }
// Eight neighbouring elements of which n are there
template <typename XT, bool VEC> __device__ __forceinline__ void load8(const XT* p, int64_t n, float* v) {
  if constexpr (VEC) {
    RowVec<XT, 8>::ld_stream(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? Elem<XT>::ld(p + i) : 0.f;
  }
}
// grid: (pieces of 64 columns of 256 rows, the rows' pieces one after another, batch).  VEC: rows of whole 16 bytes.  A thread has 8 rows of 8 neighbouring columns,
// the four lanes of a quad the 32 rows of a block.
template <typename XT, bool VEC>
__global__ __launch_bounds__(kThreads) void quantize_cols_kernel(const XT* __restrict__ x, int64_t K, int64_t N, u32x4* __restrict__ codes,
                                                                 uint8_t* __restrict__ scales, int64_t pitch, unsigned col_pieces) {
  __shared__ u32x4 s_codes[kCols][kBlocks];
  __shared__ uint8_t s_scales[kCols][kBlocks];
  const int quarter = threadIdx.x & 3, c = (threadIdx.x >> 2 & 7) * 8, b = threadIdx.x / 32;
  const int64_t piece = blockIdx.x / col_pieces, col0 = (int64_t)(blockIdx.x - piece * col_pieces) * kCols, blk0 = piece * kBlocks;
  const int64_t col = col0 + c, blk = blk0 + b, n_blk = K / kMxBlock, batch = blockIdx.y;
  x += batch * K * N;
  if (blk < n_blk && col < N) {                         // (whole quads)
    const XT* const from = x + (blk * kMxBlock + quarter * 8) * N + col;
    float v[8][8];
#pragma unroll
    for (int q = 0; q < 8; ++q) load8<XT, VEC>(from + (int64_t)q * N, N - col, v[q]);
#pragma unroll
    for (int h = 0; h < 8; ++h) {
      float w[8];
      uint32_t amax = 0;
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        w[q] = v[q][h];
        amax = max(amax, magnitude(w[q]));
      }
      amax = max(amax, (uint32_t)dpp_i32<kDppXor1>((int)amax));
      amax = max(amax, (uint32_t)dpp_i32<kDppXor2>((int)amax));
      const uint32_t byte = mx4_scale_byte(amax);
      reinterpret_cast<uint32_t*>(&s_codes[c + h][col_piece(c + h, b)])[quarter] = byte == 255u ? 0u : mx4_codes8(w, mx4_scale(byte));
      if (quarter == 0) s_scales[c + h][b] = (uint8_t)byte;
    }
  }
  __syncthreads();
  codes += batch * N * n_blk;
  scales += batch * N * pitch;
#pragma unroll
  for (int i = threadIdx.x; i < kCols * kBlocks; i += kThreads) {
    const int q = i % kBlocks;
    const int64_t n = col0 + i / kBlocks, k = blk0 + q;
    if (n >= N) continue;
    if (k < n_blk) codes[n * n_blk + k] = s_codes[i / kBlocks][col_piece(i / kBlocks, q)];
    if (k < pitch) scales[n * pitch + k] = k < n_blk ? s_scales[i / kBlocks][q] : 0;
  }
}

template <typename XT, bool VEC>
__global__ __launch_bounds__(kThreads) void dequantize_cols_kernel(const u32x4* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t K, int64_t N,
                                                                   int64_t pitch, XT* __restrict__ out, unsigned col_pieces) {
  __shared__ u32x4 s_codes[kCols][kBlocks];
  __shared__ uint8_t s_scales[kCols][kBlocks];
  const int64_t n_blk = K / kMxBlock, batch = blockIdx.y;
  const int64_t piece = blockIdx.x / col_pieces, col0 = (int64_t)(blockIdx.x - piece * col_pieces) * kCols, blk0 = piece * kBlocks;
  codes += batch * N * n_blk;
  scales += batch * N * pitch;
#pragma unroll
  for (int i = threadIdx.x; i < kCols * kBlocks; i += kThreads) {
    const int q = i % kBlocks;
    const int64_t n = col0 + i / kBlocks, k = blk0 + q;
    if (n < N && k < n_blk) {
      s_codes[i / kBlocks][col_piece(i / kBlocks, q)] = codes[n * n_blk + k];
      s_scales[i / kBlocks][q] = scales[n * pitch + k];
    }
  }
  __syncthreads();
  const int quarter = threadIdx.x & 3, c = (threadIdx.x >> 2 & 7) * 8, b = threadIdx.x / 32;
  const int64_t col = col0 + c, blk = blk0 + b;
  if (blk >= n_blk || col >= N) return;
  XT* const to = out + batch * K * N + (blk * kMxBlock + quarter * 8) * N + col;
  float v[8][8];
#pragma unroll
  for (int h = 0; h < 8; ++h) {
    float w[8];                                         // (of columns behind the last one: whatever is there, and not written)
    decode8(reinterpret_cast<const uint32_t*>(&s_codes[c + h][col_piece(c + h, b)])[quarter], scale_value(s_scales[c + h][b]), w);
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q][h] = w[q];
  }
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    if constexpr (VEC) {
      RowVec<XT, 8>::st_stream(to + (int64_t)q * N, v[q]);
    } else {
#pragma unroll
      for (int h = 0; h < 8; ++h)
        if (col + h < N) Elem<XT>::st(to + (int64_t)q * N + h, v[q][h]);
    }
  }
}

}  // namespace

int launch_mx4_quantize(const void* x, int dtype, int64_t batch, int64_t rows, int64_t cols, int axis, uint8_t* codes, uint8_t* scales,
                        hipStream_t s) {
  const int64_t K = axis == 1 ? cols : rows, pitch = mx4_pitch(K);
  if (axis == 1) {
    const int64_t n = batch * rows, blocks = std::min((n * pitch * 4 + kThreads - 1) / kThreads, kMostBlocks);
    if (dtype == BTX_BF16)
      quantize_rows_kernel<<<(unsigned)blocks, kThreads, 0, s>>>(static_cast<const bf16_t*>(x), n, K, reinterpret_cast<uint32_t*>(codes), scales, pitch);
    else
      quantize_rows_kernel<<<(unsigned)blocks, kThreads, 0, s>>>(static_cast<const float*>(x), n, K, reinterpret_cast<uint32_t*>(codes), scales, pitch);
  } else {
    const int64_t gx = (cols + kCols - 1) / kCols, gy = (pitch + kBlocks - 1) / kBlocks;
    if (gx > 65535 || !grid_fits(gx * gy, kThreads) || batch > 65535) return BTX_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)(gx * gy), (unsigned)batch);
    const bool vec = cols % 8 == 0;
    u32x4* const c = reinterpret_cast<u32x4*>(codes);
    auto go = [&](auto tag) {
      using XT = decltype(tag);
      if (vec) quantize_cols_kernel<XT, true><<<grid, kThreads, 0, s>>>(static_cast<const XT*>(x), K, cols, c, scales, pitch, (unsigned)gx);
      else quantize_cols_kernel<XT, false><<<grid, kThreads, 0, s>>>(static_cast<const XT*>(x), K, cols, c, scales, pitch, (unsigned)gx);
    };
    if (dtype == BTX_BF16) go(bf16_t{});
    else go(float{});
  }
  BTX_LAUNCH_CHECK();
  return BTX_OK;
}

int launch_mx4_begin(const void* x, const int32_t* perm, const int32_t* offsets, const Mx4Shapes& sh, uint8_t* x_codes, uint8_t* x_scales,
                     int32_t* tokens, TileInfo* tiles, hipStream_t s) {
  static_assert(kMx4MaxExperts <= kThreads, "one thread an expert");
  const int R = sh.T * sh.k, token_blocks = ceil_div(R, kThreads);
  static_assert((kMx4MostRows / kThreads + 2 + kMostBlocks) * kThreads < 1ll << 32, "the grid");
  const int64_t pitch = mx4_pitch(sh.d);
  if (sh.T * pitch >= kMx4MostScales) return BTX_ERR_UNSUPPORTED;
  const int64_t blocks = token_blocks + 1 + std::min((sh.T * pitch * 4 + kThreads - 1) / kThreads, kMostBlocks);
  const bf16_t* const xp = static_cast<const bf16_t*>(x);
  uint32_t* const codes = reinterpret_cast<uint32_t*>(x_codes);
  const int tile_rows = mx4_tile_rows(sh);
  if (tile_rows == 256)
    layer_begin_kernel<true><<<(unsigned)blocks, kThreads, 0, s>>>(xp, sh.T, sh.d, codes, x_scales, pitch, perm, R, sh.k, token_blocks, tokens, offsets,
                                                                   sh.E, tile_rows, tiles);
  else
    layer_begin_kernel<false><<<(unsigned)blocks, kThreads, 0, s>>>(xp, sh.T, sh.d, codes, x_scales, pitch, perm, R, sh.k, token_blocks, tokens, offsets,
                                                                    sh.E, tile_rows, tiles);
  BTX_LAUNCH_CHECK();
  return BTX_OK;
}

int launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, int dtype, int64_t batch, int64_t rows, int64_t cols, int axis, void* out,
                          hipStream_t s) {
  const int64_t K = axis == 1 ? cols : rows, pitch = mx4_pitch(K);
  if (axis == 1) {
    const int64_t n = batch * rows, blocks = std::min((n * (K / 8) + kThreads - 1) / kThreads, kMostBlocks);
    const uint32_t* const c = reinterpret_cast<const uint32_t*>(codes);
    if (dtype == BTX_BF16) dequantize_rows_kernel<<<(unsigned)blocks, kThreads, 0, s>>>(c, scales, n, K, pitch, static_cast<bf16_t*>(out));
    else dequantize_rows_kernel<<<(unsigned)blocks, kThreads, 0, s>>>(c, scales, n, K, pitch, static_cast<float*>(out));
  } else {
    const int64_t gx = (cols + kCols - 1) / kCols, gy = (K / kMxBlock + kBlocks - 1) / kBlocks;
    if (gx > 65535 || !grid_fits(gx * gy, kThreads) || batch > 65535) return BTX_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)(gx * gy), (unsigned)batch);
    const u32x4* const c = reinterpret_cast<const u32x4*>(codes);
    const bool vec = cols % 8 == 0;
    auto go = [&](auto tag) {
      using XT = decltype(tag);
      if (vec) dequantize_cols_kernel<XT, true><<<grid, kThreads, 0, s>>>(c, scales, K, cols, pitch, static_cast<XT*>(out), (unsigned)gx);
      else dequantize_cols_kernel<XT, false><<<grid, kThreads, 0, s>>>(c, scales, K, cols, pitch, static_cast<XT*>(out), (unsigned)gx);
    };
    if (dtype == BTX_BF16) go(bf16_t{});
    else go(float{});
  }
  BTX_LAUNCH_CHECK();
  return BTX_OK;
}

}  // namespace btx
