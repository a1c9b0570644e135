// Tensors to block-scaled 8-bit floats and back (layout: fp8.h).  Both directions are bound by the bytes they move: 2 (bf16) or 4 (fp32) of an
// element on one side, 129/128 on the other.
//   axis 1: blocks lie along the rows.  A thread has 8 consecutive elements, a DPP row of 16 lanes a block.
//   axis 0: blocks run down the columns, rows of the result are columns of the tensor: a workgroup has 128 x 128 elements, a thread 8 rows of
//           8 neighbouring columns (16 bytes a load or store of bf16, 256 a row of the workgroup's), and whole 128 bytes of every row of
//           codes go through LDS.
// block_rows 128: the 128 rows of the result that share a scale are one workgroup's.
// bf16, there and back: 2^30 elements along rows 5.9 and 5.8 TB/s, down columns 5.2 and 5.3; 4 x 4096 x 11008 down columns in 128 x 128 blocks 91 us each way;
// 4001 x 4096 down columns 11.8 us (992 workgroups, one round of the chip) and 7.5.
// Rows whose length is no multiple of 8 begin anywhere and move an element at a time: 2^28 elements in rows of 4097, bf16, there and back 3.3 and 2.2 TB/s along
// them, 2.8 and 1.9 down columns; fp32 2.9 and 2.0, 2.8 and 1.9.  (Widths are multiples of 8; a ragged number of tokens is a number of rows.)
#include "fp8.h"

#include <type_traits>

namespace btx {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int64_t kMostBlocks = 1 << 22;                // (a launch has fewer than 2^32 threads)
constexpr int kTile = kF8Block;

// Elements at, at + 1, .. + 7 of a row of `cols`, zeros where there is none; VEC: rows of whole 8.  (Without a branch around a load: behind one, the
// next waits for it.)
template <typename XT, bool VEC> __device__ __forceinline__ void load8(const XT* row, int64_t at, int64_t cols, bool there, float* v) {
  if constexpr (VEC) {
    const XT* const p = row + min(at, cols - 8);
    if constexpr (sizeof(XT) == 2) RowVec<XT, 8>::ld_stream(p, v);
    else RowVec<XT, 8>::ld(p, v);                        // (two loads, of every other 16 bytes)
    const bool is = there && at < cols;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = is ? v[i] : 0.f;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = Elem<XT>::ld(row + min(at + i, cols - 1));
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = there && at + i < cols ? v[i] : 0.f;
  }
}
template <typename XT, bool VEC> __device__ __forceinline__ void store8(XT* p, int64_t n, const float* v) {
  if (VEC && n >= 8) {
    if constexpr (sizeof(XT) == 2) RowVec<XT, 8>::st_stream(p, v);
    else RowVec<XT, 8>::st(p, v);                        // (two stores, of every other 16 bytes; streamed, 16384 x 4096 took 94 us for 61)
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) Elem<XT>::st(p + i, v[i]);
  }
}
// the zeros behind a row's scales: at most 15, one of each of a DPP row's lanes
__device__ __forceinline__ void zero_scales(uint8_t* row, int64_t n_blk, int64_t pitch, int lane16) {
  if (n_blk + lane16 < pitch) row[n_blk + lane16] = 0;
}

// ---- axis 1: [rows, K] ----------------------------------------------------------------------------------------
template <typename XT, bool VEC>
__global__ __launch_bounds__(kThreads) void f8_quantize_rows_kernel(const XT* __restrict__ x, int64_t rows, int64_t K, u32x2* __restrict__ codes,
                                                                    uint8_t* __restrict__ scales) {
  const int64_t per_row = f8_pitch(K) / 8, n_blk = per_row / 16, pitch = f8_scale_pitch(K);
  // (rows are whole DPP rows of lanes)
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < rows * per_row; i += (int64_t)gridDim.x * kThreads) {
    const int64_t r = i / per_row, p = i - r * per_row, b = p / 16;
    float v[8];
    load8<XT, VEC>(x + r * K, p * 8, K, true, v);
    uint32_t amax = 0;
#pragma unroll
    for (int q = 0; q < 8; ++q) amax = max(amax, f8_magnitude(v[q]));
    const uint32_t byte = f8_scale_byte(f8_row_max(amax));
    codes[i] = u32x2{f8_codes4(v, byte), f8_codes4(v + 4, byte)};
    uint8_t* const sc = scales + r * pitch;
    if ((threadIdx.x & 15) == 0) sc[b] = (uint8_t)byte;
    if (b + 1 == n_blk) zero_scales(sc, n_blk, pitch, threadIdx.x & 15);
  }
}

// 128 x 128 elements that share a scale; grid: (blocks along the rows, then the rows' blocks; batch)
template <typename XT, bool VEC>
__global__ __launch_bounds__(kThreads) void f8_quantize_tile_rows_kernel(const XT* __restrict__ x, int64_t rows, int64_t K, u32x2* __restrict__ codes,
                                                                         uint8_t* __restrict__ scales) {
  __shared__ uint32_t s_amax[kWaves];
  const int64_t n_blk = f8_pitch(K) / kF8Block, pitch = f8_scale_pitch(K);
  const int64_t piece = blockIdx.x / n_blk, b = blockIdx.x - piece * n_blk, batch = blockIdx.y;
  const int lane16 = threadIdx.x & 15;
  const int64_t k0 = b * kF8Block + lane16 * 8;
  constexpr int STEP = kThreads / 16, N = kTile / STEP;
  float v[N][8];
  uint32_t amax = 0;
#pragma unroll
  for (int q = 0; q < N; ++q) {
    const int64_t r = piece * kTile + q * STEP + threadIdx.x / 16;
    load8<XT, VEC>(x + (batch * rows + min(r, rows - 1)) * K, k0, K, r < rows, v[q]);
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = max(amax, f8_magnitude(v[q][i]));
  }
#pragma unroll
  for (int m = 1; m < kWave; m *= 2) amax = max(amax, (uint32_t)__shfl_xor((int)amax, m, kWave));
  if ((threadIdx.x & (kWave - 1)) == 0) s_amax[threadIdx.x / kWave] = amax;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) amax = max(amax, s_amax[w]);
  const uint32_t byte = f8_scale_byte(amax);
#pragma unroll
  for (int q = 0; q < N; ++q) {
    const int64_t r = piece * kTile + q * STEP + threadIdx.x / 16;
    if (r >= rows) break;
    const int64_t row = batch * rows + r;
    codes[(row * n_blk + b) * 16 + lane16] = u32x2{f8_codes4(v[q], byte), f8_codes4(v[q] + 4, byte)};
    uint8_t* const sc = scales + row * pitch;
    if (lane16 == 0) sc[b] = (uint8_t)byte;
    if (b + 1 == n_blk) zero_scales(sc, n_blk, pitch, lane16);
  }
}

// The eight values of eight codes; bf16: past its range or precision (below 2^-126) rounded once
__device__ __forceinline__ void decode8(const u32x2& w, uint32_t byte, float* v) {
  typedef __attribute__((ext_vector_type(2))) float f32x2;
  const float scale = byte == 255u ? __uint_as_float(0x7fc00000u) : f8_scale(byte);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[h], scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[h], scale, true);
    v[4 * h] = lo[0];
    v[4 * h + 1] = lo[1];
    v[4 * h + 2] = hi[0];
    v[4 * h + 3] = hi[1];
  }
}

template <typename XT, bool VEC>
__global__ __launch_bounds__(kThreads) void f8_dequantize_rows_kernel(const u32x2* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t rows,
                                                                      int64_t K, XT* __restrict__ out) {
  const int64_t per_row = f8_pitch(K) / 8, pitch = f8_scale_pitch(K);
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < rows * per_row; i += (int64_t)gridDim.x * kThreads) {
    const int64_t r = i / per_row, p = i - r * per_row;
    if (p * 8 >= K) continue;
    float v[8];
    decode8(codes[i], scales[r * pitch + p / 16], v);
    store8<XT, VEC>(out + r * K + p * 8, K - p * 8, v);
  }
}

// ---- axis 0: [batch, K, N] -> rows [batch, N] of K ------------------------------------------------------------
// Thread: 8 rows (kq) of 8 columns (cq); a wavefront has 4 x 16 of these pieces.
// Where 8 codes (kq) of a column lie in LDS: 16-byte chunks are XOR-swizzled by the column's eight
__device__ __forceinline__ int col_at(int c, int kq) { return c * kTile + (((kq >> 1) ^ (c >> 3 & 7)) << 4) + ((kq & 1) << 3); }

// grid: (pieces of 128 columns, then the rows' pieces; batch)
template <typename XT, bool VEC, bool SHARED>
__global__ __launch_bounds__(kThreads) void f8_quantize_cols_kernel(const XT* __restrict__ x, int64_t K, int64_t N, uint8_t* __restrict__ codes,
                                                                    uint8_t* __restrict__ scales, unsigned col_pieces) {
  __shared__ __attribute__((aligned(16))) uint8_t s_codes[kTile * kTile];
  __shared__ u32x4 s_amax[8][kTile / 8];                // of column 8 cq + h at [h][cq], or in the first of all: the four wavefronts'
  __shared__ uint8_t s_scale[kTile];
  static_assert(kWaves == 4, "u32x4");
  const int64_t b = blockIdx.x / col_pieces, col0 = (int64_t)(blockIdx.x - b * col_pieces) * kTile, batch = blockIdx.y;
  const int64_t n_blk = f8_pitch(K) / kF8Block, pitch = f8_scale_pitch(K);
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, cq = lane & 15, kq = wave * 4 + lane / 16;
  const int64_t col = col0 + cq * 8, k0 = b * kF8Block + kq * 8;
  const XT* const from = x + batch * K * N;
  float v[8][8];
#pragma unroll
  for (int q = 0; q < 8; ++q) load8<XT, VEC>(from + min(k0 + q, K - 1) * N, col, N, k0 + q < K, v[q]);
  uint32_t amax[8];
#pragma unroll
  for (int h = 0; h < 8; ++h) {
    amax[h] = 0;
#pragma unroll
    for (int q = 0; q < 8; ++q) amax[h] = max(amax[h], f8_magnitude(v[q][h]));
    amax[h] = f8_across_max(amax[h]);
  }
  if constexpr (SHARED) {
    uint32_t all = 0;
#pragma unroll
    for (int h = 0; h < 8; ++h) all = max(all, amax[h]);
    all = f8_row_max(all);
    if (lane == 0) reinterpret_cast<uint32_t*>(&s_amax[0][0])[wave] = all;
  } else if (lane < 16) {
#pragma unroll
    for (int h = 0; h < 8; ++h) reinterpret_cast<uint32_t*>(&s_amax[h][cq])[wave] = amax[h];
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 8; ++h) {
    const int c = cq * 8 + h;
    const u32x4 four = SHARED ? s_amax[0][0] : s_amax[h][cq];
    const uint32_t byte = f8_scale_byte(max(max(four[0], four[1]), max(four[2], four[3])));
    float w[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) w[q] = v[q][h];
    *reinterpret_cast<u32x2*>(s_codes + col_at(c, kq)) = u32x2{f8_codes4(w, byte), f8_codes4(w + 4, byte)};
    if (kq == 0) s_scale[c] = (uint8_t)byte;
  }
  __syncthreads();
#pragma unroll
  for (int i = threadIdx.x; i < kTile * 8; i += kThreads) {
    const int c = i / 8, q = i % 8;
    const int64_t n = col0 + c;
    if (n < N) *reinterpret_cast<u32x4*>(codes + ((batch * N + n) * n_blk + b) * kF8Block + q * 16) = *reinterpret_cast<const u32x4*>(s_codes + col_at(c, 2 * q));
  }
  if (threadIdx.x < kTile && col0 + threadIdx.x < N) {
    uint8_t* const sc = scales + (batch * N + col0 + threadIdx.x) * pitch;
    sc[b] = s_scale[threadIdx.x];
    if (b + 1 == n_blk)
      for (int64_t z = n_blk; z < pitch; ++z) sc[z] = 0;
  }
}

template <typename XT, bool VEC>
__global__ __launch_bounds__(kThreads) void f8_dequantize_cols_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t K,
                                                                      int64_t N, XT* __restrict__ out, unsigned col_pieces) {
  __shared__ __attribute__((aligned(16))) uint8_t s_codes[kTile * kTile];
  __shared__ uint8_t s_scale[kTile];
  const int64_t b = blockIdx.x / col_pieces, col0 = (int64_t)(blockIdx.x - b * col_pieces) * kTile, batch = blockIdx.y;
  const int64_t n_blk = f8_pitch(K) / kF8Block, pitch = f8_scale_pitch(K);
#pragma unroll
  for (int i = threadIdx.x; i < kTile * 8; i += kThreads) {
    const int c = i / 8, q = i % 8;
    const int64_t n = min(col0 + c, N - 1);
    *reinterpret_cast<u32x4*>(s_codes + col_at(c, 2 * q)) =
        __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(codes + ((batch * N + n) * n_blk + b) * kF8Block + q * 16));
  }
  if (threadIdx.x < kTile) s_scale[threadIdx.x] = scales[(batch * N + min(col0 + threadIdx.x, N - 1)) * pitch + b];
  __syncthreads();
  const int lane = threadIdx.x & (kWave - 1), cq = lane & 15, kq = threadIdx.x / kWave * 4 + lane / 16;
  const int64_t col = col0 + cq * 8, k0 = b * kF8Block + kq * 8;
  if (col >= N) return;
  float v[8][8];
#pragma unroll
  for (int h = 0; h < 8; ++h) {
    const int c = cq * 8 + h;
    float w[8];
    decode8(*reinterpret_cast<const u32x2*>(s_codes + col_at(c, kq)), s_scale[c], w);
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q][h] = w[q];
  }
#pragma unroll
  for (int q = 0; q < 8; ++q)
    if (k0 + q < K) store8<XT, VEC>(out + (batch * K + k0 + q) * N + col, N - col, v[q]);
}

// tiles of 128 x 128, `inner` of them beside each other in the grid
int tile_grid(int64_t inner, int64_t outer, int64_t batch, dim3* grid) {
  if (inner > (1 << 24) || outer > (1 << 24) || !grid_fits(inner * outer, kThreads) || batch > 65535) return BTX_ERR_UNSUPPORTED;
  *grid = dim3((unsigned)(inner * outer), (unsigned)batch);
  return BTX_OK;
}
int64_t tiles_of(int64_t n) { return (n + kTile - 1) / kTile; }

// go(element type, rows of whole 8 elements)
template <typename Go> void by_type(int dtype, int64_t cols, Go go) {
  auto typed = [&](auto tag) {
    if (cols % 8 == 0) go(tag, std::true_type{});
    else go(tag, std::false_type{});
  };
  if (dtype == BTX_BF16) typed(bf16_t{});
  else typed(float{});
}

}  // namespace

int launch_f8_quantize(const void* x, int dtype, int64_t batch, int64_t rows, int64_t cols, int axis, int block_rows, uint8_t* codes,
                       uint8_t* scales, hipStream_t s) {
  dim3 grid;
  if (axis == 0) {
    const int64_t pieces = tiles_of(cols);
    if (int rc = tile_grid(pieces, tiles_of(rows), batch, &grid)) return rc;
    by_type(dtype, cols, [&](auto tag, auto vec) {
      using XT = decltype(tag);
      constexpr bool VEC = decltype(vec)::value;
      const XT* const p = static_cast<const XT*>(x);
      if (block_rows > 1) f8_quantize_cols_kernel<XT, VEC, true><<<grid, kThreads, 0, s>>>(p, rows, cols, codes, scales, (unsigned)pieces);
      else f8_quantize_cols_kernel<XT, VEC, false><<<grid, kThreads, 0, s>>>(p, rows, cols, codes, scales, (unsigned)pieces);
    });
  } else if (block_rows > 1) {
    if (int rc = tile_grid(tiles_of(cols), tiles_of(rows), batch, &grid)) return rc;
    by_type(dtype, cols, [&](auto tag, auto vec) {
      using XT = decltype(tag);
      f8_quantize_tile_rows_kernel<XT, decltype(vec)::value><<<grid, kThreads, 0, s>>>(static_cast<const XT*>(x), rows, cols,
                                                                                      reinterpret_cast<u32x2*>(codes), scales);
    });
  } else {
    const int64_t n = batch * rows, blocks = std::min((n * (f8_pitch(cols) / 8) + kThreads - 1) / kThreads, kMostBlocks);
    by_type(dtype, cols, [&](auto tag, auto vec) {
      using XT = decltype(tag);
      f8_quantize_rows_kernel<XT, decltype(vec)::value><<<(unsigned)blocks, kThreads, 0, s>>>(static_cast<const XT*>(x), n, cols,
                                                                                             reinterpret_cast<u32x2*>(codes), scales);
    });
  }
  BTX_LAUNCH_CHECK();
  return BTX_OK;
}

int launch_f8_dequantize(const uint8_t* codes, const uint8_t* scales, int dtype, int64_t batch, int64_t rows, int64_t cols, int axis, void* out,
                         hipStream_t s) {
  if (axis == 0) {
    const int64_t pieces = tiles_of(cols);
    dim3 grid;
    if (int rc = tile_grid(pieces, tiles_of(rows), batch, &grid)) return rc;
    by_type(dtype, cols, [&](auto tag, auto vec) {
      using XT = decltype(tag);
      f8_dequantize_cols_kernel<XT, decltype(vec)::value><<<grid, kThreads, 0, s>>>(codes, scales, rows, cols, static_cast<XT*>(out), (unsigned)pieces);
    });
  } else {
    const int64_t n = batch * rows, blocks = std::min((n * (f8_pitch(cols) / 8) + kThreads - 1) / kThreads, kMostBlocks);
    by_type(dtype, cols, [&](auto tag, auto vec) {
      using XT = decltype(tag);
      f8_dequantize_rows_kernel<XT, decltype(vec)::value><<<(unsigned)blocks, kThreads, 0, s>>>(reinterpret_cast<const u32x2*>(codes), scales, n, cols,
                                                                                               static_cast<XT*>(out));
    });
  }
  BTX_LAUNCH_CHECK();
  return BTX_OK;
}

}  // namespace btx
