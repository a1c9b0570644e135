// The residual's addition, the root-mean-square norm of the sum and the norm in 8 bits (fp8.h), in one pass over the rows:
//     sum = h + residual, rounded to the stream's type;   rstd = 1 / sqrt(mean(sum^2) + eps);   xn = gain * sum * rstd
// Bound by the bytes: bf16 with a residual, the sum and xn 9 + 1/128 an element.  A row stays in registers between its two uses.  The squares'
// sum, rstd and the products are in fp64, as btx_moe_norm_route's are (fp64 products are as fast here as those in fp32): xn is rounded
// once.  The codes come from the product rounded to fp32, not from xn rounded to bf16.
// 16384 x 4096 in bf16 with all four 106 us (5.7 TB/s), 16 x 4096 4 us.
#include <type_traits>

#include "fp8.h"

namespace btx {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ void store_norm(float* p, const double* v) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = (float)v[i];
  RowVec<float, 8>::st(p, f);
}
__device__ __forceinline__ void store_norm(bf16_t* p, const double* v) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = (uint32_t)f64_to_bf16(v[2 * i]) | (uint32_t)f64_to_bf16(v[2 * i + 1]) << 16;
  *reinterpret_cast<u32x4*>(p) = w;
}
// v and that of the lane that a DPP step names
template <int CTRL> __device__ __forceinline__ double dpp_add_f64(double v) {
  return v + __hiloint2double(dpp_i32<CTRL>(__double2hiint(v)), dpp_i32<CTRL>(__double2loint(v)));
}
__device__ __forceinline__ double lane_f64(double v, int lane) {
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane), __builtin_amdgcn_readlane(__double2loint(v), lane));
}
__device__ __forceinline__ double wave_sum_f64(double v) {
  v = dpp_add_f64<kDppXor1>(v);
  v = dpp_add_f64<kDppXor2>(v);
  v = dpp_add_f64<kDppRor4>(v);
  v = dpp_add_f64<kDppRor8>(v);
  return (lane_f64(v, 0) + lane_f64(v, 16)) + (lane_f64(v, 32) + lane_f64(v, 48));
}
// the sum as it is kept, in eight floats
__device__ __forceinline__ void round_sum(const float*, float*) {}
__device__ __forceinline__ void round_sum(const bf16_t*, float* v) {
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const uint32_t w = pack_bf16x2(v[i], v[i + 1]);
    v[i] = bf16lo(w);
    v[i + 1] = bf16hi(w);
  }
}

// TPR: threads that share a row, a wavefront (up to 512 columns) or the workgroup; MAXC: pieces of 8 columns that each has.  (sum may be h or
// residual, whose elements a thread has read by then; those of another that it reads behind the row's end are dropped: no __restrict__.)
template <typename XT, int TPR, int MAXC>
__global__ __launch_bounds__(kThreads) void f8_norm_kernel(const XT* h, const XT* residual, const float* __restrict__ gain, float eps, int T, int d,
                                                           XT* sum, XT* __restrict__ xn, float* __restrict__ rstd, u32x2* __restrict__ codes,
                                                           uint8_t* __restrict__ scales) {
  static_assert((TPR == kWave && MAXC == 1) || TPR == kThreads, "a wavefront or the workgroup");
  __shared__ double s_part[kThreads / kWave];
  const int lane = threadIdx.x & (kWave - 1), tid = TPR == kWave ? lane : threadIdx.x;
  const int64_t t = TPR == kWave ? (int64_t)blockIdx.x * (kThreads / kWave) + threadIdx.x / kWave : blockIdx.x;
  if (t >= T) return;                                    // (whole wavefronts; with TPR the workgroup none)
  const XT* const hr = h + t * d;
  // (without a branch around a load: behind one, the next waits for it)
  auto at = [&](int m) { return min((m * TPR + tid) * 8, d - 8); };
  float v[MAXC][8];
#pragma unroll
  for (int m = 0; m < MAXC; ++m) RowVec<XT, 8>::ld(hr + at(m), v[m]);
  if (residual) {
    float r[MAXC][8];
#pragma unroll
    for (int m = 0; m < MAXC; ++m) RowVec<XT, 8>::ld(residual + t * d + at(m), r[m]);
#pragma unroll
    for (int m = 0; m < MAXC; ++m) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[m][i] += r[m][i];
      round_sum(hr, v[m]);
    }
  }
#pragma unroll
  for (int m = 0; m < MAXC; ++m)
#pragma unroll
    for (int i = 0; i < 8; ++i) v[m][i] = (m * TPR + tid) * 8 < d ? v[m][i] : 0.f;
  double square = 0.0;
#pragma unroll
  for (int m = 0; m < MAXC; ++m)
#pragma unroll
    for (int i = 0; i < 8; ++i) square = fma((double)v[m][i], (double)v[m][i], square);
  if (sum) {
#pragma unroll
    for (int m = 0; m < MAXC; ++m) {
      const int c = (m * TPR + tid) * 8;
      if (c < d) RowVec<XT, 8>::st(sum + t * d + c, v[m]);
    }
  }
  square = wave_sum_f64(square);
  if constexpr (TPR > kWave) {
    if (lane == 0) s_part[threadIdx.x / kWave] = square;
    __syncthreads();
    square = (s_part[0] + s_part[1]) + (s_part[2] + s_part[3]);
  }
  const double r = 1.0 / sqrt(square / d + (double)eps);
  if (tid == 0) rstd[t] = (float)r;
  const int64_t n_blk = f8_pitch(d) / kF8Block, pitch = f8_scale_pitch(d);
#pragma unroll
  for (int m = 0; m < MAXC; ++m) {
    if (m * TPR * 8 >= d) break;
    const int c = (m * TPR + tid) * 8, b = c / kF8Block;
    double x[8] = {};
    if (c < d) {
      float g[8];
      RowVec<float, 8>::ld(gain + c, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = (double)g[i] * (double)v[m][i] * r;
      if (xn) store_norm(xn + t * d + c, x);
    }
    if (codes) {                                         // (every lane: behind d are zeros, up to the end of the block)
      float f[8];
      uint32_t amax = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        f[i] = (float)x[i];
        amax = max(amax, f8_magnitude(f[i]));
      }
      const uint32_t byte = f8_scale_byte(f8_row_max(amax));
      if (b < n_blk) {
        codes[(t * n_blk + b) * 16 + (c & (kF8Block - 1)) / 8] = u32x2{f8_codes4(f, byte), f8_codes4(f + 4, byte)};
        uint8_t* const sc = scales + t * pitch;
        const int lane16 = tid & 15;
        if (lane16 == 0) sc[b] = (uint8_t)byte;
        if (b + 1 == n_blk && n_blk + lane16 < pitch) sc[n_blk + lane16] = 0;
      }
    }
  }
}

template <typename XT> int launch_typed(const F8NormArgs& a, hipStream_t s) {
  auto run = [&](auto tpr, auto maxc) {
    constexpr int TPR = decltype(tpr)::value;
    constexpr int ROWS = kThreads / TPR, MOST = (1 << 22) * ROWS;       // (a launch has fewer than 2^32 threads)
    for (int t0 = 0; t0 < a.T; t0 += std::min(MOST, a.T - t0)) {
      auto at = [&](auto* p, int64_t pitch) { return p ? p + t0 * pitch : p; };
      const int n = std::min(MOST, a.T - t0);
      f8_norm_kernel<XT, TPR, decltype(maxc)::value><<<ceil_div(n, ROWS), kThreads, 0, s>>>(
          at(static_cast<const XT*>(a.h), a.d), at(static_cast<const XT*>(a.residual), a.d), a.gain, a.eps, n, a.d, at(static_cast<XT*>(a.sum), a.d),
          at(static_cast<XT*>(a.xn), a.d), a.rstd + t0, reinterpret_cast<u32x2*>(at(a.codes, f8_pitch(a.d))), at(a.scales, f8_scale_pitch(a.d)));
    }
  };
  const std::integral_constant<int, kThreads> block;
  if (a.d <= kWave * 8) run(std::integral_constant<int, kWave>{}, std::integral_constant<int, 1>{});
  else if (a.d <= kThreads * 8) run(block, std::integral_constant<int, 1>{});
  else if (a.d <= 2 * kThreads * 8) run(block, std::integral_constant<int, 2>{});
  else if (a.d <= 4 * kThreads * 8) run(block, std::integral_constant<int, 4>{});
  else run(block, std::integral_constant<int, 8>{});
  BTX_LAUNCH_CHECK();
  return BTX_OK;
}

}  // namespace

int launch_f8_norm(const F8NormArgs& a, hipStream_t s) {
  return a.dtype == BTX_BF16 ? launch_typed<bf16_t>(a, s) : launch_typed<float>(a, s);
}

}  // namespace btx
