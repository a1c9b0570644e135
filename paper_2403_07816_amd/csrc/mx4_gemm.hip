// Products of the layer of 4-bit experts (serving): UP, act = silu(xq W1_e) * (xq W3_e) quantised along f, and DOWN, y = act W2_e.
// Both operands are microscaled 4-bit floats with K contiguous (mx4.h); v_mfma_scale_f32_16x16x128_f8f6f4 takes codes and scales as they
// are, exact products, sums in fp32.  A lane's 16 bytes of a fragment are one block of 32 elements of a row: lane l holds row l % 16,
// and which four blocks of K the lane groups l / 16 hold is free, as long as both operands agree.  The weights are the first operand: each
// lane then ends up with four consecutive columns of one token row.
#include "mx4.h"

namespace btx {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// one step of K = 128; S: which byte of the scale words
template <int S> __device__ __forceinline__ f32x4 mfma_mx4(const u32x4& w, const u32x4& x, const f32x4& acc, uint32_t w_scale, uint32_t x_scale) {
  const i32x8 a = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0}, b = {(int)x[0], (int)x[1], (int)x[2], (int)x[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 4, S, (int)w_scale, S, (int)x_scale);
}

struct Mx4Args {
  Mx4Matrix a, b0, b1;                  // token rows; weights (b1: W3)
  const int32_t* offsets; const int32_t* perm; int k;   // perm: row r of the product is row perm[r] / k of a (NULL: row r)
  int E, N, K;                          // columns, depth
  uint8_t* act_codes; uint8_t* act_scales; bf16_t* y;
};

// Row tiles of up to 256 experts (RowTiles has 64): lane x looks at experts 4x .. 4x + 3
struct ManyRowTiles {
  int off[5], nt[4], incl, bm;
  __device__ __forceinline__ ManyRowTiles(const int32_t* __restrict__ offsets, int E, int BM, int lane) : bm(BM) {
#pragma unroll
    for (int q = 0; q < 5; ++q) off[q] = offsets[min(4 * lane + q, E)];
    int n = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      nt[q] = (off[q + 1] - off[q] + BM - 1) / BM;
      n += nt[q];
    }
    incl = wave_incl_scan_i32(n, lane);
  }
  __device__ __forceinline__ int count() const { return __builtin_amdgcn_readlane(incl, kWave - 1); }
  // tile id < count(): its expert, and rows row0 .. row_end - 1 of which the tile takes the first bm
  __device__ __forceinline__ void find(int id, int& expert, int& row0, int& row_end) const {
    const int owner = __ffsll((long long)__ballot(incl > id)) - 1;
    int n[4], o[5], left = id - __builtin_amdgcn_readlane(incl, owner);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      n[q] = __builtin_amdgcn_readlane(nt[q], owner);
      left += n[q];
    }
#pragma unroll
    for (int q = 0; q < 5; ++q) o[q] = __builtin_amdgcn_readlane(off[q], owner);
    int q = 0;
    while (q < 3 && left >= n[q]) left -= n[q++];
    expert = 4 * owner + q;
    int begin = o[0], end = o[1];
    if (q == 1) { begin = o[1]; end = o[2]; }
    if (q == 2) { begin = o[2]; end = o[3]; }
    if (q == 3) { begin = o[3]; end = o[4]; }
    row0 = begin + left * bm;
    row_end = end;
  }
};

// ---- few rows: 16 rows x 32 columns a workgroup, whose wavefronts share K ------------------------------------
// Bound by reading the weights.  They go from memory to the registers that the products take: a lane reads 64 consecutive bytes
// of a row (4 blocks) and their four scales in a word, 512 elements of 16 rows a wavefront at a time.
constexpr int kFewRows = 16, kFewCols = 32;
template <bool UP, int NW>
__global__ __launch_bounds__(NW* kWave) void mx4_few_kernel(Mx4Args g) {
  constexpr int PANELS = UP ? 2 : 1;
  __shared__ f32x4 s_sum[NW][PANELS * 2][kWave];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const ManyRowTiles tiles(g.offsets, g.E, kFewRows, lane);
  if ((int)blockIdx.y >= tiles.count()) return;
  int e, row0, row_end;
  tiles.find(blockIdx.y, e, row0, row_end);
  const int n0 = blockIdx.x * kFewCols, r = lane & 15, grp = lane >> 4;
  const int n_blk = g.K / kMxBlock;
  const int64_t pitch = mx4_pitch(g.K);
  int64_t row = min(row0 + r, row_end - 1);
  if (g.perm) row = g.perm[row] / g.k;
  const u32x4* const a = reinterpret_cast<const u32x4*>(g.a.codes) + row * n_blk;
  const uint8_t* const a_sc = g.a.scales + row * pitch;
  const u32x4* w[PANELS * 2];
  const uint8_t* w_sc[PANELS * 2];
#pragma unroll
  for (int p = 0; p < PANELS * 2; ++p) {
    const Mx4Matrix& m = p < 2 ? g.b0 : g.b1;
    const int64_t n = (int64_t)e * g.N + n0 + 16 * (p & 1) + r;
    w[p] = reinterpret_cast<const u32x4*>(m.codes) + n * n_blk;
    w_sc[p] = m.scales + n * pitch;
  }
  f32x4 acc[PANELS * 2] = {};
  for (int b0 = 16 * wave; b0 < n_blk; b0 += 16 * NW) {
    const int at = b0 + 4 * grp;                       // (scale rows are whole 16 bytes; behind K / 32 they are zero)
    u32x4 xv[4], wv[PANELS * 2][4];
    uint32_t xs, ws[PANELS * 2];
    xs = *reinterpret_cast<const uint32_t*>(a_sc + at);
#pragma unroll
    for (int p = 0; p < PANELS * 2; ++p) ws[p] = *reinterpret_cast<const uint32_t*>(w_sc[p] + at);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const bool in = at + s < n_blk;
      xv[s] = in ? a[at + s] : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
      for (int p = 0; p < PANELS * 2; ++p) wv[p][s] = in ? w[p][at + s] : u32x4{0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int p = 0; p < PANELS * 2; ++p) {
      acc[p] = mfma_mx4<0>(wv[p][0], xv[0], acc[p], ws[p], xs);
      acc[p] = mfma_mx4<1>(wv[p][1], xv[1], acc[p], ws[p], xs);
      acc[p] = mfma_mx4<2>(wv[p][2], xv[2], acc[p], ws[p], xs);
      acc[p] = mfma_mx4<3>(wv[p][3], xv[3], acc[p], ws[p], xs);
    }
  }
#pragma unroll
  for (int p = 0; p < PANELS * 2; ++p) s_sum[wave][p][lane] = acc[p];
  __syncthreads();
  // thread t < 256: row t / 16, columns 2 (t % 16) and the next: lane 16 (c % 16 / 4) + row of fragment c / 16, element c % 4
  if (threadIdx.x >= 256) return;
  const int out_row = threadIdx.x / 16, c = 2 * (threadIdx.x % 16), m = row0 + out_row;
  const int from = 16 * ((c & 15) >> 2) + out_row, half = c >> 4, el = c & 3;
  float sum[PANELS][2] = {};
#pragma unroll
  for (int x = 0; x < NW; ++x)
#pragma unroll
    for (int p = 0; p < PANELS; ++p) {
      const f32x2* v = reinterpret_cast<const f32x2*>(&s_sum[x][2 * p + half][from]);
      sum[p][0] += v[el >> 1][0];
      sum[p][1] += v[el >> 1][1];
    }
  const bool live = m < row_end;
  if constexpr (UP) {
    const float v0 = silu_f(sum[0][0]) * sum[1][0], v1 = silu_f(sum[0][1]) * sum[1][1];
    uint32_t amax = max(magnitude(v0), magnitude(v1));
    amax = max(amax, (uint32_t)dpp_i32<kDppXor1>((int)amax));
    amax = max(amax, (uint32_t)dpp_i32<kDppXor2>((int)amax));
    amax = max(amax, (uint32_t)dpp_i32<kDppRor4>((int)amax));
    amax = max(amax, (uint32_t)dpp_i32<kDppRor8>((int)amax));
    const uint32_t byte = mx4_scale_byte(amax);
    const uint32_t code = byte == 255u ? 0u : __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v0, v1, mx4_scale(byte), 0) & 255u;
    if (live) {
      const int64_t act_pitch = mx4_pitch(g.N);
      g.act_codes[(int64_t)m * (g.N / 2) + (n0 + c) / 2] = (uint8_t)code;
      if (c == 0) g.act_scales[(int64_t)m * act_pitch + n0 / kMxBlock] = (uint8_t)byte;
      // the zeros behind the scales of a row
      if (n0 + kFewCols == g.N)
        for (int64_t z = g.N / kMxBlock + c / 2; z < act_pitch; z += 16) g.act_scales[(int64_t)m * act_pitch + z] = 0;
    }
  } else {
    if (live) *reinterpret_cast<uint32_t*>(g.y + (int64_t)m * g.N + n0 + c) = pack_bf16x2(sum[0][0], sum[0][1]);
  }
}

template <bool UP> int launch_few(const Mx4Args& g, int R, hipStream_t s) {
  const int64_t tiles = (int64_t)ceil_div(R, kFewRows) + std::min(g.E, R);    // at most: every expert may have a partly filled one
  if (tiles > 65535) return BTX_ERR_UNSUPPORTED;
  mx4_few_kernel<UP, 8><<<dim3(g.N / kFewCols, (unsigned)tiles), 8 * kWave, 0, s>>>(g);
  BTX_LAUNCH_CHECK();
  return BTX_OK;
}

}  // namespace

int launch_mx4_up(const Mx4Matrix& xq, const Mx4Matrix& W1, const Mx4Matrix& W3, const int32_t* offsets, const int32_t* perm,
                  const Mx4Shapes& sh, uint8_t* act_codes, uint8_t* act_scales, hipStream_t s) {
  const Mx4Args g{xq, W1, W3, offsets, perm, sh.k, sh.E, sh.f, sh.d, act_codes, act_scales, nullptr};
  return launch_few<true>(g, sh.T * sh.k, s);
}

int launch_mx4_down(const Mx4Matrix& act, const Mx4Matrix& W2, const int32_t* offsets, const Mx4Shapes& sh, void* y, hipStream_t s) {
  const Mx4Args g{act, W2, {nullptr, nullptr}, offsets, nullptr, 1, sh.E, sh.d, sh.f, nullptr, nullptr, static_cast<bf16_t*>(y)};
  return launch_few<false>(g, sh.T * sh.k, s);
}

}  // namespace btx
