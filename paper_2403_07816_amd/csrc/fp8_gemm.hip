// Products of matrices of block-scaled 8-bit floats (fp8.h): out = A B^T, and those of the layer of 8-bit experts (UP, act = silu(x W1_e) * (x W3_e)
// quantised along f, and DOWN, y = act W2_e).  Both operands have K contiguous.  Lane l holds row l % 16; which chunks of K the lane groups
// l / 16 hold is free, as long as both operands agree.  B is the first operand: each lane then ends up with four consecutive columns of one
// row of the result.
//   * Results in bf16 and the activations of tall tiles: v_mfma_scale_f32_16x16x128_f8f6f4 takes 128 codes of a row with their scale as they are.  Of every 8
//     neighbouring products it drops what lies 13 bits or more below the exponent of the largest before it adds them up, and then sums in
//     fp32: normally distributed rows and columns give a result 2e-5 of its norm off, where rounding it to bf16 puts it 1.7e-3 off.
//   * Results in fp32 and all other activations: the codes become bf16, exactly, with their scale (values under 2^-126: to bf16's precision there), and
//     v_mfma_f32_16x16x32_bf16 multiplies those: exact products, sums in fp32, at half the rate.
#include "fp8.h"
#include "tile_lds.h"

#include <atomic>
#include <type_traits>

namespace btx {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// one step of K = 128; SEL: which byte of the scale words
template <int SEL> __device__ __forceinline__ f32x4 mfma_f8(const u32x4& b0, const u32x4& b1, const u32x4& a0, const u32x4& a1, const f32x4& acc,
                                                            uint32_t b_scale, uint32_t a_scale) {
  const i32x8 b = {(int)b0[0], (int)b0[1], (int)b0[2], (int)b0[3], (int)b1[0], (int)b1[1], (int)b1[2], (int)b1[3]};
  const i32x8 a = {(int)a0[0], (int)a0[1], (int)a0[2], (int)a0[3], (int)a1[0], (int)a1[1], (int)a1[2], (int)a1[3]};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, acc, 0, 0, SEL, (int)b_scale, SEL, (int)a_scale);
}

// The same by way of bf16: acc += the products of 32 codes a lane
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
__device__ __forceinline__ float f8_scale_or_nan(uint32_t byte) { return byte == 255u ? __uint_as_float(0x7fc00000u) : f8_scale(byte); }
__device__ __forceinline__ bf16x8 to_bf16x8(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true),
                 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// What a launch multiplies.  Rows are those of the experts one after another (offsets, perm: row r is row perm[r] / k of a; perm NULL: row r), or, with
// offsets NULL, all R of a matrix
struct F8Args {
  F8Matrix a, b0, b1;                   // rows; weights, experts one after another (b1: W3)
  const int32_t* offsets; const int32_t* perm;
  int E, k, R, N, K;                    // N columns, depth K
  uint8_t* act_codes; uint8_t* act_scales;
  void* out; const void* residual;
  int slices; float* sums;              // K ranges of a tile; more than one, or in32: their sums [slice][R][N] go there, and not to out
  bool turned;                          // few rows: these are the result's columns, and it is written [N][R]
  bool in32;
};

struct Tile { int e, row0, row_end; };

// The row tiles of up to 256 experts, found by every wavefront for itself: lane l looks at experts 4l .. 4l + 3 (all 64 lanes active)
struct ExpertTiles {
  int o[5], n, incl, rows;
  template <typename P> __device__ __forceinline__ ExpertTiles(P offsets, int E, int tile_rows, int lane) : n(0), rows(tile_rows) {
    static_assert(kF8MaxExperts <= 4 * kWave, "four experts a lane");
#pragma unroll
    for (int i = 0; i < 5; ++i) o[i] = offsets[min(4 * lane + i, E)];
#pragma unroll
    for (int i = 0; i < 4; ++i) n += count(o[i], o[i + 1]);
    incl = wave_incl_scan_i32(n, lane);
  }
  __device__ __forceinline__ int count(int from, int to) const { return (to - from + rows - 1) / rows; }
  __device__ __forceinline__ int count() const { return __builtin_amdgcn_readlane(incl, kWave - 1); }
  // id < count()
  __device__ __forceinline__ Tile at(int id) const {
    const int lane = __ffsll((long long)__ballot(incl > id)) - 1;
    int left = id - (__builtin_amdgcn_readlane(incl, lane) - __builtin_amdgcn_readlane(n, lane));
    Tile t{4 * lane, 0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int from = __builtin_amdgcn_readlane(o[i], lane), to = __builtin_amdgcn_readlane(o[i + 1], lane), m = count(from, to);
      if (left >= 0 && left < m) t = Tile{4 * lane + i, from + left * rows, to};
      left -= m;
    }
    return t;
  }
};
inline int most_tiles(int R, int E, int tile_rows) { return (int)std::min<int64_t>((int64_t)R / tile_rows + std::min(E, R), R); }

// four columns of the result, from element `at` on
template <bool F32> __device__ __forceinline__ void store_out(const F8Args& g, int64_t at, f32x4 v) {
  if constexpr (F32) {
    if (g.residual) v += *reinterpret_cast<const f32x4*>(static_cast<const float*>(g.residual) + at);
    *reinterpret_cast<f32x4*>(static_cast<float*>(g.out) + at) = v;
  } else {
    if (g.residual) {
      const u32x2 w = *reinterpret_cast<const u32x2*>(static_cast<const bf16_t*>(g.residual) + at);
      v += f32x4{bf16lo(w[0]), bf16hi(w[0]), bf16lo(w[1]), bf16hi(w[1])};
    }
    *reinterpret_cast<u32x2*>(static_cast<bf16_t*>(g.out) + at) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  }
}

// ---- few rows -------------------------------------------------------------------------------------------------
// Bound by reading B.  It goes from memory to the registers that the products take, 256 elements (two blocks) of 16 rows a wavefront at a time: in load s
// lane group g has 16-byte chunk 4s + g, so that a load covers 64 bytes of a row.  RB blocks of 16 rows of A meet each fragment of it.
// NF x 16 rows of b: a base that the wavefront shares and a lane's offset of 32 bits, for codes and scales
template <int NF> struct FewB { const char* codes[NF]; const char* scales[NF]; uint32_t at[NF], sc_at[NF]; };
// N blocks' codes and scales of RB x 16 rows of a and NF x 16 rows of b
template <int N, int RB, int NF> struct FewStep { u32x4 a[RB][2 * N], b[NF][2 * N]; uint32_t a_s[RB], b_s[NF]; };
template <int N> __device__ __forceinline__ uint32_t few_scales(const void* p) {
  static_assert(N == 1 || N == 2, "bytes");
  if constexpr (N == 1) return *static_cast<const uint8_t*>(p);
  else return *static_cast<const uint16_t*>(p);
}
template <int N, int RB, int NF>
__device__ __forceinline__ void few_load(FewStep<N, RB, NF>& v, const FewB<NF>& b, const F8Matrix& a, const uint32_t (&row)[RB], int n_blk,
                                         int64_t a_pitch, int b0, int grp) {
  const uint32_t at = (uint32_t)b0 * kF8Block + grp * 16u;
#pragma unroll
  for (int p = 0; p < NF; ++p) {
#pragma unroll
    for (int s = 0; s < 2 * N; ++s) v.b[p][s] = *reinterpret_cast<const u32x4*>(b.codes[p] + (b.at[p] + at + s * 64u));
    v.b_s[p] = few_scales<N>(b.scales[p] + (b.sc_at[p] + b0));
  }
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
    for (int s = 0; s < 2 * N; ++s) v.a[rb][s] = *reinterpret_cast<const u32x4*>(a.codes + (int64_t)row[rb] * n_blk * kF8Block + (at + s * 64u));
    v.a_s[rb] = few_scales<N>(a.scales + row[rb] * a_pitch + b0);
  }
}
template <bool EXACT, int H, int N, int RB, int NF> __device__ __forceinline__ void few_multiply(f32x4 (*acc)[NF], const FewStep<N, RB, NF>& v) {
  if constexpr (EXACT) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {                        // 8 codes a lane
      bf16x8 bb[NF];
#pragma unroll
      for (int p = 0; p < NF; ++p) {
        const u32x4& w = v.b[p][2 * H + q / 2];
        bb[p] = to_bf16x8(w[2 * (q & 1)], w[2 * (q & 1) + 1], f8_scale_or_nan(v.b_s[p] >> (8 * H) & 255u));
      }
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const u32x4& w = v.a[rb][2 * H + q / 2];
        const bf16x8 aa = to_bf16x8(w[2 * (q & 1)], w[2 * (q & 1) + 1], f8_scale_or_nan(v.a_s[rb] >> (8 * H) & 255u));
#pragma unroll
        for (int p = 0; p < NF; ++p) acc[rb][p] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bb[p], aa, acc[rb][p], 0, 0, 0);
      }
    }
  } else {
#pragma unroll
    for (int p = 0; p < NF; ++p)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
        acc[rb][p] = mfma_f8<H>(v.b[p][2 * H], v.b[p][2 * H + 1], v.a[rb][2 * H], v.a[rb][2 * H + 1], acc[rb][p], v.b_s[p], v.a_s[rb]);
  }
}
// acc += the products of RB x 16 rows of a and NF x 16 rows of b over pairs of blocks first, first + step, ..; who would have the next pair
// has the block behind the last one.  EXACT: by way of bf16.  All loads of a step are under way before its first product; with the next step's
// under way as well there were fewer wavefronts, and it was no faster.  turn: of the pairs `first` means, to have workgroups of neighbouring
// columns at different places of their rows.
template <bool EXACT, int RB, int NF>
__device__ __forceinline__ void few_products(f32x4 (*acc)[NF], const FewB<NF>& b, const F8Matrix& a, const uint32_t (&row)[RB], int n_blk, int64_t a_pitch,
                                             int first, int step, int turn, int grp) {
  const int pairs = n_blk / 2;
#pragma unroll 1
  for (int i = first; i < pairs; i += step) {
    FewStep<2, RB, NF> v;
    const int at = i + turn;
    few_load(v, b, a, row, n_blk, a_pitch, 2 * (at < pairs ? at : at - pairs), grp);
    __builtin_amdgcn_sched_barrier(0);
    few_multiply<EXACT, 0>(acc, v);
    few_multiply<EXACT, 1>(acc, v);
  }
  if (n_blk % 2 && pairs % step == first) {
    FewStep<1, RB, NF> v;
    few_load(v, b, a, row, n_blk, a_pitch, n_blk - 1, grp);
    few_multiply<EXACT, 0>(acc, v);
  }
}
// the same, of the blocks of rows that have one
template <bool EXACT, int RB, int NF>
__device__ __forceinline__ void few_live_products(f32x4 (&acc)[RB][NF], const FewB<NF>& b, const F8Args& g, const Tile& t, int n_blk, int64_t a_pitch,
                                                  int first, int step, int turn, int grp, int r) {
  auto go = [&](auto n_tag) {
    constexpr int N = decltype(n_tag)::value;
    uint32_t row[N];
#pragma unroll
    for (int rb = 0; rb < N; ++rb) {
      row[rb] = (uint32_t)min(t.row0 + rb * 16 + r, t.row_end - 1);
      if (g.perm) row[rb] = (uint32_t)g.perm[row[rb]] / (uint32_t)g.k;
    }
    few_products<EXACT, N, NF>(acc, b, g.a, row, n_blk, a_pitch, first, step, turn, grp);
  };
  const int live = (t.row_end - t.row0 + 15) / 16;
  if (live <= 1) go(std::integral_constant<int, 1>{});
  else if (RB <= 2 || live <= 2) go(std::integral_constant<int, RB <= 2 ? RB : 2>{});
  else go(std::integral_constant<int, RB>{});
}

// the workgroup's tile of rows; false: there is none
template <int RB> __device__ __forceinline__ bool few_tile(const F8Args& g, int lane, Tile& t) {
  if (!g.offsets) {
    t = Tile{0, (int)blockIdx.y * (RB * 16), g.R};
    return true;
  }
  const ExpertTiles tiles(g.offsets, g.E, RB * 16, lane);
  if ((int)blockIdx.y >= tiles.count()) return false;
  t = tiles.at(blockIdx.y);
  return true;
}
// rows n0 .. of expert e's matrix, up to the last one
template <int NF> __device__ __forceinline__ void few_b(FewB<NF>& b, int p, const F8Matrix& m, const F8Args& g, int e, int n0, int r) {
  const int64_t pitch = f8_pitch(g.K), sc_pitch = f8_scale_pitch(g.K), n = (int64_t)e * g.N + min(n0, g.N - 1);
  const uint32_t at = (uint32_t)max(min(r, g.N - 1 - n0), 0);
  b.codes[p] = reinterpret_cast<const char*>(m.codes) + n * pitch;
  b.scales[p] = reinterpret_cast<const char*>(m.scales) + n * sc_pitch;
  b.at[p] = at * (uint32_t)pitch;
  b.sc_at[p] = at * (uint32_t)sc_pitch;
}

// FR x 16 columns, by KS wavefronts that share K.  UP: both panels, and the activations in fp32 (sums [R][N]): their blocks of 128 columns would make
// workgroups too large to spread over the chip (one token, 2 experts of 4096 x 11008: 53 us), and another launch quantises them
template <bool UP, int RB, int FR, int KS, typename OT>
__global__ __launch_bounds__(KS* kWave, 2) void f8_few_kernel(F8Args g) {
  constexpr int NF = UP ? 2 * FR : FR;
  __shared__ f32x4 s_sum[KS][RB][NF][kWave];
  const int lane = threadIdx.x & (kWave - 1), ks = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), r = lane & 15, grp = lane >> 4;
  Tile t;
  if (!few_tile<RB>(g, lane, t)) return;
  const int n0 = blockIdx.x * (FR * 16), n_blk = (int)(f8_pitch(g.K) / kF8Block);
  FewB<NF> b;
#pragma unroll
  for (int p = 0; p < NF; ++p) few_b(b, p, p < FR ? g.b0 : g.b1, g, t.e, n0 + 16 * (p % FR), r);
  f32x4 acc[RB][NF] = {};
  // (DOWN of one token, 2 experts of 4096 x 11008: 22.8 us with all workgroups at the same place of their rows, 18.9 so; UP of two to 16, 4 experts: 87-90,
  // 75-78; of 64 columns nothing was gained)
  const int turn = (UP || FR == 1) && n_blk > 1 ? 3 * blockIdx.x % (n_blk / 2) : 0;
  few_live_products<std::is_same_v<OT, float>>(acc, b, g, t, n_blk, f8_scale_pitch(g.K), ks, KS, turn, grp, r);
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int p = 0; p < NF; ++p) s_sum[ks][rb][p][lane] = acc[rb][p];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < FR * RB; ++i) {
    if (i % KS != ks) continue;
    const int rb = i / FR, p = i % FR, m = t.row0 + rb * 16 + r, n = n0 + 16 * p + 4 * grp;
    if (m >= t.row_end || n >= g.N) continue;
    auto sum = [&](int q) {
      f32x4 v = s_sum[0][rb][q][lane];
#pragma unroll
      for (int x = 1; x < KS; ++x) v += s_sum[x][rb][q][lane];
      return v;
    };
    f32x4 v = sum(p);
    const int64_t at = (int64_t)m * g.N + n;
    if constexpr (UP) {
      const f32x4 h3 = sum(FR + p);
#pragma unroll
      for (int x = 0; x < 4; ++x) v[x] = silu_f(v[x]) * h3[x];
      *reinterpret_cast<f32x4*>(g.sums + at) = v;
    } else if (g.in32) {
      *reinterpret_cast<f32x4*>(g.sums + at) = v;
    } else if (g.turned) {
      const OT* const residual = static_cast<const OT*>(g.residual);
      for (int x = 0; x < 4 && n + x < g.N; ++x) {
        const int64_t to = (int64_t)(n + x) * g.R + m;
        Elem<OT>::st(static_cast<OT*>(g.out) + to, v[x] + (residual ? Elem<OT>::ld(residual + to) : 0.f));
      }
    } else {
      store_out<std::is_same_v<OT, float>>(g, at, v);
    }
  }
}

template <bool UP, int FR, int KS, typename OT> int launch_few_shape(const F8Args& g, int tile_rows, hipStream_t s) {
  const dim3 grid((unsigned)ceil_div(g.N, FR * 16), (unsigned)(g.offsets ? most_tiles(g.R, g.E, tile_rows) : ceil_div(g.R, tile_rows)));
  if (tile_rows == 32) f8_few_kernel<UP, 2, FR, KS, OT><<<grid, KS * kWave, 0, s>>>(g);
  else if constexpr (!UP) f8_few_kernel<UP, 4, FR, KS, OT><<<grid, KS * kWave, 0, s>>>(g);    // (of one matrix)
  BTX_LAUNCH_CHECK();
  return BTX_OK;
}
// 16 columns a workgroup, whose 4 wavefronts share K, or, where there are 2048 such pieces, 64 and 2.  A compute unit reads 25 GB/s from memory, so all
// of them are needed.  DOWN of one token, 2 experts of 4096 x 11008 (512 pieces): 18.9 us with 16 columns, 24 with 32, 31 with 64; of 64 tokens,
// 32 experts of 4096 x 1376 (8192): 58, 46, 40; 2048 x 4096 (4096): 84, 66, 60; 16 experts of 1024 x 2048 (1024): 9.7, 9.0, 9.3.
// A turned product's "columns" are its many rows: 16384 (1024 pieces) x 16, K 8192, 39 us with 16 of them a workgroup, 31 with 64; 6400 20 and 25.
// (fp32 results: 16 always; bf16 values of 64 columns and 64 rows do not fit the registers)
template <typename OT> int launch_few(const F8Args& g, int tile_rows, hipStream_t s) {
  const int64_t tiles = g.offsets ? std::min(g.E, g.R) : ceil_div(g.R, tile_rows), pieces = tiles * ceil_div(g.N, 16);
  if constexpr (!std::is_same_v<OT, float>) {
    if (pieces >= (g.turned ? 1024 : 2048)) return launch_few_shape<false, 4, 2, OT>(g, tile_rows, s);
  }
  return launch_few_shape<false, 1, 4, OT>(g, tile_rows, s);
}
// (one token, 2 experts of 4096 x 11008: 37-40 us (4.7 TB/s); before products were by way of bf16, with 2 wavefronts, 4, or 16 columns and 4: 37, 40, 37;
// 64 tokens, 32 of 4096 x 1376: 85, 86, 90)
int launch_few_up(const F8Args& g, hipStream_t s) { return launch_few_shape<true, 2, 2, float>(g, 32, s); }

// (of a turned product 16 rows are a workgroup's)
static_assert((kF8MostRows / 16 + 0ll) * 4 * kWave < 1ll << 32, "a launch has fewer than 2^32 threads");

// ---- a middling number of rows: BM x 128 tiles, BM 64 or 128 -----------------------------------------------------
// Bound by reading B where rows are few, by LDS where they are many.  A k tile is a block: [row][128 bytes] of either operand, in a ring of NS stages that
// direct copies fill; 4 wavefronts have BM/2 x 64 of the result each (UP: 32 columns of either panel).  Two workgroups are on a compute unit
// and overlap what each waits for, the conversions to bf16 among it.  Rows of A that are not there are not copied.
// 64 tokens of 32 experts of 4096 x 1376, top-8: UP 89 us (4.1 TB/s), DOWN 38 (4.8); 1024 x 4096 x 4096 27 us (1.3 PFLOP/s); in fp32 4096 x 4096 x 4001 128 us
// (1.05 PFLOP/s; the conversions run at a quarter of the vector rate).
constexpr int kMidWaves = 4, kMidCols = 128;
enum MidMode { kMidUp, kMidOut, kMidExact };           // activations in fp32 (sums) and fp32 results, both by way of bf16; bf16 results
template <int BM> struct Mid {
  static constexpr int NS = BM == 128 ? 2 : 3;
  static constexpr uint32_t stage = (BM + kMidCols) * 128, scale_stage = (BM + kMidCols) * 16, scales0 = NS * stage;
  static constexpr int lds = scales0 + 2 * scale_stage;
};

template <MidMode MODE, int BM>
__global__ __launch_bounds__(kMidWaves* kWave, 2) void f8_mid_kernel(F8Args g, int n_ct) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  using M = Mid<BM>;
  constexpr bool UP = MODE == kMidUp;
  constexpr int NA = BM / 32, TM = BM / 32, TN = 4, COLS = UP ? 64 : 128, PER_K = NA + 4;      // a wavefront's copies of a k tile
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), wm = wave >> 1, wn = wave & 1;
  const int64_t row_bytes = f8_pitch(g.K), sc_pitch = f8_scale_pitch(g.K);
  const int nk_all = (int)(row_bytes / kF8Block), slices = UP ? 1 : g.slices;
  const uint32_t base = (uint32_t)(uintptr_t)smem;

  // ---- the tile.  Workgroups that are a multiple of 8 apart are on one XCD: those that read the same columns, or, of one matrix with more tiles of rows than
  // of columns, the same rows, follow each other there.  Every XCD has as many: with columns always in turn, 16384 x 128 x 8192 was one XCD's work,
  // 147 us for 32, and 16384 x 512 x 8192 149 for 72.  (In turn, where that is even: neighbouring columns are read at a time.  UP of 2 of 4 experts of
  // 4096 x 11008 95 us and 97; 64 x 4096 x 11008 16.8 and 17.7; but 256 x 4096 x 4096 17.8 and 16.0)
  Tile t;
  const int xcd = blockIdx.x % kXcds, local = blockIdx.x / kXcds;
  const int n_c = n_ct * slices;
  int c, rt;
  // columns in turn, rows of them one after another; or 8 equal runs of the tiles (past the last one: no tile), columns or rows first
  auto in_turn = [&](int n_rt) {
    c = local / n_rt * kXcds + xcd;
    rt = local % n_rt;
    return c < n_c;
  };
  auto in_runs = [&](int n_rt, bool rows_first) {
    const int tiles = n_rt * n_c, each = (tiles + kXcds - 1) / kXcds, id = xcd * each + local;
    c = rows_first ? id % n_c : id / n_rt;
    rt = rows_first ? id / n_c : id % n_rt;
    return local < each && id < tiles;
  };
  const bool even = n_c % kXcds == 0 || n_c >= 64;
  if (g.offsets) {
    const ExpertTiles tiles(g.offsets, g.E, BM, lane);
    const int n_rt = tiles.count();
    if (n_rt == 0 || !(even ? in_turn(n_rt) : in_runs(n_rt, false))) return;
    t = tiles.at(rt);
  } else {
    const int n_rt = (g.R + BM - 1) / BM;
    if (!(even && n_rt <= 2 ? in_turn(n_rt) : in_runs(n_rt, n_rt > n_ct))) return;
    t = Tile{0, rt * BM, g.R};
  }
  const int slice = c / n_ct, col0 = (c - slice * n_ct) * COLS, quads = (nk_all + 3) / 4;
  const int k_first = slice * quads / slices * 4, nk = min((slice + 1) * quads / slices * 4, nk_all) - k_first;
  // Columns begin at different places of their rows, four k tiles apart, and go round (where the scales' 16 k tiles come out even): rows that lie 4096 bytes
  // apart, of which all workgroups read the same block, use part of the memory's channels.  2 of 8 experts of 4096 x 4096, 64 tokens: 107 us and 86 so;
  // of 4 of 4096 x 11008: 140, 130
  const int turn = slices == 1 && nk % 16 == 0 ? 4 * c % nk : 0, start = k_first + turn;
  int a_left = nk - turn, b_left = a_left;               // copies up to the end of a row

  // ---- copies: a wavefront has BM / 4 rows of A and 32 of B, 8 lanes a row, 8 rows an instruction; 64 rows of A's scales, or of B's
  auto chunk = [&](int q) { return (lane & 7) ^ tile_swz(lane / 8 + 8 * (q & 1)); };
  auto row_index = [&](int at) -> uint32_t {
    const int gr = min(t.row0 + at, t.row_end - 1);
    return g.perm ? (uint32_t)g.perm[gr] / (uint32_t)g.k : (uint32_t)(gr - t.row0);
  };
  auto column = [&](int row) { return min(col0 + (UP ? row & 63 : row), g.N - 1) - col0; };
  const F8Matrix& bm = UP && wave >= 2 ? g.b1 : g.b0;
  const uint32_t to_a = base + wave * (BM / 4) * 128, to_b = base + BM * 128 + wave * 4096;
  const int64_t k0 = (int64_t)start * kF8Block;
  uint32_t a_off[NA], b_off[4], s_off;
#pragma unroll
  for (int q = 0; q < 4; ++q) b_off[q] = (uint32_t)column(wave * 32 + q * 8 + lane / 8) * (uint32_t)row_bytes + chunk(q) * 16 + (kCopyBias4 - 1024 * q);
  uint64_t b_from = uniform64(bm.codes + ((int64_t)t.e * g.N + col0) * row_bytes + k0) - kCopyBias4;
  auto copy_b = [&](uint32_t stage) {
    copy64(b_from, b_off, to_b + stage);
    b_from += kF8Block;
    if (--b_left == 0) b_from -= (int64_t)nk * kF8Block;
  };
  // (the first ones, while the rows of A are looked up)
#pragma unroll
  for (int p = 0; p < M::NS - 1; ++p)
    if (p < nk) copy_b(p * M::stage);
#pragma unroll
  for (int q = 0; q < NA; ++q) a_off[q] = row_index(wave * (BM / 4) + q * 8 + lane / 8) * (uint32_t)row_bytes + chunk(q) * 16;
  uint64_t a_from = uniform64(g.a.codes + (g.perm ? 0 : (int64_t)t.row0 * row_bytes) + k0);
  uint64_t s_from;
  const bool a_scales = wave < 2, has_scales = !a_scales || wave < BM / 64;
  if (a_scales) {
    s_off = row_index(min(wave * 64, BM - 64) + lane) * (uint32_t)sc_pitch;
    s_from = uniform64(g.a.scales + (g.perm ? 0 : (int64_t)t.row0 * sc_pitch));
  } else {
    s_off = (uint32_t)column((wave - 2) * 64 + lane) * (uint32_t)sc_pitch;
    s_from = uniform64((UP && wave == 3 ? g.b1 : g.b0).scales + ((int64_t)t.e * g.N + col0) * sc_pitch);
  }
  const int a_live = min(max((t.row_end - t.row0 - wave * (BM / 4) + 7) / 8, 0), NA);            // of its copies of A, those that have a row
  const uint32_t to_s = base + M::scales0 + (a_scales ? wave * 1024 : BM * 16 + (wave - 2) * 1024);
  auto copy_scales = [&](int c) {                        // of k tiles 16 c ..
    if (has_scales) copy16(s_from + (uint64_t)(16 * c < k_first + nk ? c : c - nk / 16) * 16, s_off, to_s + (c & 1) * M::scale_stage);
  };
  auto copy_a = [&](uint32_t stage) {
#pragma unroll
    for (int q = 0; q < NA; ++q)
      if (q < a_live) copy16(a_from, a_off[q], to_a + stage + q * 1024);
    a_from += kF8Block;
    if (--a_left == 0) a_from -= (int64_t)nk * kF8Block;
  };

  // ---- fragments: lane l has row l % 16, chunks 2g and 2g + 1 of lane group g = l / 16
  const int r = lane & 15, lg = lane >> 4;
  typedef const __attribute__((address_space(3))) u32x4* lds_frag;
  typedef const __attribute__((address_space(3))) uint32_t* lds_word;
  const uint32_t at_a = base + (wm * (BM / 2) + r) * 128 + ((2 * lg) ^ tile_swz(r)) * 16;
  const uint32_t at_b = base + (BM + wn * (UP ? 32 : 64) + r) * 128 + ((2 * lg) ^ tile_swz(r)) * 16;
  auto b_row = [](int j) { return UP ? (j >> 1) * 64 + (j & 1) * 16 : j * 16; };
  const uint32_t sc_a = base + M::scales0 + (wm * (BM / 2) + r) * 16, sc_b = base + M::scales0 + (BM + wn * (UP ? 32 : 64) + r) * 16;
  f32x4 acc[TM][TN] = {};
  uint32_t xa[TM], xb[TN];
  const bool live = t.row0 + wm * (BM / 2) < t.row_end;
  auto multiply = [&](auto q_tag, uint32_t stage) {
    constexpr int Q = decltype(q_tag)::value;
    u32x4 fa[TM][2], fb[TN][2];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int st = 0; st < 2; ++st) fb[j][st] = *(lds_frag)(uintptr_t)((at_b ^ (st << 4)) + stage + b_row(j) * 128);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int st = 0; st < 2; ++st) fa[i][st] = *(lds_frag)(uintptr_t)((at_a ^ (st << 4)) + stage + i * 2048);
    if constexpr (MODE != kMidOut) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {                      // 8 codes a lane
        bf16x8 bb[TN];
#pragma unroll
        for (int j = 0; j < TN; ++j)
          bb[j] = to_bf16x8(fb[j][q / 2][2 * (q & 1)], fb[j][q / 2][2 * (q & 1) + 1], f8_scale_or_nan(xb[j] >> (8 * Q) & 255u));
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          const bf16x8 aa = to_bf16x8(fa[i][q / 2][2 * (q & 1)], fa[i][q / 2][2 * (q & 1) + 1], f8_scale_or_nan(xa[i] >> (8 * Q) & 255u));
#pragma unroll
          for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bb[j], aa, acc[i][j], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = mfma_f8<Q>(fb[j][0], fb[j][1], fa[i][0], fa[i][1], acc[i][j], xb[j], xa[i]);
    }
  };

  // ---- k tiles.  Whoever passes the barrier of k tile kt has read all of k tile kt - 1, whose stage the copies behind it fill
  copy_scales(start >> 4);
  if (16 * ((start >> 4) + 1) < start + nk) copy_scales((start >> 4) + 1);
  uint32_t stage = 0, next = (M::NS - 1) * M::stage;     // of k tile kt, and of the one that is copied beside it
#pragma unroll
  for (int p = 0; p < M::NS - 1; ++p)
    if (p < nk) copy_a(p * M::stage);
  auto k_tile = [&](auto q_tag, int kt) {
    constexpr int Q = decltype(q_tag)::value;
    if (M::NS > 2 && kt > 0 && kt + 1 < nk) {            // the next k tile's copies may be outstanding (but for those from before the first)
      if (a_live == NA) wait_vmcnt<PER_K>(); else wait_vmcnt<4>();
    } else {
      wait_vmcnt<0>();
    }
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    if (Q == 2) {                                        // the scales of the next 16 k tiles, where those of the 16 before were (the first two are there)
      const int k = start + kt, c = k >> 4;
      if ((k & 15) == 2 && c > start >> 4 && 16 * (c + 1) < start + nk) copy_scales(c + 1);
    }
    if (kt + M::NS - 1 < nk) {
      copy_b(next);
      copy_a(next);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (live) {
      if (Q == 0) {                                      // of k tiles k .. k + 3
        const int k = start + kt;
        const uint32_t at = ((k >> 4) & 1) * M::scale_stage + (k & 12);
#pragma unroll
        for (int i = 0; i < TM; ++i) xa[i] = *(lds_word)(uintptr_t)(sc_a + at + i * 256);
#pragma unroll
        for (int j = 0; j < TN; ++j) xb[j] = *(lds_word)(uintptr_t)(sc_b + at + b_row(j) * 16);
      }
      multiply(q_tag, stage);
    }
    next = stage;
    stage = stage + M::stage == M::scales0 ? 0 : stage + M::stage;
  };
#pragma unroll 1
  for (int kt = 0; kt < nk; kt += 4) {
    k_tile(std::integral_constant<int, 0>{}, kt);
    if (kt + 1 < nk) k_tile(std::integral_constant<int, 1>{}, kt + 1);
    if (kt + 2 < nk) k_tile(std::integral_constant<int, 2>{}, kt + 2);
    if (kt + 3 < nk) k_tile(std::integral_constant<int, 3>{}, kt + 3);
  }

  // ---- acc[i][j][v] is row 16 i + l % 16, column 16 j + 4 (l / 16) + v of the wavefront's
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < (UP ? 2 : TN); ++j) {
      const int m = t.row0 + wm * (BM / 2) + i * 16 + r, n = col0 + wn * (COLS / 2) + j * 16 + 4 * lg;
      if (m >= t.row_end || n >= g.N) continue;
      const int64_t at = (int64_t)m * g.N + n;
      f32x4 v = acc[i][j];
      if constexpr (UP) {
#pragma unroll
        for (int x = 0; x < 4; ++x) v[x] = silu_f(v[x]) * acc[i][j + 2][x];
        *reinterpret_cast<f32x4*>(g.sums + at) = v;
      } else if (slices > 1 || g.in32) {
        *reinterpret_cast<f32x4*>(g.sums + (int64_t)slice * g.R * g.N + at) = v;
      } else {
        store_out<MODE == kMidExact>(g, at, v);
      }
    }
}

// ---- many rows: 256 x 256 tiles ---------------------------------------------------------------------------------
// Bound by the matrix cores and by what feeds them from LDS.  A k tile is a block: [row][128 bytes] of either operand, 8 wavefronts have 128 x 64 of the
// result each (UP: 32 columns of either panel, 128 in all: a block of the activations), 128 accumulator registers.
//   * global -> LDS copies are direct, 16 bytes a lane, two stages of both operands (128 KB); chunks are swizzled by row (tile_swz()).
//   * The two wavefronts of a SIMD alternate between a memory phase and a compute phase (16 products), half a period apart, with a barrier at
//     every boundary.  The first memory phase of a k tile reads all fragments of B and those of half of A's rows, the second the other half's: B's
//     stage and half of A's are free half a k tile early, and the copies of the k tile after the next go there.
//   * Scales: 16 bytes of every row are copied for 16 k tiles, a wavefront 64 rows with one instruction; a lane reads a word of each of its rows
//     for 4 k tiles, and the products pick the byte.
//   * Tiles are dealt so that the ones an XCD runs at a time share row and column panels in its L2; a workgroup takes tile after tile, the next
//     one's first stage is under way beside the epilogue.
//   * Of a tile's rows that are not there, 64 of a wavefront's are passed over.
// 16384 x 11008 x 4096 543 us (2.72 PFLOP/s; with codes of zero 431: the power budget), matrix cores busy 67 % of the time at 1.7 GHz; UP and DOWN of 16384 tokens,
// top-2, 2.2-2.4 and 1.1 ms.
constexpr int kTileRows = 256, kTileWaves = 8;
constexpr uint32_t kStage = 32768, kScaleStage = 8192;  // scales of 16 k tiles: 256 rows of A, 256 of B
constexpr uint32_t kB0 = 2 * kStage, kScale0 = 4 * kStage, kOffsets0 = kScale0 + 2 * kScaleStage;
constexpr int kTileLds = kOffsets0 + (kF8MaxExperts + 1) * 4;
enum TileMode { kUp, kOut };                            // activations in 8 bits; bf16

// APART: tiles of neighbouring columns begin at different places of K.  An instance of its own: with one for both, timed in turn on one card, layers that are not
// apart took 0.2-0.5 % longer (16384 tokens 3.439 and 3.444 ms, 2048 582 and 584 us, 32 experts of width 1376 1154 and 1160 us), 16384 x 11008 x 4096 as long.
template <TileMode MODE, bool APART>
__global__ __launch_bounds__(kTileWaves* kWave, 2) void f8_tile_kernel(F8Args g, int n_ct) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  constexpr bool UP = MODE == kUp;
  constexpr int TM = 8, TN = 4, TNH = UP ? 2 : 4, COLS = UP ? 128 : 256;
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int wm = wave >> 2, wn = wave & 3, grp = wm;     // the wavefronts of a SIMD are w and w + 4
  const int64_t row_bytes = f8_pitch(g.K), sc_pitch = f8_scale_pitch(g.K);
  const int nk_all = (int)(row_bytes / kF8Block), slices = UP ? 1 : g.slices;
  const uint32_t base = (uint32_t)(uintptr_t)smem;
  typedef const __attribute__((address_space(3))) int32_t* lds_int;

  // ---- the tile
  const lds_int s_offsets = (lds_int)(uintptr_t)(base + kOffsets0);
  if (g.offsets) {
    for (int i = threadIdx.x; i <= g.E; i += kTileWaves * kWave) reinterpret_cast<int32_t*>(smem + kOffsets0)[i] = g.offsets[i];
    __syncthreads();
  }
  int e, row0, row_end, col0, slice, id = blockIdx.x;
  int k_first, nk;                                       // its k tiles: k_first (a multiple of four, as words of scales are read) .. + nk - 1
  int first, left;                                       // the one that it begins at, to go round, and copies up to the last one
  auto find_tile = [&]() -> bool {                       // `id`, or the next one of this workgroup that names a tile
    auto among = [&](int n_rt, auto rows_of) -> bool {
      const int most = n_rt * n_ct + kXcds;
      int tm, tn;
      for (; id < most * slices; id += gridDim.x)
        if (tile_of(id % most, n_rt, n_ct, tm, tn)) {
          const int quads = (nk_all + 3) / 4;
          slice = id / most;
          k_first = slice * quads / slices * 4;
          nk = min((slice + 1) * quads / slices * 4, nk_all) - k_first;
          const Tile t = rows_of(tm);
          e = t.e;
          row0 = t.row0;
          row_end = t.row_end;
          col0 = tn * COLS;
          first = k_first + (APART ? 4 * tn % nk : 0);      // (whole 16 blocks, not cut)
          return true;
        }
      return false;
    };
    if (!g.offsets) return among((g.R + kTileRows - 1) / kTileRows, [&](int tm) { return Tile{0, tm * kTileRows, g.R}; });
    const ExpertTiles tiles(s_offsets, g.E, kTileRows, here(lane));
    return among(tiles.count(), [&](int tm) { return tiles.at(tm); });
  };

  // ---- copies.  Rows 0-63 and 128-191 of A are its first half (A0), which the first memory phase reads, the others the second (A1): a
  // wavefront has 16 rows of either and 32 rows of B, 8 lanes a row, 8 rows an instruction; 64 rows of A's scales, or of B's
  auto chunk = [](int ln, int q) { return (ln & 7) ^ tile_swz(ln / 8 + 8 * (q & 1)); };
  const int a_row = wm * 128 + wn * 16;
  uint32_t a_off[4], b_off[4], s_off;                    // a_off: A0, A0, A1, A1
  uint64_t a_from, a1_from, b_from, s_from;              // a, b: of the k tile behind the next (A1: the one before)
  auto row_index = [&](int at) -> uint32_t {
    const int gr = min(row0 + at, row_end - 1);
    return g.perm ? (uint32_t)g.perm[gr] / (uint32_t)g.k : (uint32_t)(gr - row0);
  };
  auto set_rows = [&] {                                  // (as indexes of rows, for now)
    const int ln = here(lane);
#pragma unroll
    for (int q = 0; q < 4; ++q) a_off[q] = row_index(a_row + (q >> 1) * 64 + (q & 1) * 8 + ln / 8);
    if (wm == 0) s_off = row_index(wn * 64 + ln);
  };
  auto set_sources = [&] {
    const int ln = here(lane);
    // (asm: one register for each of these for the whole loop, not the pair that their 64-bit products are in)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      a_off[q] = a_off[q] * (uint32_t)row_bytes + chunk(ln, q) * 16 + (kCopyBias2 - 1024 * (q & 1));
      const int row = wave * 32 + q * 8 + ln / 8, col = min(col0 + (UP ? row & 127 : row), g.N - 1) - col0;
      b_off[q] = (uint32_t)col * (uint32_t)row_bytes + chunk(ln, q) * 16 + (kCopyBias4 - 1024 * q);
      asm volatile("" : "+v"(a_off[q]), "+v"(b_off[q]));
    }
    const F8Matrix& bm = UP && wave >= 4 ? g.b1 : g.b0;
    const int64_t k0 = (int64_t)first * kF8Block;
    left = k_first + nk - first;
    a_from = uniform64(g.a.codes + (g.perm ? 0 : (int64_t)row0 * row_bytes) + k0) - kCopyBias2;
    b_from = uniform64(bm.codes + ((int64_t)e * g.N + col0) * row_bytes + k0) - kCopyBias4;
    if (wm == 0) {
      s_off *= (uint32_t)sc_pitch;
      s_from = uniform64(g.a.scales + (g.perm ? 0 : (int64_t)row0 * sc_pitch));
    } else {
      const int row = wn * 64 + ln, col = min(col0 + (UP ? row & 127 : row), g.N - 1) - col0;
      s_off = (uint32_t)col * (uint32_t)sc_pitch;
      s_from = uniform64((UP && wn >= 2 ? g.b1 : g.b0).scales + ((int64_t)e * g.N + col0) * sc_pitch);
    }
    asm volatile("" : "+v"(s_off));
  };
  const uint32_t to_a = base + a_row * 128, to_b = base + kB0 + wave * 4096, to_s = base + kScale0 + wave * 1024;
  auto copy_a0b = [&](int stage) {
    copy32(a_from, a_off[0], a_off[1], to_a + stage * kStage);
    copy64(b_from, b_off, to_b + stage * kStage);
  };
  auto advance = [&] {
    int64_t to = kF8Block;
    if constexpr (APART) {
      a1_from = a_from;
      if (--left == 0) to = (int64_t)(1 - nk) * kF8Block;
    }
    a_from += to;
    b_from += to;
  };
  auto copy_a1 = [&](int stage, uint64_t from) { copy32(from, a_off[2], a_off[3], to_a + stage * kStage + 64 * 128); };
  auto copy_scales = [&](int c) {                        // of k tiles 16 c ..
    copy16(s_from + (uint64_t)(!APART || 16 * c < k_first + nk ? c : c - nk / 16) * 16, s_off, to_s + (c & 1) * kScaleStage);
  };

  // ---- fragments: lane l has row l % 16, chunks 2g and 2g + 1 of lane group g = l / 16
  const int r = lane & 15, lg = lane >> 4;
  typedef const __attribute__((address_space(3))) u32x4* lds_frag;
  typedef const __attribute__((address_space(3))) uint32_t* lds_word;
  const uint32_t at_a = base + (wm * 128 + r) * 128 + ((2 * lg) ^ tile_swz(r)) * 16;
  const uint32_t at_b = base + kB0 + (wn * (TNH * 16) + r) * 128 + ((2 * lg) ^ tile_swz(r)) * 16;
  const uint32_t sc_a = base + kScale0 + (wm * 128 + r) * 16;
  const uint32_t sc_b = base + kScale0 + 4096 + (wn * (TNH * 16) + r) * 16;
  f32x4 acc[TM][TN];
  u32x4 fa[TM / 2][2], fb[TN][2];                        // (of one half of A)
  uint32_t xa[TM], xb[TN];
  auto read_a = [&](int stage, int half) {
#pragma unroll
    for (int i = 0; i < TM / 2; ++i)
#pragma unroll
      for (int st = 0; st < 2; ++st) fa[i][st] = *(lds_frag)(uintptr_t)((at_a ^ (st << 4)) + stage * kStage + (half * 4 + i) * 2048);
  };
  auto read_b = [&](int stage) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int st = 0; st < 2; ++st)
        fb[j][st] = *(lds_frag)(uintptr_t)((at_b ^ (st << 4)) + stage * kStage + (j / TNH) * (128 * 128) + (j % TNH) * 2048);
  };
  auto read_scales = [&](int k) {                        // of k tiles k .. k + 3
    const uint32_t at = ((k >> 4) & 1) * kScaleStage + (k & 12);
#pragma unroll
    for (int i = 0; i < TM; ++i) xa[i] = *(lds_word)(uintptr_t)(sc_a + at + i * 256);
#pragma unroll
    for (int j = 0; j < TN; ++j) xb[j] = *(lds_word)(uintptr_t)(sc_b + at + (j / TNH) * 2048 + (j % TNH) * 256);
  };
  // the products of half h of A's rows
  auto multiply = [&](auto q_tag, int h) {
    constexpr int Q = decltype(q_tag)::value;
#pragma unroll
    for (int i = 0; i < TM / 2; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
        acc[h * 4 + i][j] = mfma_f8<Q>(fb[j][0], fb[j][1], fa[i][0], fa[i][1], acc[h * 4 + i][j], xb[j], xa[h * 4 + i]);
  };
  // Copies: in the first memory phase of k tile kt A1 of kt + 1 (2 instructions), in the second A0 and B of kt + 2 (2 and 4), in front of them
  // now and then one of scales.  What they overwrite was read last in the memory phases before, and they have four phases or more to land.
  auto k_tile = [&](auto q_tag, int kt) {
    constexpr int Q = decltype(q_tag)::value, stage = Q & 1;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      // ---- memory phase
      const bool live = row0 + wm * 128 + h * 64 < row_end;    // (of this half of its rows any: a phase without products is short)
      if (Q == 0 && h == 0) read_scales(first + kt);
      if (live) {
        read_a(stage, h);
        if (h == 0) read_b(stage);
      }
      if (h == 0) {
        if (kt + 1 < nk) copy_a1(stage ^ 1, APART ? a1_from : a_from - kF8Block);
      } else {
        // the scales of the next 16 k tiles, where those of the 16 before were (the first two are there from the start)
        if (Q == 2) {
          const int k = first + kt, c = k >> 4;
          if ((k & 15) == 2 && c > first >> 4 && 16 * (c + 1) < first + nk) copy_scales(c + 1);
        }
        if (kt + 2 < nk) {
          copy_a0b(stage);
          advance();
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_waitcnt(0xC07F);                // lgkmcnt(0)
      // What the next memory phases read has landed: behind h == 0, A1 of this k tile; behind h == 1, A0 and B of the next.  What has been issued
      // since may be outstanding (scales, which are needed much later, count as if they were not).
      auto landed = [&] {
        if (h == 0) {
          if (kt + 1 < nk) wait_vmcnt<8>(); else wait_vmcnt<0>();
        } else {
          if (kt + 2 < nk) wait_vmcnt<8>(); else wait_vmcnt<2>();
        }
      };
      if (grp == 1) landed();
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
      // ---- compute phase
      if (live) multiply(q_tag, h);
#pragma unroll
      for (int i = 0; i < TM / 2; ++i)                   // here, and not where the sums are needed next: behind the next phases' barriers
#pragma unroll
        for (int j = 0; j < TN; ++j) asm volatile("" : "+v"(acc[h * 4 + i][j]));
      if (grp == 0) landed();
      __builtin_amdgcn_sched_barrier(0);
      if (!(grp == 1 && h == 1 && kt + 1 == nk)) __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  if (!find_tile()) return;
  set_rows();
  auto start = [&] {                                     // into the first stages: k tile 0; and scales
    set_sources();
    const int c = first >> 4;
    copy_scales(c);
    if (16 * (c + 1) < first + nk) copy_scales(c + 1);
    copy_a0b(0);
    copy_a1(0, a_from);
    advance();
  };
  start();
  for (;;) {
    if (nk > 1) {                                        // into the second stages, as k tile -1 would have
      copy_a0b(1);
      advance();
      wait_vmcnt<6>();
    } else {
      wait_vmcnt<0>();
    }
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    if (grp == 1) __builtin_amdgcn_s_barrier();          // group 1 is a phase behind
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll 1
    for (int kt = 0; kt < nk; kt += 4) {
      k_tile(std::integral_constant<int, 0>{}, kt);
      if (kt + 1 < nk) k_tile(std::integral_constant<int, 1>{}, kt + 1);
      if (kt + 2 < nk) k_tile(std::integral_constant<int, 2>{}, kt + 2);
      if (kt + 3 < nk) k_tile(std::integral_constant<int, 3>{}, kt + 3);
    }

    // ---- epilogue: acc[i][j][v] is row wm 128 + 16 i + l % 16, column 16 j + 4 (l / 16) + v of the wavefront's.  All of LDS is free (group
    // 0's last barrier comes after group 1's last read); the result goes through the second stages, and the first stages are filled for
    // the workgroup's next tile beside it.
    const int out_row0 = row0, out_end = row_end, out_col0 = col0, out_slice = slice;
    const int ln = here(lane), r = ln & 15, lg = ln >> 4, tid = wave * kWave + ln;
    __syncthreads();
    id += gridDim.x;
    const bool more = find_tile();
    if (more) set_rows();
    char* const out = smem + kStage;
    if constexpr (UP) {
      // a workgroup's 128 columns are one block; its codes [256 rows][128 bytes] are put together in LDS, 16-byte chunks swizzled by row
      uint32_t* const s_amax = reinterpret_cast<uint32_t*>(smem + kB0 + kStage);      // [256][4]
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        uint32_t amax = 0;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const bool there = out_col0 + wn * 32 + j * 16 + 4 * lg + x < g.N;
            acc[i][j][x] = there ? silu_f(acc[i][j][x]) * acc[i][j + 2][x] : 0.f;
            amax = max(amax, f8_magnitude(acc[i][j][x]));
          }
        amax = f8_across_max(amax);
        if (lg == 0) s_amax[(wm * 128 + i * 16 + r) * 4 + wn] = amax;
      }
      if (more) start();                                 // (behind the activations, beside which its rows were looked up)
      __syncthreads();
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const int row = wm * 128 + i * 16 + r;
        const u32x4 four = *reinterpret_cast<const u32x4*>(s_amax + row * 4);
        const uint32_t byte = f8_scale_byte(max(max(four[0], four[1]), max(four[2], four[3])));
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
          *reinterpret_cast<uint32_t*>(out + row * 128 + (((wn * 2 + j) ^ (row >> 1 & 7)) << 4) + lg * 4) = f8_codes4(v, byte);
        }
        if (wn == 0 && lg == 0 && out_row0 + row < out_end) g.act_scales[(int64_t)(out_row0 + row) * f8_scale_pitch(g.N) + out_col0 / 128] = (uint8_t)byte;
      }
      __syncthreads();
      const int64_t out_pitch = f8_pitch(g.N), out_sc_pitch = f8_scale_pitch(g.N);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int idx = q * 512 + tid, row = idx >> 3, c = idx & 7;
        if (out_row0 + row < out_end)
          *reinterpret_cast<u32x4*>(g.act_codes + (int64_t)(out_row0 + row) * out_pitch + out_col0 + c * 16) =
              *reinterpret_cast<const u32x4*>(out + row * 128 + ((c ^ (row >> 1 & 7)) << 4));
      }
      if (out_col0 + COLS >= g.N && tid < 256 && out_row0 + tid < out_end)          // the zeros behind a row's scales
        for (int64_t z = out_col0 / 128 + 1; z < out_sc_pitch; ++z) g.act_scales[(int64_t)(out_row0 + tid) * out_sc_pitch + z] = 0;
    } else {
      if (more) start();
      if (slices > 1 || g.in32) {                        // four columns a lane, as they are
        float* const to = g.sums + (int64_t)out_slice * g.R * g.N;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j) {
            const int m = wm * 128 + i * 16 + r, n = out_col0 + wn * 64 + j * 16 + 4 * lg;
            if (out_row0 + m < out_end && n < g.N) *reinterpret_cast<f32x4*>(to + (int64_t)(out_row0 + m) * g.N + n) = acc[i][j];
          }
        if (!more) return;
        __syncthreads();
        continue;
      }
      // 32 rows of the wavefront's 64 columns at a time (128 bytes a row) through its own piece of LDS, chunks swizzled by row
      char* const band = out + wave * 4096;
      const int n0 = out_col0 + wn * 64;
      bf16_t* const to = static_cast<bf16_t*>(g.out);
#pragma unroll
      for (int ib = 0; ib < TM / 2; ++ib) {
#pragma unroll
        for (int i2 = 0; i2 < 2; ++i2)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            f32x4& v = acc[2 * ib + i2][j];
            const int row = i2 * 16 + r, byte = (j * 16 + 4 * lg) * 2;
            if (g.residual) {
              const int m = out_row0 + wm * 128 + ib * 32 + row, n = n0 + j * 16 + 4 * lg;
              if (m < out_end && n < g.N) {
                const u32x2 w = *reinterpret_cast<const u32x2*>(static_cast<const bf16_t*>(g.residual) + (int64_t)m * g.N + n);
                v += f32x4{bf16lo(w[0]), bf16hi(w[0]), bf16lo(w[1]), bf16hi(w[1])};
              }
            }
            *reinterpret_cast<u32x2*>(band + row * 128 + ((byte >> 4 ^ (row & 7)) << 4) + (byte & 15)) =
                u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
          }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int row = q * 8 + ln / 8, c = ln & 7, m = out_row0 + wm * 128 + ib * 32 + row;
          const u32x4 w = *reinterpret_cast<const u32x4*>(band + row * 128 + ((c ^ (row & 7)) << 4));
          if (m < out_end && n0 + c * 8 < g.N) __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(to + (int64_t)m * g.N + n0 + c * 8));
        }
        __builtin_amdgcn_wave_barrier();
      }
    }
    if (!more) return;
    __syncthreads();                                     // the second stages are free
  }
}

// the dynamic-LDS limit, once per device (not while a stream is being captured; btx_init() does it too)
template <auto KERNEL> int raise_lds(int bytes) {
  static std::atomic<uint64_t> done{0};
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return BTX_ERR_HIP;
  if (!(done.load(std::memory_order_relaxed) >> dev & 1)) {
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess)
      return BTX_ERR_HIP;
    done.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  return BTX_OK;
}

int64_t mid_grid(int n_ct, int64_t n_rt) { return ceil_div((int64_t)n_ct, kXcds) * kXcds * n_rt; }
template <MidMode MODE, int BM> int launch_mid_tiles(const F8Args& g, hipStream_t s) {
  if (int rc = raise_lds<f8_mid_kernel<MODE, BM>>(Mid<BM>::lds)) return rc;
  const int n_ct = ceil_div(g.N, MODE == kMidUp ? 64 : kMidCols);
  const int64_t grid = mid_grid(n_ct * g.slices, g.offsets ? most_tiles(g.R, g.E, BM) : ceil_div(g.R, BM));
  if (!grid_fits(grid, kMidWaves * kWave)) return BTX_ERR_UNSUPPORTED;
  f8_mid_kernel<MODE, BM><<<(unsigned)grid, kMidWaves * kWave, Mid<BM>::lds, s>>>(g, n_ct);
  BTX_LAUNCH_CHECK();
  return BTX_OK;
}
template <MidMode MODE> int launch_mid(const F8Args& g, int tile_rows, hipStream_t s) {
  return tile_rows == 64 ? launch_mid_tiles<MODE, 64>(g, s) : launch_mid_tiles<MODE, 128>(g, s);
}

// Of so few rows, which an XCD's L2 keeps, neighbouring columns begin at different places of K, as the middling tiles' do: 301 tokens, 2 of 4 experts of 4096 x
// 11008, 172 us and 166; 500, 2 of 8 of 4096 x 4096, 133 and 118.  Of more the tiles beside each other would read them from memory again: 16384 tokens of the
// former 3.41 and 3.58 ms, 8 MB of rows as fast as together.
constexpr int64_t kApartBytes = 2 << 20;
template <TileMode MODE, bool APART> int launch_tiles_as(const F8Args& g, hipStream_t s) {
  if (int rc = raise_lds<f8_tile_kernel<MODE, APART>>(kTileLds)) return rc;
  const int n_ct = ceil_div(g.N, MODE == kUp ? 128 : 256);
  const int64_t n_rt = g.offsets ? most_tiles(g.R, g.E, kTileRows) : ceil_div(g.R, kTileRows);
  const int64_t tiles = (n_rt * n_ct + kXcds) * g.slices;
  // A workgroup for every compute unit, which takes every 256th tile: what begins its next one runs beside the last one's end.  Of less than two
  // rounds each has its own: a few ids name no tile, and their compute units take the ones behind the 256th.
  const int64_t grid = tiles <= 2 * kTileGrid ? tiles : kTileGrid;
  f8_tile_kernel<MODE, APART><<<(unsigned)grid, kTileWaves * kWave, kTileLds, s>>>(g, n_ct);
  BTX_LAUNCH_CHECK();
  return BTX_OK;
}
template <TileMode MODE> int launch_tiles(const F8Args& g, hipStream_t s) {
  const bool apart = (int64_t)(g.perm ? g.R / g.k : g.R) * f8_pitch(g.K) <= kApartBytes && g.slices == 1 && f8_pitch(g.K) % (16 * kF8Block) == 0;
  return apart ? launch_tiles_as<MODE, true>(g, s) : launch_tiles_as<MODE, false>(g, s);
}

// K ranges of the tiles: as many as fill the chip (`places` workgroups at once) where the tiles alone do not, of `shortest` k tiles or more each; no more
// than whoever adds them takes, and than there is room for
constexpr int kMostSlices = 16;
constexpr int64_t kSumBytes = (int64_t)kTileGrid * 256 * 256 * 4;        // of 256 tiles
int64_t sum_bytes(int64_t R, int N) { return std::min(R * N * 4 * kMostSlices, kSumBytes); }
int slices_of(int64_t tiles, int places, int shortest, int64_t R, int N, int K, int most) {
  const int64_t fit = sum_bytes(R, N) / (R * N * 4);
  return (int)std::max<int64_t>(std::min({places / tiles, f8_pitch(K) / kF8Block / shortest, fit, (int64_t)most, (int64_t)kMostSlices}), 1);
}

// out = residual + the sums of the slices, in order; four columns a thread
constexpr int kAddThreads = 256;
template <typename OT>
__global__ __launch_bounds__(kAddThreads) void f8_add_slices_kernel(const f32x4* __restrict__ sums, int slices, int64_t n, const OT* residual, OT* out) {
  for (int64_t i = (int64_t)blockIdx.x * kAddThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kAddThreads) {
    f32x4 v = sums[i];
    for (int s0 = 1; s0 < slices; s0 += 4) {             // four loads at a time
      f32x4 u[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) u[q] = s0 + q < slices ? sums[(int64_t)(s0 + q) * n + i] : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (s0 + q < slices) v += u[q];
    }
    if constexpr (std::is_same_v<OT, float>) {
      if (residual) v += reinterpret_cast<const f32x4*>(residual)[i];
      reinterpret_cast<f32x4*>(out)[i] = v;
    } else {
      if (residual) {
        const u32x2 w = reinterpret_cast<const u32x2*>(residual)[i];
        v += f32x4{bf16lo(w[0]), bf16hi(w[0]), bf16lo(w[1]), bf16hi(w[1])};
      }
      reinterpret_cast<u32x2*>(out)[i] = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    }
  }
}

// Which kernel, and the rows of its tiles
enum Path { kFew32, kFew64, kMid64, kMid128, kTall };
constexpr int kPathRows[] = {32, 64, 64, 128, kTileRows};
// Rows of E experts (those that have a row: about as many each), in tiles.  Counts stay on the device, so a favoured expert takes the kernel of the mean: with one
// that every token names, 301 tokens of 2 of 4 experts of 4096 x 11008 170 -> 181 us (the bf16 layer 258 -> 326), 16384 3.45 -> 3.46 ms, 64 of 8 of 32 of width
// 1376 140 -> 139 us.
struct Rows {
  int64_t busy, each;
  Rows(int64_t R, int E) : busy(std::min<int64_t>(E, R)), each((R + busy - 1) / busy) {}
  int64_t tiles(int rows) const { return busy * ((each + rows - 1) / rows); }
};
// The activations.  Few and middling rows: products by way of bf16, whose sums are exact to fp32, and fp32 activations that another launch quantises
// (2.5 us and more): a sum that is 2e-5 off is on the other side of a code's border now and then, or its block of a scale's, and over few tokens one such
// block shows (3 tokens of 4 experts of 168 x 88: 0.0053 of the result's norm, and 0.0017).  That costs little where reading the weights bounds it:
// 16 tokens of 2 of 4 experts of 4096 x 11008 122 -> 132 us, 64 131 -> 135.  Tall tiles' are on the matrix cores' own 8-bit products: 16384 tokens would
// take twice as long, and the sums' errors average out over those.  A layer's time, us, with few / 64 / 128 / tall for UP (all experts with as many rows; of one
// row two experts).  Up to 64 rows tall tiles are now and then a little faster, and not exact:
//   2 of 4 experts of 4096 x 11008, rows each:  1  62 63 77 60;  4  134 126 129 134;  16  143 122 133 135;  64  231 139 151 147;  95  303 183 171 154
//   8 of 32 of 4096 x 1376:  4  140 134 145 133;  16  146 131 137 135;  50  220 147 147 141;  95  301 181 168 148
//   2 of 8 of 2048 x 8192:  1  31 32 36 36;  16  104 95 103 102;  32  118 97 106 103;  63  169 107 116 108
//   2 of 8 of 1024 x 2048:  1  18 20 22 24;  16  25 24 27 27;  64  35 29 31 29;  128  54 34 33 32
constexpr int kUpFewRows = 3, kUpMidRows = 64, kUpMidTiles = kTileGrid;
Path up_path(int64_t R, int E, int f) {
  const Rows n(R, E);
  if (n.each <= kUpFewRows) return kFew32;
  // (64 rows of 256 experts of 2 million columns are more workgroups than a launch has)
  if (n.each <= kUpMidRows && grid_fits(mid_grid(ceil_div(f, 64), most_tiles((int)R, E, 64)), kMidWaves * kWave)) return kMid64;
  return n.tiles(128) * ceil_div(f, 64) <= kUpMidTiles ? kMid128 : kTall;
}
// Other products.  Of one matrix (sums of tiles that are cut along K are added by another launch), columns x K, rows, us:
//   1024 x 1024: 64  5.8 7.2 8.6 12;  256  5.7 7.4 9.6 15;  1024  14 7.7 10 16;  16384  77 34 28 21
//   4096 x 1376: 32  5.9 7.6 9.6 15;  96  8.7 8.5 11 17;  1024  28 12 13 20;  16384  367 207 134 86
//   4096 x 4096: 16  8.0 10 10 14;  32  9.8 11 11 15;  64  14 12 12 17;  256  47 16 18 28;  1024  75 24 30 42;  2048  155 51 42 53;  16384  1141 595 325 200
//   4096 x 11008: 16  15 14 15 20;  64  33 17 19 24;  256  120 28 28 38;  1024  192 64 67 62;  2048  399 137 102 91
//   512 x 8192: 16  11 9.9 11 15;  256  25 13 14 25;  2048  91 23 23 31        256 x 2048: 64  7.5 9.9 10 15;  1024  8.2 10 13 23;  16384  38 16 17 31
//   11008 x 4096: 1  11 13 14 15;  8  14 13 14 15;  16  16 12 15 16;  32  22 13 16 17;  256  58 23 27 34;  512  115 40 36 43;  1024  216 71 62 46
//   11008 x 2048: 16  9.0 10 10 15;  32  12 11 12 16        8192 x 8192: 4  16 17 17 18;  12  19 15 18 19        33000 x 512: 8  7.1 6.2 6.7 11;
//   48  10 7.3 7.9 10        33000 x 4096: 1  32 27 29 34;  32  44 31 31 35
// In fp32:  1024 x 2048: 64  8.4 12 14;  200  8.4 13 16        4096 x 4001: 64  15 14 16;  400  73 29 29;  1376  239 66 60;  4096  - 174 132
//   4096 x 16384: 40  38 21 24;  100  79 34 28;  400  282 107 81;  1024  - 155 148        512 x 8192: 400  25 15 19;  2048  91 34 30
// Of experts (the sums of tiles that are cut are added where the rows are combined), rows each:
//   4 of 11008 x 4096 (K x N): 4  40 47 47 45;  16  54 41 48 46;  32  76 42 50 48;  64  146 46 52 51;  150  351 90 81 62
//   32 of 1376 x 4096: 4  40 38 39 42;  16  44 40 41 43;  32  50 43 44 47;  100  138 61 52 47       8 of 2048 x 1024: 4  8.2 9.1 10 15;  16  9.4 9.0 10 15;
//   64  18 11 12 17;  256  54 15 16 25;  1024  205 34 30 30;      64 of 1024 x 2048: 4  30 31 31 34;  32  39 35 37 39;  64  61 38 40 39;  256  210 89 85 52
Path out_path(int64_t R, int E, int N, int K, bool exact) {
  const Rows n(R, E);
  const int columns = ceil_div(N, kMidCols), n_blk = (int)(f8_pitch(K) / kF8Block);
  const int64_t tiles = n.tiles(64) * columns;
  if (E == 1) {
    // (a few long columns: only cut along K do they fill the chip; short ones do as long as a compute unit has one workgroup; exact: conversions of rows
    // that are not there, and of columns twice where tiles have 64 rows)
    const bool one_round = n_blk <= 16 && ceil_div(R, 64) * ceil_div(N, 16) <= kTileGrid;
    const bool wide = columns >= 64 && !exact, few = wide ? n.each * n_blk <= 384 && (columns < 256 || n_blk < 4)
                                                          : one_round || ((n.each <= 16 || n.each * n_blk <= 1024) && (tiles >= 8 || n_blk < 48));
    if (few) return n.each <= 24 ? kFew32 : kFew64;
    if (exact && n.each > 64 && n_blk > 64 && tiles >= 64) return kMid128;
    if (tiles <= 2 * kTileGrid) return kMid64;
  } else {
    if (n.each <= 8) return kFew32;
    if (n.each <= 48 || tiles * n_blk <= 8192) return kMid64;
  }
  return n.tiles(128) * columns <= 2 * kTileGrid && n_blk <= 64 ? kMid128 : kTall;
}

// out, or the sums of g.slices ranges of K, which are set here
template <bool F32> int launch_out(F8Args& g, Path path, int most_slices, hipStream_t s) {
  using OT = std::conditional_t<F32, float, bf16_t>;
  if (path <= kFew64) return launch_few<OT>(g, kPathRows[path], s);
  const int64_t row_tiles = Rows(g.R, g.E).tiles(kPathRows[path]);
  if (path <= kMid128) {
    g.slices = slices_of(row_tiles * ceil_div(g.N, kMidCols), kTileGrid, 8, g.R, g.N, g.K, most_slices);
    return launch_mid<F32 ? kMidExact : kMidOut>(g, kPathRows[path], s);
  }
  g.slices = slices_of(row_tiles * ceil_div(g.N, 256), kTileGrid, 8, g.R, g.N, g.K, most_slices);
  if constexpr (F32) return BTX_ERR_UNSUPPORTED;
  else return launch_tiles<kOut>(g, s);
}

}  // namespace

int f8_prepare() {
  if (int rc = raise_lds<f8_tile_kernel<kUp, false>>(kTileLds)) return rc;
  if (int rc = raise_lds<f8_tile_kernel<kUp, true>>(kTileLds)) return rc;
  if (int rc = raise_lds<f8_tile_kernel<kOut, false>>(kTileLds)) return rc;
  if (int rc = raise_lds<f8_tile_kernel<kOut, true>>(kTileLds)) return rc;
  if (int rc = raise_lds<f8_mid_kernel<kMidUp, 64>>(Mid<64>::lds)) return rc;
  if (int rc = raise_lds<f8_mid_kernel<kMidUp, 128>>(Mid<128>::lds)) return rc;
  if (int rc = raise_lds<f8_mid_kernel<kMidOut, 64>>(Mid<64>::lds)) return rc;
  if (int rc = raise_lds<f8_mid_kernel<kMidOut, 128>>(Mid<128>::lds)) return rc;
  if (int rc = raise_lds<f8_mid_kernel<kMidExact, 64>>(Mid<64>::lds)) return rc;
  return raise_lds<f8_mid_kernel<kMidExact, 128>>(Mid<128>::lds);
}

// (never less for more rows, also where so many are not cut)
size_t f8_matmul_workspace_bytes(int M, int N, int K) { return f8_pitch(K) / kF8Block >= 16 ? (size_t)sum_bytes(M, N) : 0; }
int launch_f8_matmul(const F8Matmul& m, hipStream_t s) {
  F8Args g{m.a, m.b, {nullptr, nullptr}, nullptr, nullptr, 1, 1, m.M, m.N, m.K, nullptr, nullptr, m.out, m.residual, 1, static_cast<float*>(m.workspace)};
  const bool bf16 = m.dtype == BTX_BF16;
  // A result of few columns, turned: few rows of b, with the many of a for weights.  Tiles of 64 rows and 128 columns are cut along K for these, and have
  // most of their columns empty.  us, turned / not, rows x columns, K:  800 x 8  2048 5.1 7.2, 8192 9.7 9.8;  800 x 64  2048 7.9 7.8, 4096 14 10;
  // 3000 x 16  2048 5.8 7.9, 4096 7.2 10, 8192 12 13;  16384 x 16  520 6.0 5.9, 4096 15 18, 8192 26 32 (fp32 38 55);  16384 x 64  2048 15 11, 8192 42 32
  if (m.M > 64 && (m.M < 4096 ? m.N <= 64 && (int64_t)m.K * (m.N + 16) <= 180000 : m.N <= 16)) {
    const F8Args t{m.b, m.a, {nullptr, nullptr}, nullptr, nullptr, 1, 1, m.N, m.M, m.K, nullptr, nullptr, m.out, m.residual, 1, nullptr, true, false};
    return bf16 ? launch_few<bf16_t>(t, m.N <= 32 ? 32 : 64, s) : launch_few<float>(t, m.N <= 32 ? 32 : 64, s);
  }
  Path path = out_path(m.M, 1, m.N, m.K, !bf16);
  if (path == kTall && !bf16) path = kMid128;
  const int most = f8_matmul_workspace_bytes(m.M, m.N, m.K) ? kMostSlices : 1;
  if (int rc = bf16 ? launch_out<false>(g, path, most, s) : launch_out<true>(g, path, most, s)) return rc;
  if (g.slices > 1) {
    const int64_t n = (int64_t)m.M * m.N / 4;
    const unsigned blocks = (unsigned)std::min<int64_t>((n + kAddThreads - 1) / kAddThreads, 1 << 20);
    const f32x4* const sums = reinterpret_cast<const f32x4*>(g.sums);
    if (bf16) f8_add_slices_kernel<<<blocks, kAddThreads, 0, s>>>(sums, g.slices, n, static_cast<const bf16_t*>(m.residual), static_cast<bf16_t*>(m.out));
    else f8_add_slices_kernel<<<blocks, kAddThreads, 0, s>>>(sums, g.slices, n, static_cast<const float*>(m.residual), static_cast<float*>(m.out));
    BTX_LAUNCH_CHECK();
  }
  return BTX_OK;
}

int launch_f8_up(const F8Layer& l, hipStream_t s) {
  const F8Args g{l.x, l.W1, l.W3, l.offsets, l.perm, l.E, l.k, l.T * l.k, l.f, l.d, l.act_codes, l.act_scales, nullptr, nullptr, 1, static_cast<float*>(l.y)};
  const Path path = up_path(g.R, l.E, l.f);
  if (path == kTall) return launch_tiles<kUp>(g, s);
  if (int rc = path == kFew32 ? launch_few_up(g, s) : launch_mid<kMidUp>(g, kPathRows[path], s)) return rc;
  return launch_f8_quantize(g.sums, BTX_F32, 1, g.R, g.N, 1, 1, g.act_codes, g.act_scales, s);
}

// y or the sums of its slices; before these the activations of all but the tall tiles in fp32
size_t f8_y_bytes(int64_t R, int d, int f, int E) {
  const int64_t rows = std::min(R, std::max<int64_t>(kUpMidRows * E, kUpMidTiles * 128 / ceil_div(f, 64)));
  return (size_t)std::max({R * d * 2, sum_bytes(R, d), rows * f * 4});
}
// y in fp32 where it is this small (1 us at most of 64 tokens, 2 of 256 with top-4).  Rounded to bf16, as it is where writing and reading it counts, two
// experts' rows put out 2.3e-3 of its norm off, and not the 1.7e-3 that rounding out itself costs
constexpr int64_t kMost32Bytes = 16 << 20;
static_assert(kMost32Bytes <= kSumBytes, "room in y");
int launch_f8_down(const F8Layer& l, int* slices, hipStream_t s) {
  const int R = l.T * l.k, most = combine_most_slices(l.T, l.k, BTX_BF16);
  F8Args g{{l.act_codes, l.act_scales}, l.W2, {nullptr, nullptr}, l.offsets, nullptr, l.E, l.k, R, l.d, l.f, nullptr, nullptr, l.y, nullptr, 1, static_cast<float*>(l.y)};
  g.in32 = most > 1 && (int64_t)R * l.d * 4 <= kMost32Bytes;
  if (int rc = launch_out<false>(g, out_path(R, l.E, l.d, l.f, false), most, s)) return rc;
  *slices = g.in32 || g.slices > 1 ? g.slices : 0;
  return BTX_OK;
}

}  // namespace btx
