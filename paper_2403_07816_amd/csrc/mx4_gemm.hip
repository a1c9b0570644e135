// Products of the layer of 4-bit experts (serving): UP, act = silu(xq W1_e) * (xq W3_e) quantised along f, and DOWN, y = act W2_e.
// Both operands are microscaled 4-bit floats with K contiguous (mx4.h); v_mfma_scale_f32_16x16x128_f8f6f4 takes codes and scales as they
// are, exact products, sums in fp32.  A lane's 16 bytes of a fragment are one block of 32 elements of a row: lane l holds row l % 16,
// and which four blocks of K the lane groups l / 16 hold is free, as long as both operands agree.  The weights are the first operand: each
// lane then ends up with four consecutive columns of one token row.
#include "mx4.h"

#include <atomic>
#include <type_traits>

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

// ---- many rows: 256 x 256 tiles --------------------------------------------------------------------------------
// Bound by the matrix cores and by what feeds them from LDS.  A tile is [row][128 bytes] per operand and k tile (256 elements), 8 wavefronts
// have 128 x 64 of the result each (UP: 32 columns of either panel, one block of the activations), 128 accumulator registers.
//   * global -> LDS copies are direct, 16 bytes a lane; two stages of both operands (128 KB), and two of the scales, which come for two
//     k tiles at a time: 16 bytes a row (2 x 8 KB).
//   * 16-byte chunks are XOR-swizzled by row (by choosing which chunk a lane fetches), so that the 16 rows of a fragment read meet no
//     bank twice.  Step s of a k tile takes chunks 2g + s of lane group g: the two scales that a lane needs of a row are neighbours.
//   * The two wavefronts of a SIMD alternate between a memory phase (fragment reads of half a k tile) and a compute phase (32 products),
//     half a period apart, with a barrier at every boundary; the copies of the next k tile are issued in the first memory phase.
//   * Tiles are dealt so that the ones an XCD runs at a time share row and column panels in its L2.
__device__ __forceinline__ void copy16(uint64_t base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(off), "s"(base) : "memory");
}
// 4 KB: the instruction's offset counts in memory as in LDS, so the lanes' offsets are that much lower and `base` kCopyBias lower still
constexpr uint32_t kCopyBias4 = 3 * 1024;
__device__ __forceinline__ void copy64(uint64_t base, const uint32_t (&off)[4], uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1\n\tglobal_load_lds_dwordx4 %3, %1 offset:1024\n\t"
      "global_load_lds_dwordx4 %4, %1 offset:2048\n\tglobal_load_lds_dwordx4 %5, %1 offset:3072"
      :
      : "s"(lds), "s"(base), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3])
      : "memory");
}

constexpr int kSup = 16, kXcdRows = 4, kXcds = 8;       // supertile of 16 x 16 tiles; of it an XCD has 4 x 8
// tile `id` of n_rt x n_ct: 256 consecutive ids are one supertile; what is right of and below the last whole one is a list that is cut
// into 8 equal runs.  false: no tile (there are up to 8 such ids)
__device__ __forceinline__ bool tile_of(int id, int n_rt, int n_ct, int& tm, int& tn) {
  const int fr = n_rt / kSup, fc = n_ct / kSup, whole = fr * fc * kSup * kSup;
  if (id < whole) {
    constexpr int SUB_M = kSup / kXcdRows, SUB_N = kSup / (kXcds / kXcdRows);
    const int sup = id / (kSup * kSup), r = id % (kSup * kSup), xcd = r % kXcds, slot = r / kXcds;
    tm = (sup / fc) * kSup + (xcd % kXcdRows) * SUB_M + slot % SUB_M;
    tn = (sup % fc) * kSup + (xcd / kXcdRows) * SUB_N + slot / SUB_M;
    return true;
  }
  const int l0 = id - whole, w = n_ct - fc * kSup, h = n_rt - fr * kSup;
  const int right = fr * kSup * w, left = right + h * n_ct, run = (left + kXcds - 1) / kXcds;
  const int l = (l0 % kXcds) * run + l0 / kXcds;
  if (l0 / kXcds >= run || l >= left) return false;
  if (l < right) {
    tm = l / w;
    tn = fc * kSup + l % w;
  } else {
    tm = fr * kSup + (l - right) % h;
    tn = (l - right) / h;
  }
  return true;
}

constexpr int kTileRows = 256, kTileCols = 256, kTileWaves = 8, kTileK = 256;   // (UP: 128 columns of W1, 128 of W3)
constexpr uint32_t kStage = 32768, kScaleStage = 8192;
constexpr uint32_t kB0 = 2 * kStage, kScale0 = 4 * kStage;
constexpr int kTileLds = 4 * kStage + 2 * kScaleStage;

template <bool UP>
__global__ __launch_bounds__(kTileWaves* kWave, 2) void mx4_tile_kernel(Mx4Args g, int n_ct) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  constexpr int TM = 8, TN = 4, TNH = UP ? 2 : 4, COLS = UP ? 128 : 256;
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int wm = wave >> 2, wn = wave & 3, grp = wm;     // the wavefronts of a SIMD are w and w + 4
  int e, row0, row_end, tn;
  {
    const ManyRowTiles tiles(g.offsets, g.E, kTileRows, lane);
    int tm;
    if (!tile_of(blockIdx.x, tiles.count(), n_ct, tm, tn) || tm >= tiles.count()) return;
    tiles.find(tm, e, row0, row_end);
  }
  const int col0 = tn * COLS;
  const int n_blk = g.K / kMxBlock, nk = (g.K + kTileK - 1) / kTileK, tail = n_blk - (nk - 1) * 8;   // blocks of the last k tile
  const int64_t pitch = mx4_pitch(g.K), row_bytes = g.K / 2;

  // ---- copies: wavefront w has rows 32 w .. of either operand, 8 lanes a row, 8 rows an instruction
  uint32_t a_off[4], b_off[4];
  int chunk[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int row = wave * 32 + q * 8 + lane / 8;
    chunk[q] = (lane & 7) ^ ((row >> 1) & 7);
    const int gr = min(row0 + row, row_end - 1);
    const uint32_t a_row = g.perm ? (uint32_t)(g.perm[gr] / g.k) : (uint32_t)(gr - row0);
    a_off[q] = a_row * (uint32_t)row_bytes + chunk[q] * 16 + (kCopyBias4 - 1024 * q);
    const int col = min(col0 + (UP ? row & 127 : row), g.N - 1) - col0;
    b_off[q] = (uint32_t)col * (uint32_t)row_bytes + chunk[q] * 16 + (kCopyBias4 - 1024 * q);
  }
  const Mx4Matrix& bm = UP && wave >= 4 ? g.b1 : g.b0;
  uint64_t a_from = uniform64(g.a.codes + (g.perm ? 0 : (int64_t)row0 * row_bytes)) - kCopyBias4;
  uint64_t b_from = uniform64(bm.codes + ((int64_t)e * g.N + col0) * row_bytes) - kCopyBias4;
  // scales: row 64 w + lane of A's 256 rows and B's 256 columns
  uint64_t s_from;
  uint32_t s_off;
  {
    const int row = (wave & 3) * 64 + lane;
    if (wave < 4) {
      const int gr = min(row0 + row, row_end - 1);
      s_off = (uint32_t)(g.perm ? g.perm[gr] / g.k : gr - row0) * (uint32_t)pitch;
      s_from = uniform64(g.a.scales + (g.perm ? 0 : (int64_t)row0 * pitch));
    } else {
      const int col = min(col0 + (UP ? row & 127 : row), g.N - 1) - col0;
      s_off = (uint32_t)col * (uint32_t)pitch;
      const Mx4Matrix& m = UP && wave >= 6 ? g.b1 : g.b0;
      s_from = uniform64(m.scales + ((int64_t)e * g.N + col0) * pitch);
    }
  }
  const uint32_t base = (uint32_t)(uintptr_t)smem;
  uint32_t to = base + wave * 4096;                      // of A; B's is kB0 behind
  const uint32_t s_to = base + kScale0 + wave * 1024;
  auto copy_scales = [&](int pair) { copy16(s_from + (uint64_t)pair * 16, s_off, s_to + (pair & 1) * kScaleStage); };
  auto copy_tile = [&](bool last) {                      // last: chunks behind K are re-pointed at the row's first of this tile
    uint32_t ao[4], bo[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t back = last && chunk[q] >= tail ? chunk[q] * 16 : 0;
      ao[q] = a_off[q] - back;
      bo[q] = b_off[q] - back;
    }
    copy64(a_from, ao, to);
    copy64(b_from, bo, to + kB0);
  };
  auto next_tile = [&] {
    a_from += kTileK / 2;
    b_from += kTileK / 2;
    to ^= kStage;                                        // (LDS of the launch starts at a multiple of two stages)
  };

  // ---- fragments: lane l has row l % 16 and chunks 2 (l / 16) + step
  const int r = lane & 15, lg = lane >> 4;
  typedef const __attribute__((address_space(3))) u32x4* lds_frag;
  typedef const __attribute__((address_space(3))) uint32_t* lds_word;
  uint32_t at_a = base + (wm * 128 + r) * 128 + (((2 * lg) ^ ((r >> 1) & 7)) << 4);
  uint32_t at_b = base + kB0 + (wn * (TNH * 16) + r) * 128 + (((2 * lg) ^ ((r >> 1) & 7)) << 4);
  const uint32_t sc_a = base + kScale0 + (wm * 128 + r) * 16 + 4 * (lg >> 1);
  const uint32_t sc_b = base + kScale0 + (256 + wn * (TNH * 16) + r) * 16 + 4 * (lg >> 1);
  const uint32_t sc_shift = 16 * (lg & 1);
  f32x4 acc[TM][TN] = {};
  u32x4 fa[TM], fb[TN];
  uint32_t xa[TM], xb[TN];
  auto read_frags = [&](int step) {
    const uint32_t a = at_a ^ (step << 4), b = at_b ^ (step << 4);
#pragma unroll
    for (int i = 0; i < TM; ++i) fa[i] = *(lds_frag)(uintptr_t)(a + i * 2048);
#pragma unroll
    for (int j = 0; j < TN; ++j) fb[j] = *(lds_frag)(uintptr_t)(b + (j / TNH) * (128 * 128) + (j % TNH) * 2048);
  };
  auto read_scales = [&](int kt) {
    const uint32_t where = ((kt >> 1) & 1) * kScaleStage + (kt & 1) * 8;
#pragma unroll
    for (int i = 0; i < TM; ++i) xa[i] = *(lds_word)(uintptr_t)(sc_a + where + i * 256);
#pragma unroll
    for (int j = 0; j < TN; ++j) xb[j] = *(lds_word)(uintptr_t)(sc_b + where + (j / TNH) * 2048 + (j % TNH) * 256);
  };
  auto k_tile = [&](auto fast_tag, int kt) {
    constexpr bool fast = decltype(fast_tag)::value;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (h == 0 && (fast || kt + 1 < nk)) {
        next_tile();
        copy_tile(!fast && kt + 2 == nk);
        if (kt & 1) copy_scales((kt + 1) >> 1);
      }
      __builtin_amdgcn_sched_barrier(0);
      read_frags(h);
      if (h == 0) read_scales(kt);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_waitcnt(0xC07F);                // lgkmcnt(0)
      if (h == 0) {
#pragma unroll
        for (int i = 0; i < TM; ++i) xa[i] >>= sc_shift;
#pragma unroll
        for (int j = 0; j < TN; ++j) xb[j] >>= sc_shift;
      }
      if (!fast && kt + 1 == nk && 2 * lg + h >= tail) {
#pragma unroll
        for (int i = 0; i < TM; ++i) fa[i] = u32x4{0u, 0u, 0u, 0u};
      }
      if (h == 1 && grp == 1) wait_vmcnt<0>();
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
          acc[i][j] = h == 0 ? mfma_mx4<0>(fb[j], fa[i], acc[i][j], xb[j], xa[i]) : mfma_mx4<1>(fb[j], fa[i], acc[i][j], xb[j], xa[i]);
      if (h == 1 && grp == 0) wait_vmcnt<0>();
      if (h == 1) {
        at_a ^= kStage;
        at_b ^= kStage;
      }
      __builtin_amdgcn_sched_barrier(0);
      if (fast || !(grp == 1 && h == 1 && kt + 1 == nk)) __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  copy_tile(nk == 1);
  copy_scales(0);
  wait_vmcnt<0>();
  __builtin_amdgcn_s_barrier();
  if (grp == 1) __builtin_amdgcn_s_barrier();            // group 1 is a phase behind
  int kt = 0;
#pragma unroll 1
  for (; kt < nk - 2; ++kt) k_tile(std::true_type{}, kt);
#pragma unroll 1
  for (; kt < nk; ++kt) k_tile(std::false_type{}, kt);

  // ---- epilogue: acc[i][j][v] is row wm 128 + 16 i + l % 16, column 16 j + 4 (l / 16) + v of the wavefront's.  The operand stages are dead
  // (group 0's last barrier comes after group 1's last read).
  if constexpr (UP) {
    // a wavefront's 32 columns are one block; codes [256 rows][64 bytes] and scales [256][4] are put together in LDS
    __syncthreads();
    char* const s_codes = smem;
    char* const s_scales = smem + 256 * 64;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int row = wm * 128 + i * 16 + r;
      float v[2][4];
      uint32_t amax = 0;
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          v[j][x] = silu_f(acc[i][j][x]) * acc[i][j + 2][x];
          amax = max(amax, magnitude(v[j][x]));
        }
      amax = max(amax, (uint32_t)__shfl_xor((int)amax, 16, kWave));
      amax = max(amax, (uint32_t)__shfl_xor((int)amax, 32, kWave));
      const uint32_t byte = mx4_scale_byte(amax);
      const float scale = mx4_scale(byte);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        uint32_t w = 0;
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[j][0], v[j][1], scale, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[j][2], v[j][3], scale, 1);
        *reinterpret_cast<uint16_t*>(s_codes + row * 64 + wn * 16 + j * 8 + lg * 2) = byte == 255u ? 0 : (uint16_t)w;
      }
      if (lg == 0) s_scales[row * 4 + wn] = col0 + wn * 32 < g.N ? (char)byte : 0;
    }
    __syncthreads();
    const int64_t out_row = g.N / 2, out_pitch = mx4_pitch(g.N);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int idx = q * 512 + threadIdx.x, row = idx >> 2, c = idx & 3;
      if (row0 + row < row_end && col0 + c * 32 < g.N)
        *reinterpret_cast<u32x4*>(g.act_codes + (int64_t)(row0 + row) * out_row + col0 / 2 + c * 16) =
            *reinterpret_cast<const u32x4*>(s_codes + row * 64 + c * 16);
    }
    if (threadIdx.x < 256 && row0 + (int)threadIdx.x < row_end) {
      uint8_t* const to_scales = g.act_scales + (int64_t)(row0 + threadIdx.x) * out_pitch;
      *reinterpret_cast<uint32_t*>(to_scales + col0 / 32) = *reinterpret_cast<const uint32_t*>(s_scales + threadIdx.x * 4);
      if (col0 + COLS >= g.N)                            // the zeros behind them
        for (int z = col0 / 32 + 4; z < (int)out_pitch; z += 4) *reinterpret_cast<uint32_t*>(to_scales + z) = 0;
    }
  } else {
    // 32 rows of the wavefront's 64 columns at a time (128 bytes a row) through its own piece of LDS, chunks swizzled by row
    __syncthreads();
    char* const band = smem + wave * 4096;
    const int n0 = col0 + wn * 64;
#pragma unroll
    for (int ib = 0; ib < TM / 2; ++ib) {
#pragma unroll
      for (int i2 = 0; i2 < 2; ++i2)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x4& v = acc[2 * ib + i2][j];
          const int row = i2 * 16 + r, byte = (j * 16 + 4 * lg) * 2;
          *reinterpret_cast<u32x2*>(band + row * 128 + ((byte >> 4 ^ (row & 7)) << 4) + (byte & 15)) =
              u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
        }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int row = q * 8 + lane / 8, c = lane & 7, m = row0 + wm * 128 + ib * 32 + row;
        const u32x4 w = *reinterpret_cast<const u32x4*>(band + row * 128 + ((c ^ (row & 7)) << 4));
        if (m < row_end && n0 + c * 8 < g.N) __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(g.y + (int64_t)m * g.N + n0 + c * 8));
      }
    }
  }
}

// the dynamic-LDS limit, once per device (not while a stream is being captured; btx_init() does it too)
template <auto KERNEL> int raise_lds() {
  static std::atomic<uint64_t> done{0};
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return BTX_ERR_HIP;
  if (!(done.load(std::memory_order_relaxed) >> dev & 1)) {
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, kTileLds) != hipSuccess)
      return BTX_ERR_HIP;
    done.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  return BTX_OK;
}

template <bool UP> int launch_tiles(const Mx4Args& g, int R, hipStream_t s) {
  if (int rc = raise_lds<mx4_tile_kernel<UP>>()) return rc;
  const int n_ct = ceil_div(g.N, UP ? 128 : 256);
  const int64_t tiles = ((int64_t)ceil_div(R, kTileRows) + std::min(g.E, R)) * n_ct + kXcds;
  if (!grid_fits(tiles, kTileWaves * kWave)) return BTX_ERR_UNSUPPORTED;
  mx4_tile_kernel<UP><<<(unsigned)tiles, kTileWaves * kWave, kTileLds, s>>>(g, n_ct);
  BTX_LAUNCH_CHECK();
  return BTX_OK;
}

// gathered rows are found with 32-bit offsets
bool tiles_ok(const Mx4Args& g, int T) { return !g.perm || (int64_t)T * (g.K / 2) + kTileK < (int64_t)1 << 32; }
template <bool UP> int launch(const Mx4Args& g, int T, int R, hipStream_t s) {
  return R / g.E >= 64 && tiles_ok(g, T) ? launch_tiles<UP>(g, R, s) : launch_few<UP>(g, R, s);
}

}  // namespace

int mx4_prepare() {
  if (int rc = raise_lds<mx4_tile_kernel<true>>()) return rc;
  return raise_lds<mx4_tile_kernel<false>>();
}

int launch_mx4_up(const Mx4Matrix& xq, const Mx4Matrix& W1, const Mx4Matrix& W3, const int32_t* offsets, const int32_t* perm,
                  const Mx4Shapes& sh, uint8_t* act_codes, uint8_t* act_scales, hipStream_t s) {
  const Mx4Args g{xq, W1, W3, offsets, perm, sh.k, sh.E, sh.f, sh.d, act_codes, act_scales, nullptr};
  return launch<true>(g, sh.T, sh.T * sh.k, s);
}

int launch_mx4_down(const Mx4Matrix& act, const Mx4Matrix& W2, const int32_t* offsets, const Mx4Shapes& sh, void* y, hipStream_t s) {
  const Mx4Args g{act, W2, {nullptr, nullptr}, offsets, nullptr, 1, sh.E, sh.d, sh.f, nullptr, nullptr, static_cast<bf16_t*>(y)};
  return launch<false>(g, sh.T, sh.T * sh.k, s);
}

}  // namespace btx
