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

// one step of K = 128; SW, SX: which byte of the scale words
template <int SW, int SX = SW> __device__ __forceinline__ f32x4 mfma_mx4(const u32x4& w, const u32x4& x, const f32x4& acc, uint32_t w_scale, uint32_t x_scale) {
  const i32x8 a = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0}, b = {(int)x[0], (int)x[1], (int)x[2], (int)x[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 4, SW, (int)w_scale, SX, (int)x_scale);
}

struct Mx4Args {
  Mx4Matrix a, b0, b1;                  // token rows; weights (b1: W3)
  const int32_t* tokens;                // row r of the product is row tokens[r] of a (NULL: row r)
  const TileInfo* tiles;                // row tiles: the first entry's row0 is their number
  int a_rows;                           // of a (tile kernel: their scales' order, see mx4_scale_at())
  int N, K;                             // columns, depth
  uint8_t* act_codes; uint8_t* act_scales; bf16_t* y;
  int R;
  int slices;                           // DOWN in tiles: K ranges of a tile; more than one: sums [slice][R][N] in fp32, in y's place
};

// ---- few rows: up to 64 rows x 32 columns a workgroup, whose wavefronts share K ---------------------------------
// Bound by reading the weights.  They go from memory to the registers that the products take, 512 elements of 16 rows a wavefront at a time: in
// step s lane group g has chunk 4s + g, so that a load covers 64 bytes of a row; of the row's 16 scales a lane picks every fourth.  RB blocks of
// 16 rows meet each fragment of the weights.  With 4 wavefronts two or three workgroups are on a compute unit and begin and end beside each
// other (one token, 2 experts of 4096 x 11008: UP with 8 wavefronts, one workgroup at a time, 29 us).  All loads of a step are under way
// before its first product: with a block's rows loaded as its turn came, 64 tokens of 32 experts of 4096 x 1376 took 71 us, now 68, and 96
// tokens of 4 of 4096 x 11008 114 us, now 111.
constexpr int kFewCols = 32, kFewMostWaves = 8;
// (tiles of 32 rows only where R < 25 E)
static_assert(kMx4MostColumns / kFewCols <= 65535 && (kMx4MostRows / 64 + kMx4MaxExperts + 0ll) * kFewMostWaves * kWave < 1ll << 32, "the grid");
// byte g of each of four words; pick: g | (4 + g) << 8
__device__ __forceinline__ uint32_t every_fourth(const u32x4& v, uint32_t pick) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(v[3], v[2], pick), __builtin_amdgcn_perm(v[1], v[0], pick), 0x05040100u);
}
template <bool UP, int RB, int NW>
__global__ __launch_bounds__(NW* kWave, UP || RB == 4 ? 2 : 3) void mx4_few_kernel(Mx4Args g) {
  constexpr int PANELS = UP ? 2 : 1;
  __shared__ f32x4 s_sum[NW][RB][PANELS * 2][kWave];
  if ((int)blockIdx.x >= g.tiles[0].row0) return;
  const TileInfo tile = g.tiles[1 + blockIdx.x];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int n0 = blockIdx.y * kFewCols, r = lane & 15, grp = lane >> 4;
  const int n_blk = g.K / kMxBlock;
  const int64_t pitch = mx4_pitch(g.K);
  const uint32_t pick = (uint32_t)grp | (uint32_t)(4 + grp) << 8;
  const u32x4* const a = reinterpret_cast<const u32x4*>(g.a.codes);
  uint32_t row[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    row[rb] = (uint32_t)min(tile.row0 + rb * 16 + r, tile.row_end - 1);
    if (g.tokens) row[rb] = (uint32_t)g.tokens[row[rb]];
  }
  // the weights by one base for every 16 columns, and a lane's offset of 32 bits
  const char* w[PANELS * 2];
  const char* w_sc[PANELS * 2];
#pragma unroll
  for (int p = 0; p < PANELS * 2; ++p) {
    const Mx4Matrix& m = p < 2 ? g.b0 : g.b1;
    const int64_t n = (int64_t)tile.e * g.N + n0 + 16 * (p & 1);
    w[p] = reinterpret_cast<const char*>(m.codes) + n * n_blk * 16;
    w_sc[p] = reinterpret_cast<const char*>(m.scales) + n * pitch;
  }
  const uint32_t w_row = (uint32_t)r * (uint32_t)n_blk * 16, sc_row = (uint32_t)r * (uint32_t)pitch;
  f32x4 acc[RB][PANELS * 2] = {};
#pragma unroll 1
  for (int b0 = 16 * wave; b0 < n_blk; b0 += 16 * NW) {
    const int at = b0 + grp;                           // (scale rows are whole 16 bytes; behind K / 32 they are zero)
    // all loads before the first product, those of x, which are not memory's, first
    u32x4 xv[RB][4], x_sc[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      if (rb > 0 && tile.row0 + rb * 16 >= tile.row_end) break;
      x_sc[rb] = *reinterpret_cast<const u32x4*>(g.a.scales + row[rb] * pitch + b0);
#pragma unroll
      for (int s = 0; s < 4; ++s) xv[rb][s] = at + 4 * s < n_blk ? a[(int64_t)row[rb] * n_blk + at + 4 * s] : u32x4{0u, 0u, 0u, 0u};
    }
    u32x4 wv[PANELS * 2][4], w_s[PANELS * 2];
#pragma unroll
    for (int p = 0; p < PANELS * 2; ++p) {
      w_s[p] = *reinterpret_cast<const u32x4*>(w_sc[p] + (sc_row + b0));
#pragma unroll
      for (int s = 0; s < 4; ++s)
        wv[p][s] = at + 4 * s < n_blk ? *reinterpret_cast<const u32x4*>(w[p] + (w_row + (at + 4 * s) * 16u)) : u32x4{0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int p = 0; p < PANELS * 2; ++p) {
      const uint32_t ws = every_fourth(w_s[p], pick);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        if (rb > 0 && tile.row0 + rb * 16 >= tile.row_end) break;
        const uint32_t xs = every_fourth(x_sc[rb], pick);
        acc[rb][p] = mfma_mx4<0>(wv[p][0], xv[rb][0], acc[rb][p], ws, xs);
        acc[rb][p] = mfma_mx4<1>(wv[p][1], xv[rb][1], acc[rb][p], ws, xs);
        acc[rb][p] = mfma_mx4<2>(wv[p][2], xv[rb][2], acc[rb][p], ws, xs);
        acc[rb][p] = mfma_mx4<3>(wv[p][3], xv[rb][3], acc[rb][p], ws, xs);
      }
    }
  }
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int p = 0; p < PANELS * 2; ++p) s_sum[wave][rb][p][lane] = acc[rb][p];
  __syncthreads();
  // thread t of 256: rows t / 16 of every block, columns 2 (t % 16) and the next: lane 16 (c % 16 / 4) + row of fragment c / 16, element c % 4
  const int out_row = (threadIdx.x & 255) / 16, c = 2 * (threadIdx.x % 16);
  const int from = 16 * ((c & 15) >> 2) + out_row, half = c >> 4, el = c & 3;
  for (int rb = threadIdx.x / 256; rb < RB; rb += NW * kWave / 256) {
    const int m = tile.row0 + rb * 16 + out_row;
    if (m - out_row >= tile.row_end) break;
    float sum[PANELS][2] = {};
#pragma unroll
    for (int x = 0; x < NW; ++x)
#pragma unroll
      for (int p = 0; p < PANELS; ++p) {
        const f32x2* v = reinterpret_cast<const f32x2*>(&s_sum[x][rb][2 * p + half][from]);
        sum[p][0] += v[el >> 1][0];
        sum[p][1] += v[el >> 1][1];
      }
    const bool live = m < tile.row_end;
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
    } else {                                             // (y in bf16: half the bytes that are written here and read by whoever combines the rows)
      if (live) *reinterpret_cast<uint32_t*>(g.y + (int64_t)m * g.N + n0 + c) = pack_bf16x2(sum[0][0], sum[0][1]);
    }
  }
}

template <bool UP> int launch_few(const Mx4Args& g, int tile_rows, int E, hipStream_t s) {
  const int tiles = mx4_most_tiles(g.R, E, tile_rows), cols = g.N / kFewCols;
  auto go = [&](auto rb, auto nw) {
    mx4_few_kernel<UP, decltype(rb)::value, decltype(nw)::value><<<dim3((unsigned)tiles, (unsigned)cols), decltype(nw)::value * kWave, 0, s>>>(g);
  };
  auto rows = [&](auto nw) {
    if (tile_rows == 32) go(std::integral_constant<int, 2>{}, nw);
    else go(std::integral_constant<int, 4>{}, nw);
  };
  // 8 wavefronts where each has two pieces of 512 elements or more
  if (g.K >= 16 * 512) rows(std::integral_constant<int, 8>{});
  else rows(std::integral_constant<int, 4>{});
  BTX_LAUNCH_CHECK();
  return BTX_OK;
}

// ---- many rows: 256 x 256 tiles --------------------------------------------------------------------------------
// Bound by the matrix cores and by what feeds them from LDS.  A tile is [row][128 bytes] per operand and k tile (256 elements), 8 wavefronts
// have 128 x 64 of the result each (UP: 32 columns of either panel, one block of the activations), 128 accumulator registers.
//   * global -> LDS copies are direct, 16 bytes a lane, two stages of both operands (128 KB).
//   * 16-byte chunks are XOR-swizzled by row (by choosing which chunk a lane fetches), so that the 16 lanes of a fragment read's pass meet no
//     bank twice.  Step s of a k tile takes chunk 2g + s of lane group g.  (The counters have 129 cycles of conflicts in a k tile's 1018 all the same,
//     1000 in DOWN's epilogue and 1760 in UP's.)
//   * The two wavefronts of a SIMD alternate between a memory phase and a compute phase (32 products), half a period apart, with a barrier at
//     every boundary.  The first memory phase of a k tile reads all fragments of B and those of half of A's rows, the second the other
//     half's: B's stage and half of A's are free half a k tile early, and the copies of the k tile after the next go there.
//   * Scales: a lane's two of B for a k tile are neighbours and read as 16 bits.  A's, which only these kernels read, lie in an order
//     (mx4_scale_at()) in which the four of two k tiles are one word, and 16 bytes of every row for two k tiles beside each other.  (With
//     A's like B's, 12 words a lane and two k tiles dealt out by v_permlane32_swap and v_perm, the products of a k tile waited 260 cycles for it.)
//   * Tiles are dealt so that the ones an XCD runs at a time share row and column panels in its L2.
//   * Of a tile's rows that an expert does not have, 64 of a wavefront's are passed over, their reads and their products; the other wavefront of the SIMD
//     goes on sooner (96 tokens of 4 experts of 4096 x 11008 108 us -> 92, 192 of 32 of 4096 x 1376 117 -> 95, 301 of the former 121 -> 116).
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

constexpr uint32_t kCopyBias2 = 1024;
__device__ __forceinline__ void copy32(uint64_t base, uint32_t off0, uint32_t off1, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1\n\tglobal_load_lds_dwordx4 %3, %1 offset:1024"
               :
               : "s"(lds), "s"(base), "v"(off0), "v"(off1)
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

constexpr int kTileRows = 256, kTileWaves = 8, kTileK = 256;   // x 256 columns (UP: 128 of W1, 128 of W3)
constexpr uint32_t kStage = 32768, kScaleAStage = 4096, kScaleBStage = 8192;   // scales: of 2 (A) and 4 (B) k tiles
constexpr uint32_t kB0 = 2 * kStage, kScaleA0 = 4 * kStage, kScaleB0 = kScaleA0 + 2 * kScaleAStage;
constexpr int kTileLds = kScaleB0 + 2 * kScaleBStage;
constexpr int kTileGrid = 256;                          // compute units; a multiple of kXcds

// Chunk c of a row lies at chunk c ^ tile_swz(row).  A 16-byte read of 64 lanes takes four passes, of lanes 0-3, 12-15 and 20-27, of 4-11, 16-19 and
// 28-31, and so on; with chunks 2g of lane group g, (row >> 1) & 7 alone put 0-3 and 12-15 in the banks of 20-27 (16384 tokens of the
// 7B-shaped layer 2.60 / 2.45 ms).
__device__ __forceinline__ int tile_swz(int row) {
  const int i = (row >> 1) & 7;
  return i ^ ((i & 2) << 1);
}

// the same number, worked on where it is used: what follows from a lane's index for a tile's begin and end is not kept in registers over
// its k loop (spilt registers are read back behind all copies and stores on their way: 18 us a tile)
__device__ __forceinline__ int here(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

template <bool UP>
__global__ __launch_bounds__(kTileWaves* kWave, 2) void mx4_tile_kernel(Mx4Args g, int n_ct) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  constexpr int TM = 8, TN = 4, TNH = UP ? 2 : 4, COLS = UP ? 128 : 256;
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int wm = wave >> 2, wn = wave & 3, grp = wm;     // the wavefronts of a SIMD are w and w + 4
  const int nk_all = (g.K + kTileK - 1) / kTileK, slices = UP ? 1 : g.slices;
  const int64_t pitch = mx4_pitch(g.K), row_bytes = g.K / 2;
  const uint32_t base = (uint32_t)(uintptr_t)smem;

  // ---- the tile
  const int n_rt = g.tiles[0].row0, most = n_rt * n_ct + kXcds;
  int e, row0, row_end, col0, slice, id = blockIdx.x;
  int k_first, nk, tail;                                 // its k tiles: k_first (a multiple of four, as scales are copied) .. + nk - 1; blocks of the last
  auto find_tile = [&]() -> bool {                       // `id`, or the next one of this workgroup that names a tile
    int tm, tn;
    for (; id < most * slices; id += gridDim.x)
      if (tile_of(id % most, n_rt, n_ct, tm, tn)) {
        const int quads = (nk_all + 3) / 4;
        slice = id / most;
        k_first = slice * quads / slices * 4;
        nk = min((slice + 1) * quads / slices * 4, nk_all) - k_first;
        tail = min(g.K / kMxBlock - (k_first + nk - 1) * 8, 8);
        const TileInfo t = g.tiles[1 + tm];
        e = t.e;
        row0 = t.row0;
        row_end = t.row_end;
        col0 = tn * COLS;
        return true;
      }
    return false;
  };

  // ---- copies.  Rows 0-63 and 128-191 of A are its first half (A0), which the first memory phase reads, the others the second (A1): a
  // wavefront has 16 rows of either and 32 rows of B, 8 lanes a row, 8 rows an instruction; 64 rows of A's scales, or of B's (2 lanes a row).
  auto chunk = [](int ln, int q) { return (ln & 7) ^ tile_swz(ln / 8 + 8 * (q & 1)); };
  auto s_half = [](int ln) { return (ln & 1) ^ (ln >> 4 & 1); };   // the halves of rows 8 .. 15 of 16 change places (banks)
  const int a_row = wm * 128 + wn * 16;
  uint32_t a_off[4], b_off[4], s_off[2];                 // a_off: A0, A0, A1, A1
  uint64_t a_from, b_from, s_from;                       // a, b: of the k tile behind the next (A1: the one before)
  auto set_rows = [&] {                                  // (as indexes of rows, for now)
    const int ln = here(lane);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int gr = min(row0 + a_row + (q >> 1) * 64 + (q & 1) * 8 + ln / 8, row_end - 1);
      a_off[q] = (uint32_t)(g.tokens ? g.tokens[gr] : gr - row0);
    }
    if (wm == 0) {
      const int gr = min(row0 + wn * 64 + ln, row_end - 1);
      s_off[0] = (uint32_t)(g.tokens ? g.tokens[gr] : gr - row0);
    }
  };
  const uint32_t s_step = wm == 0 ? (uint32_t)g.a_rows * 16 : 32;     // to the scales of the next two k tiles (B: four)
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
    const Mx4Matrix& bm = UP && wave >= 4 ? g.b1 : g.b0;
    a_from = uniform64(g.a.codes + (g.tokens ? 0 : (int64_t)row0 * row_bytes)) - kCopyBias2 + (uint64_t)k_first * (kTileK / 2);
    b_from = uniform64(bm.codes + ((int64_t)e * g.N + col0) * row_bytes) - kCopyBias4 + (uint64_t)k_first * (kTileK / 2);
    if (wm == 0) {
      s_off[0] *= 16;
      s_off[1] = 0;
      s_from = uniform64(g.a.scales + (g.tokens ? 0 : (int64_t)row0 * 16)) + (uint64_t)(k_first / 2) * s_step;
    } else {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int row = wn * 64 + q * 32 + ln / 2, col = min(col0 + (UP ? row & 127 : row), g.N - 1) - col0;
        s_off[q] = (uint32_t)col * (uint32_t)pitch + s_half(ln) * 16;
      }
      s_from = uniform64((UP && wn >= 2 ? g.b1 : g.b0).scales + ((int64_t)e * g.N + col0) * pitch) + (uint64_t)k_first * 8;
    }
    asm volatile("" : "+v"(s_off[0]), "+v"(s_off[1]));
  };
  const uint32_t to_a = base + a_row * 128, to_b = base + kB0 + wave * 4096;
  const uint32_t to_s = base + (wm == 0 ? kScaleA0 + wn * 1024 : kScaleB0 + wn * 2048);
  // the last k tile's chunks behind K are re-pointed at the row's first of that tile
  auto back = [&](int ln, int q) -> uint32_t { return chunk(ln, q) >= tail ? chunk(ln, q) * 16 : 0; };
  auto copy_a0b = [&](int kt) {                          // a_from, b_from: of k tile kt
    if (kt + 1 == nk && tail < 8) {
      const int ln = here(lane);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (q < 2) a_off[q] -= back(ln, q);
        b_off[q] -= back(ln, q);
      }
    }
    copy32(a_from, a_off[0], a_off[1], to_a + (kt & 1) * kStage);
    copy64(b_from, b_off, to_b + (kt & 1) * kStage);
  };
  auto copy_a1 = [&](int kt, uint64_t from) {
    if (kt + 1 == nk && tail < 8) {
      const int ln = here(lane);
      a_off[2] -= back(ln, 2);
      a_off[3] -= back(ln, 3);
    }
    copy32(from, a_off[2], a_off[3], to_a + (kt & 1) * kStage + 64 * 128);
  };
  // One instruction for every two k tiles: A's scales of k tiles 2 pair, 2 pair + 1 (the wavefronts of wm 0), and of B's for four k tiles one half of
  // the rows.  (Behind the last ones: anything.  A row of B's may end in the middle of its last 32 bytes.)
  auto copy_scales_a = [&](int pair) {
    copy16(s_from + (uint64_t)min(pair, (nk - 1) / 2) * s_step, s_off[0], to_s + (pair & 1) * kScaleAStage);
  };
  auto copy_scales_b = [&](int quad, int q) {
    const int from = min(quad, (nk - 1) / 4);
    const uint32_t less = k_first * 8 + from * 32 + 16 >= (int)pitch ? s_half(here(lane)) * 16 : 0;
    copy16(s_from + (uint64_t)from * 32, (q ? s_off[1] : s_off[0]) - less, to_s + (quad & 1) * kScaleBStage + q * 1024);
  };

  // ---- fragments: lane l has row l % 16
  const int r = lane & 15, lg = lane >> 4;
  typedef const __attribute__((address_space(3))) u32x4* lds_frag;
  typedef const __attribute__((address_space(3))) uint32_t* lds_word;
  typedef const __attribute__((address_space(3))) uint16_t* lds_half;
  const uint32_t at_a = base + (wm * 128 + r) * 128 + ((2 * lg) ^ tile_swz(r)) * 16;
  const uint32_t at_b = base + kB0 + (wn * (TNH * 16) + r) * 128 + ((2 * lg) ^ tile_swz(r)) * 16;
  const uint32_t sc_a = base + kScaleA0 + (wm * 128 + r) * 16 + 4 * lg;
  const uint32_t sc_b = base + kScaleB0 + (wn * (TNH * 16) + r) * 32 + 2 * lg;
  const uint32_t sc_half = (r >> 3) * 16;                // where the first half of a row of B's is
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
  auto read_scales = [&](int kt, bool a) {
    if (a) {                                             // kt even: of it and the next
      const uint32_t at = sc_a + ((kt >> 1) & 1) * kScaleAStage;
#pragma unroll
      for (int i = 0; i < TM; ++i) xa[i] = *(lds_word)(uintptr_t)(at + i * 256);
    }
    const uint32_t at = sc_b + ((kt >> 2) & 1) * kScaleBStage + (sc_half ^ ((kt & 2) << 3)) + (kt & 1) * 8;
#pragma unroll
    for (int j = 0; j < TN; ++j) xb[j] = *(lds_half)(uintptr_t)(at + (j / TNH) * 4096 + (j % TNH) * 512);
  };
  // Copies: in the first memory phase of k tile kt A1 of kt + 1 (2 instructions), in the second A0 and B of kt + 2 (2 and 4) and in odd ones one of
  // scales.  What they overwrite was read last in the memory phases before, and they have four phases or more to land.
  auto k_tile = [&](auto odd_tag, int kt) {
    constexpr int odd = decltype(odd_tag)::value;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      // ---- memory phase
      const bool live = row0 + wm * 128 + h * 64 < row_end;    // (of this half of its rows any: a phase without products is short)
      if (live) {
        read_a(odd, h);
        if (h == 0) {
          read_b(odd);
          read_scales(kt, !odd);
        }
      }
      if (h == 0) {
        if (kt + 1 < nk) copy_a1(kt + 1, a_from - kTileK / 2);
      } else {
        if (kt + 2 < nk) {
          copy_a0b(kt + 2);
          a_from += kTileK / 2;
          b_from += kTileK / 2;
          if (odd) {
            if (wm == 0) copy_scales_a((kt + 1) / 2 + 1);
            else copy_scales_b(((kt + 1) >> 2) + 1, kt & 2 ? 0 : 1);
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_waitcnt(0xC07F);                // lgkmcnt(0)
      if (kt + 1 == nk && tail < 8) {
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          const uint32_t keep = 2 * (here(lane) >> 4) + st < tail ? ~0u : 0u;
#pragma unroll
          for (int i = 0; i < TM / 2; ++i) fa[i][st] &= keep;
        }
      }
      // What the next memory phases read has landed: behind h == 0, A1 of this k tile; behind h == 1, A0, B and scales of the next.  What has
      // been issued since may be outstanding.
      auto landed = [&] {
        if (h == 0) {
          if (kt + 1 < nk) wait_vmcnt<9 - odd>(); else wait_vmcnt<0>();
        } else {
          if (kt + 2 < nk) wait_vmcnt<8 + odd>(); else wait_vmcnt<2>();
        }
      };
      if (grp == 1) landed();
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
      // ---- compute phase
      if (live) {
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int i = 0; i < TM / 2; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j) {
            f32x4& c = acc[h * 4 + i][j];
            c = st == 0 ? mfma_mx4<0, 2 * odd>(fb[j][0], fa[i][0], c, xb[j], xa[h * 4 + i])
                        : mfma_mx4<1, 2 * odd + 1>(fb[j][1], fa[i][1], c, xb[j], xa[h * 4 + i]);
          }
      }
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
  auto start = [&] {                                     // into the first stages: k tile 0, and scales
    set_sources();
    if (wm == 0) {
      copy_scales_a(0);
    } else {
      copy_scales_b(0, 0);
      copy_scales_b(0, 1);
    }
    copy_a0b(0);
    copy_a1(0, a_from);
    a_from += kTileK / 2;
    b_from += kTileK / 2;
  };
  start();
  for (;;) {
    if (nk > 1) {                                        // into the second stages, as k tile -1 would have
      copy_a0b(1);
      a_from += kTileK / 2;
      b_from += kTileK / 2;
      if (wm == 0) copy_scales_a(1);
      else copy_scales_b(1, 0);
      wait_vmcnt<7>();
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
    for (int kt = 0; kt < nk; kt += 2) {
      k_tile(std::integral_constant<int, 0>{}, kt);
      if (kt + 1 < nk) k_tile(std::integral_constant<int, 1>{}, kt + 1);
    }

    // ---- epilogue: acc[i][j][v] is row wm 128 + 16 i + l % 16, column 16 j + 4 (l / 16) + v of the wavefront's.  All of LDS is free (group
    // 0's last barrier comes after group 1's last read); the result goes through the second stage of A, and the first stages are filled
    // for the workgroup's next tile beside it.
    const int out_row0 = row0, out_end = row_end, out_col0 = col0, out_slice = slice;
    const int ln = here(lane), r = ln & 15, lg = ln >> 4, tid = wave * kWave + ln;
    __syncthreads();
    id += gridDim.x;
    const bool more = find_tile();
    if (more) set_rows();
    char* const out = smem + kStage;
    if constexpr (UP) {
      // a wavefront's 32 columns are one block; codes [256 rows][64 bytes] and scales [256][4] are put together in LDS
      char* const s_scales = out + 256 * 64;
      if (more) start();                                 // (behind the activations: 301 tokens of 4 experts of 4096 x 11008 70 us, now 66)
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
          *reinterpret_cast<uint16_t*>(out + row * 64 + wn * 16 + j * 8 + lg * 2) = byte == 255u ? 0 : (uint16_t)w;
        }
        if (lg == 0) s_scales[row * 4 + wn] = out_col0 + wn * 32 < g.N ? (char)byte : 0;
      }
      __syncthreads();
      const int64_t out_row = g.N / 2, out_pitch = mx4_pitch(g.N);
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int idx = q * 512 + tid, row = idx >> 2, c = idx & 3;
        if (out_row0 + row < out_end && out_col0 + c * 32 < g.N)
          *reinterpret_cast<u32x4*>(g.act_codes + (int64_t)(out_row0 + row) * out_row + out_col0 / 2 + c * 16) =
              *reinterpret_cast<const u32x4*>(out + row * 64 + c * 16);
      }
      if (tid < 256 && out_row0 + tid < out_end) {
        const uint32_t four = *reinterpret_cast<const uint32_t*>(s_scales + tid * 4);
        auto put = [&](int b, uint32_t w) {              // blocks b, b + 1; b a multiple of 2
          *reinterpret_cast<uint16_t*>(g.act_scales + mx4_scale_at(g.R, out_row0 + tid, b)) = (uint16_t)w;
        };
        put(out_col0 / 32, four);
        put(out_col0 / 32 + 2, four >> 16);
        if (out_col0 + COLS >= g.N)                      // the zeros behind them
          for (int z = out_col0 / 32 + 4; z < (int)out_pitch; z += 2) put(z, 0);
      }
    } else {
      if (more) start();
      if (slices > 1) {                                  // four columns a lane, as they are
        float* const sums = reinterpret_cast<float*>(g.y) + ((int64_t)out_slice * g.R + out_row0) * g.N;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j) {
            const int m = wm * 128 + i * 16 + r, n = out_col0 + wn * 64 + j * 16 + 4 * lg;
            if (out_row0 + m < out_end && n < g.N) *reinterpret_cast<f32x4*>(sums + (int64_t)m * g.N + n) = acc[i][j];
          }
        if (!more) return;
        __syncthreads();
        continue;
      }
      // 32 rows of the wavefront's 64 columns at a time (128 bytes a row) through its own piece of LDS, chunks swizzled by row.  y in bf16: of
      // 16384 tokens of 8 slots 1.07 GB, which the combining kernel reads in 0.22 ms; in fp32 it would be twice that here and there.
      char* const band = out + wave * 4096;
      const int n0 = out_col0 + wn * 64;
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
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int row = q * 8 + ln / 8, c = ln & 7, m = out_row0 + wm * 128 + ib * 32 + row;
          const u32x4 w = *reinterpret_cast<const u32x4*>(band + row * 128 + ((c ^ (row & 7)) << 4));
          if (m < out_end && n0 + c * 8 < g.N) __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(g.y + (int64_t)m * g.N + n0 + c * 8));
        }
        __builtin_amdgcn_wave_barrier();
      }
    }
    if (!more) return;
    __syncthreads();                                     // the second stages are free
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

// K ranges of DOWN's tiles: as many as fill the chip where the tiles alone do not, of eight k tiles or more each; no more than whoever
// combines the rows adds, and than there is room for
int down_slices(const Mx4Args& g, const Mx4Shapes& sh) {
  const int64_t busy = std::min<int64_t>(sh.E, g.R), tiles = busy * ceil_div(ceil_div(g.R, busy), kTileRows) * ceil_div(g.N, 256);
  const int64_t fit = (int64_t)mx4_y_bytes(g.R, g.N) / ((int64_t)g.R * g.N * 4);
  return (int)std::max<int64_t>(std::min({kTileGrid / tiles, (int64_t)ceil_div(g.K, kTileK) / 8, fit, (int64_t)combine_most_slices(sh.T, sh.k, BTX_BF16)}), 1);
}

template <bool UP> int launch_tiles(const Mx4Args& g, int E, hipStream_t s) {
  if (int rc = raise_lds<mx4_tile_kernel<UP>>()) return rc;
  const int n_ct = ceil_div(g.N, UP ? 128 : 256);
  const int64_t tiles = ((int64_t)mx4_most_tiles(g.R, E, kTileRows) * n_ct + kXcds) * g.slices;      // (R N < 2^40: fewer than 2^26)
  // A workgroup for every compute unit, which takes every 256th tile: what begins its next one runs beside the last one's end.  Of less than two
  // rounds each has its own: a few ids name no tile, and their compute units take the ones behind the 256th.
  const int64_t grid = tiles <= 2 * kTileGrid ? tiles : kTileGrid;
  mx4_tile_kernel<UP><<<(unsigned)grid, kTileWaves * kWave, kTileLds, s>>>(g, n_ct);
  BTX_LAUNCH_CHECK();
  return BTX_OK;
}

template <bool UP> int launch(const Mx4Args& g, const Mx4Shapes& sh, hipStream_t s) {
  const int rows = mx4_tile_rows(sh);
  return rows == kTileRows ? launch_tiles<UP>(g, sh.E, s) : launch_few<UP>(g, rows, sh.E, s);
}

}  // namespace

int mx4_prepare() {
  if (int rc = raise_lds<mx4_tile_kernel<true>>()) return rc;
  return raise_lds<mx4_tile_kernel<false>>();
}

// How many rows a row tile has, by the rows an expert has on average and by what there is to multiply.
//   * 32 or 64, so that few experts have more rows than the average and a tile's: those read their weights twice.  At 24 rows both take the same
//     (96 tokens, 32 experts of 4096 x 1376, 8 a token: 79 us with 32, 81 with 64), at 16 68 and 74, at 32 125 and 90.  (16 take what 32 do,
//     down to one token.)
//   * 256 from 32 (4 experts of 4096 x 11008: 95 us with 64, 89 with 256; at 24 86 and 89; 32 of 4096 x 1376 90 and 94, at 48 102 and 96; 64 of
//     1024 x 2048 80 and 68), where there is enough to multiply: a tile of the result takes as long alone as 256 of them beside each other.
//     Either 12000 rows by 128 columns of UP or 256 of DOWN, or 2.3 10^9 products, as fewer tiles of long sums have:  2 experts of 1024 x 1024 at 768
//     rows 24 and 32 us, at 1024 31 and 32; 4 of 512 x 512 at 1024 rows 20 and 26, at 2048 27 and 26; 8 of 4096 x 1376 at 384 rows 40
//     and 45, at 512 57 and 47; one of 4096 x 11008 at 44 42 and 47, at 64 59 and 49; 2 at 88 70 and 52.
//     (Rows of x, a tile's rows and their scales are found with 32-bit offsets there: of x, set_sources()'s a_off, the last token's row, 112 bytes
//     of a chunk and kCopyBias2.)
int mx4_tile_rows(const Mx4Shapes& sh) {
  const int64_t R = (int64_t)sh.T * sh.k, avg = R / sh.E;
  const bool enough = R * (ceil_div(sh.f, 128) + ceil_div(sh.d, 256)) >= 12000 || R * sh.d * (int64_t)sh.f >= (int64_t)2300000000;
  if (avg >= 32 && enough && (int64_t)sh.T * (sh.d / 2) + kTileK / 2 + kCopyBias2 < (int64_t)1 << 32) return kTileRows;
  return avg <= 24 ? 32 : 64;
}

int launch_mx4_up(const Mx4Layer& l, const Mx4Matrix& W1, const Mx4Matrix& W3, const Mx4Shapes& sh, hipStream_t s) {
  return launch<true>(Mx4Args{l.x, W1, W3, l.tokens, l.tiles, sh.T, sh.f, sh.d, l.act_codes, l.act_scales, nullptr, sh.T * sh.k, 1}, sh, s);
}

int launch_mx4_down(const Mx4Layer& l, const Mx4Matrix& W2, const Mx4Shapes& sh, int* slices, hipStream_t s) {
  const int R = sh.T * sh.k;
  Mx4Args g{{l.act_codes, l.act_scales}, W2, {nullptr, nullptr}, nullptr, l.tiles, R, sh.d, sh.f, nullptr, nullptr, static_cast<bf16_t*>(l.y), R, 1};
  if (mx4_tile_rows(sh) == kTileRows) g.slices = down_slices(g, sh);
  *slices = g.slices;
  return launch<false>(g, sh, s);
}

}  // namespace btx
