// What the products of 256-row tiles share whose operands are rows of 128 bytes a k tile in LDS: direct copies, the rows' swizzle and the order of
// the tiles.
#pragma once
#include "common.h"

namespace btx {
namespace {

__device__ __forceinline__ void copy16(uint64_t base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(off), "s"(base) : "memory");
}
// 4 KB: the instruction's offset counts in memory as in LDS, so the lanes' offsets are that much lower and `base` kCopyBias lower still
constexpr uint32_t kCopyBias4 = 3 * 1024;
__device__ __forceinline__ void copy64(uint64_t base, const uint32_t (&off)[4], uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1\n\tglobal_load_lds_dwordx4 %3, %1 offset:1024\n\t"
      "global_load_lds_dwordx4 %4, %1 offset:2048\n\tglobal_load_lds_dwordx4 %5, %1 offset:3*1024"
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

}  // namespace
}  // namespace btx
