// Routing from logits for many experts (see group_route.hip).
#pragma once
#include <type_traits>

#include "common.h"

namespace btx {

constexpr int kGroupMaxExperts = 256, kGroupMaxK = 16, kGroupMaxGroups = 16;

struct GroupRouteArgs {
  const void* logits; int dtype; const float* bias; int T, E, k, score_fn, G, keep, group_score, renorm; float scale;
  int32_t* topk_idx; float* gates; float* scores; int32_t* counts; int32_t* offsets; int32_t* perm; int32_t* inv_pos;
  int* hist;                       // workspace: [blocks][hist_pitch] pairs of every expert
  // by the launcher: E, rounded up; experts of a group; lanes it has (log2) of a token's 16, experts a lane; rows in pieces of four; tokens of a block
  int hist_pitch, per_group, log2_lanes, per_lane, vector, tokens;
};
size_t group_route_workspace_bytes(int T, int E);
int launch_group_route(GroupRouteArgs a, hipStream_t s);

struct GroupRouteBwdArgs {
  const void* logits; int dtype; const int32_t* topk_idx; const float* dgates; const float* dscores; int T, E, k, score_fn, renorm;
  float scale; void* dlogits;
};
int launch_group_route_bwd(const GroupRouteBwdArgs& a, hipStream_t s);

// dgates[p] = sum of pair p's n_part partial sums (launch_bwd_act()), those of grouped row inv_pos[p]; 0 where that is negative
int launch_gate_grads(const float* dg_part, int n_part, const int32_t* inv_pos, int R, float* dgates, hipStream_t s);

// Counts of all pairs by expert (s_base, at most 256) -> s_off = where each expert's pairs begin; block 0 writes counts and offsets.
// Every thread of the workgroup calls it, at least one wavefront of them; s_wave: a number for every 64 experts.
__device__ __forceinline__ void group_offsets(const GroupRouteArgs& a, const int* s_base, int* s_off, int* s_wave) {
  const int lane = threadIdx.x & (kWave - 1), waves = blockDim.x / kWave, chunks = (a.E + kWave - 1) / kWave;
  for (int c = threadIdx.x / kWave; c < chunks; c += waves) {
    const int e = c * kWave + lane, n = e < a.E ? s_base[e] : 0;
    const int incl = wave_incl_scan_i32(n, lane);
    if (e < a.E) s_off[e] = incl - n;
    if (lane == kWave - 1) s_wave[c] = incl;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += blockDim.x) {
    int before = 0;
    for (int c = 0; c < e / kWave; ++c) before += s_wave[c];
    s_off[e] += before;
    if (blockIdx.x == 0) {
      a.counts[e] = s_base[e];
      a.offsets[e] = s_off[e];
      if (e == a.E - 1) a.offsets[a.E] = s_off[e] + s_base[e];
    }
  }
  __syncthreads();
}

}  // namespace btx
