// Routing from logits for mixtures of many experts: softmax or sigmoid scores, a bias that only the selection sees, groups of
// which the best are kept, top-k, renormalised and scaled gates, and the stable grouping of the (token, slot) pairs by expert.
// Up to 64 tokens one launch, else two:
//   1. group_select   16 lanes (one DPP row) take a token, four tokens a wavefront, up to 64 a workgroup at a time: scores, the groups'
//                     values and ranks, the k largest one after another; then the workgroup ranks its pairs among those of the same
//                     expert and leaves how many of each it has.
//   2. group_scatter  every workgroup adds those counts up (of the workgroups before it, and of all) and writes its pairs' places.
// The selection is the one of the scores in double precision.  It is done in float, with a bound of each value's error; a token with two
// values, or two groups, nearer to each other than that is done again in double (group_pick_f64), by its wavefront: a few in a
// thousand of ordinary logits.
#include "group_route.h"

namespace btx {
namespace {

constexpr int kLanes = 16;                     // of a token
constexpr int kTokWave = kWave / kLanes;
constexpr int kThreadsMost = 1024, kTokPass = kThreadsMost / kLanes;
constexpr int kSlots = kGroupMaxK + 1;         // the k chosen and the one behind them
constexpr float kMaskedF = -INFINITY;          // value of a masked expert
constexpr float kUlp = 1.1920929e-7f;          // 2^-23
constexpr float kTiny = 1.1754944e-38f;        // 2^-126: a score below it may be 0 in float

template <int CTRL> __device__ __forceinline__ uint32_t dpp_u32(uint32_t v) { return (uint32_t)dpp_i32<CTRL>((int)v); }
// over the 16 lanes of a row
__device__ __forceinline__ uint32_t row_max_u32(uint32_t v) {
  v = max(v, dpp_u32<kDppXor1>(v));
  v = max(v, dpp_u32<kDppXor2>(v));
  v = max(v, dpp_u32<kDppRor4>(v));
  return max(v, dpp_u32<kDppRor8>(v));
}
__device__ __forceinline__ float row_max_f32(float v) {
  v = fmaxf(v, dpp_f32<kDppXor1>(v));
  v = fmaxf(v, dpp_f32<kDppXor2>(v));
  v = fmaxf(v, dpp_f32<kDppRor4>(v));
  return fmaxf(v, dpp_f32<kDppRor8>(v));
}
// (mirrors, not rotations: both halves of every addition are the same two sums, so that all lanes have the same bits, and equal
// logits in different lanes equal scores)
constexpr int kDppHalfMirror = 0x141, kDppMirror = 0x140;   // lane i of 8 (of 16): lane 7 - i (15 - i)
__device__ __forceinline__ float row_sum_f32(float v) {
  v += dpp_f32<kDppXor1>(v);
  v += dpp_f32<kDppXor2>(v);
  v += dpp_f32<kDppHalfMirror>(v);
  return v + dpp_f32<kDppMirror>(v);
}
__device__ __forceinline__ uint32_t row_or_u32(uint32_t v) {
  v |= dpp_u32<kDppXor1>(v);
  v |= dpp_u32<kDppXor2>(v);
  v |= dpp_u32<kDppRor4>(v);
  return v | dpp_u32<kDppRor8>(v);
}
// a float's bits in an order that unsigned integers have; above 0 for every float
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t u = __float_as_uint(v);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// NaN: masked, as -inf is; +inf: the largest float
__device__ __forceinline__ float clean(float l) { return l == l ? fminf(l, 3.402823e38f) : -INFINITY; }

__device__ __forceinline__ float load_logit(const float* p) { return clean(*p); }
__device__ __forceinline__ float load_logit(const bf16_t* p) { return clean(bf16_to_f32(*p)); }
__device__ __forceinline__ void load_logits4(const float* p, float* v) {
  const f32x4 w = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = clean(w[i]);
}
__device__ __forceinline__ void load_logits4(const bf16_t* p, float* v) {
  const u32x2 w = *reinterpret_cast<const u32x2*>(p);
#pragma unroll
  for (int i = 0; i < 2; ++i) { v[2 * i] = clean(bf16lo(w[i])); v[2 * i + 1] = clean(bf16hi(w[i])); }
}

// Which experts a lane has: group g's are dealt to 2^log2_lanes lanes of the row, `per_lane` consecutive ones each
struct Deal {
  int first, n, group;       // of this lane
  __device__ __forceinline__ Deal(const GroupRouteArgs& a, int sub) {
    group = sub >> a.log2_lanes;
    const int part = sub & ((1 << a.log2_lanes) - 1), from = part * a.per_lane;
    first = group * a.per_group + from;
    n = group < a.G ? max(0, min(a.per_lane, a.per_group - from)) : 0;
  }
};

// Scores of one token: max and 1 / sum of exp for softmax
struct RowStat { float m, inv; };
template <int SCORE> __device__ __forceinline__ float score_f(float l, const RowStat& st) {
  if (SCORE == BTX_SCORE_SIGMOID) return sigmoid_f(l);
  return l == -INFINITY ? 0.f : __expf(l - st.m) * st.inv;
}
// bound of the error, in 2^-23 (and kTiny on top of it), of a score in float: the argument of exp is rounded as a product, softmax's also as
// a difference (half of |l| each, an eighth for the factor), the hardware's exp2 and reciprocal add an ulp each, softmax's sum half a one for every
// addition in line (36 at most)
template <int SCORE> __device__ __forceinline__ float score_err(float l, float s) {
  if (l == -INFINITY) return 0.f;
  if (SCORE == BTX_SCORE_SIGMOID) return s * ((1.f - s) * (fabsf(l) + 2.f) + 3.f);
  return s * (1.25f * fabsf(l) + 26.f);                                         // l: less the row's largest
}
template <int SCORE> __device__ __forceinline__ float score_err(float l, float s, const RowStat& st) {
  return score_err<SCORE>(SCORE == BTX_SCORE_SOFTMAX && l != -INFINITY ? l - st.m : l, s);
}

__device__ __forceinline__ double xor_f64(double v, int d) {
  const int lo = __shfl_xor(__double2loint(v), d, kWave), hi = __shfl_xor(__double2hiint(v), d, kWave);
  return __hiloint2double(hi, lo);
}
__device__ __forceinline__ double read_lane_f64(double v, int lane) {   // lane: of all lanes the same
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane), __builtin_amdgcn_readlane(__double2loint(v), lane));
}
// over the wavefront
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
  v = row_max_u32(v);
  uint32_t top = 0u;
#pragma unroll
  for (int r = 0; r < kWave; r += kLanes) top = max(top, (uint32_t)__builtin_amdgcn_readlane((int)v, r));
  return top;
}

// what lanes of this wavefront have put into LDS is there for the others
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The selection of one token in double, by the whole wavefront: slot[j] = expert of slot j.  logits: the token's.  64 lanes and not the
// token's 16, since such a token is the last one of its workgroup, and of the launch: over 16384 tokens of 256 experts without any, those
// of random logits took 12 us more with 16 lanes and take 2 us more with 64.
template <typename XT, int P, int SCORE>
__device__ __forceinline__ void group_pick_f64(const GroupRouteArgs& a, const XT* logits, int lane, int* slot) {
  constexpr int Q = P / kTokWave;                                       // four times the lanes have a group
  const int shift = a.log2_lanes + 2, per = (a.per_group + (1 << shift) - 1) >> shift;
  const int group = lane >> shift, from = (lane & ((1 << shift) - 1)) * per;
  const int first = group * a.per_group + from, n = group < a.G ? max(0, min(per, a.per_group - from)) : 0;
  double v[Q];
  double m = -INFINITY, sum = 0.0;
#pragma unroll
  for (int i = 0; i < Q; ++i) v[i] = i < n ? (double)load_logit(logits + first + i) : -INFINITY;
  if (SCORE == BTX_SCORE_SOFTMAX) {
#pragma unroll
    for (int i = 0; i < Q; ++i) m = fmax(m, v[i]);
    for (int d = 1; d < kWave; d *= 2) m = fmax(m, xor_f64(m, d));
#pragma unroll
    for (int i = 0; i < Q; ++i) {
      v[i] = v[i] != -INFINITY ? exp(v[i] - m) : -INFINITY;
      sum += v[i] != -INFINITY ? v[i] : 0.0;
    }
    for (int d = 1; d < kWave; d *= 2) sum += xor_f64(sum, d);
  }
#pragma unroll
  for (int i = 0; i < Q; ++i) {
    if (v[i] != -INFINITY) {
      v[i] = SCORE == BTX_SCORE_SIGMOID ? 1.0 / (1.0 + exp(-v[i])) : v[i] / sum;
      if (a.bias) v[i] += (double)a.bias[first + i];
      if (!(v[i] == v[i])) v[i] = -INFINITY;
    }
  }
  bool in = group < a.G;
  if (a.G > 1) {
    double b1 = -INFINITY, b2 = -INFINITY;
#pragma unroll
    for (int i = 0; i < Q; ++i) {
      b2 = fmax(b2, fmin(b1, v[i]));
      b1 = fmax(b1, v[i]);
    }
    for (int d = 1; d < (1 << shift); d *= 2) {
      const double o1 = xor_f64(b1, d), o2 = xor_f64(b2, d);
      b2 = fmax(fmax(b2, o2), fmin(b1, o1));
      b1 = fmax(b1, o1);
    }
    const double value = a.group_score == BTX_GROUP_TOP2 && b2 != -INFINITY ? b1 + b2 : b1;
    int better = 0;
    for (int h = 0; h < a.G; ++h) {
      const double o = read_lane_f64(value, h << shift);
      better += h != group && (o > value || (o == value && h < group));
    }
    in &= better < a.keep;
  }
  unsigned long long key[Q];                                            // 0: cannot be chosen; masked experts can, after all others
#pragma unroll
  for (int i = 0; i < Q; ++i) {
    const unsigned long long u = __double_as_longlong(v[i] == 0.0 ? 0.0 : v[i]);
    key[i] = in && i < n ? (u >> 63 ? ~u : u | 1ull << 63) : 0ull;
  }
  for (int j = 0; j < a.k; ++j) {
    unsigned long long best = key[0];
#pragma unroll
    for (int i = 1; i < Q; ++i) best = max(best, key[i]);
    const uint32_t hi = wave_max_u32((uint32_t)(best >> 32));
    const uint32_t lo = wave_max_u32((uint32_t)(best >> 32) == hi ? (uint32_t)best : 0u);
    const unsigned long long top = (unsigned long long)hi << 32 | lo;
    if (lane == __ffsll(__ballot(best == top)) - 1) {                   // the first lane of those that have it, the first of its experts
      int at = 0;
#pragma unroll
      for (int i = Q - 1; i >= 0; --i) at = key[i] == top ? i : at;
#pragma unroll
      for (int i = 0; i < Q; ++i) key[i] = i == at ? 0ull : key[i];
      slot[j] = first + at;
    }
  }
}

// grid: blocks of `tokens` tokens.  LDS: slots of the tokens of a pass; counts of [64 pairs][expert].
template <typename XT, int P, int SCORE>
__global__ __launch_bounds__(kThreadsMost) void group_select_kernel(GroupRouteArgs a) {
  __shared__ u32x4 s_key[kThreadsMost * (P / 4)];                       // of the lanes: [wavefront][four][lane]
  __shared__ int s_slot[kTokPass][kSlots];
  __shared__ int s_idx[kTokPass * kGroupMaxK];                          // of the pass' pairs
  __shared__ uint16_t s_count[kTokPass * kGroupMaxK / kWave][kGroupMaxExperts];
  __shared__ int s_base[kGroupMaxExperts], s_off[kGroupMaxExperts], s_wave[kGroupMaxExperts / kWave];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, sub = lane & (kLanes - 1), row_base = lane & ~(kLanes - 1);
  const int in_pass = threadIdx.x / kLanes, pass_tokens = blockDim.x / kLanes;
  const Deal mine(a, sub);
  const XT* const logits = static_cast<const XT*>(a.logits);
  for (int e = threadIdx.x; e < a.E; e += blockDim.x) s_base[e] = 0;
  const int t_begin = blockIdx.x * a.tokens, t_end = min(a.T, t_begin + a.tokens);
  for (int t0 = t_begin; t0 < t_end; t0 += pass_tokens) {
    const int t = t0 + in_pass;
    const int n_tok = min(pass_tokens, t_end - t0), rounds = (n_tok * a.k + kWave - 1) / kWave;
    for (int i = threadIdx.x; i < rounds * a.E; i += blockDim.x) s_count[i / a.E][i % a.E] = 0;
    if (t0 + wave * kTokWave < t_end) {                                 // (the rows behind the last token do its work again)
      const bool live = t < t_end;
      const XT* const row = logits + (size_t)min(t, t_end - 1) * a.E;
      // ---- scores ----
      float l[P], v[P];
      const XT* const from = row + mine.first;
      if (P % 4 == 0 && a.vector) {
#pragma unroll
        for (int i = 0; i + 3 < P; i += 4) {
          if (i < mine.n) load_logits4(from + i, l + i);
          else l[i] = l[i + 1] = l[i + 2] = l[i + 3] = -INFINITY;
          f32x4 b{0.f, 0.f, 0.f, 0.f};
          if (a.bias && i < mine.n) b = *reinterpret_cast<const f32x4*>(a.bias + mine.first + i);
#pragma unroll
          for (int x = 0; x < 4; ++x) v[i + x] = b[x];
        }
      } else {
#pragma unroll
        for (int i = 0; i < P; ++i) {
          l[i] = i < mine.n ? load_logit(from + i) : -INFINITY;
          v[i] = a.bias && i < mine.n ? a.bias[mine.first + i] : 0.f;
        }
      }
      float l_max = l[0];
#pragma unroll
      for (int i = 1; i < P; ++i) l_max = fmaxf(l_max, l[i]);
      l_max = row_max_f32(l_max);
      RowStat st{0.f, 0.f};
      if (SCORE == BTX_SCORE_SOFTMAX) {
        st.m = l_max == -INFINITY ? 0.f : l_max;                        // (every expert masked)
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < P; ++i) sum += __expf(l[i] - st.m);
        sum = row_sum_f32(sum);
        st.inv = sum > 0.f ? 1.f / sum : 0.f;
      }
      // No score's error is more than that of the largest logit's and a twentieth: softmax's bound rises with the logit, sigmoid's
      // s (3 + (1 - s) (|l| + 2)) up to l = 2.5, where it is 3.09, and falls to 3 from there.
      const float all_err = 1.05f * score_err<SCORE>(l_max, score_f<SCORE>(l_max, st), st);
      float b1 = kMaskedF, b2 = kMaskedF;
      float* const to = a.scores ? a.scores + (size_t)t * a.E + mine.first : nullptr;
      const bool store = to && live;
#pragma unroll
      for (int i = 0; i < P; i += 4) {
        float s[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          s[x] = score_f<SCORE>(l[i + x], st);
          const float y = fmaxf(s[x] + v[i + x], kMaskedF);             // (of a NaN, too)
          v[i + x] = l[i + x] == -INFINITY ? kMaskedF : y;
          b2 = fmaxf(b2, fminf(b1, v[i + x]));
          b1 = fmaxf(b1, v[i + x]);
        }
        if (store) {
          if (P % 4 == 0 && a.vector) {
            if (i < mine.n) *reinterpret_cast<f32x4*>(to + i) = f32x4{s[0], s[1], s[2], s[3]};
          } else {
#pragma unroll
            for (int x = 0; x < 4; ++x)
              if (i + x < mine.n) to[i + x] = s[x];
          }
        }
      }
      // ---- groups ----
      bool in = true, unsure = false;
      if (a.G > 1) {
        for (int d = 1; d < (1 << a.log2_lanes); d *= 2) {
          const float o1 = __shfl_xor(b1, d, kWave), o2 = __shfl_xor(b2, d, kWave);
          b2 = fmaxf(fmaxf(b2, o2), fminf(b1, o1));
          b1 = fmaxf(b1, o1);
        }
        // errors of the difference of two groups' values: four of scores, the roundings of v (of a lower v than the group's best: what it
        // is lower by makes up for it), of two sums and of the difference
        const float most = row_max_f32(fmaxf(b1 > kMaskedF ? fabsf(b1) : 0.f, b2 > kMaskedF ? fabsf(b2) : 0.f));
        const float e2 = kUlp * (4.f * all_err + 8.f * most) + 4.f * kTiny;
        const bool two = a.group_score == BTX_GROUP_TOP2 && b2 > kMaskedF;
        const float value = two ? b1 + b2 : b1;
        int above = 0, maybe = 0;                                       // groups that are better, or may be
        for (int h = 0; h < a.G; ++h) {
          const float d = __shfl(value, row_base + (h << a.log2_lanes), kWave) - value;
          if (h != mine.group) {
            above += d > e2;
            maybe += !(d < -e2);                                        // (also infinity less itself)
          }
        }
        in = maybe < a.keep;
        unsure = mine.group < a.G && !in && above < a.keep;
      }
      // ---- the k largest, and the next ----
      // A lane's values lie in LDS in fours, whose largest it keeps; only the four that the winner was in is looked at again.  (With all of them
      // in registers and looked at, 128 instructions a slot and not 50, 16384 tokens of 256 experts took 25 us here, now 22.)
      u32x4* const fours = s_key + wave * (P / 4) * kWave + lane;
      uint32_t most[P / 4];
#pragma unroll
      for (int q = 0; q < P / 4; ++q) {
        u32x4 w;
#pragma unroll
        for (int x = 0; x < 4; ++x) w[x] = in && 4 * q + x < mine.n ? ordered(v[4 * q + x]) : 0u;
        fours[q * kWave] = w;
        most[q] = max(max(w[0], w[1]), max(w[2], w[3]));
      }
      int* const slot = s_slot[in_pass];
      for (int j = 0; j <= a.k; ++j) {
        uint32_t best = most[0];
#pragma unroll
        for (int q = 1; q < P / 4; ++q) best = max(best, most[q]);
        const uint32_t top = row_max_u32(best);
        const uint32_t have = (uint32_t)(__ballot(best == top) >> row_base) & 0xffffu;
        if (sub == __ffs(have) - 1) {                                   // the first lane of those that have it
          int at = -1;                                                  // none is left
          if (top) {
            int q = 0;
#pragma unroll
            for (int z = P / 4 - 1; z > 0; --z) q = most[z] == top ? z : q;
            q = most[0] == top ? 0 : q;
            u32x4 w = fours[q * kWave];
            int x = 3;
#pragma unroll
            for (int z = 2; z >= 0; --z) x = w[z] == top ? z : x;
#pragma unroll
            for (int z = 0; z < 4; ++z) w[z] = z == x ? 0u : w[z];      // of equal ones the first
            reinterpret_cast<uint32_t*>(&fours[q * kWave])[x] = 0u;
            const uint32_t next = max(max(w[0], w[1]), max(w[2], w[3]));
#pragma unroll
            for (int z = 0; z < P / 4; ++z) most[z] = z == q ? next : most[z];
            at = mine.first + 4 * q + x;
          }
          slot[j] = at;
        }
      }
      wave_lds_fence();
      // lane j: slot j
      int e = -1;
      float ls = -INFINITY, ss = 0.f, ve = 0.f, room = 0.f;
      bool tied = false;
      if (sub < a.k) {
        e = slot[sub];
        const int n = slot[sub + 1];
        if (e >= 0) {
          ls = load_logit(row + e);
          ss = score_f<SCORE>(ls, st);
        }
        if (e < 0) {
          unsure = true;
        } else if (n >= 0) {                                            // nearer to the next one than the errors of both?
          const float ln = load_logit(row + n), sn = score_f<SCORE>(ln, st);
          const float be = a.bias ? a.bias[e] : 0.f, bn = a.bias ? a.bias[n] : 0.f;
          ve = ls == -INFINITY ? kMaskedF : fmaxf(ss + be, kMaskedF);
          const float vn = ln == -INFINITY ? kMaskedF : fmaxf(sn + bn, kMaskedF);
          const bool last = sub == a.k - 1;                             // behind it any that is left may be the next
          float err = score_err<SCORE>(ls, ss, st) + (last ? all_err : score_err<SCORE>(ln, sn, st));
          err += (ve > kMaskedF ? fabsf(ve) : 0.f) + (vn > kMaskedF ? fabsf(vn) : 0.f);
          room = kUlp * err + 2.f * kTiny;
          const bool near = !(ve - vn > room), same = ls == ln && be == bn;
          tied = near && same && last && !a.bias;
          unsure |= near && !(same && (!last || tied));                 // (the same value: the lower index, which came first)
        }
      }
      if (__ballot(tied)) {
        // The last slot's logit once more, left out: of all that are left, only that very logit may be so near.
        const int at = row_base + a.k - 1;
        const float l_last = __shfl(ls, at, kWave), least = __shfl(ve - room, at, kWave);
        const int any = __shfl((int)tied, at, kWave);                   // (of all lanes, those of groups that are out too)
        const bool here = in && any;
#pragma unroll
        for (int i = 0; i < P; ++i) if (here && reinterpret_cast<const uint32_t*>(&fours[i / 4 * kWave])[i % 4]) unsure |= load_logit(from + i) != l_last && !(v[i] < least);
      }
      unsigned long long again = __ballot(unsure && live);
      if (again) {
        for (int r = 0; r < kTokWave; ++r)
          if (again >> (r * kLanes) & 0xffff) {
            const int w = wave * kTokWave + r;
            group_pick_f64<XT, P, SCORE>(a, logits + (size_t)(t0 + w) * a.E, lane, s_slot[w]);
          }
        wave_lds_fence();
        if (sub < a.k && live) {
          e = slot[sub];
          ss = score_f<SCORE>(load_logit(row + e), st);
        }
      }
      // ---- gates ----
      const float sum = row_sum_f32(sub < a.k ? ss : 0.f);
      if (sub < a.k && live) {
        a.gates[(size_t)t * a.k + sub] = a.renorm ? a.scale * (ss / (sum + 1e-20f)) : a.scale * ss;
        a.topk_idx[(size_t)t * a.k + sub] = e;
        s_idx[in_pass * a.k + sub] = e;
      }
    }
    __syncthreads();
    // ---- ranks of the pass' pairs among those of their expert: a wavefront takes 64 pairs ----
    const int n_pairs = n_tok * a.k;
    for (int r = wave; r < rounds; r += blockDim.x / kWave) {
      const int p = r * kWave + lane;
      const int e = p < n_pairs ? s_idx[p] : -1;
      unsigned long long same = ~0ull;
#pragma unroll
      for (int b = 0; b < 9; ++b) {                                     // (-1 has all bits, no expert bit 8)
        const unsigned long long set = __ballot(e >> b & 1);
        same &= (e >> b & 1) ? set : ~set;
      }
      const int rank = __popcll(same & ((1ull << lane) - 1ull));
      if (e >= 0) {
        if (rank == 0) s_count[r][e] = (uint16_t)__popcll(same);
        s_idx[p] = e | rank << 16;
      }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.E; e += blockDim.x) {               // counts -> pairs of the block in front of these 64
      int n = s_base[e];
      for (int r = 0; r < rounds; ++r) {
        const int c = s_count[r][e];
        s_count[r][e] = (uint16_t)(n - s_base[e]);
        n += c;
      }
      s_off[e] = s_base[e];
      s_base[e] = n;
    }
    __syncthreads();
    for (int p = threadIdx.x; p < n_pairs; p += blockDim.x) {
      const int w = s_idx[p], e = w & 0xffff;
      a.inv_pos[(size_t)t0 * a.k + p] = (w >> 16) + s_off[e] + s_count[p / kWave][e];    // the rank inside the block
    }
    __syncthreads();
  }
  if (gridDim.x > 1) {
    for (int e = threadIdx.x; e < a.E; e += blockDim.x) a.hist[(size_t)blockIdx.x * a.hist_pitch + e] = s_base[e];
    return;
  }
  // one block: its counts are all there are
  group_offsets(a, s_base, s_off, s_wave);
  for (int p = threadIdx.x; p < a.T * a.k; p += blockDim.x) {           // (the same thread wrote inv_pos[p])
    const int pos = s_off[a.topk_idx[p]] + a.inv_pos[p];
    a.inv_pos[p] = pos;
    a.perm[pos] = p;
  }
}

// The counts are read in pieces of four experts, 16 rows or so a thread at once: one by one, 64 rows a thread, the launch took 8.8 us for
// 256 workgroups, 6.6 so.
constexpr int kScatterThreads = 1024;
__global__ __launch_bounds__(kScatterThreads) void group_scatter_kernel(GroupRouteArgs a, int blocks) {
  constexpr int kFours = kGroupMaxExperts / 4, kSegs = kScatterThreads / kFours;
  __shared__ __attribute__((aligned(16))) int s_part[kSegs][kGroupMaxExperts], s_upto[kSegs][kGroupMaxExperts];
  __shared__ int s_base[kGroupMaxExperts], s_off[kGroupMaxExperts], s_wave[kGroupMaxExperts / kWave];
  const int e4 = threadIdx.x % kFours * 4, seg = threadIdx.x / kFours;
  const size_t p1 = min((size_t)(blockIdx.x + 1) * a.tokens * a.k, (size_t)a.T * a.k);
  size_t p = (size_t)blockIdx.x * a.tokens * a.k + threadIdx.x;
  int pair_e = p < p1 ? a.topk_idx[p] : 0, rank = p < p1 ? a.inv_pos[p] : 0;   // (under way while the counts are added up)
  u32x4 all{0, 0, 0, 0}, upto{0, 0, 0, 0};
  if (e4 < a.E) {
#pragma unroll 16
    for (int b = seg; b < blocks; b += kSegs) {
      const u32x4 c = *reinterpret_cast<const u32x4*>(a.hist + (size_t)b * a.hist_pitch + e4);
      all += c;
      if (b < (int)blockIdx.x) upto += c;
    }
  }
  *reinterpret_cast<u32x4*>(&s_part[seg][e4]) = all;
  *reinterpret_cast<u32x4*>(&s_upto[seg][e4]) = upto;
  __syncthreads();
  for (int x = threadIdx.x; x < a.E; x += blockDim.x) {
    int n = 0;
#pragma unroll
    for (int s = 0; s < kSegs; ++s) n += s_part[s][x];
    s_base[x] = n;
  }
  __syncthreads();
  group_offsets(a, s_base, s_off, s_wave);                              // every block works them out, the first writes them
  for (int x = threadIdx.x; x < a.E; x += blockDim.x) {
    int n = s_off[x];
#pragma unroll
    for (int s = 0; s < kSegs; ++s) n += s_upto[s][x];
    s_off[x] = n;
  }
  __syncthreads();
  while (p < p1) {
    const int pos = s_off[pair_e] + rank;
    a.inv_pos[p] = pos;
    a.perm[pos] = (int32_t)p;
    p += blockDim.x;
    if (p < p1) {
      pair_e = a.topk_idx[p];
      rank = a.inv_pos[p];
    }
  }
}

// ---- backward ----
// dL/dlogits from dL/dgates (and dL/dscores), 16 lanes a token, four experts at a time a lane (vector) or one.  With
//   w_j = s_{e_j},  g_j = scale w_j / Z,  Z = sum w + 1e-20:   dw_j = (scale dg_j - sum_i dg_i g_i) / Z      (or scale dg_j)
//   ds = dscores + the dw at their experts;   sigmoid: dl = ds s (1 - s);   softmax: dl = s (ds - sum ds s)
// A masked expert has dw = ds = 0, whatever its dgates and dscores are (0 times an infinity is not).
// Bound by what it reads and writes; a sigmoid router without dscores reads only the chosen logits.
constexpr int kBwdThreads = 256, kBwdTokens = kBwdThreads / kLanes;
__device__ __forceinline__ void store_grad4(float* p, const float* v) { *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]}; }
__device__ __forceinline__ void store_grad4(bf16_t* p, const float* v) {
  *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
}
template <typename XT, int SCORE, bool DSCORES, bool VEC>
__global__ __launch_bounds__(kBwdThreads) void group_route_bwd_kernel(GroupRouteBwdArgs a) {
  constexpr int P = kGroupMaxExperts / kLanes, W = VEC ? 4 : 1;
  __shared__ __attribute__((aligned(16))) float s_dw[kBwdTokens][kGroupMaxExperts];
  const int lane = threadIdx.x & (kWave - 1), sub = lane & (kLanes - 1), in_block = threadIdx.x / kLanes;
  const int t = blockIdx.x * kBwdTokens + in_block;
  if (t >= a.T) return;                                                 // (whole rows of 16 lanes)
  const XT* const logits = static_cast<const XT*>(a.logits) + (size_t)t * a.E;
  constexpr bool ALL = SCORE == BTX_SCORE_SOFTMAX || DSCORES;           // every logit is needed
  float* const dw = s_dw[in_block];
#pragma unroll
  for (int i = 0; i < P; i += W) {
    const int e = (i / W * kLanes + sub) * W;
    if (e < a.E) {
#pragma unroll
      for (int x = 0; x < W; ++x) dw[e + x] = 0.f;
    }
  }
  float l[P];
  RowStat st{0.f, 0.f};
  if (ALL) {
#pragma unroll
    for (int i = 0; i < P; i += W) {
      const int e = (i / W * kLanes + sub) * W;
      if (e < a.E) {
        if constexpr (VEC) load_logits4(logits + e, l + i);
        else l[i] = load_logit(logits + e);
      } else {
#pragma unroll
        for (int x = 0; x < W; ++x) l[i + x] = -INFINITY;
      }
    }
  }
  if (SCORE == BTX_SCORE_SOFTMAX) {
    float m = l[0];
#pragma unroll
    for (int i = 1; i < P; ++i) m = fmaxf(m, l[i]);
    st.m = row_max_f32(m);
    if (st.m == -INFINITY) st.m = 0.f;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < P; ++i) sum += __expf(l[i] - st.m);
    sum = row_sum_f32(sum);
    st.inv = sum > 0.f ? 1.f / sum : 0.f;
  }
  int e = -1;
  float w = 0.f, dg = 0.f, slope = 0.f;                                 // slot sub
  if (sub < a.k) {
    e = a.topk_idx[(size_t)t * a.k + sub];
    dg = a.dgates[(size_t)t * a.k + sub];
    if ((unsigned)e < (unsigned)a.E) {
      const float x = load_logit(logits + e);
      w = score_f<SCORE>(x, st);
      const float z = __expf(-fabsf(x)), r = __builtin_amdgcn_rcpf(1.f + z);
      slope = z * r * r;                                                // s (1 - s), also where s rounds to 1
      if (x == -INFINITY) dg = 0.f;
    } else {
      e = -1;
      dg = 0.f;
    }
  }
  float d = a.scale * dg;
  if (a.renorm) {
    const float inv_z = 1.f / (row_sum_f32(w) + 1e-20f), mean = row_sum_f32(dg * (w * inv_z));
    d = a.scale * (dg - mean) * inv_z;
  }
  wave_lds_fence();
  if (e >= 0) dw[e] = SCORE == BTX_SCORE_SIGMOID && !DSCORES ? d * slope : d;
  wave_lds_fence();
  XT* const out = static_cast<XT*>(a.dlogits) + (size_t)t * a.E;
  float ds[P];
#pragma unroll
  for (int i = 0; i < P; i += W) {
    const int x0 = (i / W * kLanes + sub) * W;
#pragma unroll
    for (int x = 0; x < W; ++x) ds[i + x] = x0 < a.E ? dw[x0 + x] : 0.f;
    if (DSCORES && x0 < a.E) {
      if constexpr (VEC) {
        const f32x4 q = *reinterpret_cast<const f32x4*>(a.dscores + (size_t)t * a.E + x0);
#pragma unroll
        for (int x = 0; x < 4; ++x) ds[i + x] += l[i + x] != -INFINITY ? q[x] : 0.f;
      } else if (l[i] != -INFINITY) {
        ds[i] += a.dscores[(size_t)t * a.E + x0];
      }
    }
  }
  float mean = 0.f;
  if (SCORE == BTX_SCORE_SOFTMAX) {
#pragma unroll
    for (int i = 0; i < P; ++i) mean += ds[i] * score_f<SCORE>(l[i], st);
    mean = row_sum_f32(mean);
  }
#pragma unroll
  for (int i = 0; i < P; i += W) {
    const int x0 = (i / W * kLanes + sub) * W;
    if (x0 >= a.E) continue;
#pragma unroll
    for (int x = 0; x < W; ++x) {
      if (SCORE == BTX_SCORE_SOFTMAX) {
        ds[i + x] = score_f<SCORE>(l[i + x], st) * (ds[i + x] - mean);
      } else if (DSCORES) {
        const float z = __expf(-fabsf(l[i + x])), r = __builtin_amdgcn_rcpf(1.f + z);
        ds[i + x] *= z * r * r;
      }
    }
    if constexpr (VEC) store_grad4(out + x0, ds + i);
    else Elem<XT>::st(out + x0, ds[i]);
  }
}

// 16 lanes a pair
__global__ __launch_bounds__(kBwdThreads) void gate_grads_kernel(const float* __restrict__ part, int n_part, const int32_t* __restrict__ inv_pos, int R,
                                                                 float* __restrict__ dgates) {
  const int sub = threadIdx.x & (kLanes - 1);
  for (int64_t p = (int64_t)blockIdx.x * kBwdTokens + threadIdx.x / kLanes; p < R; p += (int64_t)gridDim.x * kBwdTokens) {
    const int r = inv_pos[p];
    float sum = 0.f;
    if (r >= 0)
      for (int i = sub; i < n_part; i += kLanes) sum += part[(size_t)r * n_part + i];
    sum = row_sum_f32(sum);
    if (sub == 0) dgates[p] = sum;
  }
}

}  // namespace

int launch_gate_grads(const float* dg_part, int n_part, const int32_t* inv_pos, int R, float* dgates, hipStream_t s) {
  const int64_t blocks = std::min<int64_t>(((int64_t)R + kBwdTokens - 1) / kBwdTokens, 1 << 20);
  gate_grads_kernel<<<(unsigned)blocks, kBwdThreads, 0, s>>>(dg_part, n_part, inv_pos, R, dgates);
  BTX_LAUNCH_CHECK();
  return BTX_OK;
}

// Tokens of a workgroup: up to 64 tokens one workgroup does without the second launch.  Then 16, one wavefront a SIMD, as long as there are compute
// units for them (301 tokens of 60 experts: 9.5 us with 16, 11.3 with 64; 1024 of 256 13.9 and 17.6), 32 and 64, and more where that would be over
// 512 workgroups, whose counts every workgroup of the second launch adds up.
constexpr int kFullChip = 256, kMostBlocks = 512;
static int block_tokens(int T) {
  if (T <= kTokPass) return kTokPass;
  for (int n = 16; n < kTokPass; n *= 2)
    if (T <= kFullChip * n) return n;
  return T <= kMostBlocks * kTokPass ? kTokPass : ceil_div(ceil_div(T, kMostBlocks), kTokPass) * kTokPass;
}
static int hist_pitch(int E) { return (E + 3) & ~3; }    // (whole pieces of 16 bytes)

size_t group_route_workspace_bytes(int T, int E) {
  if (T <= kTokPass) return 0;
  // (of the most workgroups that fewer tokens have: never less for more tokens)
  const int blocks = std::max(std::min(kFullChip, ceil_div(T, 16)), std::min(kMostBlocks, ceil_div(T, kTokPass)));
  return (size_t)blocks * hist_pitch(E) * sizeof(int);
}

int launch_group_route(GroupRouteArgs a, hipStream_t s) {
  a.per_group = a.E / a.G;
  a.log2_lanes = 0;                                     // as many lanes a group as there are for the next power of two of groups
  while (a.G << (a.log2_lanes + 1) <= kLanes) ++a.log2_lanes;
  a.per_lane = ceil_div(a.per_group, 1 << a.log2_lanes);
  a.tokens = block_tokens(a.T);
  a.hist_pitch = hist_pitch(a.E);
  if (a.per_lane > 4 || a.per_group % 4 == 0) a.per_lane = (a.per_lane + 3) & ~3;   // whole vectors, where rows have them
  const int lsize = a.dtype == BTX_BF16 ? 2 : 4;
  a.vector = a.per_group % 4 == 0 && a.per_lane % 4 == 0 && ((uintptr_t)a.logits % (4 * lsize)) == 0 &&
             (((uintptr_t)a.scores | (uintptr_t)a.bias) & 15) == 0;
  const int blocks = ceil_div(a.T, a.tokens);
  const int threads = std::min(kThreadsMost, ceil_div(std::min(a.T, a.tokens), kTokWave) * kWave);
  auto go = [&](auto tag, auto per, auto score) {
    group_select_kernel<decltype(tag), decltype(per)::value, decltype(score)::value><<<blocks, threads, 0, s>>>(a);
  };
  auto with_p = [&](auto tag, auto score) {
    if (a.per_lane <= 4) go(tag, std::integral_constant<int, 4>{}, score);
    else if (a.per_lane <= 8) go(tag, std::integral_constant<int, 8>{}, score);
    else if (a.per_lane <= 16) go(tag, std::integral_constant<int, 16>{}, score);
    else go(tag, std::integral_constant<int, 32>{}, score);
  };
  auto with_score = [&](auto tag) {
    if (a.score_fn == BTX_SCORE_SIGMOID) with_p(tag, std::integral_constant<int, BTX_SCORE_SIGMOID>{});
    else with_p(tag, std::integral_constant<int, BTX_SCORE_SOFTMAX>{});
  };
  if (a.dtype == BTX_BF16) with_score(bf16_t{});
  else with_score(float{});
  BTX_LAUNCH_CHECK();
  if (blocks > 1) {
    group_scatter_kernel<<<blocks, kScatterThreads, 0, s>>>(a, blocks);
    BTX_LAUNCH_CHECK();
  }
  return BTX_OK;
}

int launch_group_route_bwd(const GroupRouteBwdArgs& a, hipStream_t s) {
  const int lsize = a.dtype == BTX_BF16 ? 2 : 4, blocks = ceil_div(a.T, kBwdTokens);
  if (!grid_fits(blocks, kBwdThreads)) return BTX_ERR_UNSUPPORTED;
  const bool vec = a.E % 4 == 0 && (((uintptr_t)a.logits | (uintptr_t)a.dlogits) % (4 * lsize)) == 0 && ((uintptr_t)a.dscores & 15) == 0;
  auto go = [&](auto tag, auto score) {
    using XT = decltype(tag);
    constexpr int SC = decltype(score)::value;
    if (a.dscores) {
      if (vec) group_route_bwd_kernel<XT, SC, true, true><<<blocks, kBwdThreads, 0, s>>>(a);
      else group_route_bwd_kernel<XT, SC, true, false><<<blocks, kBwdThreads, 0, s>>>(a);
    } else {
      if (vec) group_route_bwd_kernel<XT, SC, false, true><<<blocks, kBwdThreads, 0, s>>>(a);
      else group_route_bwd_kernel<XT, SC, false, false><<<blocks, kBwdThreads, 0, s>>>(a);
    }
  };
  auto with_score = [&](auto tag) {
    if (a.score_fn == BTX_SCORE_SIGMOID) go(tag, std::integral_constant<int, BTX_SCORE_SIGMOID>{});
    else go(tag, std::integral_constant<int, BTX_SCORE_SOFTMAX>{});
  };
  if (a.dtype == BTX_BF16) with_score(bf16_t{});
  else with_score(float{});
  BTX_LAUNCH_CHECK();
  return BTX_OK;
}

}  // namespace btx
