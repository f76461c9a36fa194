// Routing of tokens to experts: scores, choice, the lists of the experts' rows,
// and the gradient of the weights.
//
// A token's lanes hold its logits; the choice is k times the largest key over them (lane
// moves within rows of 16), and of equals the lowest index. Up to 256 experts, 16
// slots and groups of whole lanes: a row of 16 lanes a token, four tokens a wavefront,
// neighbouring experts in a lane; otherwise, and for a few tokens, a wavefront a
// token, experts l, l + 64, … in lane l. The lists are a counting sort over at most
// kMaxBlocks blocks of tokens: the block that routes its tokens counts them per expert;
// then each block sums what the blocks before it counted and ranks its entries, 64 at a
// time, by the votes on their experts' bits, so that an expert's entries keep their
// order. Two launches; one for a few tokens.
//
// Bound by the instructions of the choice: 16384 tokens, 8 of 256 experts in 8 groups, in
// bf16: 15 µs (27 with a wavefront a token), the lists 9 (each block reads all
// blocks' counts), the gradient 9 (11).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <utility>

#include "layer_kernels.h"
#include "layer_math.hpp"

namespace gt {
namespace {

constexpr int kMaxE = 1024;
constexpr int kMaxBlocks = 256;
constexpr int kWaves = 16;       // of a routing block, a token each at a time
constexpr int kEntries = 512;    // entries ranked at a time; the most of one block that does all

struct RouteArgs {
  gt_route_args a;
  int32_t* counts;   // [block][E]
  int32_t blocks;
  int32_t tokens;    // of a block
};

// Keys are compared as signed integers in the order of the floats (−0 and 0 equal; no NaN
// comes here): whole-number maxima take one instruction where a float's take
// three, the scalar unit joins the rows of 16, and no key needs its NaN quieted.
constexpr int32_t kNone = static_cast<int32_t>(0x807fffffu);   // of −inf
__device__ __forceinline__ int32_t ordered(float v) {
  const int32_t b = __builtin_bit_cast(int32_t, v + 0.0f);
  return b ^ ((b >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float unordered(int32_t v) {
  return __builtin_bit_cast(float, v ^ ((v >> 31) & 0x7fffffff));
}
template <int CTRL>
__device__ __forceinline__ int32_t moved(int32_t v) {
  return __builtin_amdgcn_update_dpp(v, v, CTRL, 0xf, 0xf, false);
}
__device__ __forceinline__ int32_t wave_max(int32_t v) {
  v = max(v, moved<0xb1>(v));
  v = max(v, moved<0x4e>(v));
  v = max(v, moved<0x141>(v));
  v = max(v, moved<0x140>(v));
  return max(max(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16)),
             max(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48)));
}

// The value of the lane that a move within 16 lanes names.
template <int CTRL>
__device__ __forceinline__ float moved(float v) {
  const int b = __builtin_bit_cast(int, v);
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(b, b, CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float lane_of(float v, int lane) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}
// Reductions over the wavefront, all lanes active, the result in every lane.
// (0xb1, 0x4e: neighbours and pairs swapped; 0x141, 0x140: 8 and 16 lanes mirrored.)
__device__ __forceinline__ float wave_max(float v) {
  v = fmaxf(v, moved<0xb1>(v));
  v = fmaxf(v, moved<0x4e>(v));
  v = fmaxf(v, moved<0x141>(v));
  v = fmaxf(v, moved<0x140>(v));
  return fmaxf(fmaxf(lane_of(v, 0), lane_of(v, 16)), fmaxf(lane_of(v, 32), lane_of(v, 48)));
}
__device__ __forceinline__ float wave_sum(float v) {
  v += moved<0xb1>(v);
  v += moved<0x4e>(v);
  v += moved<0x141>(v);
  v += moved<0x140>(v);
  return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}

// The same over the 16 lanes of a row.
__device__ __forceinline__ int32_t row_max(int32_t v) {
  v = max(v, moved<0xb1>(v));
  v = max(v, moved<0x4e>(v));
  v = max(v, moved<0x141>(v));
  return max(v, moved<0x140>(v));
}
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, moved<0xb1>(v));
  v = fmaxf(v, moved<0x4e>(v));
  v = fmaxf(v, moved<0x141>(v));
  return fmaxf(v, moved<0x140>(v));
}
__device__ __forceinline__ float row_sum(float v) {
  v += moved<0xb1>(v);
  v += moved<0x4e>(v);
  v += moved<0x141>(v);
  return v + moved<0x140>(v);
}
// A token's lanes: a wavefront's, or a row's.
template <bool ROW, typename V>
__device__ __forceinline__ V token_max(V v) {
  if constexpr (ROW) return row_max(v);
  else return wave_max(v);
}
template <bool ROW>
__device__ __forceinline__ float token_sum(float v) {
  if constexpr (ROW) return row_sum(v);
  else return wave_sum(v);
}

// exp(x − m) where m is the largest of the values: 1 for the largest, +inf included.
__device__ __forceinline__ float exp_below(float x, float m) { return x == m ? 1.0f : expf(x - m); }

// σ(x)/σ(m) for x ≤ m, by whichever form cannot overflow: scores too small for
// a float still have their quotient.
__device__ __forceinline__ float sigmoid_ratio(float x, float m) {
  if (m > 0.0f) return (1.0f + expf(-m)) / (1.0f + expf(-x));
  return exp_below(x, m) * (1.0f + expf(m)) / (1.0f + expf(x));
}

// A token's share of each chosen logit (lane s holds slot s's, live where it has
// an expert), before `scale`, and what else the gradient needs.
struct Shares {
  float part;    // the weight over scale
  float rest;    // sigmoid: 1 − score, formed as σ(−x): the difference has no bits left from x = 17 on
  float top, total;  // softmax: the largest logit, Σ exp(logit − top) over all
};
// x: this lane's logits of the row.
template <bool ROW, int EPL>
__device__ __forceinline__ Shares shares_of(int score, int renormalise, const float (&x)[EPL],
                                            float chosen, bool live) {
  Shares r{0.0f, 0.0f, 0.0f, 1.0f};
  const float ninf = -__builtin_inff();
  if (score == GT_SCORE_SIGMOID) {
    r.rest = 1.0f / (1.0f + expf(chosen));
    r.part = live ? 1.0f / (1.0f + expf(-chosen)) : 0.0f;
    if (renormalise) {
      const float top = token_max<ROW>(live ? chosen : ninf);
      const float e = live ? sigmoid_ratio(chosen, top) : 0.0f;
      const float total = token_sum<ROW>(e);
      r.part = live ? e / total : 0.0f;
    }
    return r;
  }
  if (renormalise) {     // the softmax over the chosen alone
    const float top = token_max<ROW>(live ? chosen : ninf);
    const float e = live ? exp_below(chosen, top) : 0.0f;
    const float total = token_sum<ROW>(e);
    r.part = live ? e / total : 0.0f;
    return r;
  }
  float top = ninf;
#pragma unroll
  for (int i = 0; i < EPL; ++i) top = fmaxf(top, x[i]);
  r.top = token_max<ROW>(top);
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < EPL; ++i) sum += x[i] > ninf ? exp_below(x[i], r.top) : 0.0f;
  r.total = token_sum<ROW>(sum);
  r.part = live ? exp_below(chosen, r.top) / r.total : 0.0f;
  return r;
}

template <typename T, int EPL>
__device__ __forceinline__ void load_logits(const void* logits, int64_t at, int E, int lane,
                                            float (&x)[EPL]) {
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const int e = i * 64 + lane;
    x[i] = -__builtin_inff();
    if (e < E) {
      const float v = to_float(static_cast<const T*>(logits)[at + e]);
      if (v == v) x[i] = v;   // a NaN is never chosen and has no share
    }
  }
}

// The two largest of a run's keys.
struct Best {
  int32_t a, b;
  __device__ __forceinline__ void add(int32_t v) {
    b = max(b, min(a, v));
    a = max(a, v);
  }
  __device__ __forceinline__ void add(int32_t x, int32_t y) {   // x ≥ y, of other keys
    add(x);
    b = max(b, y);
  }
};

// What does not change from token to token: the lanes of a run and the runs of this
// lane's experts.
template <int EPL>
struct Runs {
  int size, parts, part, first;   // keys of a run, lanes a run (a power of two), this lane's part, its first run
  int mine[EPL];                  // the run of expert i·64 + lane
  float bias[EPL];
  __device__ __forceinline__ Runs(const gt_route_args& a, int lane) {
    size = a.E / a.groups;
    parts = 1;
    while (parts < 64 && 2 * parts * a.groups <= 64) parts *= 2;
    part = lane & (parts - 1);
    first = lane / parts;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      const int e = i * 64 + lane;
      mine[i] = e / size;
      bias[i] = a.bias && e < a.E ? a.bias[e] : 0.0f;
    }
  }
};

// The keys of experts outside the kept groups become −inf. keys, score: this wavefront's LDS
// (E keys, `groups` scores). A run's two largest keys by `parts` lanes each; a run
// stays if fewer than `keep` runs beat it.
template <int EPL>
__device__ __forceinline__ void keep_groups(const Runs<EPL>& runs, int E, int groups, int keep,
                                            int lane, int32_t* keys, int32_t* score,
                                            int32_t (&key)[EPL]) {
#pragma unroll
  for (int i = 0; i < EPL; ++i)
    if (i * 64 + lane < E) keys[i * 64 + lane] = key[i];
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  for (int g0 = 0; g0 < groups; g0 += 64) {
    const int g = g0 + runs.first;
    Best best{kNone, kNone};
    if (g < groups)
      for (int j = runs.part; j < runs.size; j += runs.parts) best.add(keys[g * runs.size + j]);
    if (runs.parts > 1) best.add(moved<0xb1>(best.a), moved<0xb1>(best.b));
    if (runs.parts > 2) best.add(moved<0x4e>(best.a), moved<0x4e>(best.b));
    if (runs.parts > 4) best.add(moved<0x141>(best.a), moved<0x141>(best.b));
    if (runs.parts > 8) best.add(moved<0x140>(best.a), moved<0x140>(best.b));
    if (runs.parts > 16) best.add(__shfl_xor(best.a, 16), __shfl_xor(best.b, 16));
    const float s = unordered(best.a) + unordered(best.b);   // (NaN: +inf and −inf in one run)
    if (g < groups && runs.part == 0)
      score[g] = runs.size == 1 ? best.a : s == s ? ordered(s) : kNone;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (groups <= 64) {
    const int32_t own = lane < groups ? score[lane] : kNone;
    int better = 0;
    for (int o = 0; o < groups; ++o) {
      const int32_t v = __builtin_amdgcn_readlane(own, o);
      better += v > own || (v == own && o < lane) ? 1 : 0;
    }
    const uint64_t kept = __ballot(lane < groups && better < keep);
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (!((kept >> (runs.mine[i] & 63)) & 1)) key[i] = kNone;
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      if (i * 64 + lane >= E) continue;
      const int g = runs.mine[i];
      const int32_t mine = score[g];
      int better = 0;
      for (int o = 0; o < groups; ++o) {
        const int32_t v = score[o];
        better += v > mine || (v == mine && o < g) ? 1 : 0;
      }
      if (better >= keep) key[i] = kNone;
    }
  }
}

// LDS floats a wavefront needs to keep groups.
__host__ __device__ constexpr int group_floats(int E, int groups) {
  return groups > 1 ? E + groups : 0;
}

// Scores and choice of token t, whose logits x are; lane s returns the expert of slot s
// (−1: none).
template <int EPL>
__device__ __forceinline__ int route_row(const gt_route_args& a, const Runs<EPL>& runs, int64_t t,
                                         int lane, float* lds, const float (&x)[EPL]) {
  const int E = a.E, k = a.k;
  int32_t key[EPL];
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const float v = x[i] + runs.bias[i];
    key[i] = v == v ? ordered(v) : kNone;
  }
  if (a.groups > 1)
    keep_groups<EPL>(runs, E, a.groups, a.keep, lane, reinterpret_cast<int32_t*>(lds),
                     reinterpret_cast<int32_t*>(lds) + E, key);
  int mine = -1;
  float chosen = 0.0f;
  for (int s = 0; s < k; ++s) {
    int32_t m = key[0];
#pragma unroll
    for (int i = 1; i < EPL; ++i) m = max(m, key[i]);
    m = wave_max(m);
    if (m == kNone) break;
    bool found = false;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      const uint64_t has = __ballot(key[i] == m);
      if (!found && has != 0) {
        found = true;
        const int at = __builtin_ctzll(has);
        const float logit = lane_of(x[i], at);
        if (lane == s) {
          mine = i * 64 + at;
          chosen = logit;
        }
        if (lane == at) key[i] = kNone;
      }
    }
  }
  const Shares sh = shares_of<false, EPL>(a.score, a.renormalise, x, chosen, mine >= 0);
  if (lane < k) {
    a.experts[t * k + lane] = mine;
    a.weights[t * k + lane] = a.scale * sh.part;
  }
  return mine;
}

// A wavefront's tokens t, t + kWaves, … below t1, the next one's logits loaded while the
// choice of one goes on; then(t, expert of the lane's slot).
template <typename T, int EPL, typename F>
__device__ __forceinline__ void route_rows(const gt_route_args& a, int64_t t, int64_t t1, int lane,
                                           float* lds, F then) {
  const Runs<EPL> runs(a, lane);
  float x[EPL], next[EPL];
  if (t < t1) load_logits<T, EPL>(a.logits, t * a.ldl, a.E, lane, next);
  for (; t < t1; t += kWaves) {
#pragma unroll
    for (int i = 0; i < EPL; ++i) x[i] = next[i];
    if (t + kWaves < t1) load_logits<T, EPL>(a.logits, (t + kWaves) * a.ldl, a.E, lane, next);
    then(t, route_row<EPL>(a, runs, t, lane, lds, x));
  }
}

// Scores and choice of a block's tokens, and their counts per expert.
template <typename T, int EPL>
__global__ __launch_bounds__(64 * kWaves) void route_kernel(const RouteArgs r) {
  extern __shared__ float lds[];
  __shared__ int hist[kMaxE];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int E = r.a.E;
  for (int e = threadIdx.x; e < E; e += 64 * kWaves) hist[e] = 0;
  __syncthreads();
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * r.tokens;
  const int64_t t1 = t0 + r.tokens < r.a.T ? t0 + r.tokens : r.a.T;
  route_rows<T, EPL>(r.a, t0 + wave, t1, lane, lds + wave * group_floats(E, r.a.groups),
                     [&](int64_t, int e) {
                       if (e >= 0) atomicAdd(&hist[e], 1);   // whole numbers: any order gives the same
                     });
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += 64 * kWaves)
    r.counts[static_cast<int64_t>(blockIdx.x) * E + e] = hist[e];
}

// KPL values from p, the first n of them; `none` beyond.
template <typename T, int KPL>
__device__ __forceinline__ void load_run(const T* p, int n, float none, float (&v)[KPL]) {
  T e[KPL];
  if (n >= KPL) {
    __builtin_memcpy(e, p, sizeof(e));   // at any alignment
  } else {
#pragma unroll
    for (int i = 0; i < KPL; ++i) e[i] = i < n ? p[i] : T(0);
  }
#pragma unroll
  for (int i = 0; i < KPL; ++i) v[i] = i < n ? to_float(e[i]) : none;
}

template <typename F, int... I>
__device__ __forceinline__ void for_each(F f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}

// Four tokens a wavefront, a row of 16 lanes each, KPL neighbouring experts a lane: the
// instructions of a maximum, a vote or an exponential serve four tokens, for those
// of looking through a lane's KPL keys. Serves up to 256 experts and 16 slots, groups of
// whole lanes (a power of two).
template <typename T, int KPL>
__global__ __launch_bounds__(64 * kWaves) void route_quad_kernel(const RouteArgs r) {
  __shared__ int hist[16 * KPL];
  const gt_route_args& a = r.a;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 15;
  const int E = a.E, k = a.k, e0 = l * KPL;
  for (int e = threadIdx.x; e < E; e += 64 * kWaves) hist[e] = 0;
  float bias[KPL];
  load_run<float, KPL>(a.bias + e0, a.bias ? E - e0 : 0, 0.0f, bias);
  const int parts = a.groups > 1 ? E / a.groups / KPL : 1;   // lanes of a group
  __syncthreads();
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * r.tokens;
  const int64_t t1 = t0 + r.tokens < a.T ? t0 + r.tokens : a.T;
  for (int64_t tw = t0 + wave * 4; tw < t1; tw += kWaves * 4) {
    const int64_t t = tw + (lane >> 4);
    const bool there = t < t1;
    const T* row = static_cast<const T*>(a.logits) + (there ? t : tw) * a.ldl;
    float x[KPL];
    int32_t key[KPL];
    load_run<T, KPL>(row + e0, E - e0, -__builtin_inff(), x);
#pragma unroll
    for (int i = 0; i < KPL; ++i)   // (a NaN is never chosen and has no share)
      if (x[i] != x[i]) x[i] = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < KPL; ++i) {
      const float v = x[i] + bias[i];
      key[i] = v == v ? ordered(v) : kNone;
    }
    if (a.groups > 1) {
      Best best{kNone, kNone};
#pragma unroll
      for (int i = 0; i < KPL; ++i) best.add(key[i]);
      if (parts > 1) best.add(moved<0xb1>(best.a), moved<0xb1>(best.b));
      if (parts > 2) best.add(moved<0x4e>(best.a), moved<0x4e>(best.b));
      if (parts > 4) best.add(moved<0x141>(best.a), moved<0x141>(best.b));
      const float s = unordered(best.a) + unordered(best.b);   // (NaN: +inf and −inf in one run)
      const int32_t own = e0 < E && s == s ? ordered(s) : kNone;
      int better = 0;   // lanes of better groups
      const int mine = l / parts * parts;
      auto against = [&](auto o) __attribute__((always_inline)) {
        constexpr int O = decltype(o)::value;
        if (O < E / KPL) {
          const int32_t v = moved<0x150 + O>(own);   // lane O's of each row
          better += v > own || (v == own && O < mine) ? 1 : 0;
        }
      };
      for_each(against, std::make_integer_sequence<int, 16>{});
      if (better >= a.keep * parts) {
#pragma unroll
        for (int i = 0; i < KPL; ++i) key[i] = kNone;
      }
    }
    int slot = -1;
    for (int s = 0; s < k; ++s) {
      int32_t mine = key[0];
#pragma unroll
      for (int i = 1; i < KPL; ++i) mine = max(mine, key[i]);
      const int32_t m = row_max(mine);
      if (__ballot(m != kNone) == 0) break;
      // the lowest lane that has it takes its lowest expert
      const uint32_t have = static_cast<uint32_t>(__ballot(mine == m) >> (lane & 48)) & 0xffff;
      bool open = m != kNone && l == __builtin_ctz(have);
      int e = -1;
#pragma unroll
      for (int i = 0; i < KPL; ++i) {
        const bool hit = open && key[i] == m;
        e = hit ? e0 + i : e;
        key[i] = hit ? kNone : key[i];
        open = open && !hit;
      }
      e = row_max(e);
      if (l == s) slot = e;
    }
    const bool live = slot >= 0 && there;
    const float chosen = live ? to_float(row[slot]) : 0.0f;
    const Shares sh = shares_of<true, KPL>(a.score, a.renormalise, x, chosen, live);
    if (l < k && there) {
      a.experts[t * k + l] = slot;
      a.weights[t * k + l] = a.scale * sh.part;
      if (live) atomicAdd(&hist[slot], 1);   // whole numbers: any order gives the same
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += 64 * kWaves)
    r.counts[static_cast<int64_t>(blockIdx.x) * E + e] = hist[e];
}

// total[E] in LDS → first[0 … E], the sums before each; called by the first wavefront.
__device__ __forceinline__ void scan_experts(const int* total, int E, int* first) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int e0 = 0; e0 < E; e0 += 64) {
    const int v = e0 + lane < E ? total[e0 + lane] : 0;
    const int upto = wave_prefix(v);
    if (e0 + lane < E) first[e0 + lane] = before + upto - v;
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  if (lane == 0) first[E] = before;
}

// The lanes that hold the same expert as this one (all lanes active; −1 too).
__device__ __forceinline__ uint64_t same_expert(int e) {
  uint64_t same = ~uint64_t{0};
#pragma unroll
  for (int b = 0; b < 11; ++b) {   // an expert's ten bits, and that of −1
    const bool set = (e >> b) & 1;
    const uint64_t v = __ballot(set);
    same &= set ? v : ~v;
  }
  return same;
}

// Gives each of up to kEntries entries (thread i's expert e, −1: none) its place; at[e]
// is the next place of expert e and moves on. The wavefronts take turns.
__device__ __forceinline__ int place_entry(int e, int* at) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t same = same_expert(e);
  const int rank = __popcll(same & ((uint64_t{1} << lane) - 1));
  int p = -1;
  for (int w = 0; w < kEntries / 64; ++w) {
    if (wave == w && e >= 0) {
      p = at[e] + rank;
      __builtin_amdgcn_wave_barrier();
      if (rank == 0) at[e] += __popcll(same);
    }
    __syncthreads();
  }
  return p;
}

// Each entry of a block's tokens to its place; the order after the last entry to −1; the
// offsets.
__global__ __launch_bounds__(kEntries) void place_kernel(const RouteArgs r) {
  __shared__ int total[kMaxE], before[kMaxE], first[kMaxE + 1];
  const int E = r.a.E, k = r.a.k, b = static_cast<int>(blockIdx.x);
  for (int e = threadIdx.x; e < E; e += kEntries) total[e] = before[e] = 0;
  __syncthreads();
  // the blocks' counts, by as many threads an expert as there are
  const int parts = E < kEntries ? kEntries / E : 1;
  for (int x = threadIdx.x; x < E * parts; x += kEntries) {
    const int e = x % E, part = x / E;
    int mine = 0, all = 0;
#pragma unroll 16
    for (int i = part; i < r.blocks; i += parts) {
      const int c = r.counts[static_cast<int64_t>(i) * E + e];
      all += c;
      mine += i < b ? c : 0;
    }
    atomicAdd(&total[e], all);
    atomicAdd(&before[e], mine);
  }
  __syncthreads();
  if (threadIdx.x < 64) scan_experts(total, E, first);
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += kEntries) before[e] += first[e];
  if (b == 0)
    for (int e = threadIdx.x; e <= E; e += kEntries) r.a.offsets[e] = first[e];
  __syncthreads();
  const int64_t n = r.a.T * k, i0 = static_cast<int64_t>(b) * r.tokens * k;
  const int64_t i1 = i0 + static_cast<int64_t>(r.tokens) * k < n ? i0 + static_cast<int64_t>(r.tokens) * k : n;
  for (int64_t at = i0; at < i1; at += kEntries) {
    const int64_t i = at + threadIdx.x;
    const int p = place_entry(i < i1 ? r.a.experts[i] : -1, before);
    if (i < i1) {
      if (p >= 0) r.a.order[p] = static_cast<int32_t>(i);
      r.a.place[i] = p;
      if (i >= first[E]) r.a.order[i] = -1;
    }
  }
}

// A few tokens: everything in one block. Bound by its launch and the chain of one token: 4
// tokens, 6 of 64 experts, 4.8 µs.
template <typename T, int EPL>
__global__ __launch_bounds__(64 * kWaves) void route_few_kernel(const RouteArgs r) {
  extern __shared__ float lds[];
  __shared__ int ids[kEntries];
  __shared__ int total[kMaxE], first[kMaxE + 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int E = r.a.E, k = r.a.k;
  for (int e = threadIdx.x; e < E; e += 64 * kWaves) total[e] = 0;
  __syncthreads();
  route_rows<T, EPL>(r.a, wave, r.a.T, lane, lds + wave * group_floats(E, r.a.groups),
                     [&](int64_t t, int e) {
                       if (lane < k) ids[t * k + lane] = e;
                       if (e >= 0) atomicAdd(&total[e], 1);
                     });
  __syncthreads();
  if (wave == 0) scan_experts(total, E, first);
  __syncthreads();
  for (int x = threadIdx.x; x <= E; x += 64 * kWaves) r.a.offsets[x] = first[x];
  const int n = static_cast<int>(r.a.T) * k, all = first[E];
  __syncthreads();
  const int i = threadIdx.x;
  const int p = place_entry(i < n ? ids[i < kEntries ? i : 0] : -1, first);
  if (i < n) {
    if (p >= 0) r.a.order[p] = i;
    r.a.place[i] = p;
    if (i >= all) r.a.order[i] = -1;
  }
}

// ---- the gradient; one wavefront a token

template <typename T, int EPL>
__global__ __launch_bounds__(256) void route_grad_kernel(const gt_route_grad_args a) {
  extern __shared__ float lds[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * 4 + wave;
  if (t >= a.T) return;
  const int E = a.E, k = a.k;
  float* row = lds + wave * E;
  float x[EPL];
  load_logits<T, EPL>(a.logits, t * a.ldl, E, lane, x);
  const int e = lane < k ? a.experts[t * k + lane] : -1;
  const bool live = e >= 0 && e < E;
  const float chosen = live ? to_float(static_cast<const T*>(a.logits)[t * a.ldl + e]) : 0.0f;
  const float g = live ? a.scale * a.dweights[t * k + lane] : 0.0f;
  const Shares sh = shares_of<false, EPL>(a.score, a.renormalise, x, chosen, live);
  // mean = Σ of the chosen's share·gradient
  const float mean = wave_sum(live ? sh.part * g : 0.0f);
  float d;
  if (a.score == GT_SCORE_SIGMOID)
    d = sh.part * sh.rest * (a.renormalise ? g - mean : g);
  else
    d = sh.part * (a.renormalise ? g - mean : g);
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const int c = i * 64 + lane;
    float v = 0.0f;
    if (a.score == GT_SCORE_SOFTMAX && !a.renormalise && x[i] > -__builtin_inff())
      v = -mean * exp_below(x[i], sh.top) / sh.total;
    if (c < E) row[c] = v;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (live) row[e] += d;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const int c = i * 64 + lane;
    if (c < E) static_cast<T*>(a.dlogits)[t * a.lddl + c] = from_float<T>(row[c]);
  }
}

// The same with a row of 16 lanes a token and KPL neighbouring experts a lane; the logits
// are read where all of them count, in the softmax over all experts.
template <typename T, int KPL>
__global__ __launch_bounds__(256) void route_grad_quad_kernel(const gt_route_grad_args a) {
  __shared__ float rows[16][16 * KPL];
  const int lane = threadIdx.x & 63, l = lane & 15, e0 = l * KPL;
  const int64_t tw = static_cast<int64_t>(blockIdx.x) * 16 + (threadIdx.x >> 6) * 4;
  if (tw >= a.T) return;
  const bool there = tw + (lane >> 4) < a.T;
  const int64_t t = there ? tw + (lane >> 4) : tw;
  const int E = a.E, k = a.k;
  float* row = rows[threadIdx.x >> 4];
  const T* logits = static_cast<const T*>(a.logits) + t * a.ldl;
  const int e = l < k ? a.experts[t * k + l] : -1;
  const bool live = e >= 0 && e < E;
  const float chosen = live ? to_float(logits[e]) : 0.0f;
  const float g = live ? a.scale * a.dweights[t * k + l] : 0.0f;
  const bool all = a.score == GT_SCORE_SOFTMAX && !a.renormalise;
  float x[KPL];
#pragma unroll
  for (int i = 0; i < KPL; ++i) x[i] = -__builtin_inff();
  if (all) {
    load_run<T, KPL>(logits + e0, E - e0, -__builtin_inff(), x);
#pragma unroll
    for (int i = 0; i < KPL; ++i)
      if (x[i] != x[i]) x[i] = -__builtin_inff();
  }
  const Shares sh = shares_of<true, KPL>(a.score, a.renormalise, x, chosen, live);
  const float mean = row_sum(live ? sh.part * g : 0.0f);
  float d = sh.part * (a.renormalise ? g - mean : g);
  if (a.score == GT_SCORE_SIGMOID) d *= sh.rest;
#pragma unroll
  for (int i = 0; i < KPL; ++i)
    row[e0 + i] = all && x[i] > -__builtin_inff() ? -mean * exp_below(x[i], sh.top) / sh.total : 0.0f;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (live) row[e] += d;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (!there) return;
  T out[KPL];
#pragma unroll
  for (int i = 0; i < KPL; ++i) out[i] = from_float<T>(row[e0 + i]);
  T* to = static_cast<T*>(a.dlogits) + t * a.lddl + e0;
  if (e0 + KPL <= E) {
    __builtin_memcpy(to, out, sizeof(out));   // at any alignment
  } else {
#pragma unroll
    for (int i = 0; i < KPL; ++i)
      if (e0 + i < E) to[i] = out[i];
  }
}

// Tokens of a block: whole rounds of its wavefronts, at most kMaxBlocks blocks.
int32_t block_tokens(int64_t T) {
  const int64_t each = (T + kMaxBlocks - 1) / kMaxBlocks;
  return static_cast<int32_t>((each + kWaves - 1) / kWaves * kWaves);
}

// Whether one block does all: one launch, no scratch, and the keys of its wavefronts'
// tokens in 48 KiB of LDS (beside 10 of lists, a launch's 64 without asking for more).
bool few(int64_t T, int E, int k, int groups) {
  return T == 0 || (T <= 64 && T * k <= kEntries && group_floats(E, groups) * kWaves * 4 <= 48 * 1024);
}

// Experts a lane where a row of 16 lanes a token serves, 0 where it does not.
int quad_experts(int E, int k) { return E > 256 || k > 16 ? 0 : E <= 64 ? 4 : E <= 128 ? 8 : 16; }
int quad_experts(const gt_route_args& a) {
  const int kpl = quad_experts(a.E, a.k);
  if (kpl == 0) return 0;
  const int size = a.E / a.groups, parts = size / kpl;
  const bool lanes = size % kpl == 0 && (parts & (parts - 1)) == 0 && parts <= 8;
  return a.groups == 1 || lanes ? kpl : 0;
}

template <typename T, int EPL>
hipError_t route_by(const gt_route_args& a, void* ws, hipStream_t s) {
  RouteArgs r{a, static_cast<int32_t*>(ws), 0, 0};
  const size_t lds = a.T == 0 ? 0 : group_floats(a.E, a.groups) * kWaves * sizeof(float);
  if (few(a.T, a.E, a.k, a.groups)) {
    route_few_kernel<T, EPL><<<1, 64 * kWaves, lds, s>>>(r);
    return hipGetLastError();
  }
  r.tokens = block_tokens(a.T);
  r.blocks = static_cast<int32_t>((a.T + r.tokens - 1) / r.tokens);
  const dim3 grid(static_cast<unsigned>(r.blocks)), block(64 * kWaves);
  const int quad = quad_experts(a);
  if (quad == 4) {
    route_quad_kernel<T, 4><<<grid, block, 0, s>>>(r);
  } else if (quad == 8) {
    route_quad_kernel<T, 8><<<grid, block, 0, s>>>(r);
  } else if (quad == 16) {
    route_quad_kernel<T, 16><<<grid, block, 0, s>>>(r);
  } else {
    if (lds > 48 * 1024) {   // E + groups beyond 640: a launch may use more than its default LDS
      const hipError_t e =
          hipFuncSetAttribute(reinterpret_cast<const void*>(route_kernel<T, EPL>),
                              hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(lds));
      if (e != hipSuccess) return e;
    }
    route_kernel<T, EPL><<<grid, block, lds, s>>>(r);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  place_kernel<<<grid, kEntries, 0, s>>>(r);
  return hipGetLastError();
}

template <typename T, int EPL>
hipError_t grad_by(const gt_route_grad_args& q, hipStream_t s) {
  const int quad = quad_experts(q.E, q.k);
  const int64_t most = int64_t{1} << 24;   // tokens of a launch: 2^30 work-items
  for (int64_t t = 0; t < q.T; t += most) {
    gt_route_grad_args a = q;
    a.T = std::min(most, q.T - t);
    a.logits = static_cast<const T*>(q.logits) + t * q.ldl;
    a.experts = q.experts + t * q.k;
    a.dweights = q.dweights + t * q.k;
    a.dlogits = static_cast<T*>(q.dlogits) + t * q.lddl;
    const dim3 grid(static_cast<unsigned>((a.T + 15) / 16));
    if (quad == 4)
      route_grad_quad_kernel<T, 4><<<grid, 256, 0, s>>>(a);
    else if (quad == 8)
      route_grad_quad_kernel<T, 8><<<grid, 256, 0, s>>>(a);
    else if (quad == 16)
      route_grad_quad_kernel<T, 16><<<grid, 256, 0, s>>>(a);
    else
      route_grad_kernel<T, EPL>
        <<<static_cast<unsigned>((a.T + 3) / 4), 256, 4 * a.E * sizeof(float), s>>>(a);
  }
  return hipGetLastError();
}

#define GT_BY_E(F, T_, E_, ...)                    \
  (E_ <= 64    ? F<T_, 1>(__VA_ARGS__)             \
   : E_ <= 128 ? F<T_, 2>(__VA_ARGS__)             \
   : E_ <= 256 ? F<T_, 4>(__VA_ARGS__)             \
   : E_ <= 512 ? F<T_, 8>(__VA_ARGS__)             \
               : F<T_, 16>(__VA_ARGS__))

}  // namespace

int64_t route_scratch(int64_t T, int E, int k, int groups) {
  if (few(T, E, k, groups)) return 0;
  const int64_t tokens = block_tokens(T);
  return (T + tokens - 1) / tokens * E * static_cast<int64_t>(sizeof(int32_t));
}

hipError_t launch_route(const gt_route_args& a, void* ws, hipStream_t s) {
  return a.dtype == GT_BF16 ? GT_BY_E(route_by, uint16_t, a.E, a, ws, s)
                            : GT_BY_E(route_by, float, a.E, a, ws, s);
}

hipError_t launch_route_grad(const gt_route_grad_args& a, hipStream_t s) {
  if (a.T == 0) return hipSuccess;
  return a.dtype == GT_BF16 ? GT_BY_E(grad_by, uint16_t, a.E, a, s)
                            : GT_BY_E(grad_by, float, a.E, a, s);
}

}  // namespace gt
