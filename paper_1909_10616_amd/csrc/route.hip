// Routing of tokens to experts: scores, choice, the lists of the experts' rows,
// and the gradient of the weights.
//
// One wavefront a token. Lane l holds the logits of experts l, l + 64, …; the
// choice is k times the largest key, as one 64-bit maximum over the wavefront
// of (the key made unsigned in its order, the index inverted), so that equals
// go to the lowest index. The lists are a counting sort in fixed blocks of
// entries: every block's counts per expert, their running sums, and each
// entry's rank among its block's entries of the same expert, so that an
// expert's entries keep their order.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "layer_kernels.h"
#include "layer_math.hpp"

namespace gt {
namespace {

constexpr int kMaxE = 1024;
constexpr int kMaxK = 64;
constexpr int kEntries = 512;     // entries of a sort block

struct RouteArgs {
  gt_route_args a;
  int32_t* counts;   // [block][E], then made the blocks' first positions
  int64_t blocks;
};

// Unsigned integers in the order of the floats (NaN taken as −inf before; −0 and 0
// are equal).
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint64_t o = __shfl_xor(static_cast<unsigned long long>(v), d);
    v = o > v ? o : v;
  }
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  return v;
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
  float score;   // sigmoid: the score
  float top, total;  // softmax: the largest logit, Σ exp(logit − top) over all
};
// all(f): f over this lane's logits of the row.
template <int EPL>
__device__ __forceinline__ Shares shares_of(int score, int renormalise, const float (&x)[EPL],
                                            float chosen, bool live) {
  Shares r{0.0f, 0.0f, 0.0f, 1.0f};
  const float ninf = -__builtin_inff();
  if (score == GT_SCORE_SIGMOID) {
    r.score = 1.0f / (1.0f + expf(-chosen));
    r.part = live ? r.score : 0.0f;
    if (renormalise) {
      const float top = wave_max(live ? chosen : ninf);
      const float e = live ? sigmoid_ratio(chosen, top) : 0.0f;
      const float total = wave_sum(e);
      r.part = live ? e / total : 0.0f;
    }
    return r;
  }
  if (renormalise) {     // the softmax over the chosen alone
    const float top = wave_max(live ? chosen : ninf);
    const float e = live ? exp_below(chosen, top) : 0.0f;
    const float total = wave_sum(e);
    r.part = live ? e / total : 0.0f;
    return r;
  }
  float top = ninf;
#pragma unroll
  for (int i = 0; i < EPL; ++i) top = fmaxf(top, x[i]);
  r.top = wave_max(top);
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < EPL; ++i) sum += x[i] > ninf ? exp_below(x[i], r.top) : 0.0f;
  r.total = wave_sum(sum);
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

// The keys of experts outside the kept groups become −inf. keys, runs: this
// wavefront's LDS (E keys, `groups` scores).
template <int EPL>
__device__ __forceinline__ void keep_groups(int E, int groups, int keep, int lane, float* keys,
                                            float* runs, float (&key)[EPL]) {
  const int size = E / groups;
#pragma unroll
  for (int i = 0; i < EPL; ++i)
    if (i * 64 + lane < E) keys[i * 64 + lane] = key[i];
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  for (int g = lane; g < groups; g += 64) {
    float a = -__builtin_inff(), b = a;
    for (int j = 0; j < size; ++j) {
      const float v = keys[g * size + j];
      if (v > a) {
        b = a;
        a = v;
      } else if (v > b) {
        b = v;
      }
    }
    float s = size > 1 ? a + b : a;
    if (!(s == s)) s = -__builtin_inff();   // +inf and −inf in one run
    runs[g] = s;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  // an expert's run stays if fewer than `keep` runs beat it
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const int e = i * 64 + lane;
    if (e >= E) continue;
    const int g = e / size;
    const float mine = runs[g];
    int better = 0;
    for (int o = 0; o < groups; ++o) {
      const float v = runs[o];
      better += v > mine || (v == mine && o < g) ? 1 : 0;
    }
    if (better >= keep) key[i] = -__builtin_inff();
  }
}

// Scores and choice of one token.
template <typename T, int EPL>
__device__ __forceinline__ int route_row(const gt_route_args& a, int64_t t, int lane, float* keys,
                                         float* runs) {
  const int E = a.E, k = a.k;
  float x[EPL], key[EPL];
  load_logits<T, EPL>(a.logits, t * a.ldl, E, lane, x);
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    key[i] = x[i];
    const int e = i * 64 + lane;
    if (a.bias && e < E) {
      key[i] = x[i] + a.bias[e];
      if (!(key[i] == key[i])) key[i] = -__builtin_inff();
    }
  }
  if (a.groups > 1) keep_groups<EPL>(E, a.groups, a.keep, lane, keys, runs, key);
  int mine = -1;       // lane s: the expert of slot s
  float chosen = 0.0f; // and its logit
  const uint32_t none = ordered(-__builtin_inff());
  for (int s = 0; s < k; ++s) {
    uint64_t best = 0;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      const uint64_t c = static_cast<uint64_t>(ordered(key[i])) << 32 |
                         static_cast<uint32_t>(~(i * 64 + lane));
      best = c > best ? c : best;
    }
    best = wave_max(best);
    if (static_cast<uint32_t>(best >> 32) <= none) break;
    const int e = static_cast<int>(~static_cast<uint32_t>(best));
    if (lane == s) mine = e;
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (i * 64 + lane == e) key[i] = -__builtin_inff();
  }
  const bool live = mine >= 0;
  if (live) chosen = to_float(static_cast<const T*>(a.logits)[t * a.ldl + mine]);
  const Shares sh = shares_of<EPL>(a.score, a.renormalise, x, chosen, live);
  if (lane < k) {
    a.experts[t * k + lane] = mine;
    a.weights[t * k + lane] = a.scale * sh.part;
  }
  return mine;
}

// Scores and choice; one wavefront a token.
template <typename T, int EPL>
__global__ __launch_bounds__(256) void route_kernel(const RouteArgs r) {
  extern __shared__ float lds[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * 4 + wave;
  if (t >= r.a.T) return;
  float* keys = lds + wave * (r.a.E + r.a.groups);
  route_row<T, EPL>(r.a, t, lane, keys, keys + r.a.E);
}

// Counts per expert of each block of entries.
__global__ __launch_bounds__(kEntries) void count_kernel(const RouteArgs r) {
  __shared__ int hist[kMaxE];
  const int E = r.a.E;
  for (int e = threadIdx.x; e < E; e += kEntries) hist[e] = 0;
  __syncthreads();
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kEntries + threadIdx.x;
  if (i < r.a.T * r.a.k) {
    const int e = r.a.experts[i];
    if (e >= 0) atomicAdd(&hist[e], 1);   // whole numbers: any order gives the same
  }
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += kEntries) r.counts[blockIdx.x * static_cast<int64_t>(E) + e] = hist[e];
}

// The exclusive prefix over the wavefront-held totals of up to kMaxE experts.
__device__ __forceinline__ void scan_experts(int* total, int E, int* first) {
  // total[E] in LDS → first[0 … E]; called by the first wavefront
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int e0 = 0; e0 < E; e0 += 64) {
    const int v = e0 + lane < E ? total[e0 + lane] : 0;
    int upto = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(upto, d);
      if (lane >= d) upto += o;
    }
    if (e0 + lane < E) first[e0 + lane] = before + upto - v;
    before += __shfl(upto, 63);
  }
  if (lane == 0) first[E] = before;
}

// counts[block][e] → the first position of block's entries of expert e; offsets.
__global__ __launch_bounds__(1024) void scan_kernel(const RouteArgs r) {
  __shared__ int total[kMaxE], first[kMaxE + 1];
  const int E = r.a.E;
  for (int e = threadIdx.x; e < E; e += 1024) {
    int sum = 0;
    for (int64_t b = 0; b < r.blocks; ++b) sum += r.counts[b * E + e];
    total[e] = sum;
  }
  __syncthreads();
  if (threadIdx.x < 64) scan_experts(total, E, first);
  __syncthreads();
  for (int e = threadIdx.x; e <= E; e += 1024) r.a.offsets[e] = first[e];
  for (int e = threadIdx.x; e < E; e += 1024) {
    int at = first[e];
    for (int64_t b = 0; b < r.blocks; ++b) {
      const int c = r.counts[b * E + e];
      r.counts[b * E + e] = at;
      at += c;
    }
  }
}

// Each entry of a block to its place; the order after the last entry to −1.
__global__ __launch_bounds__(kEntries) void place_kernel(const RouteArgs r) {
  __shared__ __align__(16) int ids[kEntries];
  const int64_t n = r.a.T * r.a.k;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kEntries + threadIdx.x;
  const int e = i < n ? r.a.experts[i] : -1;
  ids[threadIdx.x] = e;
  __syncthreads();
  int rank = 0;
  for (int j = 0; j < static_cast<int>(threadIdx.x); ++j) rank += ids[j] == e ? 1 : 0;
  if (i < n) {
    int p = -1;
    if (e >= 0) {
      p = r.counts[blockIdx.x * static_cast<int64_t>(r.a.E) + e] + rank;
      r.a.order[p] = static_cast<int32_t>(i);
    }
    r.a.place[i] = p;
    if (i >= r.a.offsets[r.a.E]) r.a.order[i] = -1;
  }
}

// A few tokens: everything in one block.
template <typename T, int EPL>
__global__ __launch_bounds__(1024) void route_few_kernel(const RouteArgs r) {
  extern __shared__ float lds[];
  __shared__ __align__(16) int ids[kEntries];
  __shared__ int total[kMaxE], first[kMaxE + 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int E = r.a.E, k = r.a.k;
  for (int e = threadIdx.x; e < E; e += 1024) total[e] = 0;
  float* keys = lds + wave * (E + r.a.groups);
  for (int64_t t = wave; t < r.a.T; t += 16) {
    const int mine = route_row<T, EPL>(r.a, t, lane, keys, keys + E);
    if (lane < k) ids[t * k + lane] = mine;
  }
  __syncthreads();
  const int n = static_cast<int>(r.a.T) * k;
  const int i = threadIdx.x;
  const int e = i < n ? ids[i] : -1;
  int rank = 0;
  if (e >= 0) {
    atomicAdd(&total[e], 1);
    for (int j = 0; j < i; ++j) rank += ids[j] == e ? 1 : 0;
  }
  __syncthreads();
  if (wave == 0) scan_experts(total, E, first);
  __syncthreads();
  for (int x = threadIdx.x; x <= E; x += 1024) r.a.offsets[x] = first[x];
  if (i < n) {
    const int p = e >= 0 ? first[e] + rank : -1;
    if (p >= 0) r.a.order[p] = i;
    r.a.place[i] = p;
    if (i >= first[E]) r.a.order[i] = -1;
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
  const Shares sh = shares_of<EPL>(a.score, a.renormalise, x, chosen, live);
  // mean = Σ of the chosen's share·gradient
  const float mean = wave_sum(live ? sh.part * g : 0.0f);
  float d;
  if (a.score == GT_SCORE_SIGMOID)
    d = sh.part * (1.0f - sh.score) * (a.renormalise ? g - mean : g);
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

// Whether one block does all: one launch, no scratch, and the keys of 16 tokens
// in its LDS.
bool few(int64_t T, int E, int k, int groups) {
  return T <= 64 && T * k <= kEntries && E + groups <= 640;
}

template <typename T, int EPL>
hipError_t route_by(const gt_route_args& a, void* ws, hipStream_t s) {
  const RouteArgs r{a, static_cast<int32_t*>(ws), (a.T * a.k + kEntries - 1) / kEntries};
  if (few(a.T, a.E, a.k, a.groups)) {
    route_few_kernel<T, EPL><<<1, 1024, 16 * (a.E + a.groups) * sizeof(float), s>>>(r);
    return hipGetLastError();
  }
  route_kernel<T, EPL><<<static_cast<unsigned>((a.T + 3) / 4), 256,
                         4 * (a.E + a.groups) * sizeof(float), s>>>(r);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  count_kernel<<<static_cast<unsigned>(r.blocks), kEntries, 0, s>>>(r);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  scan_kernel<<<1, 1024, 0, s>>>(r);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  place_kernel<<<static_cast<unsigned>(r.blocks), kEntries, 0, s>>>(r);
  return hipGetLastError();
}

template <typename T, int EPL>
hipError_t grad_by(const gt_route_grad_args& a, hipStream_t s) {
  route_grad_kernel<T, EPL>
      <<<static_cast<unsigned>((a.T + 3) / 4), 256, 4 * a.E * sizeof(float), s>>>(a);
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
  return (T * k + kEntries - 1) / kEntries * E * static_cast<int64_t>(sizeof(int32_t));
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
