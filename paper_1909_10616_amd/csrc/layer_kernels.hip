// Memory-bound kernels around the layer products: the join of K slices, the
// activation's gradient with its column sums, the sorted copies of the experts'
// rows and the sums back into the tokens' order. Each reads its inputs once and
// writes its outputs once; column sums go by fixed blocks of rows and are
// joined in order, so that the same call gives the same bits.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "layer_kernels.h"
#include "product.hpp"

namespace gt {
namespace {

unsigned blocks_for(int64_t n, int64_t per) {
  return static_cast<unsigned>(std::min<int64_t>((n + per - 1) / per, int64_t{1} << 20));
}

__device__ __forceinline__ int64_t clamp_offset(int32_t v, int64_t most) {
  return v < 0 ? 0 : v > most ? most : v;
}

// The group that row p belongs to: the last whose first row is ≤ p.
__device__ __forceinline__ int group_of_row(const int32_t* offsets, int groups, int64_t p) {
  int lo = 0, hi = groups;   // offsets[lo] ≤ p < offsets[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (offsets[mid] <= p)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// ---- the join of K slices

template <typename T>
__global__ __launch_bounds__(256) void reduce_kernel(const ProductArgs a) {
  const int64_t quads = (a.N + 3) / 4;
  const int64_t rows = a.groups > 0 ? clamp_offset(a.offsets[a.groups], a.M) : a.M;
  const int64_t slice = a.M * a.e.ldpart;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < rows * quads;
       i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t row = i / quads, n = (i - row * quads) * 4;
    const float* p = a.e.part + row * a.e.ldpart + n;
    f32x4 v{}, u{};
    for (int z = 0; z < a.splits; ++z) {
      v += *reinterpret_cast<const f32x4*>(p + z * slice);
      if (a.e.gated) u += *reinterpret_cast<const f32x4*>(p + z * slice + a.e.ldpart / 2);
    }
    const int group = a.groups > 0 ? group_of_row(a.offsets, a.groups, row) : 0;
    const int left = a.N - n < 4 ? static_cast<int>(a.N - n) : 4;
    const f32x4 bv = bias_quad<T>(a.e, n, group, left);
    const f32x4 bu = a.e.gated ? bias_quad<T>(a.e, n + a.N, group, left) : f32x4{};
    linear_quad<T>(a.e, a.N, row, n, group, left, a.e.gated != 0, v, u, bv, bu,
                   residual_quad<T>(a.e, row, n, left));
  }
}

// ---- the activation's gradient

// 256 threads: 64 quads of columns, kActRows rows, a quarter of them a thread.
template <typename T>
__global__ __launch_bounds__(256) void act_grad_kernel(const ActGradArgs a) {
  __shared__ f32x4 sums[2][4][64];
  const int q = threadIdx.x & 63, part = threadIdx.x >> 6;
  const int64_t n = (static_cast<int64_t>(blockIdx.y) * 64 + q) * 4;
  const int64_t r0 = static_cast<int64_t>(blockIdx.x) * kActRows;
  const int left = a.N - n < 4 ? static_cast<int>(a.N - n) : 4;
  const bool vec = a.vec != 0;
  f32x4 sg{}, su{};
  if (left > 0) {
    for (int r = part; r < kActRows; r += 4) {
      const int64_t row = r0 + r;
      if (row >= a.M) break;
      const f32x4 dy = load4(static_cast<const T*>(a.dY) + row * a.lddy + n, left, vec);
      f32x4 g = dy, u{};
      if (a.P) {
        const T* p = static_cast<const T*>(a.P) + row * a.ldp + n;
        const f32x4 gate = load4(p, left, vec);
        f32x4 up = f32x4{1.0f, 1.0f, 1.0f, 1.0f};
        if (a.gated) up = load4(p + a.N, left, vec);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float val, slope;
          act_both(a.act, gate[i], &val, &slope);
          g[i] = dy[i] * up[i] * slope;
          u[i] = dy[i] * val;
        }
      }
      if (a.dP) {
        T* out = static_cast<T*>(a.dP) + row * a.lddp + n;
        store4(out, g, left, vec);
        if (a.gated) store4(out + a.N, u, left, vec);
      }
      sg += g;
      su += u;
    }
  }
  if (!a.part) return;
  sums[0][part][q] = sg;
  sums[1][part][q] = su;
  __syncthreads();
  const int half = threadIdx.x >> 6;
  if (half >= (a.gated ? 2 : 1) || left <= 0) return;
  const f32x4 t = (sums[half][0][q] + sums[half][1][q]) + (sums[half][2][q] + sums[half][3][q]);
  const int64_t wide = a.gated ? 2 * a.N : a.N;
  float* out = a.part + blockIdx.x * wide + half * a.N + n;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < left) out[i] = t[i];
}

// ---- the join of column sums

// 256 threads: 64 columns of a group, a quarter of the partial rows each.
__global__ __launch_bounds__(256) void join_kernel(const float* part, int64_t rows, int64_t wide,
                                                   const int32_t* offsets, int64_t most, int bm,
                                                   int per, float* out) {
  __shared__ float sums[4][64];
  __shared__ int64_t span[2];
  const int g = static_cast<int>(blockIdx.y);
  int64_t r0 = 0, r1 = rows;
  if (offsets) {
    if (threadIdx.x < 64) {   // the tiles of the groups before this one
      int64_t before = 0;
      for (int i = threadIdx.x; i < g; i += 64) {
        const int64_t lo = clamp_offset(offsets[i], most), hi = clamp_offset(offsets[i + 1], most);
        before += hi > lo ? (hi - lo + bm - 1) / bm : 0;
      }
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) before += __shfl_xor(before, d);
      if (threadIdx.x == 0) {
        const int64_t lo = clamp_offset(offsets[g], most), hi = clamp_offset(offsets[g + 1], most);
        span[0] = before * per;
        span[1] = span[0] + (hi > lo ? (hi - lo + bm - 1) / bm : 0) * per;
      }
    }
    __syncthreads();
    r0 = span[0];
    r1 = span[1];
  }
  const int c = threadIdx.x & 63, quarter = threadIdx.x >> 6;
  const int64_t n = static_cast<int64_t>(blockIdx.x) * 64 + c;
  float s = 0.0f;
  if (n < wide)
    for (int64_t r = r0 + quarter; r < r1; r += 4) s += part[r * wide + n];
  sums[quarter][c] = s;
  __syncthreads();
  if (quarter == 0 && n < wide)
    out[g * wide + n] = (sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]);
}

// ---- sorted copies of rows

// One wavefront a row; VEC elements a lane where rows and pointers allow it.
template <typename T, int VEC>
__global__ __launch_bounds__(256) void gather_kernel(const T* a, int64_t lda, T* da, const T* b,
                                                     int64_t ldb, T* db, int64_t ldd, int64_t cols,
                                                     const int32_t* order, const int32_t* offsets,
                                                     int E, int64_t entries, int k, int64_t tokens) {
  const int lane = threadIdx.x & 63;
  const int64_t rows = clamp_offset(offsets[E], entries);
  const T* src = blockIdx.y == 0 ? a : b;
  const int64_t lds = blockIdx.y == 0 ? lda : ldb;
  T* dst = blockIdx.y == 0 ? da : db;
  if (!src || !dst) return;
  for (int64_t p = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6); p < rows;
       p += static_cast<int64_t>(gridDim.x) * 4) {
    const int32_t entry = order[p];
    const int64_t t = entry < 0 ? tokens : entry / k;
    for (int64_t c = static_cast<int64_t>(lane) * VEC; c < cols; c += 64 * VEC) {
      if constexpr (VEC > 1) {
        u32x4 v{};
        if (t < tokens) v = *reinterpret_cast<const u32x4*>(src + t * lds + c);
        *reinterpret_cast<u32x4*>(dst + p * ldd + c) = v;
      } else {
        dst[p * ldd + c] = t < tokens ? src[t * lds + c] : T(0);
      }
    }
  }
}

// ---- sums back into the tokens' order

template <typename T>
__global__ __launch_bounds__(256) void combine_kernel(const CombineArgs a) {
  const int64_t quads = (a.D + 3) / 4;
  const bool vec = a.vec != 0;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < a.T * quads;
       i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t t = i / quads, n = (i - t * quads) * 4;
    const int left = a.D - n < 4 ? static_cast<int>(a.D - n) : 4;
    f32x4 v{};
    for (int s = 0; s < a.k; ++s) {
      const int64_t p = a.place[t * a.k + s];
      if (p < 0 || p >= a.entries) continue;
      const f32x4 o = *reinterpret_cast<const f32x4*>(a.O + p * a.ldo + n);   // rows of whole quads
      const float w = a.weights ? a.weights[t * a.k + s] : 1.0f;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = fmaf(w, o[j], v[j]);
    }
    if (a.R) v += load4(static_cast<const T*>(a.R) + t * a.ldr + n, left, vec);
    store4(static_cast<T*>(a.out) + t * a.ldout + n, v, left, vec);
  }
}

// ---- weighted column sums of the experts' rows

// 256 threads: 64 quads of columns, kSumRows rows, a quarter of them a thread.
template <typename T>
__global__ __launch_bounds__(256) void weighted_sums_kernel(const T* rows, int64_t ld, int64_t D,
                                                            const float* weights,
                                                            const int32_t* order, int64_t entries,
                                                            const int32_t* offsets, ProductArgs a,
                                                            float* part) {
  __shared__ f32x4 sums[4][64];
  int64_t first;
  const Span sp = group_of_tile<kSumRows>(a, static_cast<int>(blockIdx.x), &first);
  if (sp.group < 0) return;
  const int q = threadIdx.x & 63, quarter = threadIdx.x >> 6;
  const int64_t n = (static_cast<int64_t>(blockIdx.y) * 64 + q) * 4;
  const int left = D - n < 4 ? static_cast<int>(D - n) : 4;
  f32x4 s{};
  if (left > 0)
    for (int r = quarter; r < kSumRows; r += 4) {
      const int64_t p = first + r;
      if (p >= sp.hi) break;
      const int64_t entry = order[p];
      const float w = entry >= 0 && entry < entries ? weights[entry] : 0.0f;
      const f32x4 v = load4(rows + p * ld + n, left, true);   // (our own rows: whole quads, aligned)
      s += v * w;
    }
  sums[quarter][q] = s;
  __syncthreads();
  if (quarter != 0) return;
  const f32x4 t = (sums[0][q] + sums[1][q]) + (sums[2][q] + sums[3][q]);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < left) part[blockIdx.x * D + n + i] = t[i];
}

// ---- the gradient of the routing weights

// One wavefront an entry.
template <typename T>
__global__ __launch_bounds__(256) void weight_grad_kernel(const WeightGradArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (i >= a.entries) return;
  const int64_t p = a.place[i];
  float s = 0.0f;
  if (p >= 0 && p < clamp_offset(a.offsets[a.E], a.entries)) {
    for (int64_t j = lane; j < a.ldot; j += 64) s += a.dot[p * a.ldot + j];
    if (a.b2) {
      const int e = group_of_row(a.offsets, a.E, p);
      const T* b = static_cast<const T*>(a.b2) + e * a.D;
      const T* y = static_cast<const T*>(a.rows) + p * a.ld;
      for (int64_t n = lane; n < a.D; n += 64) s = fmaf(to_float(b[n]), to_float(y[n]), s);
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) s += __shfl_xor(s, d);
  if (lane == 0) a.dweights[i] = s;
}

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

}  // namespace

hipError_t launch_reduce(int dtype, const ProductArgs& a, hipStream_t s) {
  const int64_t n = a.M * ((a.N + 3) / 4);
  if (n == 0) return hipSuccess;
  const dim3 grid(blocks_for(n, 256));
  if (dtype == GT_BF16)
    reduce_kernel<uint16_t><<<grid, 256, 0, s>>>(a);
  else
    reduce_kernel<float><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_act_grad(int dtype, const ActGradArgs& a, hipStream_t s) {
  if (a.M == 0) return hipSuccess;
  const dim3 grid(static_cast<unsigned>((a.M + kActRows - 1) / kActRows),
                  static_cast<unsigned>((a.N + 255) / 256));
  if (dtype == GT_BF16)
    act_grad_kernel<uint16_t><<<grid, 256, 0, s>>>(a);
  else
    act_grad_kernel<float><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_join(const float* part, int64_t rows, int64_t wide, const int32_t* offsets,
                       int groups, int64_t most, int bm, int per, float* out, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>((wide + 63) / 64), static_cast<unsigned>(groups));
  join_kernel<<<grid, 256, 0, s>>>(part, rows, wide, offsets, most, bm, per, out);
  return hipGetLastError();
}

hipError_t launch_gather(int dtype, const void* a, int64_t lda, void* da, const void* b, int64_t ldb,
                         void* db, int64_t ldd, int64_t cols, const int32_t* order,
                         const int32_t* offsets, int E, int64_t entries, int k, int64_t T,
                         hipStream_t s) {
  if (entries == 0) return hipSuccess;
  const int64_t vec = dtype == GT_BF16 ? 8 : 4;
  const bool wide = cols % vec == 0 && (!a || (lda % vec == 0 && aligned(a, 16))) &&
                    (!b || (ldb % vec == 0 && aligned(b, 16))) && ldd % vec == 0;
  const dim3 grid(blocks_for(entries, 4), 2);
#define GT_GATHER(T_, V_)                                                                          \
  gather_kernel<T_, V_><<<grid, 256, 0, s>>>(static_cast<const T_*>(a), lda, static_cast<T_*>(da), \
                                             static_cast<const T_*>(b), ldb, static_cast<T_*>(db), \
                                             ldd, cols, order, offsets, E, entries, k, T)
  if (dtype == GT_BF16) {
    if (wide)
      GT_GATHER(uint16_t, 8);
    else
      GT_GATHER(uint16_t, 1);
  } else {
    if (wide)
      GT_GATHER(float, 4);
    else
      GT_GATHER(float, 1);
  }
#undef GT_GATHER
  return hipGetLastError();
}

hipError_t launch_combine(int dtype, const CombineArgs& a, hipStream_t s) {
  const int64_t n = a.T * ((a.D + 3) / 4);
  if (n == 0) return hipSuccess;
  const dim3 grid(blocks_for(n, 256));
  if (dtype == GT_BF16)
    combine_kernel<uint16_t><<<grid, 256, 0, s>>>(a);
  else
    combine_kernel<float><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_weighted_sums(int dtype, const void* rows, int64_t ld, int64_t D,
                                const float* weights, const int32_t* order, int64_t entries,
                                const int32_t* offsets, int E, float* part, hipStream_t s) {
  if (entries == 0) return hipSuccess;
  ProductArgs a{};
  a.offsets = offsets;
  a.groups = E;
  a.M = entries;
  const dim3 grid(static_cast<unsigned>(entries / kSumRows + std::min<int64_t>(E, entries)),
                  static_cast<unsigned>((D + 255) / 256));
  if (dtype == GT_BF16)
    weighted_sums_kernel<uint16_t><<<grid, 256, 0, s>>>(static_cast<const uint16_t*>(rows), ld, D,
                                                        weights, order, entries, offsets, a, part);
  else
    weighted_sums_kernel<float><<<grid, 256, 0, s>>>(static_cast<const float*>(rows), ld, D, weights,
                                                     order, entries, offsets, a, part);
  return hipGetLastError();
}

hipError_t launch_weight_grad(int dtype, const WeightGradArgs& a, hipStream_t s) {
  if (a.entries == 0) return hipSuccess;
  const dim3 grid(static_cast<unsigned>((a.entries + 3) / 4));
  if (dtype == GT_BF16)
    weight_grad_kernel<uint16_t><<<grid, 256, 0, s>>>(a);
  else
    weight_grad_kernel<float><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace gt
