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

// ---- copies to aligned rows

// One wavefront a row, a 16-byte chunk a lane, all of a product's (or of two products')
// operands in one launch. Bound by memory: 1999×3457 and 3457×2623 in bf16 12 µs, 5.3 TB/s
// both ways.
template <typename T>
__global__ __launch_bounds__(256) void pad_kernel(const PadJobs jobs) {
  constexpr int VEC = 16 / sizeof(T);
  const PadJob& j = jobs.job[blockIdx.y];
  const int lane = threadIdx.x & 63;
  const int64_t n = j.half > 0 ? j.cols / 2 : j.cols;   // columns of a half
  for (int64_t r = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6); r < j.groups * j.rows;
       r += static_cast<int64_t>(gridDim.x) * 4) {
    const int64_t g = j.groups > 1 ? r / j.rows : 0, row = r - g * j.rows;
    const T* src = static_cast<const T*>(j.src) + g * j.sgroup + row * j.ld;
    T* dst = static_cast<T*>(j.dst) + r * j.ldd;
    for (int64_t c = static_cast<int64_t>(lane) * VEC; c < j.ldd; c += 64 * VEC) {
      const bool second = j.half > 0 && c >= j.half;
      const int64_t col = second ? c - j.half : c;
      *reinterpret_cast<u32x4*>(dst + c) = load_chunk<T, VEC>(src + (second ? n : 0) + col, n - col);
    }
  }
}

// ---- the join of K slices

// A quad of outputs a thread, the slices' sums in their order, then the product's epilogue.
// Bound by its launch: 64×4096 in 4 slices (4 MB) 4 µs.
template <typename T>
__global__ __launch_bounds__(256) void reduce_kernel(const ProductArgs a) {
  const int64_t quads = (written<T>(a.e, a.N) + 3) / 4;
  const int64_t rows = a.groups > 0 ? clamp_offset(a.offsets[a.groups], a.M) : a.M;
  const int64_t slice = a.M * a.e.ldpart;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < rows * quads;
       i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t row = i / quads, n = (i - row * quads) * 4;
    const float* p = a.e.part + row * a.e.ldpart + n;
    f32x4 v{}, u{};
    if (n < a.N) {
#pragma unroll 4
      for (int z = 0; z < a.splits; ++z) {
        v += *reinterpret_cast<const f32x4*>(p + z * slice);
        if (a.e.gated) u += *reinterpret_cast<const f32x4*>(p + z * slice + a.e.ldpart / 2);
      }
    }
    const int group = a.groups > 0 ? group_of_row(a.offsets, a.groups, row) : 0;
    const int left = a.N - n < 4 ? static_cast<int>(a.N - n) : 4;
    const f32x4 bv = bias_quad<T>(a.e, n, group, left);
    const f32x4 bu = a.e.gated ? bias_quad<T>(a.e, n + a.N, group, left) : f32x4{};
    linear_quad<T>(a.e, a.N, row, n, group, left, a.e.gated != 0, v, u, bv, bu,
                   residual_quad<T>(a.e, row, n, left));
  }
}

// The join of the last tiles' slices, 256 threads a quad each. Bound by memory and its
// launch: 14 µs for 64 tiles of 256×256 in 4 slices, in place of a round of tiles of which
// 64 units were busy (the down product of 8192 rows of 4096 × 2048 in 8 groups:
// 214 → 159 + 14 µs); 80 of 336 tiles of 128×128 in 3 slices 7 (1999×2623×3457 in bf16:
// 71 → 57 + 7; 472×9008×1024 in fp32, 28 of 284: 130 → 88 in all).
template <typename T, int TILE>
__global__ __launch_bounds__(256) void tail_kernel(const ProductArgs a) {
  constexpr int BM = kTile[TILE].BM, BN = kTile[TILE].BN;
  const bool gated = a.e.epi == kEpiGated;
  GroupTiles<BM> tiles(a);
  int rows = a.tilesM;
  if (a.groups > 0) rows = min(rows, tiles.total());
  const int nt = rows * a.tilesN;
  constexpr int BK = kTile[TILE].KB / static_cast<int>(sizeof(T));
  const Tail tail = tail_of(nt, static_cast<int>((a.K + BK - 1) / BK));
  const int at = static_cast<int>(blockIdx.y);
  if (tail.slices < 2 || at >= tail.left) return;
  int tm, tn, group = 0;
  tile_at(tail.full + at, nt, rows, a.tilesN, tm, tn);
  int64_t m0 = static_cast<int64_t>(tm) * BM, mend = a.M;
  if (a.groups > 0) {
    const Span s = tiles.find(tm, &m0);
    if (s.group < 0) return;
    group = s.group;
    mend = s.hi;
  }
  const int width = gated ? BN / 2 : BN, quads = width / 4;   // of outputs
  const int i = blockIdx.x * 256 + threadIdx.x;
  const int r = i / quads, c = i % quads * 4;
  const int64_t row = m0 + r, n = static_cast<int64_t>(tn) * width + c;
  if (r >= BM || row >= mend || n >= written<T>(a.e, a.N)) return;
  const float* p = a.tail + static_cast<int64_t>(at) * tail.slices * BM * BN + r * BN + c;
  f32x4 v{}, u{};
#pragma unroll 4
  for (int z = 0; z < tail.slices; ++z) {
    v += *reinterpret_cast<const f32x4*>(p + static_cast<int64_t>(z) * BM * BN);
    if (gated) u += *reinterpret_cast<const f32x4*>(p + static_cast<int64_t>(z) * BM * BN + BN / 2);
  }
  const int left = a.N - n < 4 ? static_cast<int>(a.N - n) : 4;
  const f32x4 bv = bias_quad<T>(a.e, n, group, left);
  const f32x4 bu = gated ? bias_quad<T>(a.e, n + a.N, group, left) : f32x4{};
  linear_quad<T>(a.e, a.N, row, n, group, left, gated, v, u, bv, bu,
                 residual_quad<T>(a.e, row, n, left));
}

// ---- the activation's gradient

// 256 threads: 64 column quads (octets, WIDE), kActRows rows, four of them a thread: all its
// loads are out before the first is used. Bound by memory: 4096×4096 in bf16 28 µs,
// 3.6 TB/s (dP stored past the caches 27, and no less for both products after it).
// dP is stored in the operands' type, since the matrix instructions of both products take no
// other: its rounding adds to the outputs' own (bf16 dX, dW 0.0024 of their norm from 64 bits,
// 0.0017 without). The column sums are of dP before it.
template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void act_grad_kernel(const ActGradArgs a) {
  constexpr int U = kActRows / 4, Q = WIDE ? 2 : 1;
  __shared__ f32x4 sums[2][Q][4][64];
  const int q = threadIdx.x & 63, part = threadIdx.x >> 6;
  const int64_t n = (static_cast<int64_t>(blockIdx.y) * 64 + q) * 4 * Q;
  const int64_t r0 = static_cast<int64_t>(blockIdx.x) * kActRows + part;
  const int64_t left64 = a.N - n;
  const int left = left64 < 4 ? static_cast<int>(left64) : 4;
  f32x4 dy[U][Q], gate[U][Q], up[U][Q];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int64_t row = r0 + 4 * i;
#pragma unroll
    for (int j = 0; j < Q; ++j) dy[i][j] = gate[i][j] = up[i][j] = f32x4{};
    if (left <= 0 || row >= a.M) continue;
    const T* d = static_cast<const T*>(a.dY) + row * a.lddy + n;
    const T* p = a.P ? static_cast<const T*>(a.P) + row * a.ldp + n : nullptr;
    if constexpr (WIDE) {
      const oct v = load8(d);
      dy[i][0] = v.a;
      dy[i][1] = v.b;
      if (a.P) {
        const oct g = load8(p);
        gate[i][0] = g.a;
        gate[i][1] = g.b;
        if (a.gated) {
          const oct u = load8(p + a.N);
          up[i][0] = u.a;
          up[i][1] = u.b;
        }
      }
    } else {
      dy[i][0] = load4(d, left);
      if (a.P) {
        gate[i][0] = load4(p, left);
        if (a.gated) up[i][0] = load4(p + a.N, left);
      }
    }
  }
  f32x4 sg[Q] = {}, su[Q] = {};
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int64_t row = r0 + 4 * i;
    f32x4 g[Q], u[Q];
#pragma unroll
    for (int j = 0; j < Q; ++j) {
      g[j] = dy[i][j];
      u[j] = f32x4{};
      if (a.P) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          float val, slope;
          act_both<T>(a.act, gate[i][j][c], &val, &slope);
          g[j][c] = dy[i][j][c] * slope;
          u[j][c] = dy[i][j][c] * val;
        }
        if (a.gated) g[j] *= up[i][j];
      }
      sg[j] += g[j];
      su[j] += u[j];
    }
    if (a.dP && left > 0 && row < a.M) {
      T* out = static_cast<T*>(a.dP) + row * a.lddp + n;
      if constexpr (WIDE) {
        store8(out, oct{g[0], g[1]});
        if (a.gated) store8(out + a.N, oct{u[0], u[1]});
      } else {
        store4(out, g[0], left);
        if (a.gated) store4(out + a.N, u[0], left);
        if (n + left == a.N)
          for (int z = 0; z < a.pad; ++z) out[(a.gated ? a.N : 0) + left + z] = T(0);
      }
    }
  }
  if (!a.part) return;
#pragma unroll
  for (int j = 0; j < Q; ++j) {
    sums[0][j][part][q] = sg[j];
    sums[1][j][part][q] = su[j];
  }
  __syncthreads();
  const int half = threadIdx.x >> 6;
  if (half >= (a.gated ? 2 : 1) || left <= 0) return;
  const int64_t wide = a.gated ? 2 * a.N : a.N;
  float* out = a.part + blockIdx.x * wide + half * a.N + n;
#pragma unroll
  for (int j = 0; j < Q; ++j) {
    const f32x4* s = &sums[half][j][0][q];
    const f32x4 t = (s[0] + s[64]) + (s[128] + s[192]);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) out[4 * j + i] = t[i];
  }
}

// ---- the join of column sums

// 1024 threads: 64 columns of a group, a sixteenth of the partial rows each. Bound by its
// launch and the rows' chain of loads: 256 rows of 4096 5 µs, 32 groups of 2048 6.
__global__ __launch_bounds__(1024) void join_kernel(const float* part, int64_t rows, int64_t wide,
                                                   const int32_t* offsets, int64_t most, int bm,
                                                   int per, float* out) {
  __shared__ float sums[16][64];
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
        // (offsets that do not ascend may name more tiles than there are)
        const int64_t own = hi > lo ? (hi - lo + bm - 1) / bm : 0;
        span[0] = before * per < rows ? before * per : rows;
        span[1] = (before + own) * per < rows ? (before + own) * per : rows;
      }
    }
    __syncthreads();
    r0 = span[0];
    r1 = span[1];
  }
  const int c = threadIdx.x & 63, part16 = threadIdx.x >> 6;
  for (int64_t n = static_cast<int64_t>(blockIdx.x) * 64 + c; n - c < wide; n += int64_t{gridDim.x} * 64) {
    float s = 0.0f;
    if (n < wide) {
#pragma unroll 4
      for (int64_t r = r0 + part16; r < r1; r += 16) s += part[r * wide + n];
    }
    sums[part16][c] = s;
    __syncthreads();
    if (part16 == 0 && n < wide) {
      float t = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) t += sums[i][c];
      out[g * wide + n] = t;
    }
    __syncthreads();
  }
}

// ---- sorted copies of rows, and what else dY's rows give

// 256 threads: a block of rows of one group, a 16-byte chunk of columns a lane, a wavefront
// every fourth row, eight of its rows at a time. Bound by memory, mostly its stores: 16384
// rows of 1024 of both in bf16, 67 MB, 28.5 µs (31.5 with four rows at a time, their
// tokens looked up in each). (WIDE: X and dY, and b2, take 16-byte loads.)
template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void sort_kernel(const SortArgs a) {
  constexpr int VEC = 16 / sizeof(T), U = 8;
  static_assert(kSortRows % (4 * U) == 0 && kSortRows <= 256);
  __shared__ float part[4][64 * VEC];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  ProductArgs g{};
  g.offsets = a.offsets;
  g.groups = a.E;
  g.M = a.entries;
  int64_t first;
  const Span sp = GroupTiles<kSortRows>(g).find(static_cast<int>(blockIdx.x), &first);
  if (sp.group < 0) return;
  const int64_t end = first + kSortRows < sp.hi ? first + kSortRows : sp.hi;
  const int64_t c0 = static_cast<int64_t>(blockIdx.y) * kSortCols;
  const int64_t c1 = c0 + kSortCols < a.ldd ? c0 + kSortCols : a.ldd;
  // row 4·i of the wavefront's in lane i: its token (T: none) and its weight
  int token = static_cast<int>(a.T);
  float weight = 0.0f;
  if (lane < kSortRows / 4 && first + wave + 4 * lane < end) {
    const int entry = a.order[first + wave + 4 * lane];
    if (entry >= 0 && entry / a.k < a.T) {
      token = entry / a.k;
      if (a.sums) weight = a.weights[entry];
    }
  }
  auto chunk = [&](const void* p, int64_t ld, int64_t row, int64_t c) __attribute__((always_inline)) {
    const T* q = static_cast<const T*>(p) + row * ld + c;
    if constexpr (WIDE) return *reinterpret_cast<const u32x4*>(q);
    return load_chunk<T, VEC>(q, a.D - c);
  };
  for (int64_t cb = c0; cb < c1; cb += 64 * VEC) {   // (once in bf16, twice in fp32)
    const int64_t c = cb + lane * VEC;
    const bool in = c < c1;
    float sum[VEC] = {}, b2[VEC] = {};
    if (a.b2 && in) {
      const u32x4 b = chunk(a.b2, a.D, sp.group, c);
      T e[VEC];
      __builtin_memcpy(e, &b, 16);
#pragma unroll
      for (int j = 0; j < VEC; ++j) b2[j] = to_float(e[j]);
    }
    int i0 = 0;
    for (int64_t p0 = first + wave; p0 < end; p0 += 4 * U, i0 += U) {
      u32x4 x[U], y[U];
      float w[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        x[u] = y[u] = u32x4{};
        const int64_t t = __builtin_amdgcn_readlane(token, i0 + u);
        w[u] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, weight), i0 + u));
        if (t >= a.T || !in) continue;
        y[u] = chunk(a.dY, a.lddy, t, c);
        if (a.X) x[u] = chunk(a.X, a.ldx, t, c);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t p = p0 + 4 * u;
        if (p >= end) continue;
        if (in) {
          *reinterpret_cast<u32x4*>(static_cast<T*>(a.dYs) + p * a.ldd + c) = y[u];
          if (a.X) *reinterpret_cast<u32x4*>(static_cast<T*>(a.Xs) + p * a.ldd + c) = x[u];
        }
        T e[VEC];
        __builtin_memcpy(e, &y[u], 16);
        float dot = 0.0f;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float v = to_float(e[j]);
          sum[j] = fmaf(w[u], v, sum[j]);
          dot = fmaf(b2[j], v, dot);
        }
        if (a.b2) {
#pragma unroll
          for (int d = 1; d < 64; d <<= 1) dot += __shfl_xor(dot, d);
          if (lane == 0) a.dot[p * a.ldot + cb / (64 * VEC)] = dot;
        }
      }
    }
    if (a.sums) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) part[wave][lane * VEC + j] = sum[j];
      __syncthreads();
      for (int i = threadIdx.x; i < 64 * VEC; i += 256)
        if (cb + i < a.D && cb + i < c1)
          a.sums[blockIdx.x * a.D + cb + i] = (part[0][i] + part[1][i]) + (part[2][i] + part[3][i]);
      __syncthreads();
    }
  }
}

// ---- sums back into the tokens' order

// A quad (octet, WIDE) of a token's columns a thread; the rows of four slots at a time. Bound
// by memory: 4096 tokens of 2 slots and 2048 columns with a residual, 101 MB, 19.3 µs,
// 5.2 TB/s; a single token 4.8, its launch and two loads in turn.
template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void combine_kernel(const CombineArgs a) {
  constexpr int Q = WIDE ? 2 : 1;
  const uint32_t per = static_cast<uint32_t>((a.D + 4 * Q - 1) / (4 * Q));
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < a.T * per;
       i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t t = i / per, n = (i - t * per) * 4 * Q;
    const int left = a.D - n < 4 ? static_cast<int>(a.D - n) : 4;
    f32x4 v[Q] = {}, r[Q] = {};
    if (a.R) {
      const T* p = static_cast<const T*>(a.R) + t * a.ldr + n;
      if constexpr (WIDE) {
        const oct o = load8(p);
        r[0] = o.a;
        r[1] = o.b;
      } else {
        r[0] = load4(p, left);
      }
    }
    for (int s0 = 0; s0 < a.k; s0 += 4) {
      f32x4 o[4][Q];
      float w[4];
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        w[s] = 0.0f;
#pragma unroll
        for (int j = 0; j < Q; ++j) o[s][j] = f32x4{};
        if (s0 + s >= a.k) continue;
        const int64_t p = a.place[t * a.k + s0 + s];
        if (p < 0 || p >= a.entries) continue;
        w[s] = a.weights ? a.weights[t * a.k + s0 + s] : 1.0f;
#pragma unroll
        for (int j = 0; j < Q; ++j)   // (rows of whole quads)
          o[s][j] = *reinterpret_cast<const f32x4*>(a.O + p * a.ldo + n + 4 * j);
      }
#pragma unroll
      for (int s = 0; s < 4; ++s)
        if (s0 + s < a.k) {
#pragma unroll
          for (int j = 0; j < Q; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c) v[j][c] = fmaf(w[s], o[s][j][c], v[j][c]);
        }
    }
#pragma unroll
    for (int j = 0; j < Q; ++j) v[j] += r[j];
    T* out = static_cast<T*>(a.out) + t * a.ldout + n;
    if constexpr (WIDE)
      store8(out, oct{v[0], v[1]});
    else
      store4(out, v[0], left);
  }
}

// ---- the gradient of the routing weights

// An entry a thread: the partial sums of its row in their order. Bound by its launch: 16384
// rows of 18 sums 4.8 µs.
__global__ __launch_bounds__(256) void weight_grad_kernel(const float* dot, int64_t ldot, int64_t n,
                                                          const int32_t* place,
                                                          const int32_t* offsets, int E,
                                                          int64_t entries, float* dweights) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= entries) return;
  const int64_t p = place[i];
  float s = 0.0f;
  if (p >= 0 && p < clamp_offset(offsets[E], entries)) {
#pragma unroll 4
    for (int64_t j = 0; j < n; ++j) s += dot[p * ldot + j];
  }
  dweights[i] = s;
}

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

}  // namespace

hipError_t launch_pad(int dtype, const PadJobs& jobs, hipStream_t s) {
  int64_t rows = 0;
  for (int i = 0; i < jobs.n; ++i) rows = std::max(rows, jobs.job[i].groups * jobs.job[i].rows);
  if (rows == 0) return hipSuccess;
  const dim3 grid(blocks_for(rows, 4), static_cast<unsigned>(jobs.n));
  if (dtype == GT_BF16)
    pad_kernel<uint16_t><<<grid, 256, 0, s>>>(jobs);
  else
    pad_kernel<float><<<grid, 256, 0, s>>>(jobs);
  return hipGetLastError();
}

hipError_t launch_reduce(int dtype, const ProductArgs& a, hipStream_t s) {
  const int64_t n = a.M * ((a.N + 7) / 4);
  if (n == 0) return hipSuccess;
  const dim3 grid(blocks_for(n, 256));
  if (dtype == GT_BF16)
    reduce_kernel<uint16_t><<<grid, 256, 0, s>>>(a);
  else
    reduce_kernel<float><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

namespace {
template <typename T, int TILE>
hipError_t tail_by(const ProductArgs& a, hipStream_t s) {
  const int64_t tiles = static_cast<int64_t>(a.tilesM) * a.tilesN;
  // (with two slices at least, half the units' number of tiles at most)
  const dim3 grid(kTile[TILE].BM * kTile[TILE].BN / 4 / 256,
                  static_cast<unsigned>(std::min<int64_t>(tiles, kUnits / 2)));
  tail_kernel<T, TILE><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}
}  // namespace
hipError_t launch_tail(int dtype, int tile, const ProductArgs& a, hipStream_t s) {
  if (dtype != GT_BF16) return tail_by<float, 1>(a, s);   // (tile 0 is bf16's)
  return tile == 0 ? tail_by<uint16_t, 0>(a, s) : tail_by<uint16_t, 1>(a, s);
}

namespace {
template <typename T>
hipError_t act_grad_by(const ActGradArgs& q, hipStream_t s) {
  const int cols = q.wide ? 512 : 256;
  const int64_t most = int64_t{kActRows} << 20;   // rows of a launch: 2^28 work-items
  for (int64_t m = 0; m < q.M; m += most) {
    ActGradArgs a = q;
    a.M = std::min(most, q.M - m);
    a.dY = static_cast<const T*>(q.dY) + m * q.lddy;
    if (q.P) a.P = static_cast<const T*>(q.P) + m * q.ldp;
    if (q.dP) a.dP = static_cast<T*>(q.dP) + m * q.lddp;
    if (q.part) a.part = q.part + m / kActRows * (q.gated ? 2 * q.N : q.N);
    const dim3 grid(blocks_for(a.M, kActRows), static_cast<unsigned>((a.N + cols - 1) / cols));
    if (a.wide)
      act_grad_kernel<T, true><<<grid, 256, 0, s>>>(a);
    else
      act_grad_kernel<T, false><<<grid, 256, 0, s>>>(a);
  }
  return hipGetLastError();
}
}  // namespace
hipError_t launch_act_grad(int dtype, const ActGradArgs& a, hipStream_t s) {
  if (a.M == 0) return hipSuccess;
  return dtype == GT_BF16 ? act_grad_by<uint16_t>(a, s) : act_grad_by<float>(a, s);
}

hipError_t launch_join(const float* part, int64_t rows, int64_t wide, const int32_t* offsets,
                       int groups, int64_t most, int bm, int per, float* out, hipStream_t s) {
  const dim3 grid(blocks_for(wide, 64), static_cast<unsigned>(groups));
  join_kernel<<<grid, 1024, 0, s>>>(part, rows, wide, offsets, most, bm, per, out);
  return hipGetLastError();
}

hipError_t launch_sort(int dtype, const SortArgs& a, hipStream_t s) {
  if (a.entries == 0) return hipSuccess;
  const int64_t vec = dtype == GT_BF16 ? 8 : 4;
  const bool wide = a.D % vec == 0 && (!a.X || (a.ldx % vec == 0 && aligned(a.X, 16))) &&
                    a.lddy % vec == 0 && aligned(a.dY, 16) && (!a.b2 || aligned(a.b2, 16));
  const dim3 grid(static_cast<unsigned>(a.entries / kSortRows + std::min<int64_t>(a.E, a.entries)),
                  static_cast<unsigned>((a.ldd + kSortCols - 1) / kSortCols));
  if (dtype == GT_BF16) {
    if (wide)
      sort_kernel<uint16_t, true><<<grid, 256, 0, s>>>(a);
    else
      sort_kernel<uint16_t, false><<<grid, 256, 0, s>>>(a);
  } else {
    if (wide)
      sort_kernel<float, true><<<grid, 256, 0, s>>>(a);
    else
      sort_kernel<float, false><<<grid, 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

hipError_t launch_combine(int dtype, const CombineArgs& a, hipStream_t s) {
  const int cols = a.wide ? 8 : 4;
  const int64_t n = a.T * ((a.D + cols - 1) / cols);
  if (n == 0) return hipSuccess;
  const dim3 grid(blocks_for(n, 256));
  if (dtype == GT_BF16) {
    if (a.wide)
      combine_kernel<uint16_t, true><<<grid, 256, 0, s>>>(a);
    else
      combine_kernel<uint16_t, false><<<grid, 256, 0, s>>>(a);
  } else {
    if (a.wide)
      combine_kernel<float, true><<<grid, 256, 0, s>>>(a);
    else
      combine_kernel<float, false><<<grid, 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

hipError_t launch_weight_grad(const float* dot, int64_t ldot, int64_t n, const int32_t* place,
                              const int32_t* offsets, int E, int64_t entries, float* dweights,
                              hipStream_t s) {
  if (entries == 0) return hipSuccess;
  weight_grad_kernel<<<static_cast<unsigned>((entries + 255) / 256), 256, 0, s>>>(
      dot, ldot, n, place, offsets, E, entries, dweights);
  return hipGetLastError();
}

}  // namespace gt
