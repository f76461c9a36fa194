// Products of up to 16 rows a workgroup with a matrix, X·W with the linear epilogue, where
// the weights are small enough that one launch without K slices beats sliced tiles and
// the launch that joins them: bound by latency.
//
// A workgroup takes 16 rows, 64 columns (gated: 64 of each half) and all of K, its
// wavefronts (16, gated 8) taking turns at its steps, straight from memory into matrix instructions: no
// LDS, no barrier until the end. W's rows hold neighbouring columns, the instruction
// wants neighbouring k: a lane loads a quad of columns of all the k that its group of
// lanes holds, and instruction j multiplies column j of every quad (bf16: pairs of rows are
// merged by one byte permutation a register). The result then lies in quads of
// neighbouring columns. The wavefronts' sums meet in LDS and are added in their order.
// 13×1021×777 in fp32: 9.8 µs, where the best tiles with the join of their K slices take
// 12.1; 64×1024×1024 in bf16 6.1 (8.0), 16×4096×4096 in 4 slices 10.2 (11.3).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "layer_kernels.h"
#include "product.hpp"

namespace gt {
namespace {

constexpr int kCols = 64;

// A step: 32 k in bf16, 16 in fp32. AL: as slim_aligned says.
template <int DT, bool G, bool AL>
__global__ __launch_bounds__(64 * slim_waves(G)) void slim_kernel(const ProductArgs a) {
  using T = typename Elem<DT>::T;
  constexpr int VEC = Elem<DT>::VEC;       // k of a lane a step
  constexpr int STEP = 4 * VEC;            // k of a wavefront a step
  constexpr int H = G ? 2 : 1, kWaves = slim_waves(G);
  constexpr int QD = DT == 1 ? 2 : 4;      // registers of a quad as it is stored
  extern __shared__ float lds[];           // [wavefront][half][row][quad ^ row]
  const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6);
  const int lx = lane & 15, grp = lane >> 4;
  int64_t m0 = static_cast<int64_t>(blockIdx.y) * 16, mend = a.M;
  int group = 0;
  if (a.groups > 0) {
    const Span s = GroupTiles<16>(a).find(static_cast<int>(blockIdx.y), &m0);
    if (s.group < 0) return;
    group = s.group;
    mend = s.hi;
  }
  const int K = static_cast<int>(a.K);
  // this lane's row of X
  bool have = m0 + lx < mend;
  int64_t row = have ? m0 + lx : m0;
  if (a.gather) {
    const int at = a.gather[row];
    row = at < 0 ? 0 : at / a.gather_div;
    have = have && at >= 0 && row < a.a_rows;
    if (!have) row = 0;
  }
  const T* X = static_cast<const T*>(a.A) + row * a.lda;
  // and its columns of W
  const int64_t n0 = static_cast<int64_t>(blockIdx.x) * kCols, n = n0 + lx * 4;
  const int valid = a.N - n >= 4 ? 4 : a.N > n ? static_cast<int>(a.N - n) : 0;
  const T* W = static_cast<const T*>(a.B) + group * a.sB + (valid ? n : 0);

  uint32_t w[H][VEC][QD];
  u32x4 x;
  auto load = [&](int step) __attribute__((always_inline)) {
    const int k = step * STEP + grp * VEC;
    if constexpr (AL) {
      x = u32x4{};
      if (have && k < K) x = *reinterpret_cast<const u32x4*>(X + k);
    } else {
      x = load_chunk<T, VEC>(X + k, have ? K - k : 0);
    }
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const T* p = W + static_cast<int64_t>(k + i) * a.ldb + h * a.N;
        const int many = k + i < K ? valid : 0;
        uint32_t q[QD] = {};
        if constexpr (AL) {
          if (many) __builtin_memcpy(q, __builtin_assume_aligned(p, 4 * sizeof(T)), 4 * sizeof(T));
        } else if (many == 4) {
          __builtin_memcpy(q, p, 4 * sizeof(T));
        } else if (many > 0) {
          T e[4] = {};
#pragma unroll
          for (int c = 0; c < 3; ++c)
            if (c < many) e[c] = p[c];
          __builtin_memcpy(q, e, sizeof(e));
        }
#pragma unroll
        for (int c = 0; c < QD; ++c) w[h][i][c] = q[c];
      }
  };
  using acc_t = f32x4;
  acc_t acc[H][4] = {};
  const int all = (K + STEP - 1) / STEP, z = static_cast<int>(blockIdx.z);
  const int first = static_cast<int>(static_cast<int64_t>(all) * z / a.splits);
  const int steps = static_cast<int>(static_cast<int64_t>(all) * (z + 1) / a.splits);
  if (first + wave < steps) load(first + wave);
  for (int s = first + wave; s < steps; s += kWaves) {
    uint32_t v[H][VEC][QD];
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int i = 0; i < VEC; ++i)
#pragma unroll
        for (int c = 0; c < QD; ++c) v[h][i][c] = w[h][i][c];
    const u32x4 xs = x;
    if (s + kWaves < steps) load(s + kWaves);
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (DT == 1) {
          u32x4 b;
#pragma unroll
          for (int p = 0; p < 4; ++p)   // k 2p and 2p + 1 of column j
            b[p] = __builtin_amdgcn_perm(v[h][2 * p + 1][j / 2], v[h][2 * p][j / 2],
                                         j & 1 ? 0x07060302u : 0x05040100u);
          acc[h][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              __builtin_bit_cast(bf16x8, b), __builtin_bit_cast(bf16x8, xs), acc[h][j], 0, 0, 0);
        } else {
          const f32x4 xf = __builtin_bit_cast(f32x4, xs);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            acc[h][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                __builtin_bit_cast(float, v[h][i][j]), xf[i], acc[h][j], 0, 0, 0);
        }
      }
  }
  // register r of instruction j: row lx, column 16·grp + 4·r + j
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      *reinterpret_cast<f32x4*>(lds + (((wave * H + h) * 16 + lx) * 16 + ((grp * 4 + r) ^ lx)) * 4) =
          f32x4{acc[h][0][r], acc[h][1][r], acc[h][2][r], acc[h][3][r]};
  __syncthreads();
  if (threadIdx.x >= 256) return;
  const int m = threadIdx.x >> 4, q = threadIdx.x & 15;
  const int64_t out = m0 + m, col = n0 + q * 4;
  if (out >= mend || col >= written<T>(a.e, a.N)) return;
  const float* mine = lds + (m * 16 + (q ^ m)) * 4;
  f32x4 v{}, u{};
#pragma unroll 8
  for (int s = 0; s < kWaves; ++s) {
    v += *reinterpret_cast<const f32x4*>(mine + s * H * 1024);
    if constexpr (G) u += *reinterpret_cast<const f32x4*>(mine + (s * H + 1) * 1024);
  }
  if (a.splits > 1) {
    part_quad<G>(a, z, out, col, v, u);
    return;
  }
  const int left = a.N - col < 4 ? static_cast<int>(a.N - col) : 4;
  const f32x4 bv = bias_quad<T>(a.e, col, group, left);
  const f32x4 bu = G ? bias_quad<T>(a.e, col + a.N, group, left) : f32x4{};
  linear_quad<T>(a.e, a.N, out, col, group, left, G, v, u, bv, bu,
                 residual_quad<T>(a.e, out, col, left));
}

template <int DT, bool G, bool AL>
hipError_t slim_by(const ProductArgs& a, hipStream_t s) {
  constexpr int lds = slim_waves(G) * (G ? 2 : 1) * 16 * kCols * 4;
  static_assert(lds <= 64 * 1024);
  const dim3 grid(static_cast<unsigned>(a.tilesN), static_cast<unsigned>(a.tilesM),
                  static_cast<unsigned>(a.splits));
  slim_kernel<DT, G, AL><<<grid, 64 * slim_waves(G), lds, s>>>(a);
  return hipGetLastError();
}

template <int DT>
hipError_t slim_of(const ProductArgs& a, hipStream_t s) {
  const bool al = slim_aligned(DT, a);
  if (a.e.gated) return al ? slim_by<DT, true, true>(a, s) : slim_by<DT, true, false>(a, s);
  return al ? slim_by<DT, false, true>(a, s) : slim_by<DT, false, false>(a, s);
}

}  // namespace

// 16-byte aligned rows of whole chunks of X, whole aligned quads of W.
bool slim_aligned(int dtype, const ProductArgs& a) {
  const int64_t vec = dtype == GT_BF16 ? 8 : 4;
  return a.K % vec == 0 && a.lda % vec == 0 && reinterpret_cast<uintptr_t>(a.A) % 16 == 0 &&
         a.N % 4 == 0 && a.ldb % 4 == 0 && a.sB % 4 == 0 &&
         reinterpret_cast<uintptr_t>(a.B) % (64 / vec) == 0;
}

hipError_t launch_slim(int dtype, const ProductArgs& a, hipStream_t s) {
  return dtype == GT_BF16 ? slim_of<1>(a, s) : slim_of<0>(a, s);
}

}  // namespace gt
