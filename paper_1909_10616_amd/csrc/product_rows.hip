// Products of a few rows with a matrix, X·W with the linear epilogue: one generated
// token through a layer, or through its experts.
//
// Bound by W's way from memory, so it is read once, straight into registers, with as
// much in flight as they hold: a workgroup takes 64 columns (gated: 64 of each half, so
// that a row of W gives whole 128-byte lines) and all of K, its 16 wavefronts a
// sixteenth of it each. Lanes hold 16 bytes of a row; they multiply by X, kept in LDS
// in fp32, on the vector units (a matrix instruction would want W transposed and
// 16 rows of X). The sums meet in the workgroup, lanes first, then wavefronts in
// order, so one launch gives the layer's output, but for narrow layers, whose few
// workgroups cannot draw W fast enough: K is sliced over more of them then.
// 1×11008×4096 gated in bf16: 39 µs, 4.6 TB/s; 1×4096×4096 past the caches 15.2 in 4
// slices, 4 of it the join.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "layer_kernels.h"
#include "product.hpp"

namespace gt {
namespace {

constexpr int kRowWaves = kRowThreads / 64;
constexpr int kRowCols = 64;
constexpr int kRowStep = 64;   // k of a wavefront's loads in flight, at most

// AL: W's rows are 16-byte aligned and whole chunks: loads by descriptor, zero beyond W.
template <int DT, int MR, bool G, bool AL>
__global__ __launch_bounds__(kRowThreads) void rows_kernel(const ProductArgs a) {
  using T = typename Elem<DT>::T;
  constexpr int VEC = Elem<DT>::VEC;
  constexpr int CW = kRowCols, CL = CW / VEC;   // columns, and lanes a row of them
  constexpr int KL = 64 / CL;           // rows of W a load
  constexpr int H = G ? 2 : 1;
  // loads of a half in flight, and as many being used
  constexpr int U = !AL || H * MR == 8 ? 2 : G ? 4 : 8;
  static_assert(kRowStep % (U * KL) == 0);
  extern __shared__ float lds[];        // X: [MR][the slice's k], then the wavefronts' sums
  const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6);
  int64_t m0 = static_cast<int64_t>(blockIdx.y) * MR, mend = a.M;
  int group = 0;
  if (a.groups > 0) {
    const Span s = GroupTiles<MR>(a).find(static_cast<int>(blockIdx.y), &m0);
    if (s.group < 0) return;
    group = s.group;
    mend = s.hi;
  }
  const int64_t n0 = static_cast<int64_t>(blockIdx.x) * CW, n = n0 + lane % CL * VEC;
  const int K = static_cast<int>(a.K);
  const T* W = static_cast<const T*>(a.B) + group * a.sB + n;
  const int valid = a.N - n >= VEC ? VEC : a.N > n ? static_cast<int>(a.N - n) : 0;
  // the wavefronts take turns of U loads, so that the workgroup reads one run of rows
  constexpr int STEP = U * KL * kRowWaves;
  const int all = (K + U * KL - 1) / (U * KL), z = static_cast<int>(blockIdx.z);   // of loads
  const int kz = all * z / a.splits * (U * KL), ke = min(K, all * (z + 1) / a.splits * (U * KL));
  const int k0 = kz + wave * U * KL;

  u32x4 w[H][U];
  const T* first = static_cast<const T*>(a.B) + group * a.sB + n0;
  const int64_t bytes = (static_cast<int64_t>(K - 1) * a.ldb + H * a.N - n0) * static_cast<int64_t>(sizeof(T));
  const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(
      reinterpret_cast<void*>(uniform_ptr(first)), 0, uni(static_cast<int>(bytes < kReach ? bytes : kReach)), 0x00020000);
  const uint32_t ldb = static_cast<uint32_t>(a.ldb) * sizeof(T);
  const uint32_t lane0 = valid ? lane / CL * ldb + static_cast<uint32_t>(n - n0) * sizeof(T) : kOutside;
  auto load = [&](int k) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int h = 0; h < H; ++h) {
        if constexpr (AL) {
          w[h][u] = __builtin_bit_cast(
              u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                         rsrc, lane0 + static_cast<uint32_t>(k + u * KL) * ldb +
                                   h * static_cast<uint32_t>(a.N) * sizeof(T), 0, 0));
        } else {
          const int row = k + u * KL + lane / CL;
          w[h][u] = load_chunk<T, VEC>(W + static_cast<int64_t>(row) * a.ldb + h * a.N, row < K ? valid : 0);
        }
      }
    }
  };
  if (k0 < ke) load(k0);
  // (whole loads' k: beyond K X is zero as W is, or an infinite X would meet W's zeros)
  const int slice = all * (z + 1) / a.splits * (U * KL) - kz;
  for (int i = threadIdx.x; i < MR * slice; i += kRowThreads) {
    const int m = i / slice, k = kz + i - m * slice;
    float x = 0.0f;
    if (m0 + m < mend && k < K) {
      int64_t row = m0 + m;
      bool ok = true;
      if (a.gather) {
        const int at = a.gather[row];
        row = at < 0 ? 0 : at / a.gather_div;
        ok = at >= 0 && row < a.a_rows;
      }
      if (ok) x = to_float(static_cast<const T*>(a.A)[row * a.lda + k]);
    }
    lds[i] = x;
  }
  __syncthreads();
  float acc[H][MR][VEC] = {};
  for (int k = k0; k < ke; k += STEP) {
    u32x4 v[H][U];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < H; ++h) v[h][u] = w[h][u];
    if (k + STEP < ke) load(k + STEP);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int row = k + u * KL + lane / CL - kz;
      float x[MR];
#pragma unroll
      for (int m = 0; m < MR; ++m) x[m] = lds[m * slice + row];
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int c = 0; c < VEC; ++c) {
          float b;
          if constexpr (DT == 1)
            b = __builtin_bit_cast(float, c & 1 ? v[h][u][c / 2] & 0xffff0000u : v[h][u][c / 2] << 16);
          else
            b = __builtin_bit_cast(f32x4, v[h][u])[c];
#pragma unroll
          for (int m = 0; m < MR; ++m) acc[h][m][c] = fmaf(x[m], b, acc[h][m][c]);
        }
    }
  }
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int m = 0; m < MR; ++m)
#pragma unroll
      for (int c = 0; c < VEC; ++c)
#pragma unroll
        for (int d = CL; d < 64; d <<= 1) acc[h][m][c] += __shfl_xor(acc[h][m][c], d);
  __syncthreads();
  // [wavefront][half][row][CW]
  if (lane < CL) {
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int m = 0; m < MR; ++m)
#pragma unroll
        for (int c = 0; c < VEC; c += 4)
          *reinterpret_cast<f32x4*>(lds + ((wave * H + h) * MR + m) * CW + lane * VEC + c) =
              f32x4{acc[h][m][c], acc[h][m][c + 1], acc[h][m][c + 2], acc[h][m][c + 3]};
  }
  __syncthreads();
  const int i = threadIdx.x;
  constexpr int QN = CW / 4;
  if (i >= MR * QN) return;
  const int m = i / QN, q = i % QN;
  const int64_t row = m0 + m, col = n0 + q * 4;
  if (row >= mend || col >= written<T>(a.e, a.N)) return;
  f32x4 v{}, u{};
#pragma unroll 4
  for (int s = 0; s < kRowWaves; ++s) {
    v += *reinterpret_cast<const f32x4*>(lds + (s * H * MR + m) * CW + q * 4);
    if constexpr (G) u += *reinterpret_cast<const f32x4*>(lds + ((s * H + 1) * MR + m) * CW + q * 4);
  }
  if (a.splits > 1) {
    part_quad<G>(a, z, row, col, v, u);
    return;
  }
  const int left = a.N - col < 4 ? static_cast<int>(a.N - col) : 4;
  const f32x4 bv = bias_quad<T>(a.e, col, group, left);
  const f32x4 bu = G ? bias_quad<T>(a.e, col + a.N, group, left) : f32x4{};
  linear_quad<T>(a.e, a.N, row, col, group, left, G, v, u, bv, bu,
                 residual_quad<T>(a.e, row, col, left));
}

template <int DT, int MR, bool G, bool AL>
hipError_t rows_by(const ProductArgs& a, hipStream_t s) {
  const size_t lds = static_cast<size_t>(rows_lds(a.K, MR, G));
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(rows_kernel<DT, MR, G, AL>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize,
                                             static_cast<int>(lds));
    if (e != hipSuccess) return e;
  }
  const dim3 grid(static_cast<unsigned>(a.tilesN), static_cast<unsigned>(a.tilesM),
                  static_cast<unsigned>(a.splits));
  rows_kernel<DT, MR, G, AL><<<grid, kRowThreads, lds, s>>>(a);
  return hipGetLastError();
}

template <int DT, int MR>
hipError_t rows_of(const ProductArgs& a, hipStream_t s) {
  constexpr int VEC = Elem<DT>::VEC;
  const bool g = a.e.gated != 0;
  const bool al = a.N % VEC == 0 && a.ldb % VEC == 0 && a.sB % VEC == 0 &&
                  reinterpret_cast<uintptr_t>(a.B) % 16 == 0 &&
                  (a.K + 1024) * a.ldb * static_cast<int64_t>(sizeof(typename Elem<DT>::T)) < kReach;
  if (g) return al ? rows_by<DT, MR, true, true>(a, s) : rows_by<DT, MR, true, false>(a, s);
  return al ? rows_by<DT, MR, false, true>(a, s) : rows_by<DT, MR, false, false>(a, s);
}
template <int DT>
hipError_t rows_of(int rows, const ProductArgs& a, hipStream_t s) {
  return rows == 1 ? rows_of<DT, 1>(a, s) : rows == 2 ? rows_of<DT, 2>(a, s) : rows_of<DT, 4>(a, s);
}

}  // namespace

int64_t rows_lds(int64_t K, int rows, bool gated) {
  const int64_t whole = (K + kRowStep - 1) / kRowStep * kRowStep;
  return std::max<int64_t>(rows * whole, int64_t{kRowWaves} * (gated ? 2 : 1) * rows * 64) * 4;
}

hipError_t launch_rows(int dtype, int rows, const ProductArgs& a, hipStream_t s) {
  return dtype == GT_BF16 ? rows_of<1>(rows, a, s) : rows_of<0>(rows, a, s);
}

}  // namespace gt
