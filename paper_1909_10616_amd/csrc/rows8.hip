// 8-bit products of up to 64 rows a workgroup, X·Wᵀ with the linear epilogue, codes straight from
// memory into matrix instructions: bound by W's way from memory.
//
// A workgroup takes 16, 32 or 64 rows, 16 columns (gated: 16 of each half) and all of K, its 8
// wavefronts taking turns at its blocks of 128, whose sums then take their scales. The codes are
// widened to bf16 for the matrix instructions, whose sums are then fp32's. A lane holds 32 neighbouring k of a row, so rows of both
// operands are read in runs of 128 bytes, at any alignment. The wavefronts' sums meet in
// LDS and are added in their order.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "fp8.hpp"
#include "layer8_kernels.h"
#include "product.hpp"

namespace gt {
namespace {

constexpr int kWaves = 8;

template <typename T, bool G, int XC, int WC, int RT>
__global__ __launch_bounds__(64 * kWaves) void rows8_kernel(const Product8 q) {
  constexpr int H = G ? 2 : 1, ROWS = 16 * RT;
  const ProductArgs& a = q.p;
  __shared__ f32x4 lds[kWaves][H][ROWS][4];   // [wavefront][half][row][quad ^ (row & 3)]
  const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6);
  const int lx = lane & 15, grp = lane >> 4;
  const int64_t m0 = static_cast<int64_t>(blockIdx.y) * ROWS, n0 = static_cast<int64_t>(blockIdx.x) * 16;
  const uint8_t* X[RT];
  const float* sx[RT];
  const uint8_t* W[H];
  const float* sw[H][4];
  // (rows past the last read the last again, for results that nobody takes)
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const int64_t m = m0 + 16 * i + lx, row = m < a.M ? m : a.M - 1;
    X[i] = static_cast<const uint8_t*>(a.A) + row * a.lda + 32 * grp;
    sx[i] = q.sa + (row >> q.xshift) * q.ldsa;
  }
#pragma unroll
  for (int h = 0; h < H; ++h) {
    const int64_t n = n0 + lx < a.N ? n0 + lx : a.N - 1;
    W[h] = static_cast<const uint8_t*>(a.B) + (h * a.N + n) * a.ldb + 32 * grp;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t c = n0 + 4 * grp + r < a.N ? n0 + 4 * grp + r : a.N - 1;
      sw[h][r] = q.sb + ((h * a.N + c) >> q.wshift) * q.ldsb;
    }
  }
  struct Step {
    i32x8 x[RT], w[H];
    float sx[RT], sw[H][4];
  };
  auto codes = [&](const uint8_t* p, int64_t k, bool whole) __attribute__((always_inline)) {
    i32x8 v;
    if (whole) {
      __builtin_memcpy(&v, p + k, 32);
    } else {   // the last block, where it ends inside
      const u32x4 lo = load_chunk<uint8_t, 16>(p + k, a.K - k - 32 * grp);
      const u32x4 hi = load_chunk<uint8_t, 16>(p + k + 16, a.K - k - 32 * grp - 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = static_cast<int>(lo[i]);
        v[4 + i] = static_cast<int>(hi[i]);
      }
    }
    return v;
  };
  auto load = [&](Step& s, int64_t b, bool whole) __attribute__((always_inline)) {
    const int64_t k = b * kBlock;
#pragma unroll
    for (int h = 0; h < H; ++h) {
      s.w[h] = codes(W[h], k, whole);
#pragma unroll
      for (int r = 0; r < 4; ++r) s.sw[h][r] = sw[h][r][b];
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      s.x[i] = codes(X[i], k, whole);
      s.sx[i] = sx[i][b];
    }
  };
  f32x4 acc[H][RT] = {};
  auto multiply = [&](const Step& s) __attribute__((always_inline)) {
    f32x4 part[H][RT] = {};
#pragma unroll
    for (int c = 0; c < 8; c += 2) {
      bf16x8 w[H];
#pragma unroll
      for (int h = 0; h < H; ++h) w[h] = widen8<WC>(s.w[h][c], s.w[h][c + 1]);
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        const bf16x8 x = widen8<XC>(s.x[i][c], s.x[i][c + 1]);
#pragma unroll
        for (int h = 0; h < H; ++h)
          part[h][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[h], x, part[h][i], 0, 0, 0);
      }
    }
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[h][i][r] = fmaf(part[h][i][r], s.sx[i] * s.sw[h][r], acc[h][i][r]);
  };
  // A wavefront's next block is on its way while it multiplies one. The blocks that are whole in a
  // loop of their own, two by two, so that no step is copied and no load checked (1×11008×4096 15.6
  // → 12.3 µs); gated, whose registers then leave one workgroup a unit, not (22.2 µs, 26.0 so).
  const int64_t whole = a.K / kBlock, blocks = (a.K + kBlock - 1) / kBlock;
  if constexpr (G) {
    Step next;
    if (wave < blocks) load(next, wave, wave < whole);
    for (int64_t b = wave; b < blocks; b += kWaves) {
      const Step s = next;
      if (b + kWaves < blocks) load(next, b + kWaves, b + kWaves < whole);
      multiply(s);
    }
  } else {
    Step step[2];
    if (wave < whole) load(step[0], wave, true);
    for (int64_t b = wave; b < whole; b += 2 * kWaves) {
      if (b + kWaves < whole) load(step[1], b + kWaves, true);
      multiply(step[0]);
      if (b + 2 * kWaves < whole) load(step[0], b + 2 * kWaves, true);
      if (b + kWaves < whole) multiply(step[1]);
    }
    if (whole < blocks && wave == whole % kWaves) {
      load(step[0], whole, false);
      multiply(step[0]);
    }
  }
  // a lane's sums: row 16·i + lx, columns 4·grp …
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int i = 0; i < RT; ++i) lds[wave][h][16 * i + lx][grp ^ (lx & 3)] = acc[h][i];
  __syncthreads();
  const int m = threadIdx.x >> 2, c = threadIdx.x & 3;
  const int64_t row = m0 + m, col = n0 + 4 * c;
  if (m >= ROWS || row >= a.M || col >= a.N) return;
  f32x4 v{}, u{};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    v += lds[w][0][m][c ^ (m & 3)];
    if constexpr (G) u += lds[w][H - 1][m][c ^ (m & 3)];
  }
  const int left = a.N - col < 4 ? static_cast<int>(a.N - col) : 4;
  linear_quad<T>(a.e, a.N, row, col, 0, left, G, v, u, bias_quad<T>(a.e, col, 0, left),
                 G ? bias_quad<T>(a.e, col + a.N, 0, left) : f32x4{}, residual_quad<T>(a.e, row, col, left));
}

template <typename T, bool G, int XC, int WC>
hipError_t by_rows(int rows, const Product8& a, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(a.p.tilesN), static_cast<unsigned>(a.p.tilesM));
  if (rows == 16) rows8_kernel<T, G, XC, WC, 1><<<grid, 64 * kWaves, 0, s>>>(a);
  else if (rows == 32) rows8_kernel<T, G, XC, WC, 2><<<grid, 64 * kWaves, 0, s>>>(a);
  else if constexpr (!G) rows8_kernel<T, G, XC, WC, 4><<<grid, 64 * kWaves, 0, s>>>(a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}
template <typename T, bool G>
hipError_t by_codes(int rows, const Product8& a, hipStream_t s) {
  if (a.acode == GT_E4M3)
    return a.bcode == GT_E4M3 ? by_rows<T, G, 0, 0>(rows, a, s) : by_rows<T, G, 0, 1>(rows, a, s);
  return a.bcode == GT_E4M3 ? by_rows<T, G, 1, 0>(rows, a, s) : by_rows<T, G, 1, 1>(rows, a, s);
}
template <typename T>
hipError_t by_gate(int rows, const Product8& a, hipStream_t s) {
  return a.p.e.gated ? by_codes<T, true>(rows, a, s) : by_codes<T, false>(rows, a, s);
}

}  // namespace

hipError_t launch_rows8(int dtype, int rows, const Product8& a, hipStream_t s) {
  return dtype == GT_BF16 ? by_gate<uint16_t>(rows, a, s) : by_gate<float>(rows, a, s);
}

}  // namespace gt
