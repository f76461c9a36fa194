// Codes of a matrix and of its transpose with their blocks' scales.
//
// A workgroup takes a square of 128×128 values, 256 threads an 8×8 of them each, read
// once: rows' scales are maxima over 16 lanes, columns' and the square's meet in LDS. A
// thread's 8 codes of a row, or of a column for the transpose, are 8 bytes.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "fp8.hpp"
#include "layer8_kernels.h"
#include "layer_kernels.h"

namespace gt {
namespace {

template <typename T, int CODE, bool SQUARE, bool Q, bool QT>
__global__ __launch_bounds__(256) void quantise_kernel(const gt_quantise_args a, int64_t tilesN,
                                                       int64_t tiles) {
  __shared__ float most[4][16][8];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int cg = threadIdx.x & 15, rg = threadIdx.x >> 4;
  const bool pow2 = a.pow2 != 0;
  for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
    const int64_t tm = t / tilesN, tn = t - tm * tilesN;
    const int64_t m0 = tm * kBlock + rg * 8, n0 = tn * kBlock + cg * 8;
    const T* x = static_cast<const T*>(a.X) + m0 * a.ldx + n0;
    raw8<T> raw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      raw[i] = raw8<T>{};
      if (m0 + i < a.M) raw[i] = raw_of<T>(x + i * a.ldx, a.N - n0);
    }
    oct v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = open8<T>(raw[i]);
    float square = 0.0f;
    if constexpr (SQUARE) {
#pragma unroll
      for (int i = 0; i < 8; ++i) square = fmaxf(square, most8(v[i]));
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) square = fmaxf(square, __shfl_xor(square, d));
      __syncthreads();
      if (lane == 0) most[wave][0][0] = square;
      __syncthreads();
      square = fmaxf(fmaxf(most[0][0][0], most[1][0][0]), fmaxf(most[2][0][0], most[3][0][0]));
      square = block_scale<CODE>(square, pow2);
      if (threadIdx.x == 0) {
        if constexpr (Q) a.S[tm * a.lds + tn] = square;
        if constexpr (QT) a.St[tn * a.ldst + tm] = square;
      }
    }
    if constexpr (Q) {
      uint8_t* q = static_cast<uint8_t*>(a.Q) + m0 * a.ldq + n0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float s = SQUARE ? square : block_scale<CODE>(max16(most8(v[i])), pow2);
        if (m0 + i >= a.M) continue;
        store_codes(q + i * a.ldq, code8<CODE>(v[i], 1.0f / s), a.N - n0);
        if (!SQUARE && cg == 0) a.S[(m0 + i) * a.lds + tn] = s;
      }
    }
    if constexpr (QT) {
      float col[8];
      if constexpr (!SQUARE) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          col[j] = 0.0f;
#pragma unroll
          for (int i = 0; i < 8; ++i) col[j] = fmaxf(col[j], fabsf(j < 4 ? v[i].a[j & 3] : v[i].b[j & 3]));
          col[j] = fmaxf(col[j], __shfl_xor(col[j], 16));
          col[j] = fmaxf(col[j], __shfl_xor(col[j], 32));
        }
        __syncthreads();
        if (lane < 16) {
#pragma unroll
          for (int j = 0; j < 8; ++j) most[wave][cg][j] = col[j];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          col[j] = fmaxf(fmaxf(most[0][cg][j], most[1][cg][j]), fmaxf(most[2][cg][j], most[3][cg][j]));
          col[j] = block_scale<CODE>(col[j], pow2);
        }
      }
      uint8_t* q = static_cast<uint8_t*>(a.Qt) + n0 * a.ldqt + m0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (n0 + j >= a.N) continue;
        const float s = SQUARE ? square : col[j];
        oct w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w.a[i] = j < 4 ? v[i].a[j & 3] : v[i].b[j & 3];
          w.b[i] = j < 4 ? v[i + 4].a[j & 3] : v[i + 4].b[j & 3];
        }
        store_codes(q + j * a.ldqt, code8<CODE>(w, 1.0f / s), a.M - m0);
        if (!SQUARE && rg == 0) a.St[(n0 + j) * a.ldst + tm] = s;
      }
    }
  }
}

template <typename T, int CODE, bool SQUARE>
hipError_t go(const gt_quantise_args& a, hipStream_t s) {
  const int64_t tilesN = (a.N + kBlock - 1) / kBlock, tiles = (a.M + kBlock - 1) / kBlock * tilesN;
  const unsigned grid = static_cast<unsigned>(std::min<int64_t>(tiles, int64_t{1} << 20));
  if (a.Q && a.Qt)
    quantise_kernel<T, CODE, SQUARE, true, true><<<grid, 256, 0, s>>>(a, tilesN, tiles);
  else if (a.Q)
    quantise_kernel<T, CODE, SQUARE, true, false><<<grid, 256, 0, s>>>(a, tilesN, tiles);
  else
    quantise_kernel<T, CODE, SQUARE, false, true><<<grid, 256, 0, s>>>(a, tilesN, tiles);
  return hipGetLastError();
}
template <typename T, int CODE>
hipError_t by_block(const gt_quantise_args& a, hipStream_t s) {
  return a.block == 1 ? go<T, CODE, false>(a, s) : go<T, CODE, true>(a, s);
}
template <typename T>
hipError_t by_code(const gt_quantise_args& a, hipStream_t s) {
  return a.code == GT_E4M3 ? by_block<T, GT_E4M3>(a, s) : by_block<T, GT_E5M2>(a, s);
}

}  // namespace

hipError_t launch_quantise(const gt_quantise_args& a, hipStream_t s) {
  return a.dtype == GT_BF16 ? by_code<uint16_t>(a, s) : by_code<float>(a, s);
}

}  // namespace gt
