// Codes of a matrix and of its transpose with their blocks' scales.
//
// A workgroup takes a square of 128×128 values, 256 threads an 8×8 of them each, read
// once: rows' scales are maxima over 16 lanes, columns' and the square's meet in LDS. A
// thread's 8 codes of a row are 8 bytes; those of a column go through LDS, so that the
// transpose is written 128 bytes of a row at a time. Bound by memory: 4096×11008 of bf16 with
// both codes 46 µs, 3.9 TB/s; 2623×3457 of fp32 in squares 14 µs, 3.9 TB/s.
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
  __shared__ uint2 turn[QT ? kBlock : 1][16];   // [column][octet of rows ^ 2·(column / 8)]
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
      if constexpr (sizeof(T) == 2) {   // (widened anew: the 32 registers they lie in are half as many)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          asm volatile("" : "+v"(raw[i].w[0]));
          v[i] = open8<T>(raw[i]);
        }
      }
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
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float s = SQUARE ? square : col[j];
        oct w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w.a[i] = j < 4 ? v[i].a[j & 3] : v[i].b[j & 3];
          w.b[i] = j < 4 ? v[i + 4].a[j & 3] : v[i + 4].b[j & 3];
        }
        turn[cg * 8 + j][rg ^ (cg * 2 & 14)] = code8<CODE>(w, 1.0f / s);
        if (!SQUARE && rg == 0 && n0 + j < a.N) a.St[(n0 + j) * a.ldst + tm] = s;
      }
      __syncthreads();
      const int64_t c0 = tn * kBlock, r0 = tm * kBlock + (threadIdx.x & 7) * 16;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = i * 32 + (threadIdx.x >> 3), at = (threadIdx.x & 7) * 2 ^ (c / 8 * 2 & 14);
        if (c0 + c >= a.N) continue;
        uint8_t* q = static_cast<uint8_t*>(a.Qt) + (c0 + c) * a.ldqt + r0;
        const uint2 lo = turn[c][at], hi = turn[c][at + 1];
        if (r0 + 16 <= a.M) {
          const u32x4 w{lo.x, lo.y, hi.x, hi.y};
          __builtin_memcpy(q, &w, 16);
        } else {
          store_codes(q, lo, a.M - r0);
          store_codes(q + 8, hi, a.M - r0 - 8);
        }
      }
      __syncthreads();
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
