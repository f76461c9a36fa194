// 8-bit floating point: scales of blocks and codes.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "gemmtune_layers.h"
#include "layer_math.hpp"

namespace gt {

constexpr int kBlock = 128;   // values that share a scale, along k

template <int CODE>
constexpr float kLargest = CODE == GT_E4M3 ? 448.0f : 57344.0f;

// The scale of a block whose largest magnitude is m. Both divisions of a code, this one and
// that of one by the scale, are the compiler's correctly rounded ones, so that codes are
// the same bits in any implementation.
template <int CODE>
__device__ __forceinline__ float block_scale(float m, bool pow2) {
  float s = m / kLargest<CODE>;
  s = s < 1.17549435e-38f ? 1.17549435e-38f : s;   // (1/s stays finite)
  if (pow2) s = __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, s) + 0x7fffffu) & 0x7f800000u);
  return m == 0.0f ? 1.0f : s;
}

// 4 codes of values already divided by their scale: |v| is at most the type's largest but for
// the rounding of the division, which the nearest code absorbs. NaN is NaN.
template <int CODE>
__device__ __forceinline__ uint32_t code4(float a, float b, float c, float d) {
  int w = 0;
  if constexpr (CODE == GT_E4M3) {
    w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  } else {
    w = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, w, false);
    w = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, w, true);
  }
  return static_cast<uint32_t>(w);
}
template <int CODE>
__device__ __forceinline__ uint2 code8(const oct& v, float r) {
  return uint2{code4<CODE>(v.a[0] * r, v.a[1] * r, v.a[2] * r, v.a[3] * r),
               code4<CODE>(v.b[0] * r, v.b[1] * r, v.b[2] * r, v.b[3] * r)};
}
// The first n of 8 codes.
__device__ __forceinline__ void store_codes(uint8_t* p, uint2 q, int64_t n) {
  if (n >= 8) {
    __builtin_memcpy(p, &q, 8);
  } else {
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (i < n) p[i] = static_cast<uint8_t>((i < 4 ? q.x : q.y) >> (8 * (i & 3)));
  }
}

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// 8 codes as bf16, which holds every one of them exactly. The matrix instructions that take
// codes keep some 13 bits below the largest of the products they add at once (a 1 beside
// 2^14 and −2^14 vanishes), 1.7e-5 of a product's norm; of bf16 operands they keep all that fp32
// holds.
template <int CODE>
__device__ __forceinline__ bf16x8 widen8(int lo, int hi) {
  bf16x2 v[4];
  if constexpr (CODE == GT_E4M3) {
    v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
    v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
    v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  } else {
    v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, 1.0f, false);
    v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, 1.0f, true);
    v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, 1.0f, false);
    v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, 1.0f, true);
  }
  return __builtin_bit_cast(bf16x8, v);
}

// The largest magnitude of 8 values (NaN left out).
__device__ __forceinline__ float most8(const oct& v) {
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = fmaxf(m, fmaxf(fabsf(v.a[i]), fabsf(v.b[i])));
  return m;
}
// A value from N lanes further on, around a row of 16 lanes.
template <int N>
__device__ __forceinline__ float turned(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + N, 0xf, 0xf, false));
}
// The maximum over rows of 16 lanes (all active).
__device__ __forceinline__ float max16(float m) {
  m = fmaxf(m, turned<8>(m));
  m = fmaxf(m, turned<4>(m));
  m = fmaxf(m, turned<2>(m));
  return fmaxf(m, turned<1>(m));
}
// The sum over the wavefront, the same bits in every lane (all active).
__device__ __forceinline__ float wave_sum(float s) {
  s += turned<8>(s);
  s += turned<4>(s);
  s += turned<2>(s);
  s += turned<1>(s);
  const int v = __builtin_bit_cast(int, s);
  const float a = __builtin_bit_cast(float, __builtin_amdgcn_readlane(v, 0));
  const float b = __builtin_bit_cast(float, __builtin_amdgcn_readlane(v, 16));
  const float c = __builtin_bit_cast(float, __builtin_amdgcn_readlane(v, 32));
  const float d = __builtin_bit_cast(float, __builtin_amdgcn_readlane(v, 48));
  return (a + b) + (c + d);
}

// The first n (≤ 0: none) of 8 values from p, zero beyond.
template <typename T>
__device__ __forceinline__ raw8<T> raw_of(const T* p, int64_t n) {
  raw8<T> r{};
  if (n >= 8) {
    __builtin_memcpy(&r, p, sizeof(r));
  } else if (n > 0) {
    T e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = i < n ? p[i] : T(0);
    __builtin_memcpy(&r, e, sizeof(r));
  }
  return r;
}
template <typename T>
__device__ __forceinline__ void store8n(T* p, const oct& v, int64_t n) {
  if (n >= 8) {
    store8(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (i < n) p[i] = from_float<T>(i < 4 ? v.a[i & 3] : v.b[i & 3]);
  }
}

}  // namespace gt
