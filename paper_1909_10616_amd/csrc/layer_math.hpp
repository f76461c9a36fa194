// Activations, and accesses of 4 consecutive values, of the layer kernels. All
// arithmetic is fp32; bf16 is rounded to nearest even, once, where it is stored.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "gemm_kernel.hpp"
#include "gemmtune_layers.h"

namespace gt {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float sigmoid_of(float x) {
  return __builtin_amdgcn_rcpf(1.0f + expf(-x));
}

// act(x)
__device__ __forceinline__ float act_value(int act, float x) {
  if (act == GT_ACT_SILU) return x * sigmoid_of(x);
  if (act == GT_ACT_GELU) return 0.5f * x * (1.0f + erff(x * 0.70710678118654752f));
  if (act == GT_ACT_RELU) return x < 0.0f ? 0.0f : x;
  return x;
}

// act(x) and act'(x)
__device__ __forceinline__ void act_both(int act, float x, float* value, float* slope) {
  if (act == GT_ACT_SILU) {
    const float s = sigmoid_of(x);
    *value = x * s;
    *slope = s * (1.0f + x * (1.0f - s));
  } else if (act == GT_ACT_GELU) {
    const float c = 0.5f * (1.0f + erff(x * 0.70710678118654752f));
    *value = x * c;
    *slope = c + x * 0.39894228040143268f * expf(-0.5f * x * x);
  } else if (act == GT_ACT_RELU) {
    *value = x < 0.0f ? 0.0f : x;
    *slope = x > 0.0f ? 1.0f : 0.0f;
  } else {
    *value = x;
    *slope = 1.0f;
  }
}

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(uint16_t v) {
  return __builtin_bit_cast(float, static_cast<uint32_t>(v) << 16);
}
template <typename T>
__device__ __forceinline__ T from_float(float v) {
  if constexpr (sizeof(T) == 4)
    return v;
  else
    return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
}

// Up to 4 values from p on, the first n of them (all at once if vec); zero beyond.
template <typename T>
__device__ __forceinline__ f32x4 load4(const T* p, int n, bool vec) {
  f32x4 v{};
  if (vec && n >= 4) {
    if constexpr (sizeof(T) == 4) {
      v = *reinterpret_cast<const f32x4*>(p);
    } else {
      const uint2 u = *reinterpret_cast<const uint2*>(p);
      v[0] = __builtin_bit_cast(float, u.x << 16);
      v[1] = __builtin_bit_cast(float, u.x & 0xffff0000u);
      v[2] = __builtin_bit_cast(float, u.y << 16);
      v[3] = __builtin_bit_cast(float, u.y & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) v[i] = to_float(p[i]);
  }
  return v;
}

template <typename T>
__device__ __forceinline__ void store4(T* p, f32x4 v, int n, bool vec) {
  if (vec && n >= 4) {
    if constexpr (sizeof(T) == 4)
      *reinterpret_cast<f32x4*>(p) = v;
    else
      *reinterpret_cast<uint2*>(p) =
          __builtin_bit_cast(uint2, __builtin_convertvector(v, bf16x4));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) p[i] = from_float<T>(v[i]);
  }
}

// The first n (≤ 0: none) of VEC values from p, at any alignment; zero beyond.
template <typename T, int VEC>
__device__ __forceinline__ u32x4 load_chunk(const T* p, int64_t n) {
  u32x4 v{};
  if (n >= VEC) {
    __builtin_memcpy(&v, p, 16);
  } else if (n > 0) {
    T e[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) e[i] = i < n ? p[i] : T(0);
    __builtin_memcpy(&v, e, 16);
  }
  return v;
}

}  // namespace gt
