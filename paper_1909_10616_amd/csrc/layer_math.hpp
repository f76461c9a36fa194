// Activations, and accesses of 4 consecutive values, of the layer kernels. All
// arithmetic is fp32; bf16 is rounded to nearest even, once, where it is stored.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "gemm_kernel.hpp"
#include "gemmtune_layers.h"

namespace gt {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

// Exponentials of the activations. x·log2 e rounds at 2^-24 of itself, and so does x²: the
// instruction's exponential of either is off by up to 4e-6 of itself at x = −80 and 7e-6 at
// x = −12. bf16 rounds at 2^-9; fp32 takes the library's exponential, and what x² lost.
template <typename T>
__device__ __forceinline__ float exp_minus(float x) {   // exp(−x)
  if constexpr (sizeof(T) == 4)
    return expf(-x);
  else
    return __builtin_amdgcn_exp2f(x * -1.4426950408889634f);
}
template <typename T>
__device__ __forceinline__ float exp_square(float x) {   // exp(−x²/2)
  if constexpr (sizeof(T) == 4) {
    const float y = fminf(fabsf(x), 16.0f), s = y * y;   // (0 from 14.5 on)
    return expf(-0.5f * s) * fmaf(-0.5f, fmaf(y, y, -s), 1.0f);
  } else {
    return __builtin_amdgcn_exp2f(x * x * -0.72134752044448171f);
  }
}

template <typename T>
__device__ __forceinline__ float sigmoid_of(float x) {
  return __builtin_amdgcn_rcpf(1.0f + exp_minus<T>(x));
}

// Φ(x), the normal distribution function, and *e = exp(−x²/2). For x < 0, Φ = q·e with
// q a polynomial in t = 1/(1 + 0.3·|x|), fitted by least squares to the scaled
// complementary error function at 4500 points of [0, 14] with weights that even
// out its relative error (1.5e-7; 5e-7 as evaluated here, beside e's): a dozen instructions and
// one exponential that the slope shares, where the library's error function
// takes two branches of about fifty.
template <typename T>
__device__ __forceinline__ float normal_cdf(float x, float* e) {
  const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(x), 0.3f, 1.0f));
  float q = 0.03567453473806381f;
  q = fmaf(q, t, -0.1572018563747406f);
  q = fmaf(q, t, 0.20635104179382324f);
  q = fmaf(q, t, -0.053681083023548126f);
  q = fmaf(q, t, 0.1285601556301117f);
  q = fmaf(q, t, 0.09991396218538284f);
  q = fmaf(q, t, 0.12075387686491013f);
  q = fmaf(q, t, 0.11962930113077164f);
  *e = exp_square<T>(x);
  const float tail = q * t * *e;
  return x < 0.0f ? tail : 1.0f - tail;
}

// act(x), of operands of type T
template <typename T>
__device__ __forceinline__ float act_value(int act, float x) {
  if (act == GT_ACT_SILU) return x * sigmoid_of<T>(x);
  if (act == GT_ACT_GELU) {
    float e;
    return x * normal_cdf<T>(x, &e);
  }
  if (act == GT_ACT_RELU) return x < 0.0f ? 0.0f : x;
  return x;
}

// act(x) and act'(x)
template <typename T>
__device__ __forceinline__ void act_both(int act, float x, float* value, float* slope) {
  if (act == GT_ACT_SILU) {
    const float s = sigmoid_of<T>(x);
    *value = x * s;
    *slope = s * (1.0f + x * (1.0f - s));
  } else if (act == GT_ACT_GELU) {
    float e;
    const float c = normal_cdf<T>(x, &e);
    *value = x * c;
    *slope = fmaf(x * 0.39894228040143268f, e, c);
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

// Up to 4 values from p on, the first n of them; zero beyond. Four are one access, at any
// alignment (which the memory system splits where it must).
template <typename T>
__device__ __forceinline__ f32x4 load4(const T* p, int n) {
  f32x4 v{};
  if (n >= 4) {
    if constexpr (sizeof(T) == 4) {
      __builtin_memcpy(&v, p, 16);
    } else {
      uint2 u;
      __builtin_memcpy(&u, p, 8);
      v[0] = __builtin_bit_cast(float, u.x << 16);
      v[1] = __builtin_bit_cast(float, u.x & 0xffff0000u);
      v[2] = __builtin_bit_cast(float, u.y << 16);
      v[3] = __builtin_bit_cast(float, u.y & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < n) v[i] = to_float(p[i]);
  }
  return v;
}

template <typename T>
__device__ __forceinline__ void store4(T* p, f32x4 v, int n) {
  if (n >= 4) {
    if constexpr (sizeof(T) == 4) {
      __builtin_memcpy(p, &v, 16);
    } else {
      const uint2 u = __builtin_bit_cast(uint2, __builtin_convertvector(v, bf16x4));
      __builtin_memcpy(p, &u, 8);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < n) p[i] = from_float<T>(v[i]);
  }
}

// 8 values, at any alignment.
struct oct {
  f32x4 a, b;
};
template <typename T>
struct raw8 {   // as they lie in memory
  u32x4 w[sizeof(T) / 2];
};
template <typename T>
__host__ __device__ __forceinline__ oct open8(const raw8<T>& r) {
  oct v;
  if constexpr (sizeof(T) == 4) {
    v.a = __builtin_bit_cast(f32x4, r.w[0]);
    v.b = __builtin_bit_cast(f32x4, r.w[1]);
  } else {
    const u32x4 u = r.w[0];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      v.a[2 * i] = __builtin_bit_cast(float, u[i] << 16);
      v.a[2 * i + 1] = __builtin_bit_cast(float, u[i] & 0xffff0000u);
      v.b[2 * i] = __builtin_bit_cast(float, u[i + 2] << 16);
      v.b[2 * i + 1] = __builtin_bit_cast(float, u[i + 2] & 0xffff0000u);
    }
  }
  return v;
}
template <typename T>
__host__ __device__ __forceinline__ oct load8(const T* p) {
  raw8<T> r;
  __builtin_memcpy(&r, p, sizeof(r));
  return open8<T>(r);
}
template <typename T>
__host__ __device__ __forceinline__ void store8(T* p, const oct& v) {
  if constexpr (sizeof(T) == 4) {
    __builtin_memcpy(p, &v.a, 16);
    __builtin_memcpy(p + 4, &v.b, 16);
  } else {
    const uint2 x = __builtin_bit_cast(uint2, __builtin_convertvector(v.a, bf16x4));
    const uint2 y = __builtin_bit_cast(uint2, __builtin_convertvector(v.b, bf16x4));
    const u32x4 w{x.x, x.y, y.x, y.y};
    __builtin_memcpy(p, &w, 16);
  }
}
template <typename T, int ACT>
__device__ __forceinline__ void act8(oct& v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v.a[i] = act_value<T>(ACT, v.a[i]);
    v.b[i] = act_value<T>(ACT, v.b[i]);
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

// The inclusive prefix sum over the wavefront (all lanes active): lane moves within rows of
// 16, then the rows' totals.
__device__ __forceinline__ int wave_prefix(int v) {
  const int lane = threadIdx.x & 63;
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);   // from 1, 2, 4, 8 lanes below
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
  const int a = __builtin_amdgcn_readlane(v, 15), b = a + __builtin_amdgcn_readlane(v, 31),
            c = b + __builtin_amdgcn_readlane(v, 47);
  return v + (lane >= 48 ? c : lane >= 32 ? b : lane >= 16 ? a : 0);
}

}  // namespace gt
