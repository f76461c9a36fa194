// Layer norm and its gradients, a row in the registers of 64 to 512 threads.
//
// Forward: the mean, then in one exchange Σ(X − mean) and Σ(X − mean)² of the values that the registers
// hold, then the outputs: each row is read once and written once. The first of the two sums is what
// the mean has lost to rounding (4096 values with a mean of 10^5 deviations: 1 % of a deviation); it is
// taken off the deviations, their variance and the mean, so that a large mean costs no digits.
// Backward: both means of a row in one exchange; every thread keeps the column sums of dw
// and db for its own columns over all rows that its workgroup takes, and a second launch
// adds the workgroups' sums in their order. Of few rows other workgroups of the same
// launch take the columns' sums.
// Bound by memory: 16384×4096 in bf16 with mean and rstd 47 to 50 µs, 5.4 to 5.7 TB/s; its gradients with
// R 104 µs, 5.2 TB/s. One row of 4096 in bf16 is latency, 2.8 µs on the GPU.
// Thread t of a row has the octets t, t + TH, …, so that 16 neighbours hold 128 columns, a
// block of codes.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "fp8.hpp"
#include "layer8_kernels.h"
#include "layer_kernels.h"

namespace gt {
namespace {

// ---- sums over a row's threads

// The sum over TH threads, the same in each; `box`: LDS that the exchange before did not use.
template <int TH>
__device__ __forceinline__ float row_sum(float s, float* box) {
  s = wave_sum(s);
  if constexpr (TH > 64) {
    if ((threadIdx.x & 63) == 0) box[threadIdx.x >> 6] = s;
    __syncthreads();
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < TH / 64; ++i) s += box[i];
  }
  return s;
}

// Two sums in one exchange.
template <int TH>
__device__ __forceinline__ void row_sums(float* s, float* q, float (*box)[16]) {
  *s = wave_sum(*s);
  *q = wave_sum(*q);
  if constexpr (TH > 64) {
    if ((threadIdx.x & 63) == 0) {
      box[0][threadIdx.x >> 6] = *s;
      box[1][threadIdx.x >> 6] = *q;
    }
    __syncthreads();
    *s = *q = 0.0f;
#pragma unroll
    for (int i = 0; i < TH / 64; ++i) {
      *s += box[0][i];
      *q += box[1][i];
    }
  }
}

template <typename W>
__device__ __forceinline__ oct open_or(const void* p, const raw8<W>& r, float none) {
  return p ? open8<W>(r) : oct{f32x4{none, none, none, none}, f32x4{none, none, none, none}};
}

__device__ __forceinline__ oct times(const oct& v, float f) { return oct{v.a * f, v.b * f}; }
__device__ __forceinline__ float sum8(const oct& v) {
  return ((v.a[0] + v.a[1]) + (v.a[2] + v.a[3])) + ((v.b[0] + v.b[1]) + (v.b[2] + v.b[3]));
}
// v − m in the first n columns, zero in the others
__device__ __forceinline__ oct centred(const oct& v, float m, int64_t n) {
  oct d;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    d.a[i] = i < n ? v.a[i] - m : 0.0f;
    d.b[i] = i + 4 < n ? v.b[i] - m : 0.0f;
  }
  return d;
}

// ---- forward

// What a mean is off by, from the mean of the deviations from it; nothing where that is no number (of a row with
// an infinity, which is its mean, or where the deviations' sum overflows).
__device__ __forceinline__ float offset(float mean) { return fabsf(mean) < __builtin_inff() ? mean : 0.0f; }
// The reciprocal deviation of a row from the mean square of its deviations from a mean that is off by `off`.
// (Fused, so that an infinite square stays one; rounding may leave less than nothing of a constant row.)
__device__ __forceinline__ float deviation(float square, float off, float eps) {
  const float v = fmaf(-off, off, square);
  return 1.0f / sqrtf((v < 0.0f ? 0.0f : v) + eps);
}

// An octet of a row's outputs from its deviations from a mean that is off by `off`.
template <typename T, int CODE>
__device__ __forceinline__ void norm_out(const gt_norm_args& a, int64_t row, int64_t c, const oct& d, float off,
                                         float rstd, const oct& w, const oct& b) {
  const int64_t left = a.N - c;
  oct y;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y.a[i] = fmaf((d.a[i] - off) * rstd, w.a[i], b.a[i]);
    y.b[i] = fmaf((d.b[i] - off) * rstd, w.b[i], b.b[i]);
  }
  if (CODE >= 0 && left < 8) {   // (what is behind the row is not among a block's values)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y.a[i] = i < left ? y.a[i] : 0.0f;
      y.b[i] = i + 4 < left ? y.b[i] : 0.0f;
    }
  }
  if (a.Y && left > 0) store8n(static_cast<T*>(a.Y) + row * a.ldy + c, y, left);
  if constexpr (CODE >= 0) {
    const float s = block_scale<CODE>(max16(left > 0 ? most8(y) : 0.0f), a.pow2 != 0);
    if (left <= 0) return;
    store_codes(static_cast<uint8_t*>(a.Q) + row * a.ldq + c, code8<CODE>(y, 1.0f / s), left);
    if (c % kBlock == 0) a.S[row * a.lds + c / kBlock] = s;
  }
}

template <typename T, typename W, int TH, int NV, int CODE>
__global__ __launch_bounds__(TH < 256 ? 256 : TH) void norm_kernel(const gt_norm_args a) {
  constexpr int RB = TH < 256 ? 256 / TH : 1;   // rows of a workgroup
  __shared__ float box[3][16];
  const int t = threadIdx.x % TH, rb = threadIdx.x / TH;
  const W* wp = static_cast<const W*>(a.w);
  const W* bp = static_cast<const W*>(a.b);
  raw8<W> w[NV], b[NV];
  raw8<T> next[NV];
  const int64_t step = int64_t{gridDim.x} * RB;
  auto col = [&](int v) { return (static_cast<int64_t>(v) * TH + t) * 8; };
  auto load = [&](int64_t row) __attribute__((always_inline)) {
    const T* x = static_cast<const T*>(a.X) + row * a.ldx;
#pragma unroll
    for (int v = 0; v < NV; ++v) next[v] = raw_of<T>(x + col(v), row < a.M ? a.N - col(v) : 0);
  };
  int64_t row = int64_t{blockIdx.x} * RB + rb;
  load(row);
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    w[v] = raw_of<W>(wp + col(v), wp ? a.N - col(v) : 0);
    b[v] = raw_of<W>(bp + col(v), bp ? a.N - col(v) : 0);
  }
  const float each = 1.0f / static_cast<float>(a.N);   // (what its rounding costs the mean goes off with the rest)
  for (; row < a.M; row += step) {
    oct x[NV];
    float s = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      x[v] = open8<T>(next[v]);
      s += sum8(x[v]);
    }
    load(row + step);
    const float mean = row_sum<TH>(s, box[0]) * each;
    float squares = 0.0f;
    s = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      x[v] = centred(x[v], mean, a.N - col(v));
      s += sum8(x[v]);
      squares += sum8(oct{x[v].a * x[v].a, x[v].b * x[v].b});
    }
    row_sums<TH>(&s, &squares, box + 1);
    const float off = offset(s * each), rstd = deviation(squares * each, off, a.eps);
    if (t == 0) {
      if (a.mean) a.mean[row] = mean + off;
      if (a.rstd) a.rstd[row] = rstd;
    }
#pragma unroll
    for (int v = 0; v < NV; ++v)
      norm_out<T, CODE>(a, row, col(v), x[v], off, rstd, open_or<W>(wp, w[v], 1.0f), open_or<W>(bp, b[v], 0.0f));
  }
}

// Rows longer than the registers: read three times.
template <typename T, typename W, int CODE>
__global__ __launch_bounds__(1024) void norm_long_kernel(const gt_norm_args a) {
  constexpr int TH = 1024;
  __shared__ float box[3][16];
  const W* wp = static_cast<const W*>(a.w);
  const W* bp = static_cast<const W*>(a.b);
  const float each = 1.0f / static_cast<float>(a.N);
  for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.X) + row * a.ldx;
    float s = 0.0f;
    for (int64_t c = threadIdx.x * 8; c < a.N; c += TH * 8) s += sum8(open8<T>(raw_of<T>(x + c, a.N - c)));
    const float mean = row_sum<TH>(s, box[0]) * each;
    float squares = 0.0f;
    s = 0.0f;
    for (int64_t c = threadIdx.x * 8; c < a.N; c += TH * 8) {
      const oct d = centred(open8<T>(raw_of<T>(x + c, a.N - c)), mean, a.N - c);
      s += sum8(d);
      squares += sum8(oct{d.a * d.a, d.b * d.b});
    }
    row_sums<TH>(&s, &squares, box + 1);
    const float off = offset(s * each), rstd = deviation(squares * each, off, a.eps);
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = mean + off;
      if (a.rstd) a.rstd[row] = rstd;
    }
    for (int64_t c0 = 0; c0 < a.N; c0 += TH * 8) {   // (all lanes, for the blocks' maxima)
      const int64_t c = c0 + threadIdx.x * 8, left = a.N - c;
      norm_out<T, CODE>(a, row, c, centred(open8<T>(raw_of<T>(x + c, left)), mean, left), off, rstd,
                        open_or<W>(wp, raw_of<W>(wp + c, wp ? left : 0), 1.0f),
                        open_or<W>(bp, raw_of<W>(bp + c, bp ? left : 0), 0.0f));
    }
  }
}

// ---- backward

// Workgroup `block` of `blocks` (TH, at least 256 threads). dw and db of a thread's columns, from
// its workgroup's rows, to the workgroup's partial row.
template <typename T, typename W, int TH, int NV, bool SUMS>
__device__ __forceinline__ void grad_rows(const gt_norm_grad_args& a, float* part, int block, int blocks) {
  constexpr int RB = TH < 256 ? 256 / TH : 1;
  __shared__ float box[2][2][16];
  __shared__ f32x4 join[SUMS && RB > 1 ? RB : 1][SUMS && RB > 1 ? 2 * TH : 1];
  const int t = threadIdx.x % TH, rb = threadIdx.x / TH;
  const W* wp = static_cast<const W*>(a.w);
  const int64_t step = static_cast<int64_t>(blocks) * RB;
  auto col = [&](int v) { return (static_cast<int64_t>(v) * TH + t) * 8; };
  raw8<W> w[NV];
  raw8<T> nx[NV], ny[NV];
  float nmean, nrstd;
  auto load = [&](int64_t row) __attribute__((always_inline)) {
    const T* x = static_cast<const T*>(a.X) + row * a.ldx;
    const T* y = static_cast<const T*>(a.dY) + row * a.lddy;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int64_t left = row < a.M ? a.N - col(v) : 0;
      nx[v] = raw_of<T>(x + col(v), left);
      ny[v] = raw_of<T>(y + col(v), left);
    }
    nmean = row < a.M ? a.mean[row] : 0.0f;
    nrstd = row < a.M ? a.rstd[row] : 0.0f;
  };
  int64_t row = static_cast<int64_t>(block) * RB + rb;
  load(row);
#pragma unroll
  for (int v = 0; v < NV; ++v) w[v] = raw_of<W>(wp + col(v), wp ? a.N - col(v) : 0);
  oct dw[SUMS ? NV : 1], db[SUMS ? NV : 1];
#pragma unroll
  for (int v = 0; v < (SUMS ? NV : 1); ++v) dw[v] = db[v] = oct{};
  const float n = static_cast<float>(a.N);
  for (int it = 0; row < a.M; row += step, it ^= 1) {
    const float mean = nmean, rstd = nrstd;
    raw8<T> x[NV], y[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      x[v] = nx[v];
      y[v] = ny[v];
    }
    // g and h of an octet
    auto both = [&](int v, oct* g, oct* h) __attribute__((always_inline)) {
      const oct xv = open8<T>(x[v]), yv = open8<T>(y[v]), wv = open_or<W>(wp, w[v], 1.0f);
      *h = oct{(xv.a - mean) * rstd, (xv.b - mean) * rstd};
      *g = oct{yv.a * wv.a, yv.b * wv.b};
    };
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      oct g, h;
      both(v, &g, &h);
      if constexpr (SUMS) {
        const oct yv = open8<T>(y[v]);
        dw[v].a += yv.a * h.a;
        dw[v].b += yv.b * h.b;
        db[v].a += yv.a;
        db[v].b += yv.b;
      }
      s1 += sum8(g);
      s2 += sum8(oct{g.a * h.a, g.b * h.b});
    }
    load(row + step);
    if (!a.dX) continue;
    raw8<T> r[NV];
    if (a.R) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
        r[v] = raw_of<T>(static_cast<const T*>(a.R) + row * a.ldr + col(v), a.N - col(v));
    }
    s1 = wave_sum(s1);
    s2 = wave_sum(s2);
    if constexpr (TH > 64) {
      float(*mine)[16] = box[it];
      if ((threadIdx.x & 63) == 0) {
        mine[0][threadIdx.x >> 6] = s1;
        mine[1][threadIdx.x >> 6] = s2;
      }
      __syncthreads();
      s1 = s2 = 0.0f;
#pragma unroll
      for (int i = 0; i < TH / 64; ++i) {
        s1 += mine[0][i];
        s2 += mine[1][i];
      }
    }
    const float m1 = s1 / n, m2 = s2 / n;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      oct g, h;
      both(v, &g, &h);
      oct d{(g.a - m1 - h.a * m2) * rstd, (g.b - m1 - h.b * m2) * rstd};
      if (a.R) {
        const oct q = open8<T>(r[v]);
        d.a += q.a;
        d.b += q.b;
      }
      const int64_t left = a.N - col(v);
      if (left > 0) store8n(static_cast<T*>(a.dX) + row * a.lddx + col(v), d, left);
    }
  }
  if constexpr (SUMS) {
    float* out = part + static_cast<int64_t>(block) * 2 * a.N;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        oct s = k == 0 ? dw[v] : db[v];
        if constexpr (RB > 1) {
          __syncthreads();
          join[rb][t] = s.a;
          join[rb][TH + t] = s.b;
          __syncthreads();
          if (rb > 0) continue;
#pragma unroll
          for (int i = 1; i < RB; ++i) {
            s.a += join[i][t];
            s.b += join[i][TH + t];
          }
        }
        if (a.N > col(v)) store8n(out + k * a.N + col(v), s, a.N - col(v));
      }
    }
  }
}

template <typename T, typename W, int TH, int NV, bool SUMS>
__global__ __launch_bounds__(TH < 256 ? 256 : TH) void norm_grad_kernel(const gt_norm_grad_args a, float* part) {
  grad_rows<T, W, TH, NV, SUMS>(a, part, static_cast<int>(blockIdx.x), static_cast<int>(gridDim.x));
}

// dw and db of 8·QL columns over all rows, QL of the NT threads a row.
template <typename T, int NT, int QL>
__device__ __forceinline__ void grad_columns(const gt_norm_grad_args& a, int block) {
  constexpr int C = 8 * QL, RL = NT / QL, PARTS = NT / (2 * C);
  __shared__ __align__(16) float sums[RL][2 * C + 4];   // [row lane][dw, then db, of C columns]
  __shared__ float parts[PARTS][2 * C];
  const int q = threadIdx.x % QL, rl = threadIdx.x / QL;
  const int64_t c = static_cast<int64_t>(block) * C + q * 8, left = a.N - c;
  const T* X = static_cast<const T*>(a.X) + c;
  const T* Y = static_cast<const T*>(a.dY) + c;
  oct dw{}, db{};
  auto add = [&](const raw8<T>& xr, const raw8<T>& yr, float mean, float rstd) __attribute__((always_inline)) {
    const oct x = open8<T>(xr), y = open8<T>(yr);
    dw.a += y.a * ((x.a - mean) * rstd);
    dw.b += y.b * ((x.b - mean) * rstd);
    db.a += y.a;
    db.b += y.b;
  };
  if (left >= 8) {   // U rows' loads at once; rows past the last count as zeros
    constexpr int U = 4;
    for (int64_t row = rl; row < a.M; row += U * RL) {
      raw8<T> x[U], y[U];
      float mean[U], rstd[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int64_t at = row + i * RL < a.M ? row + i * RL : a.M - 1;
        __builtin_memcpy(&x[i], X + at * a.ldx, sizeof(x[i]));
        __builtin_memcpy(&y[i], Y + at * a.lddy, sizeof(y[i]));
        mean[i] = a.mean[at];
        rstd[i] = a.rstd[at];
      }
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const bool live = row + i * RL < a.M;
        raw8<T> xs, ys;
#pragma unroll
        for (size_t k = 0; k < sizeof(xs.w) / sizeof(xs.w[0]); ++k) {
          xs.w[k] = live ? x[i].w[k] : u32x4{};
          ys.w[k] = live ? y[i].w[k] : u32x4{};
        }
        add(xs, ys, live ? mean[i] : 0.0f, live ? rstd[i] : 0.0f);
      }
    }
  } else if (left > 0) {
    for (int64_t row = rl; row < a.M; row += RL)
      add(raw_of<T>(X + row * a.ldx, left), raw_of<T>(Y + row * a.lddy, left), a.mean[row], a.rstd[row]);
  }
  f32x4* mine = reinterpret_cast<f32x4*>(&sums[rl][q * 8]);
  mine[0] = dw.a;
  mine[1] = dw.b;
  mine[C / 4] = db.a;
  mine[C / 4 + 1] = db.b;
  __syncthreads();
  const int j = threadIdx.x % (2 * C), p = threadIdx.x / (2 * C);
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < RL / PARTS; ++i) s += sums[p * (RL / PARTS) + i][j];
  parts[p][j] = s;
  __syncthreads();
  const int64_t n = static_cast<int64_t>(block) * C + j % C;
  float* out = j < C ? a.dw : a.db;
  if (p > 0 || n >= a.N || !out) return;
  s = 0.0f;
#pragma unroll
  for (int i = 0; i < PARTS; ++i) s += parts[i][j];
  out[n] = s;
}

// Few rows: their statistics are given, so that the columns' sums need not wait for the rows. The
// first `columns` workgroups take 8·QL columns each, the others rows: one launch, no scratch.
template <typename T, typename W, int TH, int NV, int QL>
__global__ __launch_bounds__(TH < 256 ? 256 : TH) void norm_grad_few_kernel(const gt_norm_grad_args a, int columns) {
  const int block = static_cast<int>(blockIdx.x);
  if (block < columns)
    grad_columns<T, TH < 256 ? 256 : TH, QL>(a, block);
  else
    grad_rows<T, W, TH, NV, false>(a, nullptr, block - columns, static_cast<int>(gridDim.x) - columns);
}

// Long rows: dX alone, read twice.
template <typename T, typename W>
__global__ __launch_bounds__(1024) void norm_grad_long_kernel(const gt_norm_grad_args a) {
  constexpr int TH = 1024;
  __shared__ float box[2][16];
  const W* wp = static_cast<const W*>(a.w);
  const float n = static_cast<float>(a.N);
  for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.X) + row * a.ldx;
    const T* y = static_cast<const T*>(a.dY) + row * a.lddy;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s1 = 0.0f, s2 = 0.0f;
    auto both = [&](int64_t c, oct* g, oct* h) __attribute__((always_inline)) {
      const int64_t left = a.N - c;
      const oct xv = open8<T>(raw_of<T>(x + c, left)), yv = open8<T>(raw_of<T>(y + c, left));
      const oct wv = open_or<W>(wp, raw_of<W>(wp + c, wp ? left : 0), 1.0f);
      *h = oct{(xv.a - mean) * rstd, (xv.b - mean) * rstd};
      *g = oct{yv.a * wv.a, yv.b * wv.b};
    };
    oct g, h;
    for (int64_t c = threadIdx.x * 8; c < a.N; c += TH * 8) {
      both(c, &g, &h);
      s1 += sum8(g);
      s2 += sum8(oct{g.a * h.a, g.b * h.b});
    }
    const float m1 = row_sum<TH>(s1, box[0]) / n, m2 = row_sum<TH>(s2, box[1]) / n;
    for (int64_t c = threadIdx.x * 8; c < a.N; c += TH * 8) {
      both(c, &g, &h);
      oct d{(g.a - m1 - h.a * m2) * rstd, (g.b - m1 - h.b * m2) * rstd};
      if (a.R) {
        const oct q = open8<T>(raw_of<T>(static_cast<const T*>(a.R) + row * a.ldr + c, a.N - c));
        d.a += q.a;
        d.b += q.b;
      }
      store8n(static_cast<T*>(a.dX) + row * a.lddx + c, d, a.N - c);
    }
  }
}

// … and the column sums: 256 threads, 512 columns of every gridDim.y-th run of 4 rows.
template <typename T>
__global__ __launch_bounds__(256) void norm_sums_kernel(const gt_norm_grad_args a, float* part) {
  __shared__ f32x4 join[4][2][64];
  const int q = threadIdx.x & 63, rb = threadIdx.x >> 6;
  const int64_t c = (int64_t{blockIdx.x} * 64 + q) * 8, left = a.N - c;
  oct dw{}, db{};
  for (int64_t row = int64_t{blockIdx.y} * 4 + rb; row < a.M; row += int64_t{gridDim.y} * 4) {
    const oct x = open8<T>(raw_of<T>(static_cast<const T*>(a.X) + row * a.ldx + c, left));
    const oct y = open8<T>(raw_of<T>(static_cast<const T*>(a.dY) + row * a.lddy + c, left));
    const float mean = a.mean[row], rstd = a.rstd[row];
    dw.a += y.a * ((x.a - mean) * rstd);
    dw.b += y.b * ((x.b - mean) * rstd);
    db.a += y.a;
    db.b += y.b;
  }
  float* out = part + int64_t{blockIdx.y} * 2 * a.N;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    oct s = k == 0 ? dw : db;
    __syncthreads();
    join[rb][0][q] = s.a;
    join[rb][1][q] = s.b;
    __syncthreads();
    if (rb > 0) continue;
#pragma unroll
    for (int i = 1; i < 4; ++i) {
      s.a += join[i][0][q];
      s.b += join[i][1][q];
    }
    if (left > 0) store8n(out + k * a.N + c, s, left);
  }
}

// out[n] = Σ of the partial rows, in order: 64 columns of dw (blockIdx.y 0) or db, a sixteenth of
// the rows a wavefront.
__global__ __launch_bounds__(1024) void norm_join_kernel(const float* part, int64_t rows, int64_t N,
                                                        float* dw, float* db) {
  __shared__ float sums[16][64];
  const int c = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float* out = blockIdx.y == 0 ? dw : db;
  if (!out) return;
  for (int64_t n = int64_t{blockIdx.x} * 64 + c; n - c < N; n += int64_t{gridDim.x} * 64) {
    float s = 0.0f;
    if (n < N) {
      const float* p = part + blockIdx.y * N + n;
#pragma unroll 8
      for (int64_t r = wave; r < rows; r += 16) s += p[r * 2 * N];
    }
    sums[wave][c] = s;
    __syncthreads();
    if (wave == 0 && n < N) {
      s = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) s += sums[i][c];
      out[n] = s;
    }
    __syncthreads();
  }
}

// ---- choices

// Threads a row, octets a thread. 0: a long row.
struct Rows {
  int threads, octets;
};
Rows rows_of(int64_t N) {
  const int64_t oct = (N + 7) / 8;
  for (const Rows r : {Rows{64, 1}, Rows{64, 2}, Rows{256, 1}, Rows{256, 2}, Rows{512, 2}, Rows{512, 4}})
    if (oct <= int64_t{r.threads} * r.octets) return r;
  return Rows{0, 0};
}
// As many workgroups as are resident at once, each with the parameters in its registers for all its
// rows (bf16 with fp32 parameters, 16384×4096: 2 a unit 53.2 µs, 4 45.4, 5 46.7, 6 50.2; 2048×16384: 1 27.1,
// 2 30.6, 4 37.4; 4096×4096 to codes: 2 20.3, 4 17.5, 5 17.2, 8 16.6).
unsigned grid_of(int64_t M, const Rows& r) {
  const int each = r.threads == 64 ? 4 : 1;
  const int a_unit = r.threads == 512 ? (r.octets == 4 ? 1 : 2) : r.octets == 2 && r.threads == 256 ? 5 : 8;
  return static_cast<unsigned>(std::min<int64_t>((M + each - 1) / each, kUnits * a_unit));
}

template <typename T, typename W, int CODE>
hipError_t norm_by(const gt_norm_args& a, hipStream_t s) {
  const Rows r = rows_of(a.N);
  if (r.threads == 0) {
    norm_long_kernel<T, W, CODE><<<static_cast<unsigned>(std::min<int64_t>(a.M, 4096)), 1024, 0, s>>>(a);
    return hipGetLastError();
  }
  const unsigned grid = grid_of(a.M, r);
  if (r.threads == 64 && r.octets == 1) norm_kernel<T, W, 64, 1, CODE><<<grid, 256, 0, s>>>(a);
  else if (r.threads == 64) norm_kernel<T, W, 64, 2, CODE><<<grid, 256, 0, s>>>(a);
  else if (r.threads == 256 && r.octets == 1) norm_kernel<T, W, 256, 1, CODE><<<grid, 256, 0, s>>>(a);
  else if (r.threads == 256) norm_kernel<T, W, 256, 2, CODE><<<grid, 256, 0, s>>>(a);
  else if (r.octets == 2) norm_kernel<T, W, 512, 2, CODE><<<grid, 512, 0, s>>>(a);
  else norm_kernel<T, W, 512, 4, CODE><<<grid, 512, 0, s>>>(a);
  return hipGetLastError();
}
template <typename T, typename W>
hipError_t norm_by_code(const gt_norm_args& a, hipStream_t s) {
  if (!a.Q) return norm_by<T, W, -1>(a, s);
  return a.code == GT_E4M3 ? norm_by<T, W, GT_E4M3>(a, s) : norm_by<T, W, GT_E5M2>(a, s);
}

// Each workgroup writes and the join reads 8·N bytes of sums (16384×4096 in bf16: 2 a unit 106 µs,
// 3 110, 4 125).
unsigned grad_grid(int64_t M, const Rows& r) {
  const int each = r.threads == 64 ? 4 : 1;
  return static_cast<unsigned>(std::min<int64_t>((M + each - 1) / each, kUnits * (r.threads >= 512 ? 1 : 2)));
}
// Rows too wide for the sums' registers beside their own: the sums by a kernel of their own, which
// reads X and dY again (2048×16384 in bf16 78 µs, 124 with spilled sums in one).
bool sums_apart(const Rows& r) { return r.threads == 0 || r.octets == 4; }
unsigned sums_parts(int64_t M) { return static_cast<unsigned>(std::min<int64_t>((M + 3) / 4, 64)); }

template <typename T, typename W, bool SUMS>
hipError_t grad_by(const gt_norm_grad_args& a, float* part, hipStream_t s) {
  const Rows r = rows_of(a.N);
  const unsigned grid = grad_grid(a.M, r);
  if (r.threads == 64 && r.octets == 1) norm_grad_kernel<T, W, 64, 1, SUMS><<<grid, 256, 0, s>>>(a, part);
  else if (r.threads == 64) norm_grad_kernel<T, W, 64, 2, SUMS><<<grid, 256, 0, s>>>(a, part);
  else if (r.threads == 256 && r.octets == 1) norm_grad_kernel<T, W, 256, 1, SUMS><<<grid, 256, 0, s>>>(a, part);
  else if (r.threads == 256) norm_grad_kernel<T, W, 256, 2, SUMS><<<grid, 256, 0, s>>>(a, part);
  else if (r.threads == 512 && r.octets == 2) norm_grad_kernel<T, W, 512, 2, SUMS><<<grid, 512, 0, s>>>(a, part);
  else if (r.threads == 512) norm_grad_kernel<T, W, 512, 4, false><<<grid, 512, 0, s>>>(a, part);
  else norm_grad_long_kernel<T, W><<<static_cast<unsigned>(std::min<int64_t>(a.M, 4096)), 1024, 0, s>>>(a);
  return hipGetLastError();
}

// The columns' own pass reads X and dY again, few columns a workgroup: faster than the sums' way
// through memory and their launch while its rows are few (with R, in a graph, two launches in
// brackets: bf16 100×4096 4.1 µs (9.3), 1000×1024 8.1 (10.3), 1000×4096 11.9 (19.4), 500×8192
// 13.1 (17.8), 1000×8192 21.2 (18.9); fp32 1000×4096 16.6 (18.4)), and a launch and an
// allocation less for the host (5 µs).
bool few_rows(int64_t M, int64_t N) { return rows_of(N).threads > 0 && M <= (N <= 4096 ? 1024 : 512); }
// Threads a row: 4 take 64 or 128 bytes of it. Unaligned accesses are slower in a unit's memory
// pipeline, for which narrow rows get more workgroups (bf16, 1000×1021 9.7 µs, with 4 threads
// 16.6; 1000×4095 31.8 and 21.0; aligned 1000×1024 9.4 and 8.1).
int column_threads(const gt_norm_grad_args& a) {
  const int64_t size = a.dtype == GT_F32 ? 4 : 2;
  const uint64_t bits = reinterpret_cast<uintptr_t>(a.X) | reinterpret_cast<uintptr_t>(a.dY) |
                        static_cast<uint64_t>(a.ldx * size) | static_cast<uint64_t>(a.lddy * size);
  return bits % 16 == 0 || a.N > 2048 ? 4 : 1;
}

template <typename T, typename W, int QL>
hipError_t few_by(const gt_norm_grad_args& a, int columns, bool rows, hipStream_t s) {
  const Rows r = rows_of(a.N);
  const unsigned grid = columns + (rows ? grad_grid(a.M, r) : 0);
  if (r.threads == 64 && r.octets == 1) norm_grad_few_kernel<T, W, 64, 1, QL><<<grid, 256, 0, s>>>(a, columns);
  else if (r.threads == 64) norm_grad_few_kernel<T, W, 64, 2, QL><<<grid, 256, 0, s>>>(a, columns);
  else if (r.threads == 256 && r.octets == 1) norm_grad_few_kernel<T, W, 256, 1, QL><<<grid, 256, 0, s>>>(a, columns);
  else if constexpr (QL == 4) {
    if (r.threads == 256) norm_grad_few_kernel<T, W, 256, 2, QL><<<grid, 256, 0, s>>>(a, columns);
    else if (r.octets == 2) norm_grad_few_kernel<T, W, 512, 2, QL><<<grid, 512, 0, s>>>(a, columns);
    else norm_grad_few_kernel<T, W, 512, 4, QL><<<grid, 512, 0, s>>>(a, columns);
  } else {
    return hipErrorInvalidValue;   // (column_threads: not above 2048 columns)
  }
  return hipGetLastError();
}
// The bytes from p on of rows ld apart, and others: do they share any?
bool apart(const void* p, int64_t ldp, const void* q, int64_t ldq, int64_t M, int64_t N, int64_t size) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return a + ((M - 1) * ldp + N) * size <= b || b + ((M - 1) * ldq + N) * size <= a;
}
template <typename T, typename W>
hipError_t few(const gt_norm_grad_args& a, hipStream_t s) {
  const int ql = column_threads(a), columns = static_cast<int>((a.N + 8 * ql - 1) / (8 * ql));
  const bool one = !a.dX || (apart(a.dX, a.lddx, a.dY, a.lddy, a.M, a.N, sizeof(T)) &&
                             apart(a.dX, a.lddx, a.X, a.ldx, a.M, a.N, sizeof(T)));
  auto go = ql == 1 ? few_by<T, W, 1> : few_by<T, W, 4>;
  const hipError_t e = go(a, columns, a.dX && one, s);
  return e != hipSuccess || one ? e : go(a, 0, true, s);   // (dX over dY: when its sums are taken)
}

template <typename T, typename W>
hipError_t grad(const gt_norm_grad_args& a, float* part, hipStream_t s) {
  hipError_t e = hipSuccess;
  if (a.M > 0 && (a.dw || a.db) && few_rows(a.M, a.N)) return few<T, W>(a, s);
  const bool own = sums_apart(rows_of(a.N));
  if (a.M > 0 && part && own) {   // (before dX, which may be dY)
    norm_sums_kernel<T><<<dim3(static_cast<unsigned>((a.N + 511) / 512), sums_parts(a.M)), 256, 0, s>>>(a, part);
    e = hipGetLastError();
  }
  if (e == hipSuccess && a.M > 0 && (a.dX || (part && !own)))
    e = part && !own ? grad_by<T, W, true>(a, part, s) : grad_by<T, W, false>(a, part, s);
  if (e != hipSuccess || (!a.dw && !a.db)) return e;
  const unsigned columns = static_cast<unsigned>(std::min<int64_t>((a.N + 63) / 64, int64_t{1} << 20));
  norm_join_kernel<<<dim3(columns, 2), 1024, 0, s>>>(part, norm_parts(a), a.N, a.dw, a.db);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(const gt_norm_args& a, hipStream_t s) {
  if (a.dtype == GT_F32) return norm_by_code<float, float>(a, s);
  return a.wtype == GT_F32 ? norm_by_code<uint16_t, float>(a, s) : norm_by_code<uint16_t, uint16_t>(a, s);
}

int64_t norm_parts(const gt_norm_grad_args& a) {
  if (a.M == 0 || (!a.dw && !a.db)) return 0;
  const Rows r = rows_of(a.N);
  if (few_rows(a.M, a.N)) return 0;
  return sums_apart(r) ? sums_parts(a.M) : grad_grid(a.M, r);
}

hipError_t launch_norm_grad(const gt_norm_grad_args& a, float* part, hipStream_t s) {
  if (a.dtype == GT_F32) return grad<float, float>(a, part, s);
  return a.wtype == GT_F32 ? grad<uint16_t, float>(a, part, s) : grad<uint16_t, uint16_t>(a, part, s);
}

}  // namespace gt
