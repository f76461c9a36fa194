// Tiled products of any extents with a fused epilogue, the kernels behind the
// layer operators (linear, experts and their gradients).
//
//   O[m][n] = Σ_k A(m, k)·B(k, n),  then the epilogue of O's rows.
//
// Each operand is stored along k ([x][k] rows, "KC") or along its own index
// ([k][x] rows, "XC"): X·W reads KC·XC, dP·Wᵀ KC·KC, Xᵀ·dP XC·XC, so no operand
// is ever transposed in memory. Rows may be grouped (the experts' rows, one
// after the other): along m, every group with its own B; or along k, every
// group with its own output.
//
// Tiles come through LDS in stages of 128 bytes along k (64 bf16, 32 fp32), in
// a ring of NS slots. DMA: 16-byte global→LDS loads whose buffer descriptor
// ends where the operand does, so that what lies outside (rows past the last,
// k past the end) arrives as zero. REG (operands that are not 16-byte aligned
// row by row): the same chunks through registers, checked one by one.
//
// MFMA operands are given in the order (B, A): a lane then holds 4 consecutive n
// of one row m. The epilogue turns the accumulators through LDS so that
// a wavefront reads and writes whole row segments.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "gemm_kernel.hpp"
#include "layer_math.hpp"
#include "product_args.h"

namespace gt {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// ---- helpers ---------------------------------------------------------------

__device__ __forceinline__ int uni(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uni64(int64_t v) {
  return static_cast<int64_t>(
      static_cast<uint64_t>(static_cast<uint32_t>(uni(static_cast<int>(v)))) |
      (static_cast<uint64_t>(static_cast<uint32_t>(uni(static_cast<int>(v >> 32)))) << 32));
}

// Offsets beyond any descriptor's length: such a lane reads zero.
constexpr uint32_t kOutside = 0x80000000u;
// Bytes one descriptor reaches (below kOutside).
constexpr int64_t kReach = 0x7fffff00;

// Raw buffer descriptor of [b, b + bytes), both uniform: loads beyond it return zero.
__device__ __forceinline__ i32x4 descriptor(uint64_t b, int64_t bytes) {
  const int64_t n = bytes < 0 ? 0 : bytes > kReach ? kReach : bytes;
  i32x4 d;
  d[0] = static_cast<int>(b);
  d[1] = static_cast<int>((b >> 32) & 0xffffu);
  d[2] = static_cast<int>(n);
  d[3] = 0x00020000;
  return d;
}

// 64 lanes × 16 bytes: lane j's from byte off of the descriptor's memory to LDS
// byte lds_base + 16·j. (The wait state between the write of m0 and the load is the
// s_nop; the compiler counts neither the load nor its LDS writes, the ring does.)
__device__ __forceinline__ void dma_buffer16(uint32_t off, i32x4 d, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
               :
               : "v"(off), "s"(d), "s"(uni(static_cast<int>(lds_base)))
               : "memory", "m0");
}

// The five wait states between a vector instruction's write of a scalar and a
// memory instruction that reads it, which the compiler does not count into an
// assembly statement: once for both descriptors, which are then only read.
__device__ __forceinline__ void settle(i32x4& a, i32x4& b) {
  asm volatile("s_nop 4" : "+s"(a), "+s"(b));
}

// A group and its rows (or k).
struct Span {
  int group;      // −1: none
  int64_t lo, hi;
};

__device__ __forceinline__ int64_t offset_at(const ProductArgs& a, int g, int64_t most) {
  const int64_t v = a.offsets[g];
  return v < 0 ? 0 : v > most ? most : v;
}

// The groups' tiles of BM rows: up to 64 groups a lane each, loaded once; more, 64 at a time.
template <int BM>
struct GroupTiles {
  const ProductArgs& a;
  int lo, hi, mine, upto;   // of group g0 + lane: its rows, its tiles, the tiles up to its last
  __device__ __forceinline__ explicit GroupTiles(const ProductArgs& args) : a(args) { load(0); }
  __device__ __forceinline__ void load(int g0) {
    const int g = g0 + (threadIdx.x & 63);
    lo = hi = 0;
    if (g < a.groups) {
      lo = static_cast<int>(offset_at(a, g, a.M));
      hi = static_cast<int>(offset_at(a, g + 1, a.M));
    }
    mine = hi > lo ? (hi - lo + BM - 1) / BM : 0;
    upto = wave_prefix(mine);
  }
  // All groups' tiles.
  __device__ __forceinline__ int total() {
    int n = __builtin_amdgcn_readlane(upto, 63);
    if (a.groups > 64) {
      for (int g0 = 64; g0 < a.groups; g0 += 64) {
        load(g0);
        n += __builtin_amdgcn_readlane(upto, 63);
      }
      load(0);
    }
    return n;
  }
  // The group that holds tile t, counted over all groups, and the tile's first row.
  __device__ __forceinline__ Span find(int t, int64_t* first) {
    int before = 0;
    for (int g0 = 0;;) {
      const uint64_t past = __ballot(before + upto > t);
      if (past != 0) {
        const int at = __builtin_ctzll(past);
        const int l = __builtin_amdgcn_readlane(lo, at), h = __builtin_amdgcn_readlane(hi, at);
        const int tile = t - before - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(mine, at));
        *first = l + static_cast<int64_t>(tile) * BM;
        return Span{g0 + at, l, h};
      }
      before += __builtin_amdgcn_readlane(upto, 63);
      g0 += 64;
      if (g0 >= a.groups) break;
      load(g0);
    }
    *first = 0;
    return Span{-1, 0, 0};
  }
};

// Tile t of `tiles` (rows × tilesN) → its row and column: every XCD gets a run of tiles, in
// groups of 4 tile rows.
__device__ __forceinline__ void tile_at(int t, int tiles, int rows, int tilesN, int& tm, int& tn) {
  const int q = tiles >> 3, r = tiles & 7, x = t & 7;
  t = x * q + min(x, r) + (t >> 3);
  constexpr int ROWS = 4;
  const int per = ROWS * tilesN, run = t / per, f = run * ROWS, gs = min(rows - f, ROWS);
  const int in = t - run * per;
  tm = f + in % gs;
  tn = in / gs;
}

// XOR of the 16-byte chunk index of an XC row k in LDS. bf16: the transposing
// read's rows (bswz); fp32: the 64/I lane groups of a 4-byte read, 4 rows apart, go to
// distinct parts of 256 bytes.
template <int DT, int I>
__device__ __forceinline__ int xswz(int k, int chunks) {
  if constexpr (DT == 1)
    return bswz(k, chunks);
  else
    return (I == 16 ? ((k >> 2) & 3) << 2 : ((k >> 2) & 1) << 3) & (chunks - 1);
}

// ---- epilogue --------------------------------------------------------------

// 4 outputs of a row from their sums v (and u, the up values, when gated): the
// bias (bv, bu), the activation and the residual r, every step in fp32.
template <typename T>
__device__ __forceinline__ void linear_quad(const Epilogue& e, int64_t N, int64_t row, int64_t n,
                                            int group, int left, bool gated, f32x4 v, f32x4 u,
                                            f32x4 bv, f32x4 bu, f32x4 r) {
  v += bv;
  u += bu;
  if (e.P) {
    T* p = static_cast<T*>(e.P) + row * e.ldp + n;
    store4(p, v, left);
    if (gated) store4(p + N, u, left);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = act_value<T>(e.act, v[i]);
  if (gated) v *= u;
  v += r;
  const int64_t at = group * e.sY + row * e.ldy + n;
  const bool pad = e.zero_pad != 0;   // rows of whole aligned quads
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = i < left ? v[i] : 0.0f;
  if (e.out_f32)
    store4(static_cast<float*>(e.Y) + at, v, pad ? 4 : left);
  else
    store4(static_cast<T*>(e.Y) + at, v, pad ? 4 : left);
}
// Columns that an epilogue writes: N, or up to the next 16 bytes.
template <typename T>
__device__ __forceinline__ int64_t written(const Epilogue& e, int64_t N) {
  constexpr int64_t VEC = 16 / sizeof(T);
  return e.zero_pad ? (N + VEC - 1) / VEC * VEC : N;
}
template <typename T>
__device__ __forceinline__ f32x4 bias_quad(const Epilogue& e, int64_t n, int group, int left) {
  return e.bias ? load4(static_cast<const T*>(e.bias) + group * e.sbias + n, left) : f32x4{};
}
template <typename T>
__device__ __forceinline__ f32x4 residual_quad(const Epilogue& e, int64_t row, int64_t n, int left) {
  return e.R ? load4(static_cast<const T*>(e.R) + row * e.ldr + n, left) : f32x4{};
}

// A quad of a K slice's sums (gated: and the up values') to its place in `part`. A quad
// that only pads a row has none: a half of a row of `part` ends with N's last quad, and the
// launch that joins the slices writes the padding itself.
template <bool G>
__host__ __device__ __forceinline__ void part_quad(const ProductArgs& a, int slice, int64_t row,
                                                   int64_t col, f32x4 v, f32x4 u) {
  if (col >= a.N) return;
  float* part = a.e.part + (static_cast<int64_t>(slice) * a.M + row) * a.e.ldpart + col;
  *reinterpret_cast<f32x4*>(part) = v;
  if constexpr (G) *reinterpret_cast<f32x4*>(part + a.e.ldpart / 2) = u;
}

// Where a wavefront's tile lies.
struct EpiPlace {
  int64_t row, row_end;  // its first row, and the first row that is not the group's
  int64_t col;           // its first column; its second half is BN/2 further on (gated: the up values)
  int group, slice;
  int prow, pcol;        // its tile row and column among all wavefronts'
};

struct EpiSums {
  f32x4 g, u;  // a lane's columns of dP, summed over its rows
};

// Rows that the epilogue turns at a time, a wavefront having `region` bytes of LDS for them.
constexpr int epilogue_rows(int WM, int WN, int region, int I) {
  const int fit = region / (WN * 4) / I * I, rows = fit < WM ? fit : WM;
  return rows < 64 ? rows : 64;
}
// XOR of the 16-byte chunks of such a row r: r & this.
constexpr int epilogue_xor(int WN) { return (WN / 4 < 16 ? WN / 4 : 16) - 1; }

// RP rows of a wavefront's tile of WM×WN, row h + r of it in LDS at mine + r·WN·4.
template <int DT, int EPI, int WM, int WN, int XM, int RP, int BN>
struct EpiRows {
  using T = typename Elem<DT>::T;
  static constexpr int CH = WN / 4;
  static constexpr bool G = EPI == kEpiGated;
  const ProductArgs& a;
  const EpiPlace& p;
  int h;
  const char* mine;
  int lane;

  __host__ __device__ __forceinline__ f32x4 chunk(int r, int c) const {
    return *reinterpret_cast<const f32x4*>(mine + r * (WN * 4) + ((c ^ (r & XM)) << 4));
  }
  // the column of chunk c (gated: of the gate's)
  __host__ __device__ __forceinline__ int64_t col(int c) const {
    return p.col + (G || c < CH / 2 ? 0 : BN / 2 - WN / 2) + c * 4;
  }

  // Whether the slope epilogue takes octets: columns that all exist.
  __device__ static __forceinline__ bool whole_slope(const ProductArgs& a, const EpiPlace& p) {
    return p.col + BN / 2 + WN / 2 <= a.N;
  }

  // A whole tile: 16-byte accesses, at any alignment, nothing checked.
  // The residuals of U rows are loaded before the first of them is stored (an output may
  // be the residual itself) and while the U rows before them are worked on.
  template <int ACT>
  __host__ __device__ __forceinline__ void whole() const {
    const Epilogue& e = a.e;
    constexpr int LR = (G ? CH / 2 : CH) / 2;   // lanes a row
    constexpr int STEP = 64 / LR;
    constexpr int U = EPI == kEpiPlain ? 1 : RP / STEP >= 4 ? 4 : RP / STEP >= 1 ? RP / STEP : 1;
    const int c = lane % LR * 2, first = lane / LR;
    if (STEP > RP && first >= RP) return;   // (32 gated columns: 32 rows a step, of 16)
    const int64_t n = col(c), row0 = p.row + h + first;
    oct bv{}, bu{};
    const T* R = nullptr;
    T* P = nullptr;
    if constexpr (EPI != kEpiPlain) {
      if (e.bias) {
        const T* b = static_cast<const T*>(e.bias) + p.group * e.sbias + n;
        bv = load8(b);
        if constexpr (G) bu = load8(b + a.N);
      }
      if (e.R) R = static_cast<const T*>(e.R) + row0 * e.ldr + n;
      if (e.P) P = static_cast<T*>(e.P) + row0 * e.ldp + n;
    }
    char* Y = static_cast<char*>(e.Y) + (p.group * e.sY + row0 * e.ldy + n) * (e.out_f32 ? 4 : sizeof(T));
    const int64_t ystep = STEP * e.ldy * (e.out_f32 ? 4 : sizeof(T));
    oct res[U], next[U];
    if (R) {
#pragma unroll
      for (int i = 0; i < U; ++i) next[i] = load8(R + i * STEP * e.ldr);
    }
#pragma unroll 1
    for (int r0 = first; r0 < RP; r0 += U * STEP) {
      if (R) {
#pragma unroll
        for (int i = 0; i < U; ++i) res[i] = next[i];
        R += U * STEP * e.ldr;
        if (r0 + U * STEP < RP) {
#pragma unroll
          for (int i = 0; i < U; ++i) next[i] = load8(R + i * STEP * e.ldr);
        }
      }
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int r = r0 + i * STEP;
        oct v{chunk(r, c) + bv.a, chunk(r, c + 1) + bv.b};
        oct u{};
        if constexpr (G) u = oct{chunk(r, c + CH / 2) + bu.a, chunk(r, c + CH / 2 + 1) + bu.b};
        if (P) {
          store8(P, v);
          if constexpr (G) store8(P + a.N, u);
          P += STEP * e.ldp;
        }
        if constexpr (ACT != GT_ACT_NONE) act8<T, ACT>(v);
        if constexpr (G) {
          v.a *= u.a;
          v.b *= u.b;
        }
        if (R) {
          v.a += res[i].a;
          v.b += res[i].b;
        }
        if (e.out_f32)
          store8(reinterpret_cast<float*>(Y), v);
        else
          store8(reinterpret_cast<T*>(Y), v);
        Y += ystep;
      }
    }
  }

  // Any tile: a quad a lane, every row checked.
  __device__ __forceinline__ void edge() const {
    constexpr int LR = G ? CH / 2 : CH;
    constexpr int STEP = 64 / LR;
    constexpr int U = RP / STEP >= 2 ? 2 : 1;
    const int c = lane % LR;
    const int64_t n = col(c);
    const int left = a.N - n < 4 ? static_cast<int>(a.N - n) : 4;
    if (n >= written<T>(a.e, a.N)) return;
    const f32x4 bv = bias_quad<T>(a.e, n, p.group, left);
    const f32x4 bu = G ? bias_quad<T>(a.e, n + a.N, p.group, left) : f32x4{};
#pragma unroll 1
    for (int r0 = lane / LR; r0 < RP; r0 += U * STEP) {
      f32x4 res[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int64_t row = p.row + h + r0 + i * STEP;
        res[i] = row < p.row_end ? residual_quad<T>(a.e, row, n, left) : f32x4{};
      }
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int r = r0 + i * STEP;
        const int64_t row = p.row + h + r;
        if (row < p.row_end)
          linear_quad<T>(a.e, a.N, row, n, p.group, left, G, chunk(r, c),
                         G ? chunk(r, c + CH / 2) : f32x4{}, bv, bu, res[i]);
      }
    }
  }

  __device__ __forceinline__ void part() const {
    const Epilogue& e = a.e;
    const int c = lane % CH;
    const bool up = e.gated && c >= CH / 2;
    const int64_t n = up ? p.col + (c - CH / 2) * 4 : e.gated ? p.col + c * 4 : col(c);
    if (n >= a.N) return;
    float* out = e.part + (static_cast<int64_t>(p.slice) * a.M + p.row + h) * e.ldpart + n +
                 (up ? e.ldpart / 2 : 0);
#pragma unroll 1
    for (int r = lane / CH; r < RP; r += 64 / CH)
      if (p.row + h + r < p.row_end) *reinterpret_cast<f32x4*>(out + r * e.ldpart) = chunk(r, c);
  }

  // The rows as they are into a tile of BN columns (out: its place of the first).
  __device__ __forceinline__ void tail(float* out) const {
    const int c = lane % CH, n = (c < CH / 2 ? 0 : BN / 2 - WN / 2) + c * 4;
#pragma unroll 1
    for (int r = lane / CH; r < RP; r += 64 / CH)
      *reinterpret_cast<f32x4*>(out + r * BN + n) = chunk(r, c);
  }

  // The weight of one row of RP in each lane.
  __device__ __forceinline__ float row_weight() const {
    static_assert(RP <= 64, "a row's weight in each lane");
    const Epilogue& e = a.e;
    if (lane >= RP || p.row + h + lane >= p.row_end) return 0.0f;
    const int64_t entry = e.order[p.row + h + lane];
    return entry >= 0 && entry < e.entries ? e.weights[entry] : 0.0f;
  }

  // dH arrived: H = act(P) (times up), w the row's weight;
  // dP = w·dH·act'(P) (gated: ·up, and w·dH·act(gate) for up), Hw = w·H, both stored in the
  // operands' type, which the next products' matrix instructions take; Σ dH·H and the column
  // sums are of the values before that. Octets of columns that
  // all exist, the pre-activations of U rows loaded while the U rows before them are
  // worked on. (16384 rows of 1024 × 1024, gated, bf16: 104 µs; 114 with U = 1, 141 with 4,
  // which leaves one wavefront a SIMD, 122 with the rows' loads not ahead.)
  template <int ACT>
  __device__ __forceinline__ void slope_whole(EpiSums* sums) const {
    const Epilogue& e = a.e;
    constexpr int LR = CH / 2, STEP = 64 / LR, U = RP / STEP >= 2 ? 2 : 1;
    const int c = lane % LR * 2, first = lane / LR;
    const int64_t n = col(c), row0 = p.row + h + first;
    const int64_t rows = p.row_end - row0;   // of this lane's first on
    const T* P = static_cast<const T*>(e.P) + row0 * e.ldp + n;
    T* out = static_cast<T*>(e.Y) + row0 * e.ldy + n;
    T* hout = static_cast<T*>(e.Hw) + row0 * e.ldh + n;
    float* dots = e.dot + row0 * e.ldot + p.pcol;
    raw8<T> gate[U], up[U];
    auto load = [&](int at) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int r = at + i * STEP;
        gate[i] = raw8<T>{};
        up[i] = raw8<T>{};
        if (r < RP && r < rows) {
          __builtin_memcpy(&gate[i], P + r * e.ldp, sizeof(gate[i]));
          if (e.gated) __builtin_memcpy(&up[i], P + r * e.ldp + a.N, sizeof(up[i]));
        }
      }
    };
    load(0);
    const float mine_w = row_weight();
#pragma unroll 1
    for (int at = 0; at < RP; at += U * STEP) {
      oct g[U], u[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        g[i] = open8<T>(gate[i]);
        u[i] = e.gated ? open8<T>(up[i]) : oct{f32x4{1.0f, 1.0f, 1.0f, 1.0f}, f32x4{1.0f, 1.0f, 1.0f, 1.0f}};
      }
      load(at + U * STEP);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int r = at + i * STEP;
        const float w = __shfl(mine_w, first + r);
        const bool live = r < rows;
        float dot = 0.0f;
        oct dg, du, hw;
        auto quad = [&](const f32x4& v, const f32x4& gq, const f32x4& uq, f32x4& dgq, f32x4& duq,
                        f32x4& hwq, EpiSums& sum) __attribute__((always_inline)) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float val, sl;
            act_both<T>(ACT, gq[j], &val, &sl);
            const float wv = w * v[j], H = val * uq[j];
            dot += live ? v[j] * H : 0.0f;
            dgq[j] = live ? wv * uq[j] * sl : 0.0f;
            duq[j] = live ? wv * val : 0.0f;
            hwq[j] = w * H;
          }
          sum.g += dgq;
          sum.u += duq;
        };
        quad(chunk(first + r, c), g[i].a, u[i].a, dg.a, du.a, hw.a, sums[0]);
        quad(chunk(first + r, c + 1), g[i].b, u[i].b, dg.b, du.b, hw.b, sums[1]);
        if (live) {
          store8(out + r * e.ldy, dg);
          if (e.gated) store8(out + r * e.ldy + a.N, du);
          store8(hout + r * e.ldh, hw);
        }
#pragma unroll
        for (int d = 1; d < LR; d <<= 1) dot += __shfl_xor(dot, d);
        if (c == 0 && live) dots[r * e.ldot] = dot;
      }
    }
  }

  // The same a quad a lane, every column checked; U rows at a time with their
  // pre-activations loaded first.
  __device__ __forceinline__ void slope(EpiSums* sums) const {
    const Epilogue& e = a.e;
    constexpr int LR = CH, STEP = 64 / LR, U = RP / STEP >= 2 ? 2 : 1;
    const int c = lane % LR;
    const int64_t n = col(c);
    const int left = a.N - n < 4 ? static_cast<int>(a.N - n) : 4;
    const float mine_w = row_weight();
#pragma unroll 1
    for (int r0 = lane / LR; r0 < RP; r0 += U * STEP) {
      f32x4 gate[U], up[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int64_t row = p.row + h + r0 + i * STEP;
        const T* pp = static_cast<const T*>(e.P) + row * e.ldp + n;
        gate[i] = f32x4{};
        up[i] = f32x4{1.0f, 1.0f, 1.0f, 1.0f};
        if (row >= p.row_end || left <= 0) continue;
        gate[i] = load4(pp, left);
        if (e.gated) up[i] = load4(pp + a.N, left);
      }
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int r = r0 + i * STEP;
        const int64_t row = p.row + h + r;
        const float w = __shfl(mine_w, r);
        const bool live = row < p.row_end && left > 0;
        float dot = 0.0f;
        f32x4 dg, du, hw;
        const f32x4 v = chunk(r, c);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float val, sl;
          act_both<T>(e.act, gate[i][j], &val, &sl);
          const float wv = w * v[j], H = val * up[i][j];
          const bool in = live && j < left;
          dot += in ? v[j] * H : 0.0f;
          dg[j] = in ? wv * up[i][j] * sl : 0.0f;
          du[j] = in ? wv * val : 0.0f;
          hw[j] = in ? w * H : 0.0f;
        }
        sums[0].g += dg;
        sums[0].u += du;
        if (row < p.row_end && n < written<T>(e, a.N)) {
          T* out = static_cast<T*>(e.Y) + row * e.ldy + n;
          // (rows padded with zeros: dP's end with the up half when gated)
          store4(out, dg, e.gated ? left : e.zero_pad ? 4 : left);
          if (e.gated) {
            store4(out + a.N, du, left);
            constexpr int64_t VEC = 16 / sizeof(T);
            const int64_t pad = (2 * a.N + VEC - 1) / VEC * VEC - 2 * a.N;
            if (e.zero_pad && left > 0 && n + left == a.N)
              for (int64_t z = 0; z < pad; ++z) (out + a.N)[left + z] = T(0);
          }
          store4(static_cast<T*>(e.Hw) + row * e.ldh + n, hw, left);
        }
#pragma unroll
        for (int d = 1; d < LR; d <<= 1) dot += __shfl_xor(dot, d);
        if (c == 0 && row < p.row_end) e.dot[row * e.ldot + p.pcol] = dot;
      }
    }
  }

  __device__ __forceinline__ void run(EpiSums* sums) const {
    const Epilogue& e = a.e;
    if constexpr (EPI == kEpiPart) {
      part();
    } else if constexpr (EPI == kEpiSlope) {
      if (!whole_slope(a, p))
        slope(sums);
      else if (e.act == GT_ACT_SILU)
        slope_whole<GT_ACT_SILU>(sums);
      else if (e.act == GT_ACT_GELU)
        slope_whole<GT_ACT_GELU>(sums);
      else if (e.act == GT_ACT_RELU)
        slope_whole<GT_ACT_RELU>(sums);
      else
        slope_whole<GT_ACT_NONE>(sums);
    } else {
      const bool all = p.row + WM <= p.row_end &&
                       p.col + (G ? WN / 2 : BN / 2 + WN / 2) <= a.N;
      if (!all)
        edge();
      else if (EPI == kEpiPlain || e.act == GT_ACT_NONE)
        whole<GT_ACT_NONE>();
      else if (e.act == GT_ACT_SILU)
        whole<GT_ACT_SILU>();
      else if (e.act == GT_ACT_GELU)
        whole<GT_ACT_GELU>();
      else
        whole<GT_ACT_RELU>();
    }
  }
};

// The column sums of a wavefront's rows, joined over its lanes (octets: of Q quads
// a lane, as the rows were).
template <int WN, int BN, int Q>
__device__ __forceinline__ void epilogue_sums(const ProductArgs& a, const EpiPlace& p, int lane,
                                              EpiSums* s) {
  constexpr int CH = WN / 4, LR = CH / Q;
  const int c = lane % LR * Q;
  const int64_t n = p.col + (c < CH / 2 ? 0 : BN / 2 - WN / 2) + c * 4;
  float* out = a.e.colsum + p.prow * a.e.wide + n;
#pragma unroll
  for (int q = 0; q < Q; ++q) {
#pragma unroll
    for (int d = LR; d < 64; d <<= 1)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[q].g[i] += __shfl_xor(s[q].g[i], d);
        s[q].u[i] += __shfl_xor(s[q].u[i], d);
      }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (lane < LR && n + 4 * q + i < a.N) {
        out[4 * q + i] = s[q].g[i];
        if (a.e.gated) out[a.N + 4 * q + i] = s[q].u[i];
      }
  }
}

// ---- the kernel ------------------------------------------------------------

// Bound by the matrix pipes and the clock they leave where the tiles fill the chip (bf16,
// 256×256: 4096×4096×4096 116 µs, 1,180 TFLOP/s, either gradient; 4096×11008×4096
// with bias, GELU and kept pre-activations 338; the pipes work 72 and 65 % of the units' time, at
// 1.9 and 1.7 GHz), by the operands' way into LDS in smaller
// tiles, and by the launch, its first loads and its epilogue (5 to 8 µs) where K is short.
// 8 wavefronts of 128×64 in the large tile took 135 → 115 µs against 4 of 128×128, whose
// 256 accumulators left the other registers no room.
template <int DT, int I, bool AX, bool BX, int BM, int BN, int NWM, int NWN, int KB, int NS, bool REG, int EPI>
__global__ __launch_bounds__(64 * NWM * NWN) void product_kernel(const ProductArgs a) {
  using T = typename Elem<DT>::T;
  constexpr int SZ = DT == 1 ? 2 : 4;
  constexpr int VEC = 16 / SZ;
  constexpr int BK = KB / SZ;            // k of a stage, KB bytes of it
  constexpr int CPK = KB / 16;           // 16-byte chunks of a KC row
  constexpr int NW = NWM * NWN;
  constexpr int WM = BM / NWM, WN = BN / NWN;
  constexpr int TM = WM / I, TN = WN / I;
  constexpr int HN = WN / 2;             // a wavefront's columns in each half of the tile
  constexpr int G = 64 / I;              // lane groups: 16-byte chunks of k a chunk-step
  constexpr int NCS = CPK / G;           // chunk-steps of a stage
  using acc_t = typename AccT<I>::type;
  static_assert(TM >= 1 && TN >= 2 && TN % 2 == 0, "tile too small for its wavefronts");
  static_assert(!REG || NS == 2, "the register path has two slots");
  static_assert((CPK == 8 || CPK == 4) && NCS >= 2, "stage depth");
  constexpr int INA = BM * CPK / 64, INB = BN * CPK / 64;   // 1 KiB load instructions of a stage
  constexpr int NA = (INA + NW - 1) / NW, NB = (INB + NW - 1) / NW;  // of a wavefront
  static_assert(NW % 2 == 0, "chunks of a lane");
  static_assert(INA % NW == 0 || NW % INA == 0, "loads of A");
  static_assert(INB % NW == 0 || NW % INB == 0, "loads of B");
  constexpr uint32_t KBu = KB;
  constexpr uint32_t STAGE = (BM + BN) * KBu;
  constexpr uint32_t BOFF = BM * KBu;         // B inside a slot
  // XOR of a KC row's chunks: the 16 rows of a fragment read lie in distinct 16-byte
  // banks of 256 bytes
  auto kswz = [](int r) { return CPK == 8 ? (r >> 1) & 7 : (r >> 2) & 3; };

  extern __shared__ char smem[];
  const int lane = threadIdx.x & 63;
  const int wave = uni(threadIdx.x >> 6);
  const int wm = wave % NWM, wn = wave / NWM;
  const int lI = lane % I, grp = lane / I;

  // ---- which tile: XCD-contiguous runs, in groups of 4 tile rows. With groups along m the
  // launch has tiles for every way the rows may be spread; those past the last row's
  // end here, and the others are dealt out to the XCDs without them.
  int tm, tn;
  constexpr bool TAILS = BM >= 128 && !REG && (EPI == kEpiPlain || EPI == kEpiLinear || EPI == kEpiGated);
  int slice = 0, slices = 1, tail_at = -1;   // of the last tiles
  int64_t m0, mend = a.M;
  int group = 0;
  {
    const bool grouped = a.groups > 0 && !a.along_k;
    GroupTiles<BM> tiles(a);
    int t = static_cast<int>(blockIdx.x), rows = a.tilesM;
    if (grouped) rows = min(rows, tiles.total());
    const int nt = rows * a.tilesN;
    if (TAILS && a.tail) {
      const Tail tail = tail_of(nt, static_cast<int>((a.K + BK - 1) / BK));
      if (tail.slices > 1 && t >= tail.full) {
        const int i = t - tail.full;
        if (i >= tail.left * tail.slices) return;
        slice = i / tail.left;
        slices = tail.slices;
        tail_at = (i % tail.left) * slices + slice;
        t = tail.full + i % tail.left;
      }
    }
    if (t >= nt) return;
    tile_at(t, nt, rows, a.tilesN, tm, tn);
    m0 = static_cast<int64_t>(tm) * BM;
    if (grouped) {
      const Span s = tiles.find(tm, &m0);
      group = s.group;
      mend = s.hi;
    }
  }
  const int z = static_cast<int>(blockIdx.y);
  int64_t k0 = 0, kend = a.K;   // reduction range in stored coordinates
  if (a.groups > 0 && a.along_k) {
    group = static_cast<int>(blockIdx.z);
    k0 = uni64(offset_at(a, group, a.K));
    kend = uni64(offset_at(a, group + 1, a.K));
    if (kend < k0) kend = k0;
  }
  // whether the tile's second half holds up values, B's columns N on
  const bool halves = EPI == kEpiGated || (EPI == kEpiPart && BX && !AX && a.e.gated != 0);
  const int64_t wide = halves ? a.half + a.N : a.N;   // B's columns
  const int64_t n0 = static_cast<int64_t>(tn) * (halves ? BN / 2 : BN);
  // stored column of tile column c is n0 + c, plus this for the second half
  const int64_t hoff = halves ? a.half - BN / 2 : 0;

  const T* Ag = static_cast<const T*>(a.A);
  const T* Bg = static_cast<const T*>(a.B) + (a.along_k ? 0 : group * a.sB);

  // ---- the stages of this K slice
  int st0, st1;
  {
    const int all = uni(static_cast<int>((kend - k0 + BK - 1) / BK));
    st0 = EPI == kEpiPart ? min(all, z * a.per_slice) : 0;
    st1 = EPI == kEpiPart ? min(all, st0 + a.per_slice) : all;
    if constexpr (TAILS) {
      if (slices > 1) {
        st0 = all * slice / slices;
        st1 = all * (slice + 1) / slices;
      }
    }
  }
  const int nst = st1 - st0;
  k0 += static_cast<int64_t>(st0) * BK;
  if (k0 + static_cast<int64_t>(nst) * BK < kend) kend = k0 + static_cast<int64_t>(nst) * BK;

  // ---- where each of this lane's chunks of a stage lies
  // Load instruction p fills the slots 64·p + lane of its operand's part. KC: CPK
  // chunks a row r, chunk c in slot c ^ kswz(r). XC: rows k of chunks of x, chunk c in
  // slot c ^ xswz(k).
  constexpr int CA = BM / VEC, CB = BN / VEC;   // chunks of an XC row
  uint32_t offA[NA], offB[NB];
  const T* ptrA[REG ? NA : 1];
  const T* ptrB[REG ? NB : 1];
  int limA[REG ? NA : 1], limB[REG ? NB : 1];   // elements from the pointer that are the operand's
  int kA[NA], kB[NB];                           // k of the chunk inside the stage
  const int64_t arem = a.gather ? a.a_rows : mend - m0;
#pragma unroll
  for (int i = 0; i < NA; ++i) {
    const int s = (((wave + NW * i) % INA) << 6) + lane;
    if constexpr (!AX) {
      const int r = s / CPK, c = (s % CPK) ^ kswz(r);
      kA[i] = c * VEC;
      int64_t row = r;
      bool ok = m0 + r < mend;
      if (a.gather) {
        const int at = ok ? a.gather[m0 + r] : -1;
        row = at < 0 ? 0 : at / a.gather_div;
        ok = at >= 0 && row < a.a_rows;
      }
      if constexpr (REG) {
        ptrA[i] = Ag + (a.gather ? row : m0 + (ok ? row : 0)) * a.lda + k0 + kA[i];
        limA[i] = ok ? 1 : 0;
      } else {
        offA[i] = ok ? static_cast<uint32_t>(row) * static_cast<uint32_t>(a.lda * SZ) + c * 16u : kOutside;
      }
    } else {
      const int k = s / CA, c = (s % CA) ^ xswz<DT, I>(k, CA);
      kA[i] = k;
      if constexpr (REG) {
        ptrA[i] = Ag + (k0 + k) * a.lda + m0 + c * VEC;
        const int64_t lim = mend - (m0 + c * VEC);
        limA[i] = lim > VEC ? VEC : static_cast<int>(lim);
      } else {
        offA[i] = static_cast<uint32_t>(k) * static_cast<uint32_t>(a.lda * SZ) + c * 16u;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    const int s = (((wave + NW * i) % INB) << 6) + lane;
    if constexpr (!BX) {
      const int r = s / CPK, c = (s % CPK) ^ kswz(r);
      kB[i] = c * VEC;
      const bool ok = n0 + r < wide;
      if constexpr (REG) {
        ptrB[i] = Bg + (ok ? n0 + r : 0) * a.ldb + k0 + kB[i];
        limB[i] = ok ? 1 : 0;
      } else {
        offB[i] = ok ? static_cast<uint32_t>(r) * static_cast<uint32_t>(a.ldb * SZ) + c * 16u : kOutside;
      }
    } else {
      const int k = s / CB, c = (s % CB) ^ xswz<DT, I>(k, CB);
      const bool second = c * VEC >= BN / 2;
      const int64_t col = n0 + c * VEC + (second ? hoff : 0);
      const int64_t end = halves && !second ? a.N : wide;
      kB[i] = k;
      if constexpr (REG) {
        ptrB[i] = Bg + (k0 + k) * a.ldb + col;
        const int64_t lim = end - col;
        limB[i] = lim > VEC ? VEC : static_cast<int>(lim);
      } else {
        offB[i] = static_cast<uint32_t>(k) * static_cast<uint32_t>(a.ldb * SZ) +
                  static_cast<uint32_t>((col - n0) * SZ);
        if (col >= end) offB[i] = kOutside;
      }
    }
  }

  const uint32_t lds0 = static_cast<uint32_t>(uni(static_cast<int>(lds_off(smem))));
  u32x4 regA[REG ? NA : 1], regB[REG ? NB : 1];

  // DMA: the next stage to load, as the operands' addresses at its first k, the bytes from
  // there to each operand's last element, and the k left.
  uint64_t ga = 0, gb = 0;
  int64_t remA = 0, remB = 0, left = kend - k0;
  const int64_t stepA = (AX ? BK * a.lda : BK) * SZ, stepB = (BX ? BK * a.ldb : BK) * SZ;
  i32x4 da{}, db{};
  int here = 0;   // k left, at most a stage's
  if constexpr (!REG) {
    ga = uniform_ptr(AX ? Ag + k0 * a.lda + m0 : Ag + (a.gather ? 0 : m0 * a.lda) + k0);
    gb = uniform_ptr(BX ? Bg + k0 * a.ldb + n0 : Bg + n0 * a.ldb + k0);
    // (rows end on whole chunks: what pads an operand's last one is its own)
    auto whole = [](int64_t v) { return (v + VEC - 1) / VEC * VEC; };
    remA = uni64((AX ? (left - 1) * a.lda + whole(mend) - m0 : (arem - 1) * a.lda + whole(left)) * SZ);
    remB = uni64((BX ? (left - 1) * a.ldb + whole(wide) - n0 : (wide - n0 - 1) * a.ldb + whole(left)) * SZ);
  }
  auto next_stage = [&]() __attribute__((always_inline)) {
    ga += stepA;
    gb += stepB;
    remA -= stepA;
    remB -= stepB;
    left -= BK;
  };
  // (A stage past the last reads nothing: its descriptors are empty.)
  auto descriptors = [&]() __attribute__((always_inline)) {
    da = descriptor(ga, left > 0 ? remA : 0);
    db = descriptor(gb, left > 0 ? remB : 0);
    settle(da, db);
    here = left < BK ? static_cast<int>(left) : BK;
  };
  // Load instruction i of the stage (A's, then B's) into the slot at LDS address `base`.
  // KC rows that end inside the stage are zero beyond.
  auto dma = [&](uint32_t base, int i) __attribute__((always_inline)) {
    // (a KC chunk has the same k in all of a lane's instructions: NW is even)
    if (i < NA) {
      const uint32_t off = !AX && kA[0] >= here ? kOutside : offA[i];
      dma_buffer16(off, da, base + static_cast<uint32_t>((wave + NW * i) % INA) * 1024u);
    } else {
      const int j = i - NA;
      const uint32_t off = !BX && kB[0] >= here ? kOutside : offB[j];
      dma_buffer16(off, db, base + BOFF + static_cast<uint32_t>((wave + NW * j) % INB) * 1024u);
    }
  };
  // REG: stage st (from this slice's first) into registers.
  auto issue = [&](int st) __attribute__((always_inline)) {
    if constexpr (REG) {
      const int64_t kk = static_cast<int64_t>(st) * BK;       // from k0
      const int64_t rest = left - kk;                         // k left
#pragma unroll
      for (int i = 0; i < NA; ++i) {
        const T* p = ptrA[i] + (AX ? kk * a.lda : kk);
        const int64_t n = AX ? (kA[i] < rest ? limA[i] : 0) : (limA[i] ? rest - kA[i] : 0);
        regA[i] = load_chunk<T, VEC>(p, n);
      }
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const T* p = ptrB[i] + (BX ? kk * a.ldb : kk);
        const int64_t n = BX ? (kB[i] < rest ? limB[i] : 0) : (limB[i] ? rest - kB[i] : 0);
        regB[i] = load_chunk<T, VEC>(p, n);
      }
    }
  };
  // REG: the loaded stage into its slot.
  auto commit = [&](int slot) __attribute__((always_inline)) {
    if constexpr (REG) {
      char* base = smem + slot * STAGE;
#pragma unroll
      for (int i = 0; i < NA; ++i)
        *reinterpret_cast<u32x4*>(base + ((wave + NW * i) % INA) * 1024 + lane * 16) = regA[i];
#pragma unroll
      for (int i = 0; i < NB; ++i)
        *reinterpret_cast<u32x4*>(base + BOFF + ((wave + NW * i) % INB) * 1024 + lane * 16) = regB[i];
    }
  };

  // ---- fragments: I rows (columns) × 16 bytes of k a lane, chunk-step cs at k chunks cs·G …
  // tile column of fragment j: half j / (TN/2) of the tile
  auto bcol = [&](int j) { return (j < TN / 2 ? 0 : BN / 2) + wn * HN + (j % (TN / 2)) * I; };
  const uint32_t sw = static_cast<uint32_t>(kswz(lI));
  uint32_t fa[AX ? TM : NCS], fb[BX ? TN : NCS];
  // XC bf16: in a group of 16 lanes, lane i addresses row i >> 2, columns 4·(i & 3)
  const int i16 = lane & 15, g16 = lane >> 4;
  const int krow = DT == 1 ? 8 * grp + (i16 >> 2) : 4 * grp;
  const int kcol = DT == 1 ? (I == 32 ? 16 * (g16 & 1) : 0) + 4 * (i16 & 3) : lI;
  if constexpr (AX) {
#pragma unroll
    for (int t = 0; t < TM; ++t) {
      const int x = wm * WM + t * I + kcol;
      fa[t] = krow * (BM * SZ) + ((x / VEC) ^ xswz<DT, I>(krow, CA)) * 16 + (x % VEC) * SZ;
    }
  } else {
#pragma unroll
    for (int c = 0; c < NCS; ++c)
      fa[c] = (wm * WM + lI) * KBu + ((static_cast<uint32_t>(grp + c * G) ^ sw) << 4);
  }
  if constexpr (BX) {
#pragma unroll
    for (int t = 0; t < TN; ++t) {
      const int x = bcol(t) + kcol;
      fb[t] = BOFF + krow * (BN * SZ) + ((x / VEC) ^ xswz<DT, I>(krow, CB)) * 16 + (x % VEC) * SZ;
    }
  } else {
#pragma unroll
    for (int c = 0; c < NCS; ++c)
      fb[c] = BOFF + (wn * HN + lI) * KBu + ((static_cast<uint32_t>(grp + c * G) ^ sw) << 4);
  }
  auto read_x = [&](const char* st, uint32_t at, int cs, int rowb) __attribute__((always_inline)) {
    u32x4 v;
    if constexpr (DT == 1) {
      s16x4 h[2];
#pragma unroll
      for (int hh = 0; hh < 2; ++hh)
        h[hh] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)(st + at + (cs * G * 8 + 4 * hh) * rowb));
      v = __builtin_bit_cast(u32x4, __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        v[q] = *reinterpret_cast<const unsigned*>(st + at + (cs * G * 4 + q) * rowb);
    }
    return v;
  };
  u32x4 va[2][TM], vb[2][TN];
  // Fragment r of chunk-step cs (B's, then A's) of the slot at st.
  auto frag = [&](const char* st, int cs, int set, int r) __attribute__((always_inline)) {
    if (r < TN) {
      if constexpr (BX)
        vb[set][r] = read_x(st, fb[r], cs, BN * SZ);
      else
        vb[set][r] = *reinterpret_cast<const u32x4*>(st + fb[cs] + (bcol(r) - wn * HN) * KB);
    } else {
      const int t = r - TN;
      if constexpr (AX)
        va[set][t] = read_x(st, fa[t], cs, BM * SZ);
      else
        va[set][t] = *reinterpret_cast<const u32x4*>(st + fa[cs] + t * (I * KB));
    }
  };

  acc_t acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = acc_t{};
  constexpr int CNT = NA + NB;                          // loads of a wavefront and stage
  constexpr int FIRST = CNT / 2;                        // of them in the first window
  constexpr int FR = TM + TN;                           // fragments of a chunk-step
  constexpr int MF = (DT == 1 ? 1 : 4) * TM * TN;       // MFMAs of a chunk-step
  auto mfma1 = [&](int set, int q) __attribute__((always_inline)) {
    const int x = DT == 1 ? 0 : q / (TM * TN), i = q % (TM * TN) / TN, j = q % TN;
    if constexpr (DT == 1)
      acc[i][j] = mfma_bf16(__builtin_bit_cast(bf16x8, vb[set][j]),
                            __builtin_bit_cast(bf16x8, va[set][i]), acc[i][j]);
    else
      acc[i][j] = mfma_f32(__builtin_bit_cast(f32x4, vb[set][j])[x],
                           __builtin_bit_cast(f32x4, va[set][i])[x], acc[i][j]);
  };
  // The MFMAs of one chunk-step (fragments `set`) with, between them, the reads of the other
  // set (chunk-step cs of the slot at st) and loads LO … HI − 1 of a stage into
  // the slot at `base`. A wavefront that waits for room in the memory pipeline issues
  // no MFMAs, so both go out a few at a time.
  auto chunk_step = [&](int set, const char* st, int cs, uint32_t base, auto lo, auto hi)
      __attribute__((always_inline)) {
    constexpr int LO = decltype(lo)::value, HI = REG ? LO : decltype(hi)::value;
    constexpr int SPAN = MF >= 16 ? MF * 3 / 4 : MF >= 4 ? MF / 2 : 1;
#pragma unroll
    for (int q = 0; q < MF; ++q) {
#pragma unroll
      for (int r = 0; r < FR; ++r)
        if (r * SPAN / FR == q) frag(st, cs, set ^ 1, r);
      if constexpr (HI > LO) {
#pragma unroll
        for (int i = LO; i < HI; ++i)
          if ((i - LO) * SPAN / (HI - LO) == q) dma(base, i);
      }
      __builtin_amdgcn_sched_barrier(0);
      mfma1(set, q);
    }
  };
  using i0 = std::integral_constant<int, 0>;
  using iF = std::integral_constant<int, FIRST>;
  using iC = std::integral_constant<int, CNT>;

  // ---- the ring. Boundary of stage l, before its last chunk-step: stage l + 1 has
  // landed and every wavefront has read all of stage l, whose slot stage l + NS takes:
  // its first loads in that chunk-step, the others in the first of stage l + 1.
  // One loop for all stages (stages past the last are loaded as nothing, and their
  // fragments are not used): with loops of their own for the last ones the
  // compiler moves 256 accumulators about between them, or spills them.
  if (nst > 0) {
    if constexpr (REG) {
      issue(0);
      commit(0);
      issue(1);
      __syncthreads();
    } else {
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        descriptors();
#pragma unroll
        for (int i = 0; i < (s == NS - 1 ? FIRST : CNT); ++i) dma(lds0 + s * STAGE, i);
        if (s < NS - 1) next_stage();
      }
      waitcnt_vm<(NS - 2) * CNT + FIRST>();
      ring_barrier();
    }
#pragma unroll
    for (int r = 0; r < FR; ++r) frag(smem, 0, 0, r);
    uint32_t cur = 0;   // byte offset of the stage's slot
    for (int l = 0; l < nst; ++l) {
      const uint32_t nx = cur + STAGE == NS * STAGE ? 0 : cur + STAGE;
      const uint32_t before = cur == 0 ? (NS - 1) * STAGE : cur - STAGE;
      chunk_step(0, smem + cur, 1, lds0 + before, iF{}, iC{});
#pragma unroll
      for (int c = 1; c + 1 < NCS; ++c) chunk_step(c & 1, smem + cur, c + 1, 0, i0{}, i0{});
      if constexpr (REG) {
        commit(nx / STAGE);
        __syncthreads();
        issue(l + 2);
      } else {
        next_stage();
        descriptors();
        waitcnt_vm<(NS - 2) * CNT>();
        waitcnt_lgkm0();
        ring_barrier();
      }
      chunk_step((NCS - 1) & 1, smem + nx, 0, lds0 + cur, i0{}, iF{});
      cur = nx;
    }
    waitcnt_vm<0>();
  }

  // ---- epilogue: the wavefront's accumulators through its own share of LDS, RP
  // rows at a time, 16-byte chunks XOR-ed by the row.
  constexpr int REGION = NS * STAGE / NW;
  constexpr int XM = epilogue_xor(WN), RP = epilogue_rows(WM, WN, REGION, I);
  static_assert(RP >= I && WM % RP == 0, "epilogue rows");
  __syncthreads();
  char* mine = smem + wave * REGION;
  const EpiPlace place{m0 + wm * WM, mend, n0 + wn * HN, group, z,
                       tm * NWM + wm, tn * NWN + wn};
  EpiSums sums[2] = {};
#pragma unroll
  for (int h = 0; h < WM / RP; ++h) {
#pragma unroll
    for (int i = 0; i < RP / I; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < AccT<I>::N / 4; ++q) {
          // accumulators 4q … 4q + 3: columns j·I + 8q + 4·grp … (I = 16: 4·grp …) of row lI
          const int r = i * I + lI, c = (j * I + 8 * q) / 4 + grp;
          const acc_t& v = acc[h * (RP / I) + i][j];
          *reinterpret_cast<f32x4*>(mine + r * (WN * 4) + ((c ^ (r & XM)) << 4)) =
              f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
        }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    const EpiRows<DT, EPI, WM, WN, XM, RP, BN> rows{a, place, h * RP, mine, lane};
    if constexpr (TAILS) {
      if (tail_at >= 0)
        rows.tail(a.tail + static_cast<int64_t>(tail_at) * BM * BN + (wm * WM + h * RP) * BN + wn * HN);
      else
        rows.run(sums);
    } else {
      rows.run(sums);
    }
    __builtin_amdgcn_wave_barrier();
  }
  if constexpr (EPI == kEpiSlope) {
    if (a.e.colsum) {
      if (EpiRows<DT, EPI, WM, WN, XM, RP, BN>::whole_slope(a, place))
        epilogue_sums<WN, BN, 2>(a, place, lane, sums);
      else
        epilogue_sums<WN, BN, 1>(a, place, lane, sums);
    }
  }
}

}  // namespace gt
