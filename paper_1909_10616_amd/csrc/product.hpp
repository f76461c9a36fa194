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

// Raw buffer descriptor of [base, base + bytes): loads beyond it return zero.
__device__ __forceinline__ i32x4 descriptor(const void* base, int64_t bytes) {
  const uint64_t b = uniform_ptr(base);
  const int64_t n = bytes < 0 ? 0 : bytes > kReach ? kReach : bytes;
  i32x4 d;
  d[0] = static_cast<int>(b);
  d[1] = static_cast<int>((b >> 32) & 0xffffu);
  d[2] = uni(static_cast<int>(n));
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

// The group whose tiles of BM rows hold tile row t, counted over all groups, and
// *first, the first row of that tile. One wavefront-wide prefix sum per 64 groups.
template <int BM>
__device__ __forceinline__ Span group_of_tile(const ProductArgs& a, int t, int64_t* first) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int g0 = 0; g0 < a.groups; g0 += 64) {
    const int g = g0 + lane;
    int lo = 0, hi = 0;
    if (g < a.groups) {
      lo = static_cast<int>(offset_at(a, g, a.M));
      hi = static_cast<int>(offset_at(a, g + 1, a.M));
    }
    const int mine = hi > lo ? (hi - lo + BM - 1) / BM : 0;
    int upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(upto, d);
      if (lane >= d) upto += o;
    }
    const uint64_t past = __ballot(before + upto > t);
    if (past != 0) {
      const int at = __builtin_ctzll(past);
      const int l = __shfl(lo, at), h = __shfl(hi, at);
      const int tile = t - before - (__shfl(upto, at) - __shfl(mine, at));
      *first = uni(l) + static_cast<int64_t>(uni(tile)) * BM;
      return Span{uni(g0 + at), uni(l), uni(h)};
    }
    before += __shfl(upto, 63);
  }
  *first = 0;
  return Span{-1, 0, 0};
}

// XOR of the 16-byte chunk index of an XC row k in LDS. bf16: the transposing
// read's rows (bswz); fp32: the lane groups of a 4-byte read, 4 rows apart, go to the
// four 64-byte quarters of 256 bytes.
template <int DT>
__device__ __forceinline__ int xswz(int k, int chunks) {
  if constexpr (DT == 1)
    return bswz(k, chunks);
  else
    return (((k >> 2) & 3) << 2) & (chunks - 1);
}

// ---- epilogue --------------------------------------------------------------

// 4 outputs of a row from their sums v (and u, the up values, when gated): the
// bias, the activation and the residual, every step in fp32.
template <typename T>
__device__ __forceinline__ void linear_quad(const Epilogue& e, int64_t N, int64_t row, int64_t n,
                                            int group, f32x4 v, f32x4 u) {
  const bool vec = e.vec != 0;
  const int left = N - n < 4 ? static_cast<int>(N - n) : 4;
  if (e.bias) {
    const T* b = static_cast<const T*>(e.bias) + group * e.sbias + n;
    v += load4(b, left, vec);
    if (e.gated) u += load4(b + N, left, vec);
  }
  if (e.P) {
    T* p = static_cast<T*>(e.P) + row * e.ldp + n;
    store4(p, v, left, vec);
    if (e.gated) store4(p + N, u, left, vec);
  }
  if (e.act != GT_ACT_NONE) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = act_value(e.act, v[i]);
  }
  if (e.gated) v *= u;
  if (e.R) v += load4(static_cast<const T*>(e.R) + row * e.ldr + n, left, vec);
  const int64_t at = group * e.sY + row * e.ldy + n;
  if (e.out_f32)
    store4(static_cast<float*>(e.Y) + at, v, left, vec);
  else
    store4(static_cast<T*>(e.Y) + at, v, left, vec);
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

// RP rows of a wavefront's tile, row h + r of it in LDS at mine + r·WN·4.
template <int DT, int WN, int XM, int RP, int BN>
__device__ __forceinline__ void epilogue_rows(const ProductArgs& a, const EpiPlace& p, int h,
                                              const char* mine, int lane, EpiSums& sums) {
  using T = typename Elem<DT>::T;
  const Epilogue& e = a.e;
  constexpr int CH = WN / 4;
  auto chunk = [&](int r, int c) {
    return *reinterpret_cast<const f32x4*>(mine + r * (WN * 4) + ((c ^ (r & XM)) << 4));
  };
  // the column of chunk c (not gated)
  auto col = [&](int c) { return p.col + (c < CH / 2 ? 0 : BN / 2 - WN / 2) + c * 4; };
  if (e.mode == kEpiPart) {
    const int c = lane % CH;
    const bool up = e.gated && c >= CH / 2;
    const int64_t n = up ? p.col + (c - CH / 2) * 4 : e.gated ? p.col + c * 4 : col(c);
    float* const base = e.part + static_cast<int64_t>(p.slice) * a.M * e.ldpart + n +
                        (up ? e.ldpart / 2 : 0);
    for (int r = lane / CH; r < RP; r += 64 / CH) {
      const int64_t row = p.row + h + r;
      if (row < p.row_end && n < a.N) *reinterpret_cast<f32x4*>(base + row * e.ldpart) = chunk(r, c);
    }
  } else if (e.mode == kEpiLinear) {
    if (e.gated) {
      const int c = lane % (CH / 2);
      const int64_t n = p.col + c * 4;
      for (int r = lane / (CH / 2); r < RP; r += 128 / CH) {
        const int64_t row = p.row + h + r;
        if (row < p.row_end && n < a.N)
          linear_quad<T>(e, a.N, row, n, p.group, chunk(r, c), chunk(r, c + CH / 2));
      }
    } else {
      const int c = lane % CH;
      const int64_t n = col(c);
      for (int r = lane / CH; r < RP; r += 64 / CH) {
        const int64_t row = p.row + h + r;
        if (row < p.row_end && n < a.N)
          linear_quad<T>(e, a.N, row, n, p.group, chunk(r, c), f32x4{});
      }
    }
  } else {
    // dH arrived: H = act(P) (times up), w the row's weight;
    // dP = w·dH·act'(P) (gated: ·up, and w·dH·act(gate) for up), Hw = w·H
    const int c = lane % CH;
    const int64_t n = col(c);
    const int left = a.N - n < 4 ? static_cast<int>(a.N - n) : 4;
    const bool vec = e.vec != 0;
    for (int r = lane / CH; r < RP; r += 64 / CH) {
      const int64_t row = p.row + h + r;
      const bool live = row < p.row_end && left > 0;
      float dot = 0.0f;
      if (live) {
        const f32x4 v = chunk(r, c);
        const int64_t entry = e.order[row];
        const float w = entry >= 0 && entry < e.entries ? e.weights[entry] : 0.0f;
        const T* pp = static_cast<const T*>(e.P) + row * e.ldp + n;
        const f32x4 gate = load4(pp, left, vec);
        f32x4 up = f32x4{1.0f, 1.0f, 1.0f, 1.0f};
        if (e.gated) up = load4(pp + a.N, left, vec);
        f32x4 val, slope;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x, y;
          act_both(e.act, gate[i], &x, &y);
          val[i] = x;
          slope[i] = y;
        }
        const f32x4 wv = v * w, H = val * up;
#pragma unroll
        for (int i = 0; i < 4; ++i) dot += i < left ? v[i] * H[i] : 0.0f;
        const f32x4 dg = wv * up * slope;
        T* out = static_cast<T*>(e.Y) + row * e.ldy + n;
        store4(out, dg, left, vec);
        sums.g += dg;
        if (e.gated) {
          const f32x4 du = wv * val;
          store4(out + a.N, du, left, vec);
          sums.u += du;
        }
        store4(static_cast<T*>(e.Hw) + row * e.ldh + n, H * w, left, vec);
      }
#pragma unroll
      for (int d = 1; d < CH; d <<= 1) dot += __shfl_xor(dot, d);
      if (c == 0 && row < p.row_end) e.dot[row * e.ldot + p.pcol] = dot;
    }
  }
}

// The column sums of a wavefront's rows, joined over its lanes.
template <int WN, int BN>
__device__ __forceinline__ void epilogue_sums(const ProductArgs& a, const EpiPlace& p, int lane,
                                              EpiSums& s) {
  constexpr int CH = WN / 4;
#pragma unroll
  for (int d = CH; d < 64; d <<= 1)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s.g[i] += __shfl_xor(s.g[i], d);
      s.u[i] += __shfl_xor(s.u[i], d);
    }
  const int c = lane % CH;
  const int64_t n = p.col + (c < CH / 2 ? 0 : BN / 2 - WN / 2) + c * 4;
  if (lane >= CH) return;
  float* out = a.e.colsum + p.prow * a.e.wide + n;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (n + i < a.N) {
      out[i] = s.g[i];
      if (a.e.gated) out[a.N + i] = s.u[i];
    }
}

// ---- the kernel ------------------------------------------------------------

// Measured (bf16, one MI355X): see the instances' list in product_inst.hip.
template <int DT, bool AX, bool BX, int BM, int BN, int NWM, int NWN, int NS, bool REG>
__global__ __launch_bounds__(64 * NWM * NWN) void product_kernel(const ProductArgs a) {
  using T = typename Elem<DT>::T;
  constexpr int SZ = DT == 1 ? 2 : 4;
  constexpr int VEC = 16 / SZ;
  constexpr int BK = 128 / SZ;           // k of a stage
  constexpr int NW = NWM * NWN;
  constexpr int WM = BM / NWM, WN = BN / NWN;
  constexpr int TM = WM / 16, TN = WN / 16;
  constexpr int HN = WN / 2;             // a wavefront's columns in each half of the tile
  static_assert(TM >= 1 && TN >= 2 && TN % 2 == 0, "tile too small for its wavefronts");
  static_assert(!REG || NS == 2, "the register path has two slots");
  constexpr int INA = BM / 8, INB = BN / 8;   // 1 KiB load instructions of a stage
  constexpr int NA = (INA + NW - 1) / NW, NB = (INB + NW - 1) / NW;  // of a wavefront
  static_assert(INA % NW == 0 || NW % INA == 0, "loads of A");
  static_assert(INB % NW == 0 || NW % INB == 0, "loads of B");
  constexpr uint32_t STAGE = (BM + BN) * 128u;
  constexpr uint32_t BOFF = BM * 128u;        // B inside a slot

  extern __shared__ char smem[];
  const int lane = threadIdx.x & 63;
  const int wave = uni(threadIdx.x >> 6);
  const int wm = wave % NWM, wn = wave / NWM;
  const int l16 = lane & 15, g4 = lane >> 4;

  // ---- which tile: XCD-contiguous runs, in groups of 4 tile rows
  int tm, tn;
  {
    const int nt = a.tilesM * a.tilesN;
    int t = static_cast<int>(blockIdx.x);
    const int q = nt >> 3, r = nt & 7, x = t & 7;
    t = x * q + min(x, r) + (t >> 3);
    constexpr int G = 4;
    const int per = G * a.tilesN, grp = t / per, f = grp * G, gs = min(a.tilesM - f, G);
    const int in = t - grp * per;
    tm = f + in % gs;
    tn = in / gs;
  }
  const int z = static_cast<int>(blockIdx.y);
  int64_t m0 = static_cast<int64_t>(tm) * BM, mend = a.M;
  int64_t k0 = 0, kend = a.K;   // reduction range in stored coordinates
  int group = 0;
  if (a.groups > 0) {
    if (a.along_k) {
      group = static_cast<int>(blockIdx.z);
      k0 = uni64(offset_at(a, group, a.K));
      kend = uni64(offset_at(a, group + 1, a.K));
      if (kend < k0) kend = k0;
    } else {
      const Span s = group_of_tile<BM>(a, tm, &m0);
      if (s.group < 0) return;
      group = s.group;
      mend = s.hi;
    }
  }
  const bool gated = a.e.gated != 0;
  const int64_t wide = (gated && a.e.mode != kEpiSlope) ? 2 * a.N : a.N;  // B's columns
  const bool halves = wide != a.N;
  const int64_t n0 = static_cast<int64_t>(tn) * (halves ? BN / 2 : BN);
  // stored column of tile column c is n0 + c, plus this for the second half
  const int64_t hoff = halves ? a.N - BN / 2 : 0;

  const T* Ag = static_cast<const T*>(a.A);
  const T* Bg = static_cast<const T*>(a.B) + (a.along_k ? 0 : group * a.sB);

  // ---- the stages of this K slice
  int st0, st1;
  {
    const int64_t all = (kend - k0 + BK - 1) / BK;
    st0 = uni(static_cast<int>(all * z / a.splits));
    st1 = uni(static_cast<int>(all * (z + 1) / a.splits));
  }
  const int nst = st1 - st0;
  k0 += static_cast<int64_t>(st0) * BK;

  // ---- where each of this lane's chunks of a stage lies
  // Load instruction p fills the slots 64·p + lane of its operand's part. KC: 8
  // chunks a row r, chunk c in slot c ^ ((r >> 1) & 7), so that the 16 rows of a
  // fragment read lie in distinct 16-byte banks of 256 bytes. XC: rows k of
  // chunks of x, chunk c in slot c ^ xswz(k).
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
      const int r = s >> 3, c = (s & 7) ^ ((r >> 1) & 7);
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
      const int k = s / CA, c = (s % CA) ^ xswz<DT>(k, CA);
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
      const int r = s >> 3, c = (s & 7) ^ ((r >> 1) & 7);
      kB[i] = c * VEC;
      const bool ok = n0 + r < wide;
      if constexpr (REG) {
        ptrB[i] = Bg + (ok ? n0 + r : 0) * a.ldb + k0 + kB[i];
        limB[i] = ok ? 1 : 0;
      } else {
        offB[i] = ok ? static_cast<uint32_t>(r) * static_cast<uint32_t>(a.ldb * SZ) + c * 16u : kOutside;
      }
    } else {
      const int k = s / CB, c = (s % CB) ^ xswz<DT>(k, CB);
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

  // Stage st (from this slice's first) towards slot `slot`.
  auto issue = [&](int st, int slot) __attribute__((always_inline)) {
    const int64_t kk = static_cast<int64_t>(st) * BK;       // from k0
    const int64_t left = kend - k0 - kk;                    // k left, > 0
    if constexpr (REG) {
#pragma unroll
      for (int i = 0; i < NA; ++i) {
        const T* p = ptrA[i] + (AX ? kk * a.lda : kk);
        const int64_t n = AX ? (kA[i] < left ? limA[i] : 0) : (limA[i] ? left - kA[i] : 0);
        regA[i] = load_chunk<T, VEC>(p, n);
      }
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const T* p = ptrB[i] + (BX ? kk * a.ldb : kk);
        const int64_t n = BX ? (kB[i] < left ? limB[i] : 0) : (limB[i] ? left - kB[i] : 0);
        regB[i] = load_chunk<T, VEC>(p, n);
      }
    } else {
      // from the stage's origin to the operand's last element
      const T* ga = AX ? Ag + (k0 + kk) * a.lda + m0 : Ag + (a.gather ? 0 : m0 * a.lda) + k0 + kk;
      const T* gb = BX ? Bg + (k0 + kk) * a.ldb + n0 : Bg + n0 * a.ldb + k0 + kk;
      i32x4 da = descriptor(ga, (AX ? (left - 1) * a.lda + mend - m0 : (arem - 1) * a.lda + left) * SZ);
      i32x4 db = descriptor(gb, (BX ? (left - 1) * a.ldb + wide - n0 : (wide - n0 - 1) * a.ldb + left) * SZ);
      settle(da, db);
      const uint32_t base = lds0 + static_cast<uint32_t>(slot) * STAGE;
      const bool tail = left < BK;   // KC rows end inside this stage: zero beyond
#pragma unroll
      for (int i = 0; i < NA; ++i) {
        const uint32_t off = !AX && tail && kA[i] >= left ? kOutside : offA[i];
        dma_buffer16(off, da, base + static_cast<uint32_t>((wave + NW * i) % INA) * 1024u);
      }
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const uint32_t off = !BX && tail && kB[i] >= left ? kOutside : offB[i];
        dma_buffer16(off, db, base + BOFF + static_cast<uint32_t>((wave + NW * i) % INB) * 1024u);
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

  // ---- fragments: 16 rows (columns) × 16 bytes of k a lane
  // tile column of fragment j: half j / (TN/2) of the tile
  auto bcol = [&](int j) { return (j < TN / 2 ? 0 : BN / 2) + wn * HN + (j % (TN / 2)) * 16; };
  const uint32_t sw = static_cast<uint32_t>(l16 >> 1);
  uint32_t fa[AX ? TM : 2], fb[BX ? TN : 2];
  // XC bf16: in lane group g4, lane i addresses row 8·g4 + (i >> 2), columns 4·(i & 3)
  const int krow = DT == 1 ? 8 * g4 + (l16 >> 2) : 4 * g4;
  const int kcol = DT == 1 ? 4 * (l16 & 3) : l16;
  if constexpr (AX) {
#pragma unroll
    for (int t = 0; t < TM; ++t) {
      const int x = wm * WM + t * 16 + kcol;
      fa[t] = krow * (BM * SZ) + ((x / VEC) ^ xswz<DT>(krow, CA)) * 16 + (x % VEC) * SZ;
    }
  } else {
    fa[0] = (wm * WM + l16) * 128u + ((static_cast<uint32_t>(g4) ^ sw) << 4);
    fa[1] = fa[0] ^ 64u;
  }
  if constexpr (BX) {
#pragma unroll
    for (int t = 0; t < TN; ++t) {
      const int x = bcol(t) + kcol;
      fb[t] = BOFF + krow * (BN * SZ) + ((x / VEC) ^ xswz<DT>(krow, CB)) * 16 + (x % VEC) * SZ;
    }
  } else {
    fb[0] = BOFF + l16 * 128u + ((static_cast<uint32_t>(g4) ^ sw) << 4);
    fb[1] = fb[0] ^ 64u;
  }
  auto read_x = [&](const char* st, uint32_t at, int cs, int rowb) __attribute__((always_inline)) {
    u32x4 v;
    if constexpr (DT == 1) {
      s16x4 h[2];
#pragma unroll
      for (int hh = 0; hh < 2; ++hh)
        h[hh] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)(st + at + (cs * 32 + 4 * hh) * rowb));
      v = __builtin_bit_cast(u32x4, __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        v[q] = *reinterpret_cast<const unsigned*>(st + at + (cs * 16 + q) * rowb);
    }
    return v;
  };
  u32x4 va[2][TM], vb[2][TN];
  auto frags = [&](int slot, int cs, int set) __attribute__((always_inline)) {
    const char* st = smem + slot * STAGE;
#pragma unroll
    for (int t = 0; t < TN; ++t) {
      if constexpr (BX)
        vb[set][t] = read_x(st, fb[t], cs, BN * SZ);
      else
        vb[set][t] = *reinterpret_cast<const u32x4*>(st + fb[cs] + bcol(t) * 128);
    }
#pragma unroll
    for (int t = 0; t < TM; ++t) {
      if constexpr (AX)
        va[set][t] = read_x(st, fa[t], cs, BM * SZ);
      else
        va[set][t] = *reinterpret_cast<const u32x4*>(st + fa[cs] + t * 2048);
    }
  };

  f32x4 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{};
  auto mfmas = [&](int set) __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < (DT == 1 ? 1 : 4); ++q)
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          if constexpr (DT == 1)
            acc[i][j] = mfma_bf16(__builtin_bit_cast(bf16x8, vb[set][j]),
                                  __builtin_bit_cast(bf16x8, va[set][i]), acc[i][j]);
          else
            acc[i][j] = mfma_f32(__builtin_bit_cast(f32x4, vb[set][j])[q],
                                 __builtin_bit_cast(f32x4, va[set][i])[q], acc[i][j]);
        }
  };

  // ---- the ring. Boundary of stage l, before its last MFMAs: stage l + 1 has
  // landed and every wavefront has read all of stage l, whose slot stage l + NS takes.
  constexpr int CNT = NA + NB;
  if (nst > 0) {
    if constexpr (REG) {
      issue(0, 0);
      commit(0);
      if (nst > 1) issue(1, 1);
      __syncthreads();
    } else {
      const int pro = min(NS, nst);
      for (int s = 0; s < pro; ++s) issue(s, s);
      if (pro == NS)
        waitcnt_vm<(NS - 1) * CNT>();
      else
        waitcnt_vm<0>();
      ring_barrier();
    }
    frags(0, 0, 0);
    int cur = 0;
    for (int l = 0; l < nst; ++l) {
      frags(cur, 1, 1);
      mfmas(0);
      const int nx = cur + 1 == NS ? 0 : cur + 1;
      if (l + 1 < nst) {
        if constexpr (REG) {
          commit(nx);
          __syncthreads();
          if (l + 2 < nst) issue(l + 2, cur);
        } else {
          if (l + NS <= nst)
            waitcnt_vm<(NS - 2) * CNT>();
          else
            waitcnt_vm<0>();
          waitcnt_lgkm0();
          ring_barrier();
          if (l + NS < nst) issue(l + NS, cur);
        }
        frags(nx, 0, 0);
      }
      mfmas(1);
      cur = nx;
    }
  }

  // ---- epilogue: the wavefront's accumulators through its own share of LDS, RP
  // rows at a time, 16-byte chunks XOR-ed by the row.
  constexpr int REGION = NS * STAGE / NW;
  constexpr int CH = WN / 4;                       // 16-byte fp32 chunks of a row
  constexpr int XM = (CH < 16 ? CH : 16) - 1;
  constexpr int RPX = REGION / (WN * 4) / 16 * 16;
  constexpr int RP = RPX < WM ? RPX : WM;
  static_assert(RP >= 16 && WM % RP == 0, "epilogue rows");
  __syncthreads();
  char* mine = smem + wave * REGION;
  const EpiPlace place{m0 + wm * WM, mend, n0 + wn * HN, group, z,
                       tm * NWM + wm, tn * NWN + wn};
  EpiSums sums{};
#pragma unroll
  for (int h = 0; h < WM / RP; ++h) {
#pragma unroll
    for (int i = 0; i < RP / 16; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int r = i * 16 + l16, c = j * 4 + g4;
        *reinterpret_cast<f32x4*>(mine + r * (WN * 4) + ((c ^ (r & XM)) << 4)) = acc[h * (RP / 16) + i][j];
      }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    epilogue_rows<DT, WN, XM, RP, BN>(a, place, h * RP, mine, lane, sums);
    __builtin_amdgcn_wave_barrier();
  }
  if (a.e.mode == kEpiSlope && a.e.colsum) epilogue_sums<WN, BN>(a, place, lane, sums);
}

}  // namespace gt
