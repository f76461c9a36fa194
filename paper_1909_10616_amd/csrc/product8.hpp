// Tiled products of 8-bit codes with the layers' fused epilogue.
//
//   O[m][n] = Σ_b sa[m][b]·sb[n][b]·Σ_{k in block b} A[m][k]·B[n][k],  blocks of 128 k.
//
// A stage of the LDS ring is a block: 128 bytes of every row of both operands and their scales.
// The block's sum of a 16×16 tile is one matrix instruction that takes codes (EXACT: four
// that take them widened to bf16, see widen8), begun at zero, and its four values a lane
// then meet the scales on the vector pipe while the next instructions run: 16 of the 32
// cycles that the instruction takes. Loads go straight into LDS as in product.hpp, whose
// descriptors, tile order and epilogue these kernels share.
//
// Bound by the matrix instructions and what they wait for at a stage's boundary: 4096×4096×4096
// in 256×256 tiles 65 … 74 µs (up to 2.1 PFLOP/s), 4096×11008×4096 200 µs (1.85), with fp32
// results in 128×128 tiles 4096×4096×4096 145 µs. 256×256 tiles read each operand's byte from
// LDS half as often as 128×128 (96 µs); fewer rows take the smaller tiles, which fill the chip.
//
// Matrix operands are given in the order (B, A): a lane holds 4 consecutive n of one row m.
#pragma once
#include <hip/hip_runtime.h>

#include <atomic>
#include <cstdint>

#include "fp8.hpp"
#include "layer8_kernels.h"
#include "product.hpp"

namespace gt {

// Raises a kernel's dynamic LDS limit, once per kernel and device (attr: where it has been).
inline hipError_t raise_lds(const void* fn, size_t lds, std::atomic<uint64_t>& attr) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = dev >= 0 && dev < 64 ? uint64_t{1} << dev : 0;
  if (bit && (attr.load(std::memory_order_acquire) & bit)) return hipSuccess;
  e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(lds));
  if (e == hipSuccess) attr.fetch_or(bit, std::memory_order_release);
  return e;
}

// 64 lanes × 4 bytes, lane j's from its address to LDS byte lds_base + 4·j.
__device__ __forceinline__ void dma_scale(const float* p, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off"
               :
               : "v"(p), "s"(uni(static_cast<int>(lds_base)))
               : "memory", "m0");
}

// UNI: the columns of a wavefront in either half of the tile share their scale.
template <int DT, bool EXACT, int AC, int BC, int TILE, int EPI, bool UNI>
__global__ __launch_bounds__(64 * tile8(TILE).NWM * tile8(TILE).NWN, 2) void product8_kernel(const Product8 q) {
  constexpr Tile8 S = tile8(TILE);
  constexpr int BM = S.BM, BN = S.BN, NWM = S.NWM, NWN = S.NWN, NW = NWM * NWN;
  constexpr int WM = BM / NWM, WN = BN / NWN, HN = WN / 2;
  constexpr int TM = WM / 16, TN = WN / 16, MF = TM * TN;
  constexpr int NA = BM / 8 / NW, NB = BN / 8 / NW;      // 1 KiB loads of a wavefront and stage
  constexpr int CNT = NA + NB + 1;                        // … and one of scales
  constexpr int FIRST = TN;                               // of them behind the boundary
  constexpr uint32_t BOFF = BM * 128, SOFF = BOFF + BN * 128, STAGE = SOFF + (BM + BN) * 4;
  static_assert(BM + BN == 64 * NW && NB % 2 == 0 && TN % 2 == 0);
  static_assert(STAGE == kStage8(TILE));
  auto kswz = [](int r) { return (r >> 1) & 7; };

  extern __shared__ char smem[];
  const ProductArgs& a = q.p;
  const int lane = threadIdx.x & 63;
  const int wave = uni(threadIdx.x >> 6);
  const int wm = wave % NWM, wn = wave / NWM;
  const int lx = lane & 15, grp = lane >> 4;

  int tm, tn;
  tile_at(static_cast<int>(blockIdx.x), a.tilesM * a.tilesN, a.tilesM, a.tilesN, tm, tn);
  const int z = static_cast<int>(blockIdx.y);
  const int64_t m0 = static_cast<int64_t>(tm) * BM;
  // whether the tile's second half holds up values, B's rows N on
  const bool halves = EPI == kEpiGated || (EPI == kEpiPart && a.e.gated != 0);
  const int64_t n0 = static_cast<int64_t>(tn) * (halves ? BN / 2 : BN);
  const int64_t n1 = halves ? a.N + n0 : n0 + BN / 2;          // B's row of the second half's first
  const int64_t end0 = a.N, end1 = halves ? 2 * a.N : a.N;     // rows of either half end here

  // ---- the stages of this K slice
  const int all = static_cast<int>((a.K + kBlock - 1) / kBlock);
  const int st0 = EPI == kEpiPart ? min(all, z * a.per_slice) : 0;
  const int st1 = EPI == kEpiPart ? min(all, st0 + a.per_slice) : all;
  const int nst = st1 - st0;
  const int64_t k0 = static_cast<int64_t>(st0) * kBlock;

  // ---- where this lane's chunks lie: load p fills rows 8p … 8p + 7, chunk c in slot c ^ kswz(r).
  // Rows that do not exist lie behind the descriptors' ends.
  const int lr = lane >> 3;   // row of the eight
  const int r0 = wave * 8 + lr, kc = ((lane & 7) ^ kswz(r0)) * 16;   // (rows 16 apart swap alike)
  const uint32_t lda = static_cast<uint32_t>(a.lda), ldb = static_cast<uint32_t>(a.ldb);
  const uint32_t offA = static_cast<uint32_t>(r0) * lda + kc, offB = static_cast<uint32_t>(r0) * ldb + kc;
  static_assert(NW % 2 == 0, "rows of a lane's chunks are 16 apart");
  // this lane's scales, of place 64·wave + lane among A's and B's: A's of a wavefront's rows lie
  // by lx, so that a lane reads its TM as quads
  const float* scale;
  {
    const int r = wave * 64 + lane, c = r - BM;
    if (r < BM) {
      const int64_t row = m0 + r / WM * WM + r % TM * 16 + r % WM / TM, m = row < a.M ? row : a.M - 1;
      scale = q.sa + (m >> q.xshift) * q.ldsa;
    } else {
      int64_t n = c < BN / 2 ? n0 + c : n1 + c - BN / 2;
      const int64_t end = c < BN / 2 ? end0 : end1;
      n = n < end ? n : end - 1;
      scale = q.sb + (n >> q.wshift) * q.ldsb;
    }
  }

  // ---- loads of the next stage
  const uint32_t lds0 = static_cast<uint32_t>(uni(static_cast<int>(lds_off(smem))));
  uint64_t ga = uniform_ptr(static_cast<const uint8_t*>(a.A) + m0 * a.lda + k0);
  uint64_t gb = uniform_ptr(static_cast<const uint8_t*>(a.B) + n0 * a.ldb + k0);
  uint64_t gc = uniform_ptr(static_cast<const uint8_t*>(a.B) + n1 * a.ldb + k0);
  int64_t left = a.K - k0;
  // (rows begin at 16-byte aligned addresses: the last one's last chunk begins inside it)
  const int64_t whole = (left + 15) / 16 * 16;
  int64_t remA = uni64((a.M - m0 - 1) * a.lda + whole);
  int64_t remB = uni64((end0 - n0 - 1) * a.ldb + whole);
  int64_t remC = uni64((end1 - n1 - 1) * a.ldb + whole);
  int kb = st0;
  i32x4 da{}, db{}, dc{};
  auto descriptors = [&]() __attribute__((always_inline)) {
    const bool live = kb < st1;
    da = descriptor(ga, live ? remA : 0);
    db = descriptor(gb, live ? remB : 0);
    dc = descriptor(gc, live ? remC : 0);
    asm volatile("s_nop 4" : "+s"(da), "+s"(db), "+s"(dc));   // (as settle)
  };
  auto next_stage = [&]() __attribute__((always_inline)) {
    ga += kBlock;
    gb += kBlock;
    gc += kBlock;
    remA -= kBlock;
    remB -= kBlock;
    remC -= kBlock;
    left -= kBlock;
    ++kb;
  };
  auto dma = [&](uint32_t base, int i) __attribute__((always_inline)) {
    if (i < NA) {
      dma_buffer16((kc < left ? offA : kOutside) + i * (8 * NW) * lda, da,
                   base + static_cast<uint32_t>(wave + NW * i) * 1024u);
    } else if (i < NA + NB) {
      const int j = i - NA;
      dma_buffer16((kc < left ? offB : kOutside) + (j % (NB / 2)) * (8 * NW) * ldb, j < NB / 2 ? db : dc,
                   base + BOFF + static_cast<uint32_t>(wave + NW * j) * 1024u);
    } else {
      dma_scale(scale + (kb < all ? kb : all - 1), base + SOFF + static_cast<uint32_t>(wave) * 256u);
    }
  };
  // K ends inside a chunk of stage all − 1: what follows in its rows is not theirs.
  const int odd = static_cast<int>(a.K & 15);
  auto trim = [&](char* st) __attribute__((always_inline)) {
    const int c = static_cast<int>(a.K - 1 - static_cast<int64_t>(all - 1) * kBlock) >> 4;
    for (int r = threadIdx.x; r < BM + BN; r += 64 * NW) {
      u32x4* p = reinterpret_cast<u32x4*>(st + r * 128 + ((c ^ kswz(r)) << 4));
      u32x4 v = *p;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int n = odd - 4 * w;   // bytes of this word that are K's
        v[w] = n >= 4 ? v[w] : n <= 0 ? 0u : v[w] & ((1u << (8 * n)) - 1u);
      }
      *p = v;
    }
    __syncthreads();
  };

  // ---- fragments
  auto bcol = [&](int j) { return (j < TN / 2 ? 0 : BN / 2) + wn * HN + (j % (TN / 2)) * 16; };
  const uint32_t sw = static_cast<uint32_t>(kswz(lx));
  const uint32_t lo = ((static_cast<uint32_t>(grp) ^ sw) << 4) + lx * 128;
  const uint32_t hi = ((static_cast<uint32_t>(grp + 4) ^ sw) << 4) + lx * 128;
  auto read = [&](const char* st, int row) __attribute__((always_inline)) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(st + lo + row * 128);
    const u32x4 y = *reinterpret_cast<const u32x4*>(st + hi + row * 128);
    return i32x8{static_cast<int>(x[0]), static_cast<int>(x[1]), static_cast<int>(x[2]), static_cast<int>(x[3]),
                 static_cast<int>(y[0]), static_cast<int>(y[1]), static_cast<int>(y[2]), static_cast<int>(y[3])};
  };
  auto read_a = [&](const char* st, int i) __attribute__((always_inline)) { return read(st, wm * WM + i * 16); };
  auto read_b = [&](const char* st, int j) __attribute__((always_inline)) { return read(st + BOFF, bcol(j)); };
  constexpr int AHEAD = !EXACT && TM >= 4 ? 2 : 1;   // rows of fragments computed behind the boundary
  constexpr int BUFS = 2 * AHEAD;
  static_assert(TM % BUFS == 0);
  i32x8 va[BUFS], vb[TN];
  // scales: A's of rows i·16 + lx, B's of the tile's halves, or of 4 columns
  float sa[TM], sh[2];
  f32x4 sb[UNI ? 1 : TN];
  auto read_sa = [&](const char* st) __attribute__((always_inline)) {
    const float* s = reinterpret_cast<const float*>(st + SOFF) + wm * WM + lx * TM;
    if constexpr (TM >= 4) {
#pragma unroll
      for (int i = 0; i < TM; i += 4) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(s + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) sa[i + k] = v[k];
      }
    } else {
#pragma unroll
      for (int i = 0; i < TM; ++i) sa[i] = s[i];
    }
  };
  auto read_sb = [&](const char* st) __attribute__((always_inline)) {
    const float* s = reinterpret_cast<const float*>(st + SOFF);
    if constexpr (UNI) {
      sh[0] = s[BM + wn * HN];
      sh[1] = s[BM + BN / 2 + wn * HN];
    } else {
#pragma unroll
      for (int j = 0; j < TN; ++j) sb[j] = *reinterpret_cast<const f32x4*>(s + BM + bcol(j) + 4 * grp);
    }
  };

  f32x4 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{};
  constexpr int LAG = UNI ? 4 : 2;   // instructions between a sum and its scaling, as registers allow
  f32x4 part[LAG + 1];
  // step t of a stage: the last AHEAD i's are taken together, column by column
  auto row_of = [&](int t) { return t < MF - AHEAD * TN ? t / TN : TM - AHEAD + t % AHEAD; };
  auto col_of = [&](int t) { return t < MF - AHEAD * TN ? t % TN : (t - (MF - AHEAD * TN)) / AHEAD; };
  auto apply = [&](int t) __attribute__((always_inline)) {
    const int i = row_of(t), j = col_of(t);
    const f32x4& p = part[t % (LAG + 1)];
    if constexpr (UNI) {
      const float s = sa[i] * sh[j < TN / 2 ? 0 : 1];
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[i][j][r] = fmaf(p[r], s, acc[i][j][r]);
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[i][j][r] = fmaf(p[r], sa[i] * sb[j][r], acc[i][j][r]);
    }
    // (here, between the matrix instructions: the compiler would put all of a stage behind the last)
    asm volatile("" : "+v"(acc[i][j]));
  };
  bf16x8 wa[EXACT ? 4 : 1], wb[EXACT ? TN : 1][4];

  if (nst > 0) {
    descriptors();
#pragma unroll
    for (int i = 0; i < CNT; ++i) dma(lds0, i);
    next_stage();
    descriptors();
#pragma unroll
    for (int i = 0; i < FIRST; ++i) dma(lds0 + STAGE, i);
    waitcnt_vm<FIRST>();
    ring_barrier();
    if (odd && st0 == all - 1) trim(smem);
#pragma unroll
    for (int j = 0; j < TN; ++j) vb[j] = read_b(smem, j);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) va[i] = read_a(smem, i);
    read_sa(smem);
    read_sb(smem);
    uint32_t cur = 0;
    for (int l = 0; l < nst; ++l) {
      const uint32_t nx = STAGE - cur;
      if constexpr (EXACT) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int c = 0; c < 4; ++c) wb[j][c] = widen8<BC>(vb[j][2 * c], vb[j][2 * c + 1]);
      }
      constexpr int EDGE = MF - AHEAD * TN;   // the first step behind the boundary
#pragma unroll
      for (int t = 0; t < MF; ++t) {
        const int i = row_of(t), j = col_of(t);
        if (t == EDGE) {
          // every wavefront has read all of stage l, and stage l + 1 has landed
          waitcnt_vm<0>();
          waitcnt_lgkm0();
          ring_barrier();
          next_stage();
          descriptors();
          if (odd && st0 + l + 1 == all - 1) trim(smem + nx);
        }
        // A's fragments AHEAD of their use (behind the boundary the next stage's first)
        if (t < EDGE) {
          if (j == 0) va[(i + AHEAD) % BUFS] = read_a(smem + cur, i + AHEAD);
        } else if (t < EDGE + AHEAD) {
          va[t - EDGE] = read_a(smem + nx, t - EDGE);
        }
        if (t >= EDGE) {
          if (t - EDGE < FIRST) dma(lds0 + cur, t - EDGE);
        } else {
#pragma unroll
          for (int k = FIRST + t; k < CNT; k += EDGE) dma(lds0 + nx, k);
        }
        if constexpr (EXACT) {
          if (j == 0) {
#pragma unroll
            for (int c = 0; c < 4; ++c) wa[c] = widen8<AC>(va[i % BUFS][2 * c], va[i % BUFS][2 * c + 1]);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (EXACT) {
          f32x4 p{};
#pragma unroll
          for (int c = 0; c < 4; ++c) p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb[j][c], wa[c], p, 0, 0, 0);
          part[t % (LAG + 1)] = p;
        } else {
          part[t % (LAG + 1)] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(vb[j], va[i % BUFS], f32x4{}, BC, AC, 0,
                                                                                0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (t >= LAG) apply(t - LAG);
        // B's column j is done with after its last row
        if (t >= EDGE && (t - EDGE) % AHEAD == AHEAD - 1) vb[j] = read_b(smem + nx, j);
      }
#pragma unroll
      for (int t = MF - LAG; t < MF; ++t) apply(t);
      read_sa(smem + nx);
      read_sb(smem + nx);
      cur = nx;
    }
    waitcnt_vm<0>();
  }

  // ---- epilogue, as product.hpp's
  constexpr int REGION = 2 * STAGE / NW;
  constexpr int XM = epilogue_xor(WN), RP = epilogue_rows(WM, WN, REGION, 16);
  static_assert(RP >= 16 && WM % RP == 0 && REGION % 16 == 0, "epilogue rows");
  __syncthreads();
  char* mine = smem + wave * REGION;
  const EpiPlace place{m0 + wm * WM, a.M, n0 + wn * HN, 0, z, tm * NWM + wm, tn * NWN + wn};
  EpiSums sums[2] = {};
#pragma unroll
  for (int h = 0; h < WM / RP; ++h) {
#pragma unroll
    for (int i = 0; i < RP / 16; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int r = i * 16 + lx, c = j * 4 + grp;
        *reinterpret_cast<f32x4*>(mine + r * (WN * 4) + ((c ^ (r & XM)) << 4)) = acc[h * (RP / 16) + i][j];
      }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    EpiRows<DT, EPI, WM, WN, XM, RP, BN>{a, place, h * RP, mine, lane}.run(sums);
    __builtin_amdgcn_wave_barrier();
  }
}

}  // namespace gt
