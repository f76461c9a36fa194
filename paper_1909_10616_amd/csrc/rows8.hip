// 8-bit products of up to 64 rows a workgroup, X·Wᵀ with the linear epilogue, codes straight from
// memory into matrix instructions: bound by W's way from memory.
//
// A workgroup takes 16, 32 or 64 rows, 16 columns (gated: 16 of each half) and all of K, its 8
// wavefronts taking turns at its blocks of 128, whose sums then take their scales. The codes are
// widened to bf16 for the matrix instructions, whose sums are then fp32's. A lane holds 32
// neighbouring k of a row, so rows of both operands are read in runs of 128 bytes, at any
// alignment. The wavefronts' sums meet in LDS and are added in their order. 1×11008×4096 takes
// 12.3 µs on the GPU, 3.7 TB/s.
#include <hip/hip_runtime.h>

#include <atomic>
#include <cstdint>

#include "fp8.hpp"
#include "layer8_kernels.h"
#include "product8.hpp"

namespace gt {
namespace {

constexpr int kWaves = 8;

// The wavefronts' sums (a lane's: row 16·i + lx, columns 4·grp …) added in their order, and the
// epilogue. lds: [wavefront][half][row][quad ^ (row & 3)].
template <typename T, bool G, int RT>
__device__ __forceinline__ void join_rows(const Product8& q, f32x4* lds, const f32x4 (&acc)[G ? 2 : 1][RT], int64_t m0,
                                          int64_t n0) {
  constexpr int H = G ? 2 : 1, ROWS = 16 * RT;
  const ProductArgs& a = q.p;
  const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6);
  const int lx = lane & 15, grp = lane >> 4;
  auto at = [&](int w, int h, int row, int quad) { return lds + (((w * H + h) * ROWS + row) * 4 + (quad ^ (row & 3))); };
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int i = 0; i < RT; ++i) *at(wave, h, 16 * i + lx, grp) = acc[h][i];
  __syncthreads();
  const int m = threadIdx.x >> 2, c = threadIdx.x & 3;
  const int64_t row = m0 + m, col = n0 + 4 * c;
  if (m >= ROWS || row >= a.M || col >= a.N) return;
  f32x4 v{}, u{};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    v += *at(w, 0, m, c);
    if constexpr (G) u += *at(w, 1, m, c);
  }
  const int left = a.N - col < 4 ? static_cast<int>(a.N - col) : 4;
  linear_quad<T>(a.e, a.N, row, col, 0, left, G, v, u, bias_quad<T>(a.e, col, 0, left),
                 G ? bias_quad<T>(a.e, col + a.N, 0, left) : f32x4{}, residual_quad<T>(a.e, row, col, left));
}

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
  join_rows<T, G, RT>(q, &lds[0][0][0][0], acc, m0, n0);
}

// The same where 16-byte loads serve the rows: each wavefront's blocks come through LDS of its
// own, 128 bytes of a row by 8 neighbouring lanes, NS blocks ahead. (A fragment read straight
// from memory has neighbouring lanes in different rows, which the memory pipeline takes
// four times as long for: 64×4096×4096 16.3 µs so, 9.5 through LDS; 16×4096×4096 7.8 and 6.8.)
template <int RT, bool G>
constexpr int kSlot = (16 * RT + (G ? 32 : 16)) * 128 + 512;
template <int RT>
constexpr int kAhead = RT == 4 ? 1 : 2;
template <int RT, bool G>
constexpr int kStaged = kWaves * kAhead<RT> * kSlot<RT, G>;

template <typename T, bool G, int XC, int WC, int RT>
__global__ __launch_bounds__(64 * kWaves) void staged8_kernel(const Product8 q) {
  constexpr int H = G ? 2 : 1, ROWS = 16 * RT, NS = kAhead<RT>;
  constexpr int NX = 2 * RT, NW = 2 * H, CNT = NX + NW + 2;   // loads of a block
  constexpr uint32_t WOFF = ROWS * 128, SOFF = WOFF + 16 * H * 128, SLOT = kSlot<RT, G>;
  static_assert(kStaged<RT, G> >= static_cast<int>(kWaves * H * ROWS * 64), "room for the sums");
  const ProductArgs& a = q.p;
  extern __shared__ char smem[];
  const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6);
  const int lx = lane & 15, grp = lane >> 4;
  const int64_t m0 = static_cast<int64_t>(blockIdx.y) * ROWS, n0 = static_cast<int64_t>(blockIdx.x) * 16;
  auto kswz = [](int r) { return (r >> 1) & 7; };

  // load p: rows 8p …, chunk c in slot c ^ kswz(r); rows that do not exist lie behind the
  // descriptors' ends
  const int lr = lane >> 3;
  const uint32_t lda = static_cast<uint32_t>(a.lda), ldb = static_cast<uint32_t>(a.ldb);
  const int kc[2] = {((lane & 7) ^ kswz(lr)) * 16, ((lane & 7) ^ kswz(lr + 8)) * 16};   // (rows 16 apart swap alike)
  const float *sx, *sw;
  {
    const int64_t m = m0 + lane < a.M ? m0 + lane : a.M - 1;
    sx = q.sa + (m >> q.xshift) * q.ldsa;
    const int64_t n = n0 + lx < a.N ? n0 + lx : a.N - 1;
    sw = q.sb + (((G && lane >= 16 ? a.N : 0) + n) >> q.wshift) * q.ldsb;
  }
  const int64_t blocks = (a.K + kBlock - 1) / kBlock, whole = (a.K + 15) / 16 * 16;
  const uint32_t lds0 = static_cast<uint32_t>(uni(static_cast<int>(lds_off(smem)))) + wave * (NS * SLOT);
  char* mine = smem + wave * (NS * SLOT);
  const uint8_t* A = static_cast<const uint8_t*>(a.A) + m0 * a.lda;
  const uint8_t* B = static_cast<const uint8_t*>(a.B) + n0 * a.ldb;
  auto issue = [&](int64_t b, uint32_t base) __attribute__((always_inline)) {
    const bool live = b < blocks;
    const int64_t k = live ? b * kBlock : 0, left = live ? a.K - k : 0;
    i32x4 da = descriptor(uniform_ptr(A + k), live ? (a.M - m0 - 1) * a.lda + whole - k : 0);
    i32x4 db = descriptor(uniform_ptr(B + k), live ? (a.N - n0 - 1) * a.ldb + whole - k : 0);
    i32x4 dc = G ? descriptor(uniform_ptr(B + a.N * a.ldb + k), live ? (a.N - n0 - 1) * a.ldb + whole - k : 0) : db;
    asm volatile("s_nop 4" : "+s"(da), "+s"(db), "+s"(dc));
#pragma unroll
    for (int i = 0; i < NX; ++i)
      dma_buffer16((kc[i & 1] < left ? lr * lda + kc[i & 1] : kOutside) + i * 8 * lda, da, base + i * 1024u);
#pragma unroll
    for (int i = 0; i < NW; ++i)
      dma_buffer16((kc[i & 1] < left ? lr * ldb + kc[i & 1] : kOutside) + (i & 1) * 8 * ldb, i < 2 ? db : dc,
                   base + WOFF + i * 1024u);
    const int64_t at = live ? b : blocks - 1;
    dma_scale(sx + at, base + SOFF);
    dma_scale(sw + at, base + SOFF + 256u);
  };
  auto read = [&](const char* st, int row) __attribute__((always_inline)) {
    const char* p = st + (row + lx) * 128;
    const u32x4 x = *reinterpret_cast<const u32x4*>(p + ((grp ^ kswz(lx)) << 4));
    const u32x4 y = *reinterpret_cast<const u32x4*>(p + (((grp + 4) ^ kswz(lx)) << 4));
    return i32x8{static_cast<int>(x[0]), static_cast<int>(x[1]), static_cast<int>(x[2]), static_cast<int>(x[3]),
                 static_cast<int>(y[0]), static_cast<int>(y[1]), static_cast<int>(y[2]), static_cast<int>(y[3])};
  };
  // K ends inside a chunk: what follows in its row is not the row's
  auto trim = [&](i32x8 v, int left) __attribute__((always_inline)) {
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      const int n = left - 16 * (grp + (w < 4 ? 0 : 4)) - 4 * (w & 3);   // bytes of this word that are K's
      v[w] = n >= 4 ? v[w] : n <= 0 ? 0 : static_cast<int>(static_cast<uint32_t>(v[w]) & ((1u << (8 * n)) - 1u));
    }
    return v;
  };
  f32x4 acc[H][RT] = {};
#pragma unroll
  for (int s = 0; s < NS; ++s) issue(wave + s * kWaves, lds0 + s * SLOT);
  uint32_t slot = 0;
  for (int64_t b = wave; b < blocks; b += kWaves) {
    waitcnt_vm<(NS - 1) * CNT>();
    asm volatile("" ::: "memory");
    const char* st = mine + slot;
    i32x8 w[H], x[RT];
    f32x4 sws[H];
    float sxs[RT];
#pragma unroll
    for (int h = 0; h < H; ++h) {
      w[h] = read(st + WOFF, 16 * h);
      sws[h] = *reinterpret_cast<const f32x4*>(st + SOFF + 256 + (16 * h + 4 * grp) * 4);
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      x[i] = read(st, 16 * i);
      sxs[i] = *reinterpret_cast<const float*>(st + SOFF + (16 * i + lx) * 4);
    }
    waitcnt_lgkm0();
    asm volatile("" ::: "memory");
    issue(b + NS * kWaves, lds0 + slot);
    slot = slot + SLOT == NS * SLOT ? 0 : slot + SLOT;
    if ((a.K & 15) && b == blocks - 1) {
      const int left = static_cast<int>(a.K - b * kBlock);
#pragma unroll
      for (int h = 0; h < H; ++h) w[h] = trim(w[h], left);
#pragma unroll
      for (int i = 0; i < RT; ++i) x[i] = trim(x[i], left);
    }
    f32x4 part[H][RT] = {};
#pragma unroll
    for (int c = 0; c < 8; c += 2) {
      bf16x8 wv[H];
#pragma unroll
      for (int h = 0; h < H; ++h) wv[h] = widen8<WC>(w[h][c], w[h][c + 1]);
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        const bf16x8 xv = widen8<XC>(x[i][c], x[i][c + 1]);
#pragma unroll
        for (int h = 0; h < H; ++h)
          part[h][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[h], xv, part[h][i], 0, 0, 0);
      }
    }
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[h][i][r] = fmaf(part[h][i][r], sxs[i] * sws[h][r], acc[h][i][r]);
  }
  waitcnt_vm<0>();   // (loads of nothing, into the room of the sums)
  __syncthreads();
  join_rows<T, G, RT>(q, reinterpret_cast<f32x4*>(smem), acc, m0, n0);
}

template <typename T, bool G, int XC, int WC, int RT>
hipError_t go(bool staged, const Product8& a, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(a.p.tilesN), static_cast<unsigned>(a.p.tilesM));
  if (!staged) {
    rows8_kernel<T, G, XC, WC, RT><<<grid, 64 * kWaves, 0, s>>>(a);
    return hipGetLastError();
  }
  static std::atomic<uint64_t> attr{0};
  const hipError_t e = raise_lds(reinterpret_cast<const void*>(staged8_kernel<T, G, XC, WC, RT>), kStaged<RT, G>, attr);
  if (e != hipSuccess) return e;
  staged8_kernel<T, G, XC, WC, RT><<<grid, 64 * kWaves, kStaged<RT, G>, s>>>(a);
  return hipGetLastError();
}
template <typename T, bool G, int XC, int WC>
hipError_t by_rows(int rows, bool staged, const Product8& a, hipStream_t s) {
  if (rows == 16) return go<T, G, XC, WC, 1>(staged, a, s);
  if (rows == 32) return go<T, G, XC, WC, 2>(staged, a, s);
  if constexpr (!G) return go<T, G, XC, WC, 4>(staged, a, s);
  return hipErrorInvalidValue;
}
template <typename T, bool G>
hipError_t by_codes(int rows, bool staged, const Product8& a, hipStream_t s) {
  if (a.acode == GT_E4M3)
    return a.bcode == GT_E4M3 ? by_rows<T, G, 0, 0>(rows, staged, a, s) : by_rows<T, G, 0, 1>(rows, staged, a, s);
  return a.bcode == GT_E4M3 ? by_rows<T, G, 1, 0>(rows, staged, a, s) : by_rows<T, G, 1, 1>(rows, staged, a, s);
}
template <typename T>
hipError_t by_gate(int rows, bool staged, const Product8& a, hipStream_t s) {
  return a.p.e.gated ? by_codes<T, true>(rows, staged, a, s) : by_codes<T, false>(rows, staged, a, s);
}

}  // namespace

hipError_t launch_rows8(int dtype, int rows, bool staged, const Product8& a, hipStream_t s) {
  return dtype == GT_BF16 ? by_gate<uint16_t>(rows, staged, a, s) : by_gate<float>(rows, staged, a, s);
}

}  // namespace gt
