// Parts of the layer products' epilogue, run on the CPU a lane at a time over arrays that end
// where the memory that may be touched ends: an access beyond them is a segmentation fault.
//   layers_epilogue part | whole
#include <sys/mman.h>
#include <unistd.h>

#include <cstdio>
#include <cstring>
#include <vector>

#include "product.hpp"

using namespace gt;

namespace {

// n values of T, the last one right before a page that cannot be accessed.
template <typename T>
struct Fenced {
  T* p;
  explicit Fenced(int64_t n) {
    const int64_t page = sysconf(_SC_PAGESIZE), bytes = n * static_cast<int64_t>(sizeof(T));
    const int64_t whole = (bytes + page - 1) / page * page;
    void* m = mmap(nullptr, whole + page, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0);
    if (m == MAP_FAILED || mprotect(static_cast<char*>(m) + whole, page, PROT_NONE) != 0) _exit(2);
    p = reinterpret_cast<T*>(static_cast<char*>(m) + whole - bytes);
  }
};

int failed(const char* what, int64_t N, int64_t at, float got, float want) {
  std::printf("%s, N = %lld: cell %lld holds %g, not %g\n", what, static_cast<long long>(N),
              static_cast<long long>(at), got, want);
  return 1;
}

// Every quad that the kernels of a few rows come to, the padding's too, column by column: all
// cells hold their own sums in the end, and none past the last is written.
template <bool G>
int parts(int64_t N) {
  const int64_t rows = 3, slices = 2, half = (N + 3) / 4 * 4, ld = half * (G ? 2 : 1);
  ProductArgs a{};
  a.M = rows;
  a.N = N;
  a.e.ldpart = ld;
  const Fenced<float> part(slices * rows * ld);
  a.e.part = part.p;
  for (int64_t c = 0; c < N + 8; c += 4)
    for (int z = 0; z < slices; ++z)
      for (int64_t row = 0; row < rows; ++row) {
        f32x4 v, u;
        for (int i = 0; i < 4; ++i) {
          v[i] = static_cast<float>(1 + (z * rows + row) * ld + c + i);
          u[i] = static_cast<float>(1 + (z * rows + row) * ld + half + c + i);
        }
        part_quad<G>(a, z, row, c, v, u);
      }
  for (int64_t i = 0; i < slices * rows * ld; ++i)
    if (part.p[i] != static_cast<float>(1 + i))
      return failed(G ? "gated slices" : "slices", N, i, part.p[i], static_cast<float>(1 + i));
  return 0;
}

float value(uint16_t v) { return __builtin_bit_cast(float, static_cast<uint32_t>(v) << 16); }
float value(float v) { return v; }
template <typename T>
T small(int v) {   // exact in both types
  const float f = static_cast<float>(v);
  if constexpr (sizeof(T) == 4) return f;
  else return static_cast<uint16_t>(__builtin_bit_cast(uint32_t, f) >> 16);
}

// The last wavefront's part of a whole tile: sums of small whole numbers, bias, residual and kept
// pre-activations, all of which end with the tile.
template <int DT, int TILE, bool REG, int EPI>
int whole() {
  using T = typename Elem<DT>::T;
  constexpr TileShape t = tile_shape(DT, TILE);
  constexpr bool G = EPI == kEpiGated;
  constexpr int KB = REG ? 128 : t.KB, NS = REG ? 2 : t.NS, NW = t.NWM * t.NWN;
  constexpr int WM = t.BM / t.NWM, WN = t.BN / t.NWN, CH = WN / 4;
  constexpr int RP = epilogue_rows(WM, WN, NS * (t.BM + t.BN) * KB / NW, t.I), XM = epilogue_xor(WN);
  constexpr int64_t M = t.BM, N = G ? t.BN / 2 : t.BN, wide = G ? 2 * N : N;
  ProductArgs a{};
  a.M = M;
  a.N = N;
  a.e.epi = EPI;
  const Fenced<T> R(M * N), P(M * wide), bias(wide), Y(M * N);
  const Fenced<float> lds(RP * WN);
  for (int64_t i = 0; i < M * N; ++i) R.p[i] = small<T>(static_cast<int>(i % 31));
  for (int64_t i = 0; i < wide; ++i) bias.p[i] = small<T>(static_cast<int>(i % 7));
  a.e.R = R.p;
  a.e.P = P.p;
  a.e.bias = bias.p;
  a.e.Y = Y.p;
  a.e.ldr = a.e.ldy = N;
  a.e.ldp = wide;
  a.e.out_f32 = DT == 0;
  const EpiPlace place{M - WM, M, (t.NWN - 1) * WN / 2, 0, 0, t.NWM - 1, t.NWN - 1};
  auto sum = [&](int64_t row, int64_t col) { return static_cast<float>((row + 3 * col) % 5); };
  for (int h = 0; h < WM; h += RP) {
    for (int r = 0; r < RP; ++r)
      for (int x = 0; x < WN; ++x) {
        // tile column x of the wavefront: of its first half, or of the second (gated: an up value)
        const int64_t col = x < WN / 2 ? place.col + x : (G ? N : t.BN / 2) + place.col + x - WN / 2;
        lds.p[r * WN + (((x / 4) ^ (r & XM)) * 4 + x % 4)] = sum(place.row + h + r, col);
      }
    for (int lane = 0; lane < 64; ++lane)
      EpiRows<DT, EPI, WM, WN, XM, RP, t.BN>{a, place, h, reinterpret_cast<const char*>(lds.p), lane}
          .template whole<GT_ACT_NONE>();
  }
  for (int64_t row = M - WM; row < M; ++row)
    for (int x = 0; x < (G ? WN / 2 : WN); ++x) {
      const int64_t n = x < WN / 2 ? place.col + x : t.BN / 2 + place.col + x - WN / 2;
      const float p = sum(row, n) + static_cast<float>(n % 7);
      const float u = G ? sum(row, N + n) + static_cast<float>((N + n) % 7) : 1.0f;
      const float want = p * u + static_cast<float>((row * N + n) % 31);
      const float got = value(Y.p[row * N + n]);
      if (got != want) return failed("Y", N, row * N + n, got, want);
      if (value(P.p[row * wide + n]) != p) return failed("P", N, row * wide + n, value(P.p[row * wide + n]), p);
      if (G && value(P.p[row * wide + N + n]) != u)
        return failed("P", N, row * wide + N + n, value(P.p[row * wide + N + n]), u);
    }
  static_assert(CH >= 4);
  return 0;
}

template <int DT, int TILE, bool REG>
int both() {
  std::printf("type %d, tile %d, registers %d\n", DT, TILE, REG);
  std::fflush(stdout);
  return whole<DT, TILE, REG, kEpiLinear>() + whole<DT, TILE, REG, kEpiGated>();
}

}  // namespace

int main(int argc, char** argv) {
  if (argc == 2 && std::strcmp(argv[1], "part") == 0) {
    int bad = 0;
    for (int64_t N = 1; N <= 72; ++N) bad += parts<false>(N) + parts<true>(N);
    return bad != 0;
  }
  if (argc == 2 && std::strcmp(argv[1], "whole") == 0)   // every form that product_inst.hip builds
    return (both<0, 1, false>() + both<0, 2, false>() + both<0, 2, true>() + both<0, 3, false>() +
            both<0, 3, true>() + both<1, 0, false>() + both<1, 1, false>() + both<1, 2, false>() +
            both<1, 2, true>() + both<1, 3, false>() + both<1, 3, true>()) != 0;
  return 2;
}
