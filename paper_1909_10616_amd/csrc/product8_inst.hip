// One translation unit of the 8-bit products: a tile and both operands' codes
// (-DP8_TILE=<0|1|2> -DP8_AC=<0|1> -DP8_BC=<0|1>).
#include "product8.hpp"

#if !defined(P8_TILE) || !defined(P8_AC) || !defined(P8_BC)
#error "compile with -DP8_TILE=<0|1|2> -DP8_AC=<0|1> -DP8_BC=<0|1>"
#endif

#define P8_CAT(t, a, b) product8_##t##_##a##_##b
#define P8_NAME(t, a, b) P8_CAT(t, a, b)

namespace gt {
namespace {

template <int DT, bool EXACT, int EPI, bool UNI>
hipError_t go(const Product8& a, hipStream_t s) {
  constexpr auto* fn = product8_kernel<DT, EXACT, P8_AC, P8_BC, P8_TILE, EPI, UNI>;
  constexpr Tile8 t = tile8(P8_TILE);
  static std::atomic<uint64_t> attr{0};
  constexpr size_t lds = 2 * kStage8(P8_TILE);
  const hipError_t e = raise_lds(reinterpret_cast<const void*>(fn), lds, attr);
  if (e != hipSuccess) return e;
  const dim3 grid(static_cast<unsigned>(a.p.tilesM) * static_cast<unsigned>(a.p.tilesN),
                  static_cast<unsigned>(a.p.splits));
  hipLaunchKernelGGL(fn, grid, dim3(64 * t.NWM * t.NWN), lds, s, a);
  return hipGetLastError();
}

template <int DT, bool EXACT, bool UNI>
hipError_t by_epilogue(const Product8& a, hipStream_t s) {
  if (a.p.e.epi == kEpiGated) return go<DT, EXACT, kEpiGated, UNI>(a, s);
  if (a.p.e.epi == kEpiLinear) return go<DT, EXACT, kEpiLinear, UNI>(a, s);
  // (a K slice's sums have no type)
  if constexpr (DT == 1) return go<1, EXACT, kEpiPart, UNI>(a, s);
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t P8_NAME(P8_TILE, P8_AC, P8_BC)(int dtype, bool exact, bool uni, const Product8& a, hipStream_t s) {
  if (!exact) {
    if (dtype != GT_BF16) return hipErrorInvalidValue;
    return uni ? by_epilogue<1, false, true>(a, s) : by_epilogue<1, false, false>(a, s);
  }
#if P8_TILE > 0
  if (dtype == GT_BF16 || a.p.e.epi == kEpiPart) return by_epilogue<1, true, false>(a, s);
  return by_epilogue<0, true, false>(a, s);
#else
  return hipErrorInvalidValue;
#endif
}

}  // namespace gt
