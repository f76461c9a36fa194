// One translation unit of the layer products: the tiles of one operand type and
// layout (-DLP_DT=<0|1>, -DLP_LAY=<0|1|2>).
#include "product.hpp"

#if !defined(LP_DT) || !defined(LP_LAY)
#error "compile with -DLP_DT=<0|1> -DLP_LAY=<0|1|2>"
#endif

#define LP_CAT(a, b) product_##a##_##b
#define LP_NAME(a, b) LP_CAT(a, b)

namespace gt {
namespace {

// The dynamic LDS limit is raised once per kernel and device (attr: the devices
// where it has been).
template <typename F>
hipError_t launch_with_lds(F fn, std::atomic<uint64_t>& attr, const ProductArgs& a, dim3 grid,
                           dim3 block, size_t lds, hipStream_t s) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = dev >= 0 && dev < 64 ? uint64_t{1} << dev : 0;
  if (!bit || !(attr.load(std::memory_order_acquire) & bit)) {
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(fn),
                            hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(lds));
    if (e != hipSuccess) return e;
    attr.fetch_or(bit, std::memory_order_release);
  }
  hipLaunchKernelGGL(fn, grid, block, lds, s, a);
  return hipGetLastError();
}

template <int TILE, bool REG, int EPI>
hipError_t go(const ProductArgs& a, hipStream_t s) {
  constexpr TileShape t = tile_shape(LP_DT, TILE);
  constexpr int KB = REG ? 128 : t.KB, NS = REG ? 2 : t.NS;
  constexpr auto* fn = product_kernel<LP_DT, t.I, LP_LAY == kXtP, LP_LAY != kPWt, t.BM, t.BN, t.NWM,
                                      t.NWN, KB, NS, REG, EPI>;
  const dim3 grid(static_cast<unsigned>(a.tilesM) * static_cast<unsigned>(a.tilesN) +
                      (a.tail ? kUnits : 0),
                  static_cast<unsigned>(a.splits),
                  a.along_k ? static_cast<unsigned>(a.groups) : 1u);
  static std::atomic<uint64_t> attr{0};
  return launch_with_lds(fn, attr, a, grid, dim3(64 * t.NWM * t.NWN),
                         static_cast<size_t>(NS) * (t.BM + t.BN) * KB, s);
}

template <int TILE, bool REG>
hipError_t by_epilogue(const ProductArgs& a, hipStream_t s) {
  if (a.e.epi == kEpiPart) return go<TILE, REG, kEpiPart>(a, s);
#if LP_LAY == 0
  if (a.e.epi == kEpiLinear) return go<TILE, REG, kEpiLinear>(a, s);
  if (a.e.epi == kEpiGated) return go<TILE, REG, kEpiGated>(a, s);
#else
  if (a.e.epi == kEpiPlain) return go<TILE, REG, kEpiPlain>(a, s);
#endif
#if LP_LAY == 1
  if (a.e.epi == kEpiSlope) return go<TILE, REG, kEpiSlope>(a, s);
#endif
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t LP_NAME(LP_DT, LP_LAY)(int tile, bool reg, const ProductArgs& a, hipStream_t s) {
#if LP_DT == 1
  if (tile == 0 && !reg) return by_epilogue<0, false>(a, s);
#endif
  if (tile == 1 && !reg) return by_epilogue<1, false>(a, s);
  if (tile == 2) return reg ? by_epilogue<2, true>(a, s) : by_epilogue<2, false>(a, s);
#if LP_LAY != 2
  if (tile == 3) return reg ? by_epilogue<3, true>(a, s) : by_epilogue<3, false>(a, s);
#endif
  return hipErrorInvalidValue;
}

}  // namespace gt
