// Launchers of the norm, of the quantising kernels and of the 8-bit products.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "gemmtune_layers.h"
#include "product_args.h"

namespace gt {

hipError_t launch_quantise(const gt_quantise_args& a, hipStream_t s);

hipError_t launch_norm(const gt_norm_args& a, hipStream_t s);

// Partial rows of the column sums (0 where neither dw nor db is wanted), each of N of dw and
// N of db.
int64_t norm_parts(const gt_norm_grad_args& a);
hipError_t launch_norm_grad(const gt_norm_grad_args& a, float* part, hipStream_t s);

// An 8-bit product: p.A and p.B are codes, rows lda and ldb bytes apart, both along k; row r
// of A has its scales at sa + (r >> xshift)·ldsa, B's likewise. p.N: columns of Y; B has the up
// values' rows from N on when gated.
struct Product8 {
  ProductArgs p;
  const float* sa;
  const float* sb;
  int64_t ldsa, ldsb;
  int32_t xshift, wshift;
  int32_t acode, bcode;
};

// The tiles: rows, columns, wavefronts along each; bytes of LDS of a stage, its codes and scales.
struct Tile8 {
  int BM, BN, NWM, NWN;
};
constexpr int kTiles8 = 3;
constexpr Tile8 tile8(int tile) {
  return tile == 0 ? Tile8{256, 256, 2, 4} : tile == 1 ? Tile8{128, 128, 2, 2} : Tile8{64, 64, 2, 1};
}
constexpr unsigned kStage8(int tile) { return (tile8(tile).BM + tile8(tile).BN) * 132u; }
// exact: sums of all that fp32 holds (not tile 0), else what the 8-bit instructions keep, of a bf16 Y;
// uni: the rows of B in either half of a wavefront's columns share their scales.
hipError_t launch_product8(int dtype, int tile, bool exact, bool uni, const Product8& a, hipStream_t s);

// Few rows: `rows` (16, 32 or 64) a workgroup; staged: both operands at 16-byte aligned rows that
// 32-bit offsets reach.
hipError_t launch_rows8(int dtype, int rows, bool staged, const Product8& a, hipStream_t s);

}  // namespace gt

// The form that a call takes, so that tests can hold every one: rows a workgroup of the kernels of a few
// rows (0: tiles), the tile (−1), K slices (0: no form serves), whether all of its sums are fp32's.
extern "C" int gt_linear_fp8_form(const gt_linear_fp8_args* a, int32_t form[4]);
