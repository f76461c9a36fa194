// Launchers of the layer operators' helper kernels. dtype: gt_dtype of the
// operands; ld*: elements between rows.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "gemmtune_layers.h"
#include "product_args.h"

namespace gt {

// A launch has fewer work-items along a dimension than this; the runtime takes more modulo
// 2^32 and reports nothing.
constexpr int64_t kMaxItems = int64_t{1} << 32;

// Sums the K slices of a product (a.e.part) in slice order and applies the linear
// epilogue of a.e to every row (with groups along m: below the last offset).
hipError_t launch_reduce(int dtype, const ProductArgs& a, hipStream_t s);

// A matrix (or `groups` of them) copied to rows of whole 16-byte chunks, zero beyond its
// columns; half > 0: its two halves of cols / 2 columns each begin at 0 and half.
struct PadJob {
  const void* src;
  void* dst;
  int64_t groups, rows, cols;
  int64_t ld, sgroup;     // of src
  int64_t ldd, half;      // of dst, groups one after the other
};
constexpr int kPadJobs = 4;   // of two products
struct PadJobs {
  PadJob job[kPadJobs];
  int n;
};
constexpr int kBytes = 2;   // in place of a dtype: single bytes
hipError_t launch_pad(int dtype, const PadJobs& jobs, hipStream_t s);

// Rows a block of the gradient kernel sums into one row of its partial sums.
constexpr int kActRows = 16;
// dP = dY·act'(P) (gated: both halves), and each block's column sums of it into
// part[block][wide] (part NULL: not wanted; dP NULL: only the sums).
struct ActGradArgs {
  int64_t M, N;
  int act, gated;
  const void* dY;
  int64_t lddy;
  const void* P;
  int64_t ldp;
  void* dP;
  int64_t lddp;
  float* part;
  bool wide;   // whole octets of columns
  int pad;   // columns of dP beyond its last that are written as zero
};
hipError_t launch_act_grad(int dtype, const ActGradArgs& a, hipStream_t s);

// out[g][n] = Σ of part's rows of group g, in order. Rows: with offsets, group
// g's rows of tiles of `bm` rows, `per` partial rows each, of the `rows` that there are;
// without, all `rows`.
hipError_t launch_join(const float* part, int64_t rows, int64_t wide, const int32_t* offsets,
                       int groups, int64_t most, int bm, int per, float* out, hipStream_t s);

// The sorted entries' rows of X and dY, in rows of whole 16-byte chunks, zero beyond D:
// Xs[p] = X[order[p] / k] (X NULL: not wanted), dYs[p] likewise; and of each block of kSortRows
// rows of a group and kSortCols columns
//   sums[block row][D]: Σ w·dY over its rows (NULL: not wanted)
//   dot[p][block column]: b2[e]·dY over its columns (b2 NULL: not wanted).
constexpr int kSortRows = 64;
constexpr int kSortCols = 512;
struct SortArgs {
  const void *X, *dY, *b2;
  int64_t ldx, lddy;
  void *Xs, *dYs;
  int64_t ldd, D, T, entries;
  int E, k;
  const float* weights;
  const int32_t *order, *offsets;
  float *sums, *dot;
  int64_t ldot;
};
hipError_t launch_sort(int dtype, const SortArgs& a, hipStream_t s);

// out[t] = R[t] + Σ_s w[t][s]·O[place[t][s]] (w NULL: 1; R NULL: 0), s ascending.
struct CombineArgs {
  int64_t T, D, entries;
  int k;
  bool wide;   // whole octets of columns
  const float* O;
  int64_t ldo;
  const float* weights;
  const int32_t* place;
  const void* R;
  int64_t ldr;
  void* out;
  int64_t ldout;
};
hipError_t launch_combine(int dtype, const CombineArgs& a, hipStream_t s);

// dweights[entry] = Σ of the n values at dot[place], 0 for an entry without a place.
hipError_t launch_weight_grad(const float* dot, int64_t ldot, int64_t n, const int32_t* place,
                              const int32_t* offsets, int E, int64_t entries, float* dweights,
                              hipStream_t s);

// Routing (gt_route): launches and scratch.
int64_t route_scratch(int64_t T, int E, int k, int groups);
hipError_t launch_route(const gt_route_args& a, void* ws, hipStream_t s);
hipError_t launch_route_grad(const gt_route_grad_args& a, hipStream_t s);

}  // namespace gt
