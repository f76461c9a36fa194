// The entry points of the norm, the quantising and the 8-bit products: checks of the
// arguments, the choice of a form, and the launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include "gemmtune_layers.h"
#include "layer8_kernels.h"
#include "layer_checks.h"
#include "layer_kernels.h"

namespace gt {

#define P8_DECLARE(t, a, b) hipError_t product8_##t##_##a##_##b(int, bool, bool, const Product8&, hipStream_t);
P8_DECLARE(0, 0, 0)
P8_DECLARE(0, 0, 1)
P8_DECLARE(0, 1, 0)
P8_DECLARE(0, 1, 1)
P8_DECLARE(1, 0, 0)
P8_DECLARE(1, 0, 1)
P8_DECLARE(1, 1, 0)
P8_DECLARE(1, 1, 1)
#undef P8_DECLARE

hipError_t launch_product8(int dtype, int tile, bool exact, bool uni, const Product8& a, hipStream_t s) {
  using Fn = hipError_t (*)(int, bool, bool, const Product8&, hipStream_t);
  constexpr Fn kFn[kTiles8][2][2] = {{{product8_0_0_0, product8_0_0_1}, {product8_0_1_0, product8_0_1_1}},
                                     {{product8_1_0_0, product8_1_0_1}, {product8_1_1_0, product8_1_1_1}}};
  return kFn[tile][a.acode][a.bcode](dtype, exact, uni, a, s);
}

namespace {

bool code_ok(int c) { return c == GT_E4M3 || c == GT_E5M2; }
bool block_ok(int b) { return b == 1 || b == 128; }
int64_t blocks(int64_t n) { return (n + 127) / 128; }
// Codes of rows×cols values with their scales, `block` rows to a scale.
int codes(const void* q, const float* s, int64_t ldq, int64_t lds, int64_t rows, int64_t cols, int block,
          const char* name) {
  GT_CHECK(matrix(q, true, ldq, rows, cols, 1, name));
  return matrix(s, true, lds, block == 1 ? rows : blocks(rows), blocks(cols), 4,
                (std::string("the scales of ") + name).c_str());
}

// ---- quantising

int quantise_impl(const gt_quantise_args* a, void* stream) {
  if (!a) return fail("gt_quantise: null arguments");
  GT_CHECK(extent(a->M, 0, "M"));
  GT_CHECK(extent(a->N, 1, "N"));
  if (!dtype_ok(a->dtype) || !code_ok(a->code) || !block_ok(a->block))
    return fail("gt_quantise: unknown dtype, code or block");
  if (a->M == 0) return GT_OK;
  if (!a->X || (!a->Q && !a->Qt)) return fail("gt_quantise: null X, or nothing wanted");
  if ((a->Q && !a->S) || (a->Qt && !a->St)) return fail("gt_quantise: codes need their scales");
  GT_CHECK(matrix(a->X, true, a->ldx, a->M, a->N, size_of(a->dtype), "X"));
  if (a->Q) GT_CHECK(codes(a->Q, a->S, a->ldq, a->lds, a->M, a->N, a->block, "Q"));
  if (a->Qt) GT_CHECK(codes(a->Qt, a->St, a->ldqt, a->ldst, a->N, a->M, a->block, "Qt"));
  GT_TRY(launch_quantise(*a, static_cast<hipStream_t>(stream)), "quantising");
  return GT_OK;
}

// ---- norm

int norm_impl(const gt_norm_args* a, void* stream) {
  if (!a) return fail("gt_norm: null arguments");
  GT_CHECK(extent(a->M, 0, "M"));
  GT_CHECK(extent(a->N, 1, "N"));
  if (!dtype_ok(a->dtype) || !dtype_ok(a->wtype) || !code_ok(a->code))
    return fail("gt_norm: unknown dtype or code");
  if (!out_ok(a->wtype, a->dtype)) return fail("gt_norm: w and b are in dtype or in fp32");
  if (!(a->eps >= 0.0f) || std::isinf(a->eps)) return fail("gt_norm: eps is finite and not negative");
  if (a->M == 0) return GT_OK;
  if (!a->X) return fail("gt_norm: null X");
  if (!a->Y && !a->Q && !a->mean && !a->rstd) return fail("gt_norm: nothing wanted");
  if (a->Q && !a->S) return fail("gt_norm: codes need their scales");
  const int64_t sz = size_of(a->dtype);
  GT_CHECK(matrix(a->X, true, a->ldx, a->M, a->N, sz, "X"));
  GT_CHECK(vector(a->w, size_of(a->wtype), "w"));
  GT_CHECK(vector(a->b, size_of(a->wtype), "b"));
  GT_CHECK(matrix(a->Y, false, a->ldy, a->M, a->N, sz, "Y"));
  GT_CHECK(vector(a->mean, 4, "mean"));
  GT_CHECK(vector(a->rstd, 4, "rstd"));
  if (a->Y == a->X && a->ldy != a->ldx) return fail("gt_norm: Y may be X only in the same rows");
  if (a->Q) GT_CHECK(codes(a->Q, a->S, a->ldq, a->lds, a->M, a->N, 1, "Q"));
  GT_TRY(launch_norm(*a, static_cast<hipStream_t>(stream)), "norm");
  return GT_OK;
}

int norm_grad_checks(const gt_norm_grad_args* a, bool pointers) {
  if (!a) return fail("gt_norm_backward: null arguments");
  GT_CHECK(extent(a->M, 0, "M"));
  GT_CHECK(extent(a->N, 1, "N"));
  if (!dtype_ok(a->dtype) || !dtype_ok(a->wtype)) return fail("gt_norm_backward: unknown dtype");
  if (!out_ok(a->wtype, a->dtype)) return fail("gt_norm_backward: w is in dtype or in fp32");
  if (pointers && a->M > 0 && (!a->dY || !a->X || !a->mean || !a->rstd))
    return fail("gt_norm_backward: null dY, X, mean or rstd");
  const int64_t sz = size_of(a->dtype);
  GT_CHECK(matrix(a->dY, true, a->lddy, a->M, a->N, sz, "dY"));
  GT_CHECK(matrix(a->X, true, a->ldx, a->M, a->N, sz, "X"));
  GT_CHECK(vector(a->w, size_of(a->wtype), "w"));
  GT_CHECK(vector(a->mean, 4, "mean"));
  GT_CHECK(vector(a->rstd, 4, "rstd"));
  GT_CHECK(matrix(a->dX ? a->R : nullptr, false, a->ldr, a->M, a->N, sz, "R"));
  GT_CHECK(matrix(a->dX, false, a->lddx, a->M, a->N, sz, "dX"));
  if (a->dX && ((a->dX == a->R && a->lddx != a->ldr) || (a->dX == a->dY && a->lddx != a->lddy)))
    return fail("gt_norm_backward: dX may be R or dY only in the same rows");
  GT_CHECK(vector(a->dw, 4, "dw"));
  return vector(a->db, 4, "db");
}

int norm_backward_workspace_impl(const gt_norm_grad_args* a, int64_t* bytes) {
  if (!bytes) return fail("gt_norm_backward_workspace: null argument");
  GT_CHECK(norm_grad_checks(a, false));
  *bytes = up(norm_parts(*a) * 2 * a->N * 4, 256);
  return GT_OK;
}

int norm_backward_impl(const gt_norm_grad_args* a, void* ws, int64_t ws_bytes, void* stream) {
  GT_CHECK(norm_grad_checks(a, true));
  const int64_t need = up(norm_parts(*a) * 2 * a->N * 4, 256);
  GT_CHECK(scratch_ok(ws, ws_bytes, need));
  GT_TRY(launch_norm_grad(*a, need ? static_cast<float*>(ws) : nullptr, static_cast<hipStream_t>(stream)),
         "gradients of the norm");
  return GT_OK;
}

// ---- linear of codes

int linear8_checks(const gt_linear_fp8_args* a, bool pointers) {
  if (!a) return fail("gt_linear_fp8: null arguments");
  GT_CHECK(extent(a->M, 0, "M"));
  GT_CHECK(extent(a->N, 1, "N"));
  GT_CHECK(extent(a->K, 1, "K"));
  if (!dtype_ok(a->dtype) || !dtype_ok(a->out_dtype) || !act_ok(a->act))
    return fail("gt_linear_fp8: unknown dtype or activation");
  if (!code_ok(a->xcode) || !code_ok(a->wcode) || !block_ok(a->xblock) || !block_ok(a->wblock))
    return fail("gt_linear_fp8: unknown code or block");
  if (!out_ok(a->out_dtype, a->dtype)) return fail("gt_linear_fp8: Y is in dtype or in fp32");
  const int64_t wide = a->act & GT_ACT_GATED ? 2 * a->N : a->N;
  GT_CHECK(extent(wide, 1, "2N"));
  if (pointers && a->M > 0 && (!a->X || !a->sx || !a->W || !a->sw || !a->Y))
    return fail("gt_linear_fp8: null X, W, their scales or Y");
  if (a->out_dtype != a->dtype && a->R == a->Y && a->R)
    return fail("gt_linear_fp8: R may be Y only in the same type");
  if (a->R && a->R == a->Y && a->ldr != a->ldy)
    return fail("gt_linear_fp8: R may be Y only in the same rows");
  const int64_t sz = size_of(a->dtype);
  GT_CHECK(codes(a->X, a->sx, a->ldx, a->ldsx, a->M, a->K, a->xblock, "X"));
  GT_CHECK(codes(a->W, a->sw, a->ldw, a->ldsw, wide, a->K, a->wblock, "W"));
  GT_CHECK(vector(a->bias, sz, "bias"));
  GT_CHECK(matrix(a->R, false, a->ldr, a->M, a->N, sz, "R"));
  return matrix(a->Y, true, a->ldy, a->M, a->N, size_of(a->out_dtype), "Y");
}

struct Linear8 {
  Product8 q{};
  int rows = 0;   // > 0: the kernel of a few rows, so many a workgroup
  int tile = 0;
  bool exact = false, uni = false;
};

Linear8 linear8(const gt_linear_fp8_args& g) {
  Linear8 l;
  Product8& q = l.q;
  ProductArgs& a = q.p;
  a.A = g.X;
  a.B = g.W;
  a.lda = g.ldx;
  a.ldb = g.ldw;
  a.M = g.M;
  a.N = g.N;
  a.K = g.K;
  a.half = g.N;
  q.sa = g.sx;
  q.sb = g.sw;
  q.ldsa = g.ldsx;
  q.ldsb = g.ldsw;
  q.xshift = g.xblock == 1 ? 0 : 7;
  q.wshift = g.wblock == 1 ? 0 : 7;
  q.acode = g.xcode;
  q.bcode = g.wcode;
  Epilogue& e = a.e;
  e.act = g.act & ~GT_ACT_GATED;
  e.gated = g.act & GT_ACT_GATED ? 1 : 0;
  e.epi = e.gated ? kEpiGated : kEpiLinear;
  e.out_f32 = g.out_dtype == GT_F32 ? 1 : 0;
  e.Y = g.Y;
  e.ldy = g.ldy;
  e.bias = g.bias;
  e.R = g.R;
  e.ldr = g.ldr;
  e.ldpart = up(a.N, 4) * (e.gated ? 2 : 1);
  a.splits = 1;
  l.exact = g.out_dtype == GT_F32;
  l.uni = g.wblock == 128 && (!e.gated || a.N % 128 == 0);
  const bool tiles = a.M > 64 && aligned(a.A, 16) && aligned(a.B, 16) && a.lda % 16 == 0 && a.ldb % 16 == 0 &&
                     256 * std::max(a.lda, a.ldb) < kMaxExtent && a.K < kMaxExtent - 1024;
  if (tiles) {
    l.tile = l.exact || a.M <= 1024 ? 1 : 0;
    const Tile8 t = tile8(l.tile);
    const int64_t wide = e.gated ? 2 * a.N : a.N, tm = (a.M + t.BM - 1) / t.BM, tn = (wide + t.BN - 1) / t.BN;
    if (tm * tn * 64 * t.NWM * t.NWN < kMaxItems) {
      a.tilesM = static_cast<int>(tm);
      a.tilesN = static_cast<int>(tn);
      return l;
    }
  }
  l.rows = g.M <= 16 ? 16 : g.M <= 32 || e.gated ? 32 : 64;
  a.tilesN = static_cast<int>((a.N + 15) / 16);
  a.tilesM = static_cast<int>((a.M + l.rows - 1) / l.rows);
  return l;
}

int linear_fp8_workspace_impl(const gt_linear_fp8_args* a, int64_t* bytes) {
  if (!bytes) return fail("gt_linear_fp8_workspace: null argument");
  GT_CHECK(linear8_checks(a, false));
  *bytes = 0;
  return GT_OK;
}

int linear_fp8_impl(const gt_linear_fp8_args* a, void* ws, int64_t ws_bytes, void* stream) {
  GT_CHECK(linear8_checks(a, true));
  GT_CHECK(scratch_ok(ws, ws_bytes, 0));
  if (a->M == 0) return GT_OK;
  const Linear8 l = linear8(*a);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  GT_TRY(l.rows > 0 ? launch_rows8(a->dtype, l.rows, l.q, s)
                    : launch_product8(a->dtype, l.tile, l.exact, l.uni, l.q, s),
         "8-bit product");
  return GT_OK;
}

}  // namespace
}  // namespace gt

extern "C" {

using namespace gt;

int gt_quantise(const gt_quantise_args* a, void* stream) {
  return guarded([&] { return quantise_impl(a, stream); });
}
int gt_linear_fp8_workspace(const gt_linear_fp8_args* a, int64_t* bytes) {
  return guarded([&] { return linear_fp8_workspace_impl(a, bytes); });
}
int gt_linear_fp8(const gt_linear_fp8_args* a, void* ws, int64_t ws_bytes, void* stream) {
  return guarded([&] { return linear_fp8_impl(a, ws, ws_bytes, stream); });
}
int gt_norm(const gt_norm_args* a, void* stream) {
  return guarded([&] { return norm_impl(a, stream); });
}
int gt_norm_backward_workspace(const gt_norm_grad_args* a, int64_t* bytes) {
  return guarded([&] { return norm_backward_workspace_impl(a, bytes); });
}
int gt_norm_backward(const gt_norm_grad_args* a, void* ws, int64_t ws_bytes, void* stream) {
  return guarded([&] { return norm_backward_impl(a, ws, ws_bytes, stream); });
}

}  // extern "C"
