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
P8_DECLARE(2, 0, 0)
P8_DECLARE(2, 0, 1)
P8_DECLARE(2, 1, 0)
P8_DECLARE(2, 1, 1)
#undef P8_DECLARE

hipError_t launch_product8(int dtype, int tile, bool exact, bool uni, const Product8& a, hipStream_t s) {
  using Fn = hipError_t (*)(int, bool, bool, const Product8&, hipStream_t);
  constexpr Fn kFn[kTiles8][2][2] = {{{product8_0_0_0, product8_0_0_1}, {product8_0_1_0, product8_0_1_1}},
                                     {{product8_1_0_0, product8_1_0_1}, {product8_1_1_0, product8_1_1_1}},
                                     {{product8_2_0_0, product8_2_0_1}, {product8_2_1_0, product8_2_1_1}}};
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
  int rows = 0;   // > 0: the kernels of a few rows, so many a workgroup
  bool staged = false;   // … through LDS
  int tile = 0;
  bool exact = false, uni = false;
  PadJobs pad{};                     // operands copied to aligned rows first …
  int64_t pad_a = 0, pad_b = 0;      // … their bytes
  int64_t part = 0;                  // bytes of the K slices' sums
  int64_t scratch() const { return up(pad_a, 256) + up(pad_b, 256) + up(part, 256); }
};

// A form and its time in µs.
struct Form {
  int rows, tile, splits;
  double cost;
  int64_t tm, tn;
};

// What a stage (128 k) of a tile takes, in µs, where few tiles run (alone) and where they fill the
// chip (full), the launch and epilogue of such rounds, and how many tiles fill it. Fitted to
// 100 shapes from 1×1024×1024 to 4096×11008×4096, each in every form (bf16, K = 4096: 256×256
// tiles 53 µs for 16 of them, 73 for 256; 128×128 29 for 32, 45 for 512; 64×64 25 for 64, 34
// for 1024): 93 choices are within 5 % of the best form, 98 within 10 %.
struct Cost8 {
  double alone, full, fixed, fixed_full;
  int64_t fill;
};
constexpr Cost8 kCost8[2][kTiles8] = {
    {{1.45, 1.95, 8.0, 10.0, 256}, {0.78, 1.15, 4.6, 8.0, 512}, {0.68, 0.86, 2.9, 6.3, 1024}},
    {{0, 0, 0, 0, 0}, {1.21, 2.0, 5.2, 11.0, 512}, {1.1, 1.3, 3.0, 9.0, 1024}}};   // exact
double tiles_cost(const Cost8& c, int64_t tiles, double stages) {
  const int64_t rounds = tiles / c.fill, rest = tiles % c.fill;
  double t = 0.0;
  if (rounds > 0) t = rounds * (stages * c.full + 0.6 * c.fixed_full) + 0.4 * c.fixed_full;
  if (rest > 0) {
    const double share = static_cast<double>(rest) / c.fill;
    t += stages * (c.alone + (c.full - c.alone) * share * std::sqrt(share)) +
         (c.fixed + (c.fixed_full - c.fixed) * share) * (rounds > 0 ? 0.6 : 1.0);
  }
  return t;
}
// The same of the kernels of a few rows: a wavefront's block of 128 k for each round of 256 workgroups,
// and W's way from memory. (few: through LDS, or X a few rows that all lanes share.)
double rows_cost(int rows, bool gated, bool few, int64_t groups, int64_t steps, double memory) {
  // [few][gated][rows / 32]
  constexpr double kEach[2][2][3] = {{{1.28, 2.1, 3.43}, {1.85, 3.0, 0.0}}, {{0.85, 1.25, 1.7}, {1.41, 2.0, 0.0}}};
  const double each = kEach[few][gated][rows / 32];
  return 3.0 + std::hypot(each * static_cast<double>(steps) * std::max(1.0, static_cast<double>(groups) / kUnits), memory);
}

// The form by the time it should take: the tiles' rounds or the operands' way from memory, which
// overlap in part, K slices' sums and the launch that joins them, copies to aligned rows.
// What no tile serves (rows too long for 32-bit offsets) is left to the kernel of a few rows.
void choose(Linear8* l) {
  ProductArgs& a = l->q.p;
  const bool gated = a.e.gated != 0;
  const int64_t wide = gated ? 2 * a.N : a.N, all = blocks(a.K), ldd = up(a.K, 16);
  const bool ok_a = aligned(a.A, 16) && a.lda % 16 == 0, ok_b = aligned(a.B, 16) && a.ldb % 16 == 0;
  const bool tiles = 256 * std::max(ok_a ? a.lda : ldd, ok_b ? a.ldb : ldd) < kMaxExtent;
  const double copied = static_cast<double>((ok_a ? 0 : a.M * ldd) + (ok_b ? 0 : wide * ldd));
  const double copy = copied > 0 ? 5.0 + 2.0 * copied / 5.0e6 : 0.0;
  const double memory = static_cast<double>(a.M * a.K + wide * a.K) / 5.2e6;
  // (a row or four take no more from memory directly: 1×11008×4096 gated 22.2 µs, 24.4 through LDS)
  const bool staged = a.M > 4 && ok_a && ok_b && 64 * std::max(a.lda, a.ldb) < kMaxExtent;
  Form best{0, 0, 1, 0.0, 0, 0};
  auto offer = [&](const Form& f) {
    if (best.cost == 0.0 || f.cost < best.cost) best = f;
  };
  for (int t = l->exact ? 1 : 0; tiles && t < kTiles8; ++t) {
    const Tile8 s = tile8(t);
    const int64_t tm = (a.M + s.BM - 1) / s.BM, tn = (wide + s.BN - 1) / s.BN;
    if (tm * tn * 64 * s.NWM * s.NWN >= kMaxItems) continue;
    for (int z = 1; z <= 16 && (z == 1 || 2 * z <= all); z *= 2) {
      const double stages = static_cast<double>((all + z - 1) / z);
      double cost = copy + std::hypot(tiles_cost(kCost8[l->exact][t], tm * tn * z, stages), memory);
      // (two launches and the scratch are 18 µs of the host's)
      if (z > 1) cost = std::max(18.0, cost + 4.5 + 2.0 * z * a.M * wide * 4 / 6.0e6);
      offer(Form{0, t, z, cost, tm, tn});
    }
  }
  for (const int r : {16, 32, 64}) {
    if (r == 64 && gated) continue;
    const int64_t tm = (a.M + r - 1) / r, tn = (a.N + 15) / 16;
    if (tm >= 65536 || tn * 512 >= kMaxItems) continue;
    offer(Form{r, 0, 1, rows_cost(r, gated, staged || a.M <= 4, tm * tn, (all + 7) / 8, memory), tm, tn});
  }
  l->rows = best.rows;
  l->staged = staged;
  l->tile = best.tile;
  a.splits = best.cost > 0.0 ? best.splits : 0;   // (0: no form serves)
  a.tilesM = static_cast<int>(best.tm);
  a.tilesN = static_cast<int>(best.tn);
  if (a.splits == 0) return;
  a.per_slice = static_cast<int>((all + a.splits - 1) / a.splits);
  l->part = a.splits > 1 ? a.splits * a.M * a.e.ldpart * 4 : 0;
  if (l->rows > 0) return;
  auto pad = [&](const void* p, int64_t rows, int64_t* ld, int64_t* bytes) {
    PadJob& j = l->pad.job[l->pad.n++];
    j = PadJob{p, nullptr, 1, rows, a.K, *ld, 0, ldd, 0};
    *ld = ldd;
    *bytes = rows * ldd;
  };
  if (!ok_a) pad(a.A, a.M, &a.lda, &l->pad_a);
  if (!ok_b) pad(a.B, wide, &a.ldb, &l->pad_b);
}

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
  l.exact = g.out_dtype == GT_F32 || g.exact != 0;
  l.uni = g.wblock == 128 && (!e.gated || a.N % 128 == 0);
  choose(&l);
  return l;
}

int linear_fp8_workspace_impl(const gt_linear_fp8_args* a, int64_t* bytes) {
  if (!bytes) return fail("gt_linear_fp8_workspace: null argument");
  GT_CHECK(linear8_checks(a, false));
  *bytes = a->M > 0 ? linear8(*a).scratch() : 0;
  return GT_OK;
}

int linear_fp8_form_impl(const gt_linear_fp8_args* a, int32_t* form) {
  if (!form) return fail("gt_linear_fp8_form: null argument");
  GT_CHECK(linear8_checks(a, false));
  const Linear8 l = linear8(*a);
  form[0] = l.rows;
  form[1] = l.rows > 0 ? -1 : l.tile;
  form[2] = l.q.p.splits;
  form[3] = l.rows > 0 || l.exact;
  return GT_OK;
}

int linear_fp8_impl(const gt_linear_fp8_args* a, void* ws, int64_t ws_bytes, void* stream) {
  GT_CHECK(linear8_checks(a, true));
  if (a->M == 0) return GT_OK;
  Linear8 l = linear8(*a);
  ProductArgs& p = l.q.p;
  if (p.splits == 0) return fail("gt_linear_fp8: too many rows");
  GT_CHECK(scratch_ok(ws, ws_bytes, l.scratch()));
  const hipStream_t s = static_cast<hipStream_t>(stream);
  char* at = static_cast<char*>(ws);
  int n = 0;
  auto place = [&](const void** operand, int64_t bytes) {
    if (bytes == 0) return;
    *operand = l.pad.job[n++].dst = at;
    at += up(bytes, 256);
  };
  place(&p.A, l.pad_a);
  place(&p.B, l.pad_b);
  if (n > 0) GT_TRY(launch_pad(kBytes, l.pad, s), "copy to aligned rows");
  const int epi = p.e.epi;
  if (p.splits > 1) {
    p.e.part = reinterpret_cast<float*>(at);
    p.e.epi = kEpiPart;
  }
  GT_TRY(l.rows > 0 ? launch_rows8(a->dtype, l.rows, l.staged, l.q, s)
                    : launch_product8(a->dtype, l.tile, l.exact, l.uni, l.q, s),
         "8-bit product");
  p.e.epi = epi;
  if (p.splits > 1) GT_TRY(launch_reduce(a->dtype, p, s), "joining the K slices");
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
int gt_linear_fp8_form(const gt_linear_fp8_args* a, int32_t* form) {
  return guarded([&] { return linear_fp8_form_impl(a, form); });
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
