// The layer operators' entry points: checks of the arguments, the choice of a
// tile and of K slices for every product, and the launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include "gemmtune_layers.h"
#include "internal.h"
#include "layer_checks.h"
#include "layer_kernels.h"
#include "product_args.h"

namespace gt {
namespace {

// ---- one product: its tile, its K slices, its launches

struct Product {
  ProductArgs a{};
  int dtype = GT_F32, layout = kXW;
  // the operands are this library's own arrays: 16-byte aligned rows of whole chunks,
  // and, where k runs along them, zero beyond the last
  bool own_a = false, own_b = false;
  int tile = 1;
  bool reg = false;
  int rows = 0;           // > 0: the kernel for a few rows, so many a workgroup
  PadJobs pad{};          // operands copied to aligned rows first …
  int64_t pad_a = 0, pad_b = 0, part = 0;   // … and the bytes of that and of partial sums
  bool tails = false;     // `part` is the last tiles'

  int64_t pads() const { return up(pad_a, 256) + up(pad_b, 256); }
  int64_t scratch() const { return pads() + up(part, 256); }
};

// One operand as it is stored: whether 16-byte loads serve it (aligned rows of whole
// chunks, what one descriptor must reach within its range), and as the copy that they
// do serve.
struct Stored {
  bool ok;
  PadJob job;
  int64_t bytes;
};
Stored stored(const void* ptr, int64_t ld, int64_t sgroup, int64_t groups, int64_t rows, int64_t cols,
              int64_t half, int64_t reach_rows, bool own, int64_t sz) {
  const int64_t vec = 16 / sz, reach = int64_t{1} << 31;
  Stored s{};
  s.ok = aligned(ptr, 16) && ld % vec == 0 && (groups == 1 || sgroup % vec == 0) &&
         (own || (cols % vec == 0 && half % vec == 0)) && reach_rows * ld * sz < reach;
  PadJob& j = s.job;
  j.src = ptr;
  j.groups = groups;
  j.rows = rows;
  j.cols = cols;
  j.ld = ld;
  j.sgroup = sgroup;
  j.half = half ? up(half, vec) : 0;
  j.ldd = half ? 2 * j.half : up(cols, vec);
  s.bytes = groups * rows * j.ldd * sz;
  if (reach_rows * j.ldd * sz >= reach) s.bytes = -1;   // no copy of it would do
  return s;
}

// The part of the groups that get no row, were the rows spread evenly.
double no_row(const ProductArgs& a) {
  return std::pow(1.0 - 1.0 / a.groups, static_cast<double>(a.M));
}

// Rows a workgroup of the kernel for a few rows takes, 0 where it does not serve: up to 4
// rows, or up to 4 a group on average (the groups that get a row, were the rows
// spread evenly), that fit its LDS.
int few_rows(const Product& p) {
  const ProductArgs& a = p.a;
  if (p.layout != kXW || a.M < 1) return 0;
  double each = static_cast<double>(a.M);
  if (a.groups > 0) {
    if (a.M > 4 * a.groups) return 0;
    each = a.M / (a.groups * (1.0 - no_row(a)));
  }
  const int rows = each <= 1.3 ? 1 : each <= 2.3 ? 2 : each <= 4.0 ? 4 : 0;
  if (rows == 0 || rows_lds(a.K, rows, p.a.e.epi == kEpiGated) > 128 * 1024) return 0;
  if ((a.N + 63) / 64 * kRowThreads >= kMaxItems) return 0;
  return a.M / rows + a.groups < 65536 ? rows : 0;
}

// K slices of that kernel. A workgroup, one a compute unit, draws its columns of W from
// memory at 24 GB/s (30 gated, 35 in fp32, where a row gives two lines of memory) after
// 3 µs, the whole chip at 5.2 TB/s, so W comes sooner if more of them share it, for the
// launch that joins their sums and its host time: taken where a sixth is to be won
// (bf16, W past the caches: 1×4096×4096 by 64 workgroups 22.5 µs, 256 in 4 slices
// 15.2; 1×4096×11008 52.2 and 25.3; 1×11008×4096, 172 workgroups, 23.5 and in 2 slices 29.3).
int rows_slices(const Product& p) {
  const ProductArgs& a = p.a;
  const bool gated = a.e.epi == kEpiGated;
  const double each = static_cast<double>(a.K) * (gated ? 128 : 64) * size_of(p.dtype);
  const double rows = a.groups > 0 ? std::min<double>(a.groups * (1.0 - no_row(a)), a.M)
                                   : static_cast<double>((a.M + p.rows - 1) / p.rows);
  const double shares = rows * a.tilesN, rate = p.dtype != GT_BF16 ? 35e3 : gated ? 30e3 : 24e3;
  int best = 1;
  double least = 0.0, alone = 0.0;
  for (int z : {1, 2, 3, 4, 6, 8, 16}) {
    const double rounds = std::ceil(shares * z / 256.0);
    const double t = 3.0 * rounds + (z > 1 ? 4.5 : 0.0) +
                     std::hypot(rounds * each / z / rate, shares * each / 5.2e6);
    if (z == 1) alone = t;
    if (z == 1 || (t < least && t < alone * 5 / 6)) {
      best = z;
      least = t;
    }
  }
  return best;
}

// The kernel of 16 rows a workgroup: its tile rows at most.
constexpr int kSlimRows = 16;
int64_t slim_rows(const ProductArgs& a) {
  return a.groups > 0 ? a.M / kSlimRows + std::min<int64_t>(a.groups, a.M)
                      : (a.M + kSlimRows - 1) / kSlimRows;
}
// And its time in µs in z K slices (0: it does not serve): the steps of a wavefront for every
// workgroup that a compute unit gets, or W once for every tile row, at 10 TB/s while
// the last cache holds it. Fitted to 60 shapes from 1×7×3 to 512×4096×4096, plain and gated,
// with 1 to 16 slices; it is chosen up to 64 rows or so, or more of small matrices
// (13×1021×777 in fp32: 9.8 µs, the best tile with its join 12.1; 64×1024×1024 in bf16 6.1
// and 8.0; 256×1024×1024 6.5 and 8.3; but 64×11008×4096 59 and 25).
double slim_cost(const Product& p, int64_t z) {
  const ProductArgs& a = p.a;
  const int64_t rows = slim_rows(a), cols = (a.N + 63) / 64;
  const bool bf16 = p.dtype == GT_BF16, gated = a.e.epi == kEpiGated;
  if (a.M < 1 || rows >= 65536 || rows * cols >= kMaxExtent || cols * 64 * slim_waves(gated) >= kMaxItems)
    return 0.0;
  if (a.K >= kMaxExtent / 2) return 0.0;   // (its k are 32-bit numbers, past the last by a step)
  const int64_t step = bf16 ? 32 : 16, steps = (a.K + step - 1) / step, waves = slim_waves(gated);
  if (z > 1 && steps < 16 * z) return 0.0;
  const double each = static_cast<double>(((steps + z - 1) / z + waves - 1) / waves);
  const double queue = static_cast<double>((rows * cols * z + 255) / 256);
  // [type][gated][aligned]
  constexpr double kStep[2][2][2] = {{{1.8, 1.7}, {2.3, 1.65}}, {{3.0, 1.45}, {3.5, 1.25}}};
  const double per = kStep[bf16][gated][slim_aligned(p.dtype, a)];
  const double matrix = static_cast<double>(a.K) * a.N * (gated ? 2 : 1) * size_of(p.dtype);
  const double memory = std::max(rows * matrix / (matrix <= 64e6 ? 10e6 : 6e6), matrix / 5.2e6);
  return 4.2 + std::hypot(each * per * queue, memory) +
         (z > 1 ? 4.5 + 2.0 * z * a.M * a.N * (gated ? 2 : 1) * 4 / 6.0e6 : 0.0);
}

// What a tile takes a compute unit, in µs: a stage (128 bytes of k) alone and
// when others share the unit, its launch and epilogue, and how many share it. Fitted to
// 48 shapes from 1×4096×4096 to 2048×4096×4096, 14 of them odd, in every layout and
// type, each at every tile and 1 to 32 K slices (bf16, K = 4096, one slice:
// 256×256 tiles 76 µs for 16 of them, 114 for 256; 128×128 43, 75 for 512; 64×64 28, 114
// for 2048; 16×128 22, 221 for 4096). Of 254 choices four in five are within 5 % of the best form
// measured, nine in ten within 10 %; the furthest are few rows whose K slices would save 3 to 5 µs
// in a graph and cost as much of host time in a second launch without one.
struct TileCost {
  double alone, shared, fixed;
  int resident;
};
constexpr TileCost kCost[2][kTiles] = {
    {{0, 0, 0, 1}, {2.05, 2.0, 6, 2}, {0.71, 0.59, 5, 3}, {0.49, 0.41, 5, 2}},         // fp32
    {{1.62, 1.62, 8, 1}, {0.64, 0.55, 4.3, 2}, {0.375, 0.25, 4.2, 3}, {0.28, 0.235, 4.3, 2}}  // bf16
};

// What a stage of the register path takes, in stages by descriptor loads: bf16 and fp32 by
// layout (kXW, kPWt, kXtP) and tile (64×64, 16×128), fitted to 14 shapes from
// 13×1021×777 to 1999×2623×3457. bf16 rows that lie along the reduction's other side
// are transposed a value at a time.
constexpr double kReg[2][3][2] = {{{1.4, 2.0}, {1.4, 2.0}, {1.4, 2.0}},
                                  {{2.5, 4.6}, {1.5, 2.5}, {3.3, 4.6}}};

// Tile, K slices and copies by the time they should take: the stages of the tiles that a
// compute unit gets (256 of them; tiles that share a unit run in rounds) and the operands'
// way from memory, which overlap in part, a K slice's partial sums and the launch that
// joins them, the copies of operands that 16-byte loads do not serve and their launch.
void choose(Product* p, bool may_split) {
  ProductArgs& a = p->a;
  a.half = a.N;
  a.e.ldpart = up(a.N, 4) * (a.e.epi == kEpiGated ? 2 : 1);
  if ((p->rows = few_rows(*p)) > 0) {
    a.tilesN = static_cast<int>((a.N + 63) / 64);
    a.tilesM = static_cast<int>(a.groups > 0 ? a.M / p->rows + std::min<int64_t>(a.groups, a.M)
                                             : (a.M + p->rows - 1) / p->rows);
    a.splits = may_split ? rows_slices(*p) : 1;
    p->part = a.splits > 1 ? a.splits * a.M * a.e.ldpart * 4 : 0;
    return;
  }
  const int64_t sz = size_of(p->dtype), bk = 128 / sz;
  const bool gated = a.e.epi == kEpiGated;
  const int64_t wide = gated ? 2 * a.N : a.N;
  const bool ax = p->layout == kXtP, bx = p->layout != kPWt;
  const int64_t bgroups = a.groups > 0 && !a.along_k ? a.groups : 1;
  const Stored sa = stored(a.A, a.lda, 0, 1, ax ? a.K : a.gather ? a.a_rows : a.M, ax ? a.M : a.K, 0,
                           ax ? 64 : a.gather ? a.a_rows : 256, p->own_a, sz);
  const Stored sb = stored(a.B, a.ldb, a.sB, bgroups, bx ? a.K : a.N, bx ? wide : a.K,
                           bx && gated ? a.N : 0, bx ? 64 : 256, p->own_b, sz);
  const bool may_tail = !a.along_k && a.e.epi != kEpiSlope;
  const bool copies = (!sa.ok && sa.bytes > 0) || (!sb.ok && sb.bytes > 0);
  const bool can_dma = (sa.ok || sa.bytes >= 0) && (sb.ok || sb.bytes >= 0);
  const int64_t stages = std::max<int64_t>(1, ((a.along_k ? a.K / std::max(1, a.groups) : a.K) + bk - 1) / bk);
  double best = 0.0;
  for (int t = 0; t < kTiles; ++t) {
    const TileShape& s = kTile[t];
    if (t == 0 && p->dtype != GT_BF16) continue;
    if (t == 3 && p->layout == kXtP) continue;
    const int64_t tn = (wide + s.BN - 1) / s.BN;
    int64_t tm = (a.M + s.BM - 1) / s.BM;
    int64_t most = tm;
    if (a.groups > 0 && !a.along_k) {
      const int64_t g = std::min<int64_t>(a.groups, a.M);
      most = a.M / s.BM + g;
      // rows spread over the groups: half a tile lost in each, one tile at least
      tm = std::max<int64_t>(g, a.M / s.BM + g / 2);
    }
    const int64_t tiles = tm * tn * (a.along_k ? a.groups : 1);
    const TileShape waves = tile_shape(p->dtype, t);
    if (most * tn >= kMaxExtent || (most * tn + kUnits) * 64 * waves.NWM * waves.NWN >= kMaxItems) continue;
    const TileCost& c = kCost[p->dtype == GT_BF16 ? 1 : 0][t];
    const double memory = static_cast<double>(a.M * a.K + std::min(bgroups, std::max<int64_t>(1, a.M)) * a.K * wide) * sz / 5.2e6;
    for (int reg = 0; reg < 2; ++reg) {
      if (reg ? (t < 2 || (sa.ok && sb.ok)) : !can_dma) continue;
      const double copy = !reg && copies ? 5.0 + 2.0 * ((sa.ok ? 0 : sa.bytes) + (sb.ok ? 0 : sb.bytes)) / 5.0e6 : 0.0;
      for (int64_t z = 1; z <= 64; z *= 2) {
        if (z > 1 && (!may_split || stages / z < 4)) break;
        const double each = static_cast<double>((stages + z - 1) / z) * (reg ? kReg[p->dtype == GT_BF16 ? 1 : 0][p->layout][t - 2] : 1.0);
        const int64_t queue = (tiles * z + 255) / 256;
        const int64_t rounds = (queue + c.resident - 1) / c.resident;
        const double busy = rounds > 1 ? c.shared * c.resident * rounds : std::max(c.alone, c.shared * queue);
        double cost = copy + std::hypot(each * busy, memory) + c.fixed * rounds;
        if (z > 1) cost += 4.5 + 2.0 * z * a.M * wide * 4 / 6.0e6;
        bool tails = false;
        // the last tiles in slices (with groups, whose tiles are a guess, of the largest only)
        if ((t == 0 || (t == 1 && a.groups == 0)) && z == 1 && may_tail && tiles < kMaxExtent) {
          const Tail tail = tail_of(static_cast<int>(tiles), static_cast<int>(stages));
          const int64_t q = tail.full / kUnits, slice = (stages + tail.slices - 1) / tail.slices;
          // (where two share a unit, one tile or a slice may be left alone)
          const double work = c.resident == 1 ? c.shared * (stages * q + slice)
                              : q % 2 == 1    ? c.shared * (stages * (q - 1) + 2 * slice) +
                                                 c.alone * (stages - slice)
                                              : c.shared * stages * q + c.alone * slice;
          const double cut = copy + std::hypot(work, memory) + c.fixed * ((q + c.resident) / c.resident) + 6.0 +
                             2.0 * tail.left * tail.slices * s.BM * s.BN * 4 / 5.0e6;
          if (tail.slices > 1 && cut < cost) {
            tails = true;
            cost = cut;
          }
        }
        if (best == 0.0 || cost < best) {
          best = cost;
          p->tile = t;
          p->reg = reg != 0;
          p->tails = tails;
          a.splits = static_cast<int>(z);
          a.tilesM = static_cast<int>(most);
          a.tilesN = static_cast<int>(tn);
        }
      }
    }
  }
  if (p->layout == kXW) {
    for (int64_t z = 1; z <= 16; z *= 2) {
      if (z > 1 && !may_split) break;
      const double cost = slim_cost(*p, z);
      if (cost > 0.0 && cost < best) {
        best = cost;
        p->rows = kSlimRows;
        a.splits = static_cast<int>(z);
      }
    }
  }
  p->part = a.splits > 1 ? a.splits * a.M * a.e.ldpart * 4 : 0;
  if (p->rows > 0) {
    p->reg = p->tails = false;
    a.tilesN = static_cast<int>((a.N + 63) / 64);
    a.tilesM = static_cast<int>(slim_rows(a));
    return;
  }
  if (!p->reg) {
    if (!sa.ok && sa.bytes > 0) {
      p->pad.job[p->pad.n++] = sa.job;
      p->pad_a = sa.bytes;
      a.lda = sa.job.ldd;
    }
    if (!sb.ok && sb.bytes > 0) {
      p->pad.job[p->pad.n++] = sb.job;
      p->pad_b = sb.bytes;
      a.ldb = sb.job.ldd;
      a.sB = sb.job.rows * sb.job.ldd;
      if (sb.job.half) a.half = sb.job.half;
    }
  }
  const TileShape& s = kTile[p->tile];
  const int64_t kb = (p->reg ? 128 : s.KB) / sz, all = (a.K + kb - 1) / kb;
  a.per_slice = static_cast<int>((all + a.splits - 1) / std::max(1, a.splits));
  if (p->tails) p->part = static_cast<int64_t>(kUnits) * s.BM * s.BN * 4;
}

hipError_t launch(const Product& p, const ProductArgs& a, hipStream_t s) {
  return p.rows == kSlimRows ? launch_slim(p.dtype, a, s)
         : p.rows > 0        ? launch_rows(p.dtype, p.rows, a, s)
                             : launch_product(p.dtype, p.layout, p.tile, p.reg, a, s);
}

// A product's copies to aligned rows into its pads() bytes at `at`: their jobs, and the
// operands that they become.
void place_pads(const Product& p, char* at, ProductArgs* a, PadJobs* jobs) {
  int n = 0;
  auto place = [&](int64_t bytes) {
    PadJob& j = jobs->job[jobs->n++] = p.pad.job[n++];
    j.dst = at;
    at += up(bytes, 256);
    return j.dst;
  };
  if (p.pad_a) a->A = place(p.pad_a);
  if (p.pad_b) a->B = place(p.pad_b);
}

// Whether a form serves a product (called before the first launch of its operator).
int planned(const Product& p) {
  return p.a.M > 0 && p.a.splits < 1 ? fail("layer product: too many tiles") : GT_OK;
}

// Launches a product; ws: its scratch() bytes.
int run(const Product& p, void* ws, hipStream_t s) {
  ProductArgs a = p.a;
  if (a.M == 0) return GT_OK;
  char* at = static_cast<char*>(ws);
  if (p.pads() > 0) {
    PadJobs jobs{};
    place_pads(p, at, &a, &jobs);
    GT_TRY(launch_pad(p.dtype, jobs, s), "copy to aligned rows");
    at += p.pads();
  }
  if (a.splits > 1) {
    a.e.part = reinterpret_cast<float*>(at);
    const int epi = a.e.epi;
    a.e.epi = kEpiPart;
    GT_TRY(launch(p, a, s), "layer product");
    a.e.epi = epi;
    GT_TRY(launch_reduce(p.dtype, a, s), "joining the K slices");
    return GT_OK;
  }
  if (p.tails) a.tail = reinterpret_cast<float*>(at);
  GT_TRY(launch(p, a, s), "layer product");
  if (p.tails) GT_TRY(launch_tail(p.dtype, p.tile, a, s), "joining the last tiles");
  return GT_OK;
}

// ---- linear

int linear_checks(const gt_linear_args* a, bool pointers) {
  if (!a) return fail("gt_linear: null arguments");
  GT_CHECK(extent(a->M, 0, "M"));
  GT_CHECK(extent(a->N, 1, "N"));
  GT_CHECK(extent(a->K, 1, "K"));
  if (!dtype_ok(a->dtype) || !dtype_ok(a->out_dtype) || !act_ok(a->act))
    return fail("gt_linear: unknown dtype or activation");
  if (!out_ok(a->out_dtype, a->dtype)) return fail("gt_linear: Y is in dtype or in fp32");
  const int64_t wide = a->act & GT_ACT_GATED ? 2 * a->N : a->N;
  GT_CHECK(extent(wide, 1, "2N"));
  if (pointers && a->M > 0 && (!a->X || !a->W || !a->Y)) return fail("gt_linear: null X, W or Y");
  if (a->out_dtype != a->dtype && a->R == a->Y && a->R)
    return fail("gt_linear: R may be Y only in the same type");
  const int64_t sz = size_of(a->dtype);
  GT_CHECK(matrix(a->X, true, a->ldx, a->M, a->K, sz, "X"));
  GT_CHECK(matrix(a->W, true, a->ldw, a->K, wide, sz, "W"));
  GT_CHECK(vector(a->bias, sz, "bias"));
  GT_CHECK(matrix(a->R, false, a->ldr, a->M, a->N, sz, "R"));
  GT_CHECK(matrix(a->Y, true, a->ldy, a->M, a->N, size_of(a->out_dtype), "Y"));
  return matrix(a->P, false, a->ldp, a->M, wide, sz, "P");
}

Product linear_product(const gt_linear_args& q) {
  Product p;
  p.dtype = q.dtype;
  p.layout = kXW;
  ProductArgs& a = p.a;
  a.A = q.X;
  a.B = q.W;
  a.lda = q.ldx;
  a.ldb = q.ldw;
  a.M = q.M;
  a.N = q.N;
  a.K = q.K;
  Epilogue& e = a.e;
  e.act = q.act & ~GT_ACT_GATED;
  e.gated = q.act & GT_ACT_GATED ? 1 : 0;
  e.epi = e.gated ? kEpiGated : kEpiLinear;
  e.out_f32 = q.out_dtype == GT_F32 ? 1 : 0;
  e.Y = q.Y;
  e.ldy = q.ldy;
  e.P = q.P;
  e.ldp = q.ldp;
  e.bias = q.bias;
  e.R = q.R;
  e.ldr = q.ldr;
  choose(&p, true);
  return p;
}

// ---- the gradients of linear

int linear_grad_checks(const gt_linear_grad_args* a, bool pointers) {
  if (!a) return fail("gt_linear_backward: null arguments");
  GT_CHECK(extent(a->M, 0, "M"));
  GT_CHECK(extent(a->N, 1, "N"));
  GT_CHECK(extent(a->K, 1, "K"));
  if (!dtype_ok(a->dtype) || !dtype_ok(a->dw_dtype) || !act_ok(a->act))
    return fail("gt_linear_backward: unknown dtype or activation");
  if (!out_ok(a->dw_dtype, a->dtype)) return fail("gt_linear_backward: dW is in dtype or in fp32");
  const int64_t wide = a->act & GT_ACT_GATED ? 2 * a->N : a->N;
  GT_CHECK(extent(wide, 1, "2N"));
  if (pointers && a->M > 0) {
    if (!a->dY) return fail("gt_linear_backward: null dY");
    if (a->act != GT_ACT_NONE && !a->P) return fail("gt_linear_backward: the activation needs P");
    if ((a->dX && !a->W) || (a->dW && !a->X))
      return fail("gt_linear_backward: dX needs W, dW needs X");
  }
  const int64_t sz = size_of(a->dtype);
  const bool act = a->act != GT_ACT_NONE;
  GT_CHECK(matrix(a->dY, true, a->lddy, a->M, a->N, sz, "dY"));
  GT_CHECK(matrix(a->X, a->dW, a->ldx, a->M, a->K, sz, "X"));
  GT_CHECK(matrix(a->W, a->dX, a->ldw, a->K, wide, sz, "W"));
  GT_CHECK(matrix(act ? a->P : nullptr, act, a->ldp, a->M, wide, sz, "P"));
  GT_CHECK(matrix(a->dX, false, a->lddx, a->M, a->K, sz, "dX"));
  GT_CHECK(matrix(a->dW, false, a->lddw, a->K, wide, size_of(a->dw_dtype), "dW"));
  return vector(a->db, 4, "db");
}

struct LinearGrad {
  bool own_dP = false;    // dP is not dY itself
  int64_t lddp = 0, wide = 0;
  Product dx, dw;
  // scratch
  void *dP = nullptr, *rest = nullptr;   // rest: the products' partial sums, one after the other
  char* pads = nullptr;                  // both products' copies to aligned rows
  float* sums = nullptr;
  int64_t bytes = 0;
};

void output(Epilogue* e, void* y, int64_t ldy, bool f32) {
  e->epi = kEpiPlain;
  e->Y = y;
  e->ldy = ldy;
  e->out_f32 = f32 ? 1 : 0;
}

LinearGrad linear_grad(const gt_linear_grad_args& q, void* ws) {
  LinearGrad g;
  const int64_t sz = size_of(q.dtype);
  g.wide = q.act & GT_ACT_GATED ? 2 * q.N : q.N;
  g.own_dP = q.act != GT_ACT_NONE;
  g.lddp = g.own_dP ? up(g.wide, 16 / sz) : q.lddy;
  Scratch s(ws);
  const bool products = q.dX || q.dW;
  if (g.own_dP && products) g.dP = s.take(q.M * g.lddp * sz);
  const void* dP = g.own_dP ? g.dP : q.dY;
  if (q.db) g.sums = s.take<float>((q.M + kActRows - 1) / kActRows * g.wide * 4);
  int64_t rest = 0;
  if (q.dX) {   // dP (M×wide) · Wᵀ
    g.dx.dtype = q.dtype;
    g.dx.layout = kPWt;
    ProductArgs& a = g.dx.a;
    a.A = dP;
    a.lda = g.lddp;
    a.B = q.W;
    a.ldb = q.ldw;
    a.M = q.M;
    a.N = q.K;
    a.K = g.wide;
    output(&a.e, q.dX, q.lddx, q.dtype == GT_F32);
    g.dx.own_a = g.own_dP;
    choose(&g.dx, true);
    rest = std::max(rest, g.dx.part);
  }
  if (q.dW) {   // Xᵀ · dP
    g.dw.dtype = q.dtype;
    g.dw.layout = kXtP;
    ProductArgs& a = g.dw.a;
    a.A = q.X;
    a.lda = q.ldx;
    a.B = dP;
    a.ldb = g.lddp;
    a.M = q.K;
    a.N = g.wide;
    a.K = q.M;
    output(&a.e, q.dW, q.lddw, q.dw_dtype == GT_F32);
    g.dw.own_b = g.own_dP;
    choose(&g.dw, true);
    rest = std::max(rest, g.dw.part);
  }
  if (g.dx.pads() + g.dw.pads() > 0) g.pads = s.take<char>(g.dx.pads() + g.dw.pads());
  if (rest) g.rest = s.take(rest);
  g.bytes = s.used;
  return g;
}

// ---- experts

int experts_checks(int64_t T, int64_t D, int64_t H, int E, int k, int dtype, int act) {
  GT_CHECK(extent(T, 0, "T"));
  GT_CHECK(extent(D, 1, "D"));
  GT_CHECK(extent(H, 1, "H"));
  if (act & GT_ACT_GATED) GT_CHECK(extent(2 * H, 1, "2H"));
  if (E < 1 || E > 1024 || k < 1 || k > 64) return fail("experts: E is 1 … 1024, k 1 … 64");
  if (T * k >= kMaxEntries) return fail("experts: T·k out of range");
  if (!dtype_ok(dtype) || !act_ok(act)) return fail("experts: unknown dtype or activation");
  if (T * k > kMaxElements / std::max(D, 2 * H) || D > kMaxElements / (2 * H) / E)
    return fail("experts: the rows or the matrices are too large");
  return GT_OK;
}
// The experts' matrices (sw apart) and the lists.
int stack(const void* p, bool needed, int64_t ld, int64_t sw, int64_t rows, int64_t cols, int E,
          int64_t sz, const char* name) {
  if (!p && !needed) return GT_OK;
  GT_CHECK(matrix(p, true, ld, rows, cols, sz, name));
  if (sw < 0) return fail(std::string("negative stride between the experts of ") + name);
  return sw > kMaxElements / E ? fail(std::string(name) + " is too large") : GT_OK;
}
int lists(const float* weights, const int32_t* offsets, const int32_t* order, const int32_t* place) {
  GT_CHECK(vector(weights, 4, "weights"));
  GT_CHECK(vector(offsets, 4, "offsets"));
  GT_CHECK(vector(order, 4, "order"));
  return vector(place, 4, "place");
}

int experts_args_checks(const gt_experts_args* a, bool pointers) {
  if (!a) return fail("gt_experts: null arguments");
  GT_CHECK(experts_checks(a->T, a->D, a->H, a->E, a->k, a->dtype, a->act));
  const int64_t wide = a->act & GT_ACT_GATED ? 2 * a->H : a->H;
  if (pointers && a->T > 0 &&
      (!a->X || !a->W1 || !a->W2 || !a->Y || !a->weights || !a->offsets || !a->order || !a->place))
    return fail("gt_experts: null X, W1, W2, Y or list");
  const int64_t sz = size_of(a->dtype);
  GT_CHECK(matrix(a->X, true, a->ldx, a->T, a->D, sz, "X"));
  GT_CHECK(stack(a->W1, true, a->ldw1, a->sw1, a->D, wide, a->E, sz, "W1"));
  GT_CHECK(stack(a->W2, true, a->ldw2, a->sw2, a->H, a->D, a->E, sz, "W2"));
  GT_CHECK(vector(a->b1, sz, "b1"));
  GT_CHECK(vector(a->b2, sz, "b2"));
  GT_CHECK(matrix(a->R, false, a->ldr, a->T, a->D, sz, "R"));
  GT_CHECK(matrix(a->Y, true, a->ldy, a->T, a->D, sz, "Y"));
  GT_CHECK(matrix(a->P, false, a->ldp, a->T * a->k, wide, sz, "P"));
  return lists(a->weights, a->offsets, a->order, a->place);
}

struct Experts {
  Product up, down;
  void *H = nullptr, *rest = nullptr;
  float* O = nullptr;
  int64_t bytes = 0, ldo = 0;
};

Experts experts(const gt_experts_args& q, void* ws) {
  Experts x;
  const int64_t sz = size_of(q.dtype), R = q.T * q.k;
  const int64_t wide = q.act & GT_ACT_GATED ? 2 * q.H : q.H;
  const int64_t ldh = up(q.H, 16 / sz);
  x.ldo = up(q.D, 4);
  Scratch s(ws);
  x.H = s.take(R * ldh * sz);
  x.O = s.take<float>(R * x.ldo * 4);
  {   // the rows' tokens are read from X where they lie; the activated rows are stored in the
      // operands' type, which the down product's matrix instructions take
    x.up.dtype = q.dtype;
    x.up.layout = kXW;
    ProductArgs& a = x.up.a;
    a.A = q.X;
    a.lda = q.ldx;
    a.B = q.W1;
    a.ldb = q.ldw1;
    a.sB = q.sw1;
    a.M = R;
    a.N = q.H;
    a.K = q.D;
    a.offsets = q.offsets;
    a.groups = q.E;
    a.gather = q.order;
    a.gather_div = q.k;
    a.a_rows = q.T;
    Epilogue& e = a.e;
    e.act = q.act & ~GT_ACT_GATED;
    e.gated = q.act & GT_ACT_GATED ? 1 : 0;
    e.epi = e.gated ? kEpiGated : kEpiLinear;
    e.out_f32 = q.dtype == GT_F32 ? 1 : 0;
    e.Y = x.H;
    e.ldy = ldh;
    e.P = q.P;
    e.ldp = q.ldp;
    e.bias = q.b1;
    e.sbias = wide;
    e.zero_pad = 1;
    choose(&x.up, true);
  }
  {
    x.down.dtype = q.dtype;
    x.down.layout = kXW;
    ProductArgs& a = x.down.a;
    a.A = x.H;
    a.lda = ldh;
    a.B = q.W2;
    a.ldb = q.ldw2;
    a.sB = q.sw2;
    a.M = R;
    a.N = q.D;
    a.K = q.H;
    a.offsets = q.offsets;
    a.groups = q.E;
    Epilogue& e = a.e;
    e.epi = kEpiLinear;
    e.out_f32 = 1;
    e.Y = x.O;
    e.ldy = x.ldo;
    e.bias = q.b2;
    e.sbias = q.D;
    x.down.own_a = true;
    choose(&x.down, true);
  }
  const int64_t rest = std::max(x.up.scratch(), x.down.scratch());
  if (rest) x.rest = s.take(rest);
  x.bytes = s.used;
  return x;
}

int experts_grad_checks(const gt_experts_grad_args* a, bool pointers) {
  if (!a) return fail("gt_experts_backward: null arguments");
  GT_CHECK(experts_checks(a->T, a->D, a->H, a->E, a->k, a->dtype, a->act));
  const int64_t wide = a->act & GT_ACT_GATED ? 2 * a->H : a->H;
  if (pointers && a->T > 0) {
    if (!a->dY || !a->W2 || !a->P || !a->weights || !a->offsets || !a->order || !a->place)
      return fail("gt_experts_backward: null dY, W2, P or list");
    if ((a->dX && !a->W1) || (a->dW1 && !a->X))
      return fail("gt_experts_backward: dX needs W1, dW1 needs X");
  }
  if (pointers && a->T == 0 && !a->offsets) return fail("gt_experts_backward: null offsets");
  const int64_t sz = size_of(a->dtype);
  GT_CHECK(matrix(a->dY, true, a->lddy, a->T, a->D, sz, "dY"));
  GT_CHECK(matrix(a->X, a->dW1, a->ldx, a->T, a->D, sz, "X"));
  GT_CHECK(stack(a->W1, a->dX, a->ldw1, a->sw1, a->D, wide, a->E, sz, "W1"));
  GT_CHECK(stack(a->W2, true, a->ldw2, a->sw2, a->H, a->D, a->E, sz, "W2"));
  GT_CHECK(vector(a->b2, sz, "b2"));
  GT_CHECK(matrix(a->P, true, a->ldp, a->T * a->k, wide, sz, "P"));
  GT_CHECK(matrix(a->dX, false, a->lddx, a->T, a->D, sz, "dX"));
  GT_CHECK(vector(a->dW1, sz, "dW1"));
  GT_CHECK(vector(a->dW2, sz, "dW2"));
  GT_CHECK(vector(a->db1, 4, "db1"));
  GT_CHECK(vector(a->db2, 4, "db2"));
  GT_CHECK(vector(a->dweights, 4, "dweights"));
  return lists(a->weights, a->offsets, a->order, a->place);
}

struct ExpertsGrad {
  int64_t R, wide, ldd, ldp, ldh, ldo, ndot = 0, nb2 = 0;
  int64_t colrows = 0, sumrows = 0;   // partial rows of db1 and of db2
  Product dh, dw2, dx, dw1;
  void *Xs = nullptr, *dYs = nullptr, *dP = nullptr, *Hw = nullptr, *rest = nullptr;
  float *dXs = nullptr, *dot = nullptr, *colsum = nullptr, *sums = nullptr;
  int64_t bytes = 0;
};

ExpertsGrad experts_grad(const gt_experts_grad_args& q, void* ws) {
  ExpertsGrad g;
  const int64_t sz = size_of(q.dtype), vec = 16 / sz;
  g.R = q.T * q.k;
  g.wide = q.act & GT_ACT_GATED ? 2 * q.H : q.H;
  g.ldd = up(q.D, vec);
  g.ldp = up(g.wide, vec);
  g.ldh = up(q.H, vec);
  g.ldo = up(q.D, 4);
  const bool hidden = q.dX || q.dW1 || q.dW2 || q.db1 || q.dweights;
  Scratch s(ws);
  g.dYs = s.take(g.R * g.ldd * sz);
  if (q.dW1) g.Xs = s.take(g.R * g.ldd * sz);
  if (hidden) {
    g.dP = s.take(g.R * g.ldp * sz);
    g.Hw = s.take(g.R * g.ldh * sz);
  }
  auto common = [&](Product& p, Layout layout) -> ProductArgs& {
    p.dtype = q.dtype;
    p.layout = layout;
    p.a.offsets = q.offsets;
    p.a.groups = q.E;
    p.a.along_k = layout == kXtP ? 1 : 0;
    return p.a;
  };
  if (hidden) {   // dH = dY·W2ᵀ, with what follows from it
    ProductArgs& a = common(g.dh, kPWt);
    a.A = g.dYs;
    a.lda = g.ldd;
    a.B = q.W2;
    a.ldb = q.ldw2;
    a.sB = q.sw2;
    a.M = g.R;
    a.N = q.H;
    a.K = q.D;
    Epilogue& e = a.e;
    e.epi = kEpiSlope;
    e.act = q.act & ~GT_ACT_GATED;
    e.gated = q.act & GT_ACT_GATED ? 1 : 0;
    e.Y = g.dP;
    e.ldy = g.ldp;
    e.P = const_cast<void*>(q.P);
    e.ldp = q.ldp;
    e.Hw = g.Hw;
    e.ldh = g.ldh;
    e.weights = q.weights;
    e.order = q.order;
    e.entries = g.R;
    e.wide = g.wide;
    e.zero_pad = 1;
    g.dh.own_a = true;
    choose(&g.dh, false);
    const TileShape t = tile_shape(q.dtype, g.dh.tile);
    // Σ dH·H of a row's tiles, then b2·dY of its columns' blocks
    g.ndot = static_cast<int64_t>(a.tilesN) * t.NWN;
    g.nb2 = q.b2 && q.dweights ? (g.ldd + 64 * vec - 1) / (64 * vec) : 0;
    e.ldot = g.ndot + g.nb2;
    g.dot = e.dot = s.take<float>(g.R * e.ldot * 4);
    g.colrows = static_cast<int64_t>(a.tilesM) * t.NWM;
    if (q.db1) g.colsum = e.colsum = s.take<float>(g.colrows * g.wide * 4);
  }
  if (q.dW2) {
    ProductArgs& a = common(g.dw2, kXtP);
    a.A = g.Hw;
    a.lda = g.ldh;
    a.B = g.dYs;
    a.ldb = g.ldd;
    a.M = q.H;
    a.N = q.D;
    a.K = g.R;
    output(&a.e, q.dW2, q.D, q.dtype == GT_F32);
    a.e.sY = q.H * q.D;
    g.dw2.own_a = g.dw2.own_b = true;
    choose(&g.dw2, false);
  }
  if (q.dX) {
    ProductArgs& a = common(g.dx, kPWt);
    a.A = g.dP;
    a.lda = g.ldp;
    a.B = q.W1;
    a.ldb = q.ldw1;
    a.sB = q.sw1;
    a.M = g.R;
    a.N = q.D;
    a.K = g.wide;
    g.dXs = s.take<float>(g.R * g.ldo * 4);
    output(&a.e, g.dXs, g.ldo, true);
    g.dx.own_a = true;
    choose(&g.dx, false);
  }
  if (q.dW1) {
    ProductArgs& a = common(g.dw1, kXtP);
    a.A = g.Xs;
    a.lda = g.ldd;
    a.B = g.dP;
    a.ldb = g.ldp;
    a.M = q.D;
    a.N = g.wide;
    a.K = g.R;
    output(&a.e, q.dW1, g.wide, q.dtype == GT_F32);
    a.e.sY = q.D * g.wide;
    g.dw1.own_a = g.dw1.own_b = true;
    choose(&g.dw1, false);
  }
  const int64_t rest = std::max({g.dh.scratch(), g.dw2.scratch(), g.dx.scratch(), g.dw1.scratch()});
  if (rest) g.rest = s.take(rest);
  g.sumrows = g.R / kSortRows + std::min<int64_t>(q.E, g.R);
  if (q.db2) g.sums = s.take<float>(g.sumrows * q.D * 4);
  g.bytes = s.used;
  return g;
}

}  // namespace

hipError_t product_0_0(int, bool, const ProductArgs&, hipStream_t);
hipError_t product_0_1(int, bool, const ProductArgs&, hipStream_t);
hipError_t product_0_2(int, bool, const ProductArgs&, hipStream_t);
hipError_t product_1_0(int, bool, const ProductArgs&, hipStream_t);
hipError_t product_1_1(int, bool, const ProductArgs&, hipStream_t);
hipError_t product_1_2(int, bool, const ProductArgs&, hipStream_t);

hipError_t launch_product(int dtype, int layout, int tile, bool reg, const ProductArgs& a,
                          hipStream_t s) {
  static constexpr decltype(&product_0_0) table[2][3] = {{product_0_0, product_0_1, product_0_2},
                                                         {product_1_0, product_1_1, product_1_2}};
  return table[dtype == GT_BF16 ? 1 : 0][layout](tile, reg, a, s);
}

}  // namespace gt

namespace {

using namespace gt;

int linear_workspace_impl(const gt_linear_args* a, int64_t* bytes) {
  if (!bytes) return fail("gt_linear_workspace: null argument");
  GT_CHECK(linear_checks(a, false));
  *bytes = linear_product(*a).scratch();
  return GT_OK;
}

int linear_impl(const gt_linear_args* a, void* ws, int64_t ws_bytes, void* stream) {
  GT_CHECK(linear_checks(a, true));
  Product p = linear_product(*a);
  GT_CHECK(planned(p));
  GT_CHECK(scratch_ok(ws, ws_bytes, p.scratch()));
  return run(p, ws, static_cast<hipStream_t>(stream));
}

int linear_backward_workspace_impl(const gt_linear_grad_args* a, int64_t* bytes) {
  if (!bytes) return fail("gt_linear_backward_workspace: null argument");
  GT_CHECK(linear_grad_checks(a, false));
  *bytes = linear_grad(*a, nullptr).bytes;
  return GT_OK;
}

int linear_backward_impl(const gt_linear_grad_args* a, void* ws, int64_t ws_bytes, void* stream) {
  GT_CHECK(linear_grad_checks(a, true));
  const hipStream_t s = static_cast<hipStream_t>(stream);
  LinearGrad g = linear_grad(*a, ws);
  for (const Product* p : {&g.dx, &g.dw}) GT_CHECK(planned(*p));
  GT_CHECK(scratch_ok(ws, ws_bytes, g.bytes));
  if (g.dP || a->db) {
    ActGradArgs q{};
    q.M = a->M;
    q.N = a->N;
    q.act = a->act & ~GT_ACT_GATED;
    q.gated = a->act & GT_ACT_GATED ? 1 : 0;
    q.dY = a->dY;
    q.lddy = a->lddy;
    q.P = g.own_dP ? a->P : nullptr;
    q.ldp = a->ldp;
    q.dP = g.dP;
    q.lddp = g.lddp;
    q.part = g.sums;
    q.pad = static_cast<int>(g.lddp - g.wide);
    q.wide = a->N % 8 == 0;
    GT_TRY(launch_act_grad(a->dtype, q, s), "gradient of the activation");
    if (a->db)
      GT_TRY(launch_join(g.sums, (a->M + kActRows - 1) / kActRows, g.wide, nullptr, 1, 0, 1, 1, a->db, s),
             "gradient of the bias");
  }
  if (g.pads) {
    PadJobs jobs{};
    place_pads(g.dx, g.pads, &g.dx.a, &jobs);
    place_pads(g.dw, g.pads + g.dx.pads(), &g.dw.a, &jobs);
    g.dx.pad_a = g.dx.pad_b = g.dw.pad_a = g.dw.pad_b = 0;
    GT_TRY(launch_pad(a->dtype, jobs, s), "copies to aligned rows");
  }
  if (a->dX) GT_CHECK(run(g.dx, g.rest, s));
  if (a->dW) GT_CHECK(run(g.dw, g.rest, s));
  return GT_OK;
}

int route_checks(const gt_route_args* a, bool pointers) {
  if (!a) return fail("gt_route: null arguments");
  GT_CHECK(extent(a->T, 0, "T"));
  if (a->E < 1 || a->E > 1024 || a->groups < 1 || a->E % a->groups != 0 || a->keep < 1 ||
      a->keep > a->groups)
    return fail("gt_route: E is 1 … 1024 in equal groups, keep 1 … groups");
  if (a->k < 1 || a->k > 64 || a->k > a->keep * (a->E / a->groups))
    return fail("gt_route: k is 1 … 64, at most the experts of the kept groups");
  if (a->T * a->k >= kMaxExtent) return fail("gt_route: T·k out of range");
  if (!dtype_ok(a->dtype) || (a->score != GT_SCORE_SOFTMAX && a->score != GT_SCORE_SIGMOID))
    return fail("gt_route: unknown dtype or score");
  if (pointers && (!a->offsets || (a->T > 0 && (!a->logits || !a->weights || !a->experts ||
                                                !a->order || !a->place))))
    return fail("gt_route: null logits or output");
  GT_CHECK(matrix(a->logits, true, a->ldl, a->T, a->E, size_of(a->dtype), "the logits"));
  GT_CHECK(vector(a->bias, 4, "bias"));
  GT_CHECK(vector(a->experts, 4, "experts"));
  return lists(a->weights, a->offsets, a->order, a->place);
}

int route_workspace_impl(const gt_route_args* a, int64_t* bytes) {
  if (!bytes) return fail("gt_route_workspace: null argument");
  GT_CHECK(route_checks(a, false));
  *bytes = route_scratch(a->T, a->E, a->k, a->groups);
  return GT_OK;
}

int route_impl(const gt_route_args* a, void* ws, int64_t ws_bytes, void* stream) {
  GT_CHECK(route_checks(a, true));
  GT_CHECK(scratch_ok(ws, ws_bytes, route_scratch(a->T, a->E, a->k, a->groups)));
  GT_TRY(launch_route(*a, ws, static_cast<hipStream_t>(stream)), "routing");
  return GT_OK;
}

int route_backward_impl(const gt_route_grad_args* a, void* stream) {
  if (!a) return fail("gt_route_backward: null arguments");
  GT_CHECK(extent(a->T, 0, "T"));
  if (a->E < 1 || a->E > 1024 || a->k < 1 || a->k > 64 || a->k > a->E)
    return fail("gt_route_backward: E is 1 … 1024, k 1 … min(64, E)");
  if (!dtype_ok(a->dtype) || (a->score != GT_SCORE_SOFTMAX && a->score != GT_SCORE_SIGMOID))
    return fail("gt_route_backward: unknown dtype or score");
  if (a->T > 0 && (!a->logits || !a->experts || !a->dweights || !a->dlogits))
    return fail("gt_route_backward: null argument");
  const int64_t sz = size_of(a->dtype);
  GT_CHECK(matrix(a->logits, true, a->ldl, a->T, a->E, sz, "the logits"));
  GT_CHECK(matrix(a->dlogits, true, a->lddl, a->T, a->E, sz, "dlogits"));
  GT_CHECK(vector(a->experts, 4, "experts"));
  GT_CHECK(vector(a->dweights, 4, "dweights"));
  GT_TRY(launch_route_grad(*a, static_cast<hipStream_t>(stream)), "gradient of the routing");
  return GT_OK;
}

int experts_workspace_impl(const gt_experts_args* a, int64_t* bytes) {
  if (!bytes) return fail("gt_experts_workspace: null argument");
  GT_CHECK(experts_args_checks(a, false));
  *bytes = experts(*a, nullptr).bytes;
  return GT_OK;
}

int experts_impl(const gt_experts_args* a, void* ws, int64_t ws_bytes, void* stream) {
  GT_CHECK(experts_args_checks(a, true));
  if (a->T == 0) return GT_OK;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  Experts x = experts(*a, ws);
  for (const Product* p : {&x.up, &x.down}) GT_CHECK(planned(*p));
  GT_CHECK(scratch_ok(ws, ws_bytes, x.bytes));
  GT_CHECK(run(x.up, x.rest, s));
  GT_CHECK(run(x.down, x.rest, s));
  CombineArgs c{};
  c.T = a->T;
  c.D = a->D;
  c.entries = a->T * a->k;
  c.k = a->k;
  c.O = x.O;
  c.ldo = x.ldo;
  c.weights = a->weights;
  c.place = a->place;
  c.R = a->R;
  c.ldr = a->ldr;
  c.out = a->Y;
  c.ldout = a->ldy;
  c.wide = a->D % 8 == 0;
  GT_TRY(launch_combine(a->dtype, c, s), "summing the experts' outputs");
  return GT_OK;
}

int experts_backward_workspace_impl(const gt_experts_grad_args* a, int64_t* bytes) {
  if (!bytes) return fail("gt_experts_backward_workspace: null argument");
  GT_CHECK(experts_grad_checks(a, false));
  *bytes = experts_grad(*a, nullptr).bytes;
  return GT_OK;
}

int experts_backward_impl(const gt_experts_grad_args* a, void* ws, int64_t ws_bytes, void* stream) {
  GT_CHECK(experts_grad_checks(a, true));
  const hipStream_t s = static_cast<hipStream_t>(stream);
  ExpertsGrad g = experts_grad(*a, ws);
  for (const Product* p : {&g.dh, &g.dw2, &g.dx, &g.dw1}) GT_CHECK(planned(*p));
  GT_CHECK(scratch_ok(ws, ws_bytes, g.bytes));
  SortArgs q{};
  q.X = a->dW1 ? a->X : nullptr;
  q.dY = a->dY;
  q.b2 = g.nb2 ? a->b2 : nullptr;
  q.ldx = a->ldx;
  q.lddy = a->lddy;
  q.Xs = g.Xs;
  q.dYs = g.dYs;
  q.ldd = g.ldd;
  q.D = a->D;
  q.T = a->T;
  q.entries = g.R;
  q.E = a->E;
  q.k = a->k;
  q.weights = a->weights;
  q.order = a->order;
  q.offsets = a->offsets;
  q.sums = g.sums;
  q.dot = g.dot ? g.dot + g.ndot : nullptr;
  q.ldot = g.ndot + g.nb2;
  GT_TRY(launch_sort(a->dtype, q, s), "sorting the rows");
  if (g.dP) GT_CHECK(run(g.dh, g.rest, s));
  if (a->db1)
    GT_TRY(launch_join(g.colsum, g.colrows, g.wide, a->offsets, a->E, g.R, kTile[g.dh.tile].BM,
                       tile_shape(a->dtype, g.dh.tile).NWM, a->db1, s),
           "gradient of b1");
  if (a->db2)
    GT_TRY(launch_join(g.sums, g.sumrows, a->D, a->offsets, a->E, g.R, kSortRows, 1, a->db2, s),
           "gradient of b2");
  if (a->dweights)
    GT_TRY(launch_weight_grad(g.dot, g.ndot + g.nb2, g.ndot + g.nb2, a->place, a->offsets, a->E, g.R,
                              a->dweights, s),
           "gradient of the weights");
  if (a->dW2) GT_CHECK(run(g.dw2, g.rest, s));
  if (a->dX) {
    GT_CHECK(run(g.dx, g.rest, s));
    CombineArgs c{};
    c.T = a->T;
    c.D = a->D;
    c.entries = g.R;
    c.k = a->k;
    c.O = g.dXs;
    c.ldo = g.ldo;
    c.place = a->place;
    c.out = a->dX;
    c.ldout = a->lddx;
    c.wide = a->D % 8 == 0;
    GT_TRY(launch_combine(a->dtype, c, s), "summing the experts' gradients");
  }
  if (a->dW1) GT_CHECK(run(g.dw1, g.rest, s));
  return GT_OK;
}

}  // namespace

extern "C" {

int gt_linear_workspace(const gt_linear_args* a, int64_t* bytes) {
  return guarded([&] { return linear_workspace_impl(a, bytes); });
}
int gt_linear(const gt_linear_args* a, void* ws, int64_t ws_bytes, void* stream) {
  return guarded([&] { return linear_impl(a, ws, ws_bytes, stream); });
}
int gt_linear_backward_workspace(const gt_linear_grad_args* a, int64_t* bytes) {
  return guarded([&] { return linear_backward_workspace_impl(a, bytes); });
}
int gt_linear_backward(const gt_linear_grad_args* a, void* ws, int64_t ws_bytes, void* stream) {
  return guarded([&] { return linear_backward_impl(a, ws, ws_bytes, stream); });
}
int gt_route_workspace(const gt_route_args* a, int64_t* bytes) {
  return guarded([&] { return route_workspace_impl(a, bytes); });
}
int gt_route(const gt_route_args* a, void* ws, int64_t ws_bytes, void* stream) {
  return guarded([&] { return route_impl(a, ws, ws_bytes, stream); });
}
int gt_route_backward(const gt_route_grad_args* a, void* stream) {
  return guarded([&] { return route_backward_impl(a, stream); });
}
int gt_experts_workspace(const gt_experts_args* a, int64_t* bytes) {
  return guarded([&] { return experts_workspace_impl(a, bytes); });
}
int gt_experts(const gt_experts_args* a, void* ws, int64_t ws_bytes, void* stream) {
  return guarded([&] { return experts_impl(a, ws, ws_bytes, stream); });
}
int gt_experts_backward_workspace(const gt_experts_grad_args* a, int64_t* bytes) {
  return guarded([&] { return experts_backward_workspace_impl(a, bytes); });
}
int gt_experts_backward(const gt_experts_grad_args* a, void* ws, int64_t ws_bytes, void* stream) {
  return guarded([&] { return experts_backward_impl(a, ws, ws_bytes, stream); });
}

}  // extern "C"
