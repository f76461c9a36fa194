// The layer operators' entry points: checks of the arguments, the choice of a
// tile and of K slices for every product, and the launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <string>

#include "gemmtune_layers.h"
#include "internal.h"
#include "layer_kernels.h"
#include "product_args.h"

namespace gt {
namespace {

constexpr int64_t kMaxExtent = int64_t{1} << 31;

int fail(const std::string& what) {
  set_error(what);
  return GT_EINVAL;
}
int hip_fail(hipError_t e, const char* what) {
  set_error(std::string(what) + ": " + hipGetErrorString(e));
  return GT_EHIP;
}
#define GT_TRY(call, what)                              \
  do {                                                  \
    const hipError_t e_ = (call);                       \
    if (e_ != hipSuccess) return hip_fail(e_, what);    \
  } while (0)

int64_t size_of(int dtype) { return dtype == GT_BF16 ? 2 : 4; }
bool dtype_ok(int d) { return d == GT_F32 || d == GT_BF16; }
bool act_ok(int a) { return (a & ~(GT_ACT_GATED | 3)) == 0; }
bool aligned(const void* p, int64_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
int64_t up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }
// An array inside the caller's scratch, 256-byte aligned.
struct Scratch {
  char* base;
  int64_t used = 0;
  explicit Scratch(void* p) : base(static_cast<char*>(p)) {}
  template <typename T = void>
  T* take(int64_t bytes) {
    const int64_t at = used;
    used += up(bytes, 256);
    return reinterpret_cast<T*>(base + at);
  }
};

// ---- one product: its tile, its K slices, its launches

struct Product {
  ProductArgs a{};
  int dtype = GT_F32, layout = kXW;
  int tile = 1;
  bool reg = false;
  int64_t part = 0;      // bytes of partial sums
};

// Whether the 16-byte loads serve both operands: rows of whole aligned chunks,
// and what one descriptor must reach of them within its range.
bool chunks_serve(const Product& p) {
  const ProductArgs& a = p.a;
  const int64_t sz = size_of(p.dtype), vec = 16 / sz;
  const int64_t reach = int64_t{1} << 31;
  const int64_t wide = a.e.epi == kEpiGated ? 2 * a.N : a.N;
  if (!aligned(a.A, 16) || !aligned(a.B, 16) || a.lda % vec || a.ldb % vec || a.sB % vec) return false;
  const bool ax = p.layout == kXtP, bx = p.layout != kPWt;
  if ((ax ? a.M : a.K) % vec || (bx ? wide : a.K) % vec || (wide != a.N && a.N % vec)) return false;
  if ((ax ? 64 : a.gather ? a.a_rows : 256) * a.lda * sz >= reach) return false;
  return (bx ? 64 : 256) * a.ldb * sz < reach;
}

// Tile and K slices by the time they should take. A stage of a tile (128 bytes
// of k) costs a compute unit the larger of its MFMAs and of its operands' way
// into LDS; workgroups beyond one per compute unit queue up; a K slice adds its
// partial sums' way through memory and the launch that joins them.
void choose(Product* p, bool may_split) {
  ProductArgs& a = p->a;
  const int64_t bk = 128 / size_of(p->dtype);
  const int64_t wide = a.e.epi == kEpiGated ? 2 * a.N : a.N;
  p->reg = !chunks_serve(*p);
  const int64_t stages = std::max<int64_t>(1, (a.along_k ? a.K / std::max(1, a.groups) : a.K) / bk);
  double best = 0.0;
  for (int t = 0; t < kTiles; ++t) {
    const TileShape& s = kTile[t];
    if (t == 0 && (p->dtype != GT_BF16 || p->reg)) continue;
    if (t == 3 && p->layout == kXtP) continue;
    const int64_t tn = (wide + s.BN - 1) / s.BN;
    int64_t tm = (a.M + s.BM - 1) / s.BM;
    int64_t most = tm;
    if (a.groups > 0 && !a.along_k) {
      const int64_t g = std::min<int64_t>(a.groups, a.M);
      most = a.M / s.BM + g;
      const int64_t each = (a.M + g - 1) / std::max<int64_t>(1, g);
      tm = g * ((each + s.BM - 1) / s.BM);
    }
    const int64_t tiles = tm * tn * (a.along_k ? a.groups : 1);
    if (most * tn >= kMaxExtent) continue;
    // cycles of a stage: 4096 (bf16) or 256 (fp32) operations a cycle at 60 %,
    // 24 operand bytes a cycle
    const double ops = 2.0 * s.BM * s.BN * bk;
    const double stage = std::max(ops / (p->dtype == GT_BF16 ? 4096 * 0.6 : 256 * 0.8),
                                  (s.BM + s.BN) * 128.0 / 24);
    for (int64_t z = 1; z <= 64; z *= 2) {
      if (z > 1 && (!may_split || stages / z < 4)) break;
      const int64_t queue = (tiles * z + 255) / 256;
      double cost = queue * (((stages + z - 1) / z + 2) * stage) + 2000;
      if (z > 1) cost += 6000 + 2.0 * z * a.M * wide * 4 / 1700;   // bytes at 4 TB/s, in cycles
      if (best == 0.0 || cost < best) {
        best = cost;
        p->tile = t;
        a.splits = static_cast<int>(z);
        a.tilesM = static_cast<int>(most);
        a.tilesN = static_cast<int>(tn);
      }
    }
  }
  a.e.ldpart = up(a.N, 4) * (wide == a.N ? 1 : 2);
  const int64_t all = (a.K + bk - 1) / bk;
  a.per_slice = static_cast<int>((all + a.splits - 1) / std::max(1, a.splits));
  p->part = a.splits > 1 ? a.splits * a.M * a.e.ldpart * 4 : 0;
}

int run(Product& p, float* part, hipStream_t s) {
  ProductArgs a = p.a;
  if (a.M == 0) return GT_OK;
  if (a.splits < 1) return fail("layer product: too many tiles");
  if (a.splits > 1) {
    a.e.epi = kEpiPart;
    a.e.part = part;
  }
  GT_TRY(launch_product(p.dtype, p.layout, p.tile, p.reg, a, s), "layer product");
  if (a.splits > 1) GT_TRY(launch_reduce(p.dtype, a, s), "joining the K slices");
  return GT_OK;
}

// Rows of n elements of sz bytes (pointer and leading dimension; null: none): 2
// if all take accesses of 8 elements, 1 of 4, 0 of one.
int width(int64_t n, std::initializer_list<std::pair<const void*, int64_t>> rows, int64_t sz) {
  for (int w = 2; w >= 1; --w) {
    const int64_t e = 4 * w, bytes = std::min<int64_t>(16, e * sz);
    bool ok = n % e == 0;
    for (const auto& r : rows) ok = ok && (!r.first || (aligned(r.first, bytes) && r.second % e == 0));
    if (ok) return w;
  }
  return 0;
}

int extent(int64_t v, int64_t least, const char* name) {
  if (v < least || v >= kMaxExtent) return fail(std::string(name) + " out of range");
  return GT_OK;
}
int row(const void* p, int64_t ld, int64_t cols, const char* name) {
  if (p && ld < cols) return fail(std::string("leading dimension of ") + name + " below its row");
  if (p && ld >= kMaxExtent) return fail(std::string("leading dimension of ") + name + " too large");
  return GT_OK;
}
int scratch_ok(const void* ws, int64_t have, int64_t need) {
  if (need == 0) return GT_OK;
  if (have < need) {
    set_error("workspace of " + std::to_string(have) + " bytes, " + std::to_string(need) + " needed");
    return GT_ESMALL;
  }
  if (!ws || !aligned(ws, 256)) return fail("workspace must be 256-byte aligned device memory");
  return GT_OK;
}
#define GT_CHECK(call)          \
  do {                          \
    const int rc_ = (call);     \
    if (rc_ != GT_OK) return rc_; \
  } while (0)

// ---- linear

int linear_checks(const gt_linear_args* a, bool pointers) {
  if (!a) return fail("gt_linear: null arguments");
  GT_CHECK(extent(a->M, 0, "M"));
  GT_CHECK(extent(a->N, 1, "N"));
  GT_CHECK(extent(a->K, 1, "K"));
  if (!dtype_ok(a->dtype) || !dtype_ok(a->out_dtype) || !act_ok(a->act))
    return fail("gt_linear: unknown dtype or activation");
  const int64_t wide = a->act & GT_ACT_GATED ? 2 * a->N : a->N;
  GT_CHECK(extent(wide, 1, "2N"));
  if (pointers && a->M > 0 && (!a->X || !a->W || !a->Y)) return fail("gt_linear: null X, W or Y");
  if (a->out_dtype != a->dtype && a->R == a->Y && a->R)
    return fail("gt_linear: R may be Y only in the same type");
  GT_CHECK(row(a->X, a->ldx, a->K, "X"));
  GT_CHECK(row(a->W, a->ldw, wide, "W"));
  GT_CHECK(row(a->R, a->ldr, a->N, "R"));
  GT_CHECK(row(a->Y, a->ldy, a->N, "Y"));
  return row(a->P, a->ldp, wide, "P");
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
  e.vec = std::min(width(q.N, {{q.P, q.ldp}, {q.bias, 0}, {q.R, q.ldr}}, size_of(q.dtype)),
                   width(q.N, {{q.Y, q.ldy}}, size_of(q.out_dtype)));
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
  const int64_t wide = a->act & GT_ACT_GATED ? 2 * a->N : a->N;
  GT_CHECK(extent(wide, 1, "2N"));
  if (pointers && a->M > 0) {
    if (!a->dY) return fail("gt_linear_backward: null dY");
    if (a->act != GT_ACT_NONE && !a->P) return fail("gt_linear_backward: the activation needs P");
    if ((a->dX && !a->W) || (a->dW && !a->X))
      return fail("gt_linear_backward: dX needs W, dW needs X");
  }
  GT_CHECK(row(a->dY, a->lddy, a->N, "dY"));
  GT_CHECK(row(a->X, a->ldx, a->K, "X"));
  GT_CHECK(row(a->W, a->ldw, wide, "W"));
  GT_CHECK(row(a->act != GT_ACT_NONE ? a->P : nullptr, a->ldp, wide, "P"));
  GT_CHECK(row(a->dX, a->lddx, a->K, "dX"));
  return row(a->dW, a->lddw, wide, "dW");
}

struct LinearGrad {
  bool own_dP = false;    // dP is not dY itself
  int64_t lddp = 0, wide = 0;
  Product dx, dw;
  // scratch
  void* dP = nullptr;
  float *part = nullptr, *sums = nullptr;
  int64_t bytes = 0;
};

void output(Epilogue* e, void* y, int64_t ldy, bool f32, int64_t n, int64_t sz) {
  e->epi = kEpiPlain;
  e->Y = y;
  e->ldy = ldy;
  e->out_f32 = f32 ? 1 : 0;
  e->vec = width(n, {{y, ldy}}, f32 ? 4 : sz);
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
  int64_t part = 0;
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
    output(&a.e, q.dX, q.lddx, q.dtype == GT_F32, q.K, sz);
    choose(&g.dx, true);
    part = std::max(part, g.dx.part);
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
    output(&a.e, q.dW, q.lddw, q.dw_dtype == GT_F32, g.wide, sz);
    choose(&g.dw, true);
    part = std::max(part, g.dw.part);
  }
  if (part) g.part = s.take<float>(part);
  g.bytes = s.used;
  return g;
}

// ---- experts

int experts_checks(int64_t T, int64_t D, int64_t H, int E, int k, int dtype, int act) {
  GT_CHECK(extent(T, 0, "T"));
  GT_CHECK(extent(D, 1, "D"));
  GT_CHECK(extent(act & GT_ACT_GATED ? 2 * H : H, 1, "H"));
  if (E < 1 || E > 1024 || k < 1 || k > 64) return fail("experts: E is 1 … 1024, k 1 … 64");
  if (T * k >= kMaxExtent) return fail("experts: T·k out of range");
  if (!dtype_ok(dtype) || !act_ok(act)) return fail("experts: unknown dtype or activation");
  return GT_OK;
}

int experts_args_checks(const gt_experts_args* a, bool pointers) {
  if (!a) return fail("gt_experts: null arguments");
  GT_CHECK(experts_checks(a->T, a->D, a->H, a->E, a->k, a->dtype, a->act));
  const int64_t wide = a->act & GT_ACT_GATED ? 2 * a->H : a->H;
  if (pointers && a->T > 0 &&
      (!a->X || !a->W1 || !a->W2 || !a->Y || !a->weights || !a->offsets || !a->order || !a->place))
    return fail("gt_experts: null X, W1, W2, Y or list");
  GT_CHECK(row(a->X, a->ldx, a->D, "X"));
  GT_CHECK(row(a->W1, a->ldw1, wide, "W1"));
  GT_CHECK(row(a->W2, a->ldw2, a->D, "W2"));
  GT_CHECK(row(a->R, a->ldr, a->D, "R"));
  GT_CHECK(row(a->Y, a->ldy, a->D, "Y"));
  if (a->sw1 < 0 || a->sw2 < 0) return fail("gt_experts: negative stride between experts");
  return row(a->P, a->ldp, wide, "P");
}

struct Experts {
  Product up, down;
  void* H = nullptr;
  float *O = nullptr, *part = nullptr;
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
  {   // the rows' tokens are read from X where they lie
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
    e.vec = width(q.H, {{q.P, q.ldp}, {q.b1, 0}, {x.H, ldh}}, sz);
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
    e.vec = std::min(width(q.D, {{q.b2, 0}}, sz), width(q.D, {{x.O, x.ldo}}, 4));
    choose(&x.down, true);
  }
  const int64_t part = std::max(x.up.part, x.down.part);
  if (part) x.part = s.take<float>(part);
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
  GT_CHECK(row(a->dY, a->lddy, a->D, "dY"));
  GT_CHECK(row(a->X, a->ldx, a->D, "X"));
  GT_CHECK(row(a->W1, a->ldw1, wide, "W1"));
  GT_CHECK(row(a->W2, a->ldw2, a->D, "W2"));
  GT_CHECK(row(a->P, a->ldp, wide, "P"));
  if (a->sw1 < 0 || a->sw2 < 0) return fail("gt_experts_backward: negative stride between experts");
  return row(a->dX, a->lddx, a->D, "dX");
}

struct ExpertsGrad {
  int64_t R, wide, ldd, ldp, ldh, ldo;
  Product dh, dw2, dx, dw1;
  void *Xs = nullptr, *dYs = nullptr, *dP = nullptr, *Hw = nullptr;
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
    e.vec = width(q.H, {{q.P, q.ldp}, {g.dP, g.ldp}, {g.Hw, g.ldh}}, sz);
    choose(&g.dh, false);
    const TileShape& t = kTile[g.dh.tile];
    e.ldot = static_cast<int64_t>(a.tilesN) * t.NWN;
    g.dot = e.dot = s.take<float>(g.R * e.ldot * 4);
    if (q.db1) g.colsum = e.colsum = s.take<float>(static_cast<int64_t>(a.tilesM) * t.NWM * g.wide * 4);
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
    output(&a.e, q.dW2, q.D, q.dtype == GT_F32, q.D, sz);
    a.e.sY = q.H * q.D;
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
    output(&a.e, g.dXs, g.ldo, true, q.D, sz);
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
    output(&a.e, q.dW1, g.wide, q.dtype == GT_F32, g.wide, sz);
    a.e.sY = q.D * g.wide;
    choose(&g.dw1, false);
  }
  if (q.db2) g.sums = s.take<float>((g.R / kSumRows + std::min<int64_t>(q.E, g.R)) * q.D * 4);
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

using namespace gt;

extern "C" {

int gt_linear_workspace(const gt_linear_args* a, int64_t* bytes) {
  if (!bytes) return fail("gt_linear_workspace: null argument");
  GT_CHECK(linear_checks(a, false));
  *bytes = linear_product(*a).part;
  return GT_OK;
}

int gt_linear(const gt_linear_args* a, void* ws, int64_t ws_bytes, void* stream) {
  GT_CHECK(linear_checks(a, true));
  Product p = linear_product(*a);
  GT_CHECK(scratch_ok(ws, ws_bytes, p.part));
  return run(p, static_cast<float*>(ws), static_cast<hipStream_t>(stream));
}

int gt_linear_backward_workspace(const gt_linear_grad_args* a, int64_t* bytes) {
  if (!bytes) return fail("gt_linear_backward_workspace: null argument");
  GT_CHECK(linear_grad_checks(a, false));
  *bytes = linear_grad(*a, nullptr).bytes;
  return GT_OK;
}

int gt_linear_backward(const gt_linear_grad_args* a, void* ws, int64_t ws_bytes, void* stream) {
  GT_CHECK(linear_grad_checks(a, true));
  const hipStream_t s = static_cast<hipStream_t>(stream);
  LinearGrad g = linear_grad(*a, ws);
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
    q.vec = width(a->N, {{a->dY, a->lddy}, {q.P, a->ldp}, {g.dP, g.lddp}}, size_of(a->dtype));
    GT_TRY(launch_act_grad(a->dtype, q, s), "gradient of the activation");
    if (a->db)
      GT_TRY(launch_join(g.sums, (a->M + kActRows - 1) / kActRows, g.wide, nullptr, 1, 0, 1, 1, a->db, s),
             "gradient of the bias");
  }
  if (a->dX) GT_CHECK(run(g.dx, g.part, s));
  if (a->dW) GT_CHECK(run(g.dw, g.part, s));
  return GT_OK;
}

int gt_route_workspace(const gt_route_args* a, int64_t* bytes) {
  if (!a || !bytes) return fail("gt_route_workspace: null argument");
  if (a->T < 0 || a->T >= kMaxExtent || a->E < 1 || a->E > 1024 || a->k < 1 || a->k > 64)
    return fail("gt_route: T, E or k out of range");
  *bytes = route_scratch(a->T, a->E, a->k, a->groups);
  return GT_OK;
}

int gt_route(const gt_route_args* a, void* ws, int64_t ws_bytes, void* stream) {
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
  if (!a->offsets ||
      (a->T > 0 && (!a->logits || !a->weights || !a->experts || !a->order || !a->place)))
    return fail("gt_route: null logits or output");
  GT_CHECK(row(a->logits, a->ldl, a->E, "the logits"));
  GT_CHECK(scratch_ok(ws, ws_bytes, route_scratch(a->T, a->E, a->k, a->groups)));
  GT_TRY(launch_route(*a, ws, static_cast<hipStream_t>(stream)), "routing");
  return GT_OK;
}

int gt_route_backward(const gt_route_grad_args* a, void* stream) {
  if (!a) return fail("gt_route_backward: null arguments");
  GT_CHECK(extent(a->T, 0, "T"));
  if (a->E < 1 || a->E > 1024 || a->k < 1 || a->k > 64 || a->k > a->E)
    return fail("gt_route_backward: E is 1 … 1024, k 1 … min(64, E)");
  if (!dtype_ok(a->dtype) || (a->score != GT_SCORE_SOFTMAX && a->score != GT_SCORE_SIGMOID))
    return fail("gt_route_backward: unknown dtype or score");
  if (a->T > 0 && (!a->logits || !a->experts || !a->dweights || !a->dlogits))
    return fail("gt_route_backward: null argument");
  GT_CHECK(row(a->logits, a->ldl, a->E, "the logits"));
  GT_CHECK(row(a->dlogits, a->lddl, a->E, "dlogits"));
  GT_TRY(launch_route_grad(*a, static_cast<hipStream_t>(stream)), "gradient of the routing");
  return GT_OK;
}

int gt_experts_workspace(const gt_experts_args* a, int64_t* bytes) {
  if (!bytes) return fail("gt_experts_workspace: null argument");
  GT_CHECK(experts_args_checks(a, false));
  *bytes = experts(*a, nullptr).bytes;
  return GT_OK;
}

int gt_experts(const gt_experts_args* a, void* ws, int64_t ws_bytes, void* stream) {
  GT_CHECK(experts_args_checks(a, true));
  if (a->T == 0) return GT_OK;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  Experts x = experts(*a, ws);
  GT_CHECK(scratch_ok(ws, ws_bytes, x.bytes));
  GT_CHECK(run(x.up, x.part, s));
  GT_CHECK(run(x.down, x.part, s));
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
  c.vec = width(a->D, {{a->R, a->ldr}, {a->Y, a->ldy}}, size_of(a->dtype));
  GT_TRY(launch_combine(a->dtype, c, s), "summing the experts' outputs");
  return GT_OK;
}

int gt_experts_backward_workspace(const gt_experts_grad_args* a, int64_t* bytes) {
  if (!bytes) return fail("gt_experts_backward_workspace: null argument");
  GT_CHECK(experts_grad_checks(a, false));
  *bytes = experts_grad(*a, nullptr).bytes;
  return GT_OK;
}

int gt_experts_backward(const gt_experts_grad_args* a, void* ws, int64_t ws_bytes, void* stream) {
  GT_CHECK(experts_grad_checks(a, true));
  const hipStream_t s = static_cast<hipStream_t>(stream);
  ExpertsGrad g = experts_grad(*a, ws);
  GT_CHECK(scratch_ok(ws, ws_bytes, g.bytes));
  GT_TRY(launch_gather(a->dtype, a->dW1 ? a->X : nullptr, a->ldx, g.Xs, a->dY, a->lddy, g.dYs, g.ldd,
                       a->D, a->order, a->offsets, a->E, g.R, a->k, a->T, s),
         "sorting the rows");
  if (g.dP) GT_CHECK(run(g.dh, nullptr, s));
  if (a->db1)
    GT_TRY(launch_join(g.colsum, 0, g.wide, a->offsets, a->E, g.R, kTile[g.dh.tile].BM,
                       kTile[g.dh.tile].NWM, a->db1, s),
           "gradient of b1");
  if (a->db2) {
    GT_TRY(launch_weighted_sums(a->dtype, g.dYs, g.ldd, a->D, a->weights, a->order, g.R, a->offsets,
                                a->E, g.sums, s),
           "gradient of b2");
    GT_TRY(launch_join(g.sums, 0, a->D, a->offsets, a->E, g.R, kSumRows, 1, a->db2, s),
           "gradient of b2");
  }
  if (a->dweights) {
    WeightGradArgs w{};
    w.entries = g.R;
    w.D = a->D;
    w.E = a->E;
    w.dot = g.dot;
    w.ldot = g.dh.a.e.ldot;
    w.place = a->place;
    w.offsets = a->offsets;
    w.rows = g.dYs;
    w.ld = g.ldd;
    w.b2 = a->b2;
    w.dweights = a->dweights;
    GT_TRY(launch_weight_grad(a->dtype, w, s), "gradient of the weights");
  }
  if (a->dW2) GT_CHECK(run(g.dw2, nullptr, s));
  if (a->dX) {
    GT_CHECK(run(g.dx, nullptr, s));
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
    c.vec = width(a->D, {{a->dX, a->lddx}}, size_of(a->dtype));
    GT_TRY(launch_combine(a->dtype, c, s), "summing the experts' gradients");
  }
  if (a->dW1) GT_CHECK(run(g.dw1, nullptr, s));
  return GT_OK;
}

}  // extern "C"
