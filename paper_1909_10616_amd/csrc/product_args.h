// Arguments of the layer products and their launch.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace gt {

// What becomes of the product's rows; each is a kernel of its own, so that none carries
// the others' code (a launch fetches its instructions cold).
enum Epi : int {
  kEpiPlain = 0,   // Y alone
  kEpiPart = 1,    // a K slice's sums, as they are, into `part`
  kEpiLinear = 2,  // + bias, activation, + residual, P kept
  kEpiGated = 3,   // the same with a gate and an up half
  kEpiSlope = 4,   // the product is dH of the experts: dP, w·H, Σ dH·H, column sums of dP
};

struct Epilogue {
  int32_t epi;
  int32_t act;       // gt_act
  int32_t gated;     // columns n and N + n are a gate and its up value
  int32_t out_f32;   // Y in fp32, else in the operands' type
  int32_t zero_pad;  // columns of Y from N to the next 16 bytes are written as zero
  void* Y;           // [rows][ldy]; group g at Y + g·sY (groups along k)
  int64_t ldy, sY;
  void* P;           // kept pre-activations or the given ones (kEpiSlope), or null
  int64_t ldp;
  const void* bias;  // per group sbias apart
  int64_t sbias;
  const void* R;
  int64_t ldr;
  float* part;       // [slice][row][ldpart]: columns n, and ldpart/2 + n for up values
  int64_t ldpart;
  // kEpiSlope
  void* Hw;               // [row][ldh]: w·act(P)
  int64_t ldh;
  const float* weights;   // of entry order[row]
  const int32_t* order;
  int64_t entries;        // entries of `order` and `weights`
  float* dot;             // [row][ldot]: Σ over a wavefront's columns of dH·H
  int64_t ldot;
  float* colsum;          // [tile row·WAVES_M + wave row][wide]: sums of dP over its rows
  int64_t wide;
};

struct ProductArgs {
  const void* A;
  const void* B;
  int64_t lda, ldb;     // elements between stored rows
  int64_t M, N, K;      // N: columns of Y
  int64_t half;         // gated: columns of B before the up half's first
  const int32_t* offsets;  // group g: rows (or k) offsets[g] … offsets[g + 1] − 1
  int32_t groups;       // 0: no groups
  int32_t along_k;      // groups along k
  int64_t sB;           // elements between the groups' B
  const int32_t* gather;   // KC A: row r is A's row gather[r] / gather_div
  int32_t gather_div;
  int32_t splits;       // K slices (grid y)
  int32_t per_slice;    // stages of a slice
  int64_t a_rows;       // rows A has (gather)
  int32_t tilesM, tilesN;
  float* tail;          // sums of K slices of the last tiles, or null: see Tail
  Epilogue e;
};

// The large tiles that are left when the compute units have had the same number each would keep a few of them busy for as long again. They are cut into K slices
// instead, as many as the units take at once (at most kTailSlices, and no fewer than 4
// stages each); their sums go to `tail`, [tile of the left][slice][BM][BN], and a
// launch of its own joins them. The kernel finds out itself, since with groups
// the host does not know the tiles.
constexpr int kUnits = 256;
constexpr int kTailSlices = 8;
struct Tail {
  int full, left, slices;   // whole tiles, tiles in slices, slices of each (1: whole too)
};
__host__ __device__ inline Tail tail_of(int tiles, int stages) {
  Tail t{tiles / kUnits * kUnits, tiles % kUnits, 1};
  if (t.left > 0) {
    t.slices = kUnits / t.left;
    if (t.slices > kTailSlices) t.slices = kTailSlices;
    if (t.slices > stages / 4) t.slices = stages / 4;
    if (t.slices < 1) t.slices = 1;
  }
  return t;
}

// How the operands lie: A and B along k or along their own index.
enum Layout : int { kXW = 0, kPWt = 1, kXtP = 2 };  // KC·XC, KC·KC, XC·XC

// The tiles that are built: rows, columns, wavefronts along each, bytes of k in a stage,
// ring slots, MFMA size.
struct TileShape {
  int BM, BN, NWM, NWN, KB, NS, I;
};
constexpr int kTiles = 4;
constexpr TileShape kTile[kTiles] = {
    {256, 256, 2, 4, 128, 2, 32},  // 0: bf16, DMA only
    {128, 128, 2, 2, 128, 2, 32},  // 1: DMA only
    {64, 64, 2, 2, 128, 3, 16},    // 2
    {16, 128, 1, 4, 128, 4, 16},   // 3: not for kXtP
};
// In fp32 two wavefronts a SIMD hide the small tile's barriers behind each other's MFMAs
// (dX of 1000×1024×1024 29.0 → 26.8 µs, 64×4096×4096 in one slice 103 → 92); in bf16, with
// an eighth of the MFMA time, they gain here and lose there.
constexpr TileShape tile_shape(int dtype, int tile) {
  TileShape t = kTile[tile];
  if (dtype == 0 && tile == 2) t.NWM = 4;
  return t;
}

// Launches the product kernel of a tile (reg: the register path) with the epilogue
// a.e.epi: kXW has kEpiPart, kEpiLinear and kEpiGated, kPWt kEpiPlain, kEpiPart and
// kEpiSlope, kXtP kEpiPlain and kEpiPart. The grid is (tilesM·tilesN, splits, groups
// along k or 1).
hipError_t launch_product(int dtype, int layout, int tile, bool reg, const ProductArgs& a,
                          hipStream_t s);

// Joins the K slices of the last tiles (a.tail) with the epilogue a.e.epi.
hipError_t launch_tail(int dtype, int tile, const ProductArgs& a, hipStream_t s);

// The product of a few rows (1, 2 or 4 a workgroup; of a group, with groups along m) with a
// matrix, kXW with kEpiLinear or kEpiGated, in one launch: tilesN of 64 columns, tilesM of
// `rows` rows. The LDS it takes holds the rows.
constexpr int kRowThreads = 1024;
int64_t rows_lds(int64_t K, int rows, bool gated);
hipError_t launch_rows(int dtype, int rows, const ProductArgs& a, hipStream_t s);
constexpr int slim_waves(bool gated) { return gated ? 8 : 16; }   // (as registers allow)
bool slim_aligned(int dtype, const ProductArgs& a);
hipError_t launch_slim(int dtype, const ProductArgs& a, hipStream_t s);

}  // namespace gt
