// Checks of arguments, errors and scratch memory, as all layer operators' entry points have them.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <exception>
#include <string>

#include "gemmtune_layers.h"
#include "internal.h"

namespace gt {

constexpr int64_t kMaxExtent = int64_t{1} << 31;
constexpr int64_t kMaxEntries = int64_t{1} << 29;    // rows of experts: counted by tiles of them in 32 bits
constexpr int64_t kMaxElements = int64_t{1} << 45;   // of one array: no size below leaves 64 bits

inline int fail(const std::string& what) {
  set_error(what);
  return GT_EINVAL;
}
inline int hip_fail(hipError_t e, const char* what) {
  set_error(std::string(what) + ": " + hipGetErrorString(e));
  return GT_EHIP;
}
#define GT_TRY(call, what)                              \
  do {                                                  \
    const hipError_t e_ = (call);                       \
    if (e_ != hipSuccess) return hip_fail(e_, what);    \
  } while (0)

inline int64_t size_of(int dtype) { return dtype == GT_BF16 ? 2 : 4; }
inline bool dtype_ok(int d) { return d == GT_F32 || d == GT_BF16; }
// What the epilogues store: the operands' type, or fp32.
inline bool out_ok(int out, int dtype) { return out == dtype || out == GT_F32; }
inline bool act_ok(int a) { return (a & ~(GT_ACT_GATED | 3)) == 0; }
inline bool aligned(const void* p, int64_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
inline int64_t up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }
// An array inside the caller's scratch, 256-byte aligned.
struct Scratch {
  uintptr_t base;   // (0 in a query)
  int64_t used = 0;
  explicit Scratch(void* p) : base(reinterpret_cast<uintptr_t>(p)) {}
  template <typename T = void>
  T* take(int64_t bytes) {
    const int64_t at = used;
    used += up(bytes, 256);
    return reinterpret_cast<T*>(base + at);
  }
};

inline int extent(int64_t v, int64_t least, const char* name) {
  if (v < least || v >= kMaxExtent) return fail(std::string(name) + " out of range");
  return GT_OK;
}
// A matrix that is there, or has to be (needed): rows of cols, ld apart, of sz-byte elements.
inline int matrix(const void* p, bool needed, int64_t ld, int64_t rows, int64_t cols, int64_t sz,
                  const char* name) {
  if (!p && !needed) return GT_OK;
  if (ld < cols) return fail(std::string("leading dimension of ") + name + " below its row");
  if (ld >= kMaxExtent || rows > kMaxElements / ld)
    return fail(std::string(name) + " is too large");
  if (!aligned(p, sz)) return fail(std::string(name) + " is not aligned to its elements");
  return GT_OK;
}
inline int vector(const void* p, int64_t sz, const char* name) {
  return aligned(p, sz) ? GT_OK : fail(std::string(name) + " is not aligned to its elements");
}
inline int scratch_ok(const void* ws, int64_t have, int64_t need) {
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

// Messages allocate host memory: no C++ exception crosses the C ABI.
template <class F>
inline int guarded(F f) {
  try {
    return f();
  } catch (const std::exception&) {
    return GT_EINVAL;
  }
}

}  // namespace gt
