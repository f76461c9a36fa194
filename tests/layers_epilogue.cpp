// Parts of the layer products' epilogue, run on the CPU a lane at a time over arrays that end
// where the memory that may be touched ends: an access beyond them is a segmentation fault.
//   layers_epilogue part
#include <sys/mman.h>
#include <unistd.h>

#include <cstdio>
#include <cstring>
#include <vector>

#include "product.hpp"

using namespace gt;

namespace {

// n values of T, the last one right before a page that cannot be accessed.
template <typename T>
struct Fenced {
  T* p;
  explicit Fenced(int64_t n) {
    const int64_t page = sysconf(_SC_PAGESIZE), bytes = n * static_cast<int64_t>(sizeof(T));
    const int64_t whole = (bytes + page - 1) / page * page;
    void* m = mmap(nullptr, whole + page, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0);
    if (m == MAP_FAILED || mprotect(static_cast<char*>(m) + whole, page, PROT_NONE) != 0) _exit(2);
    p = reinterpret_cast<T*>(static_cast<char*>(m) + whole - bytes);
  }
};

int failed(const char* what, int64_t N, int64_t at, float got, float want) {
  std::printf("%s, N = %lld: cell %lld holds %g, not %g\n", what, static_cast<long long>(N),
              static_cast<long long>(at), got, want);
  return 1;
}

// Every quad that the kernels of a few rows come to, the padding's too, column by column: all
// cells hold their own sums in the end, and none past the last is written.
template <bool G>
int parts(int64_t N) {
  const int64_t rows = 3, slices = 2, half = (N + 3) / 4 * 4, ld = half * (G ? 2 : 1);
  ProductArgs a{};
  a.M = rows;
  a.N = N;
  a.e.ldpart = ld;
  const Fenced<float> part(slices * rows * ld);
  a.e.part = part.p;
  for (int64_t c = 0; c < N + 8; c += 4)
    for (int z = 0; z < slices; ++z)
      for (int64_t row = 0; row < rows; ++row) {
        f32x4 v, u;
        for (int i = 0; i < 4; ++i) {
          v[i] = static_cast<float>(1 + (z * rows + row) * ld + c + i);
          u[i] = static_cast<float>(1 + (z * rows + row) * ld + half + c + i);
        }
        part_quad<G>(a, z, row, c, v, u);
      }
  for (int64_t i = 0; i < slices * rows * ld; ++i)
    if (part.p[i] != static_cast<float>(1 + i))
      return failed(G ? "gated slices" : "slices", N, i, part.p[i], static_cast<float>(1 + i));
  return 0;
}

}  // namespace

int main(int argc, char** argv) {
  if (argc == 2 && std::strcmp(argv[1], "part") == 0) {
    int bad = 0;
    for (int64_t N = 1; N <= 72; ++N) bad += parts<false>(N) + parts<true>(N);
    return bad != 0;
  }
  return 2;
}
