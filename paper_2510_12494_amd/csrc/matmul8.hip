// The product of two matrices in 8 bits on gfx950: C = A B^T (+ bias, ReLU).
//
// Both operands carry a power of two for each block of 128 along the sum, which
// is what one v_mfma_scale_f32_16x16x128_f8f6f4 takes: the matrix cores apply the
// powers themselves, and a product of two e4m3 values times them is exact in
// float32, so the only roundings are those of the float32 sums and of the result.
#include <algorithm>

#include "ops8.h"
#include "product.h"

namespace vfl {
namespace {

typedef Tile<kE4m3, 256, 256, 2, 4, 128, 2> Large;
typedef Tile<kE4m3, 128, 128, 2, 2, 128, 2> Small;
typedef Tile<kE4m3Wide, 128, 128, 2, 2, 128, 2> Wide;     // of float32 results

// How a product is cut up: its tile and the parts of its sum.
struct Cut {
  bool large;
  int64_t tm, tn;
  int steps, parts, per;
};

Cut cut(Elt e, int64_t m, int64_t n, int64_t k) {
  Cut c;
  c.steps = (int)((k + kBlock8 - 1) / kBlock8);
  c.large = e == BF16 && tiles_of(m, 256) * tiles_of(n, 256) >= 192;
  const int by = c.large ? 256 : 128;
  c.tm = tiles_of(m, by);
  c.tn = tiles_of(n, by);
  const int64_t all = c.tm * c.tn;
  int64_t parts = 1;
  if (all < 256) parts = std::max<int64_t>(1, std::min<int64_t>(512 / all, c.steps / 4));
  c.per = (int)((c.steps + parts - 1) / parts);
  c.parts = (c.steps + c.per - 1) / c.per;
  return c;
}

Operand operand(const Mat8& m, int64_t rows) {
  return {(const char*)m.p, m.ld, rows - 1, m.scale, m.scale_ld};
}

template <class TL, typename T>
hipError_t matmul8(const Matmul8Job& j, const Cut& c, hipStream_t st) {
  ProductArgs a{};
  a.a = operand(j.a, j.m);
  a.b = operand(j.b, j.n);
  a.m = j.m;
  a.n = (int)j.n;
  a.tm = (uint32_t)c.tm;
  a.tn = (uint32_t)c.tn;
  a.steps = c.steps;
  a.per = c.per;
  if (c.parts == 1) {
    a.c = j.c.p;
    a.ldc = j.c.ld;
    a.bias = j.bias;
    a.relu = j.relu;
    return product<TL, T>(a, 1, st);
  }
  a.c = j.part;
  a.ldc = part_ld(j.n);
  const hipError_t e = product<TL, float>(a, c.parts, st);
  return e != hipSuccess ? e : join<T>(j.part, c.parts, j.m, j.n, j.bias, j.relu, j.c, st);
}

}  // namespace

size_t matmul8_workspace(int64_t m, int64_t n, int64_t k) {
  size_t most = 0;
  for (Elt e : {F32, BF16}) {
    const Cut c = cut(e, m, n, k);
    if (c.parts > 1) most = std::max(most, (size_t)c.parts * (size_t)m * (size_t)part_ld(n) * sizeof(float));
  }
  return most;
}

hipError_t launch_matmul8(Elt e, const Matmul8Job& j, hipStream_t st) {
  const Cut c = cut(e, j.m, j.n, j.k);
  if (e == F32) return matmul8<Wide, float>(j, c, st);
  return c.large ? matmul8<Large, uint16_t>(j, c, st) : matmul8<Small, uint16_t>(j, c, st);
}

}  // namespace vfl
