// The product of two matrices in 8 bits on gfx950: C = A B^T (+ bias, ReLU).
//
// Both operands carry a power of two for each block of 128 along the sum, which
// is what one v_mfma_scale_f32_16x16x128_f8f6f4 takes: the matrix cores apply the
// powers themselves.  That instruction's sums are shorter than float32's (gemm.h),
// which a bf16 result's own rounding hides; float32 results take values widened to
// bf16, whose products are exact in float32, so that the only roundings are those of
// float32 sums and of the result.
#include <algorithm>

#include "ops8.h"
#include "product.h"

namespace vfl {
namespace {

// 16 wavefronts of 64 x 64: four a SIMD, whose reads of LDS hide behind each
// other's products (8192 x 8192 x 4096: 237 us, 2.32 PFLOP/s; eight of 128 x 64 265)
typedef Tile<kE4m3, 256, 256, 4, 4, 128, 2> Large;
typedef Tile<kE4m3, 128, 128, 2, 2, 128, 2> Small;
typedef Tile<kE4m3Wide, 128, 128, 2, 2, 128, 2> Wide;     // of float32 results

// Few rows, or little work: a workgroup takes 16 columns of 16 MT rows, its wavefronts
// the blocks of the sum in turn, straight from global memory into the MFMA's operands;
// their results meet in LDS.  The rows of B are read once (for each 16 MT rows of A), 128
// bytes of 16 of them a wavefront, and that or the latency of one such step bounds it: 1 x
// 1024 x 1024 3.3 us (5.8 with the call, 9.1 in tiles); 16 x 8192 x 8192 18 us, 3.7 TB/s.
struct RowsArgs {
  Operand a, b;
  void* c;
  int64_t ldc;
  const float* bias;
  int m, n, steps, relu;
};
constexpr int kRowWaves = 8;
template <Type TY, int MT, typename T>
__global__ __launch_bounds__(64 * kRowWaves) void k_rows(RowsArgs j) {
  __shared__ f32x4 sums[kRowWaves][MT][64];
  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n0 = (int)blockIdx.x * 16, m0 = (int)blockIdx.y * 16 * MT;
  const int64_t col = min(n0 + i, j.n - 1);
  const VFL_GLOBAL char* const pb = glb(j.b.p) + col * j.b.ld + 16 * g;
  const VFL_GLOBAL uint8_t* const sb = glb(j.b.scale) + col;
  const VFL_GLOBAL char* pa[MT];
  const VFL_GLOBAL uint8_t* sa[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int64_t row = min(m0 + 16 * t + i, j.m - 1);
    pa[t] = glb(j.a.p) + row * j.a.ld + 16 * g;
    sa[t] = glb(j.a.scale) + row;
  }
  f32x4 acc[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  constexpr int U = MT > 1 ? 2 : 4;     // steps in flight
  uint32_t ends = 0;                    // bits of values past an end of bf16
  for (int s0 = wave; s0 < j.steps; s0 += U * kRowWaves) {
    u32x4 b[U][2], a[U][MT][2];
    uint32_t eb[U], ea[U][MT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      // past the last step: the last one again, which is not added
      const int64_t s = min(s0 + u * kRowWaves, j.steps - 1);
#pragma unroll
      for (int h = 0; h < 2; ++h) b[u][h] = *(const VFL_GLOBAL u32x4*)(pb + s * 128 + 64 * h);
      eb[u] = sb[s * j.b.scale_ld];
#pragma unroll
      for (int t = 0; t < MT; ++t) {
#pragma unroll
        for (int h = 0; h < 2; ++h) a[u][t][h] = *(const VFL_GLOBAL u32x4*)(pa[t] + s * 128 + 64 * h);
        ea[u][t] = sa[t][s * j.a.scale_ld];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s0 + u * kRowWaves >= j.steps) break;
      if constexpr (TY == kE4m3) {
        struct Pair { u32x4 x, y; };
        const i32x8 vb = __builtin_bit_cast(i32x8, (Pair{b[u][0], b[u][1]}));
#pragma unroll
        for (int t = 0; t < MT; ++t)
          acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
              __builtin_bit_cast(i32x8, (Pair{a[u][t][0], a[u][t][1]})), vb, acc[t], 0, 0, 0, (int)ea[u][t], 0, (int)eb[u]);
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          bf16x8 wb[2];
          widen_e4m3(b[u][h], eb[u], wb);
          ends |= bits_at_an_end(b[u][h], eb[u]);
#pragma unroll
          for (int t = 0; t < MT; ++t) {
            bf16x8 wa[2];
            widen_e4m3(a[u][t][h], ea[u][t], wa);
            ends |= bits_at_an_end(a[u][t][h], ea[u][t]);
            acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa[0], wb[0], acc[t], 0, 0, 0);
            acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa[1], wb[1], acc[t], 0, 0, 0);
          }
        }
      }
    }
  }
  if constexpr (TY == kE4m3Wide) {
    if (__any((ends & kMagnitudes) != 0)) {          // the sum again, by parts (gemm.h)
#pragma unroll
      for (int t = 0; t < MT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
      for (int64_t s = wave; s < j.steps; s += kRowWaves)
#pragma unroll 1
        for (int p = 0; p < kEndsParts; ++p) {
          const EndsPart part(p);
#pragma unroll 1
          for (int h = 0; h < 2; ++h) {
            bf16x8 wb[2];
            const u32x4 vb = *(const VFL_GLOBAL u32x4*)(pb + s * 128 + 64 * h);
            EndsPart::widen(vb, sb[s * j.b.scale_ld], part.columns, -part.by, wb);
#pragma unroll
            for (int t = 0; t < MT; ++t) {
              bf16x8 wa[2];
              const u32x4 va = *(const VFL_GLOBAL u32x4*)(pa[t] + s * 128 + 64 * h);
              EndsPart::widen(va, sa[t][s * j.a.scale_ld], part.rows, part.by, wa);
              acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa[0], wb[0], acc[t], 0, 0, 0);
              acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa[1], wb[1], acc[t], 0, 0, 0);
            }
          }
        }
    }
  }
#pragma unroll
  for (int t = 0; t < MT; ++t) sums[wave][t][lane] = acc[t];
  __syncthreads();
  for (int at = threadIdx.x; at < MT * 64; at += 64 * kRowWaves) {
    const int t = at >> 6, l = at & 63;
    f32x4 v = sums[0][t][l];
#pragma unroll
    for (int w = 1; w < kRowWaves; ++w) v += sums[w][t][l];
    const int c = n0 + (l & 15);
    if (c >= j.n) continue;
    const float bias = j.bias ? j.bias[c] : 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = m0 + 16 * t + 4 * (l >> 4) + r;
      const float x = v[r] + bias;
      if (row < j.m) st1<T>((T*)j.c + (int64_t)row * j.ldc + c, j.relu && x < 0.f ? 0.f : x);
    }
  }
}

// Products that k_rows takes: of few rows, and those of few workgroups and steps, to
// which a tile's start and the joining of parts would come dearer (us, k_rows and
// tiles, bf16: 64 x 1024 x 1024 7.1, 11.0; 256 x 1024 x 1024 6.9, 11.8; 1024 x 1024 x
// 1024 12.7, 16.0; 64 x 4096 x 4096 12.3, 16.3; beyond: 64 x 1024 x 8192 20.6, 15.9;
// 32 x 8192 x 8192 24.6, 23.3; and where the tiles are many: 32768 x 64 x 500 15.8, 9.6).
constexpr int kRowSteps = 32, kRowWork = 8192;
constexpr int64_t kRowColumns = (int64_t)1 << 26;    // its grid is below 2^32 threads

enum Kind { kRowsOne, kRowsTwo, kRowsFour, kLargeTile, kSmallTile };
struct Choice : Cut { Kind kind; };

// Steps timed over 8192 x 8192 x 4096.  The two kinds of tile, us: 8192 x 8192 x 4096
// 237 large, 287 small; 2944 cubed 41, 47; 1024 x 8192 x 8192 89, 64; 4096 x 2048 x 1024
// 19.8, 15.8.
Choice choose(Elt e, int64_t m, int64_t n, int64_t k) {
  const int steps = (int)tiles_of(k, kBlock8);
  if ((m <= 16 && n <= kRowColumns) ||
      (steps <= kRowSteps && tiles_of(m, 64) * tiles_of(n, 16) * steps <= kRowWork &&
       tiles_of(m, 128) * tiles_of(n, 128) < 128))
    return {Cut{0, 0, steps, 1, steps, 0.0}, m <= 16 ? kRowsOne : m <= 32 ? kRowsTwo : kRowsFour};
  const Cut small = cut_up(m, n, 128, 128, steps, e == F32 ? StepTime{0.98, 1.2, 2} : StepTime{0.5, 0.75, 2});
  if (e == F32) return {small, kSmallTile};
  const Cut large = cut_up(m, n, 256, 256, steps, StepTime{1.75, 1.75, 1});
  return large.us < small.us ? Choice{large, kLargeTile} : Choice{small, kSmallTile};
}

Operand operand(const Mat8& m, int64_t rows) {
  return {(const char*)m.p, m.ld, rows - 1, m.scale, m.scale_ld};
}

template <class TL, typename T>
hipError_t tiles8(const Matmul8Job& j, const Cut& c, hipStream_t st) {
  ProductArgs a{};
  a.a = operand(j.a, j.m);
  a.b = operand(j.b, j.n);
  a.m = j.m;
  a.n = (int)j.n;
  a.tm = (uint32_t)c.tm;
  a.tn = (uint32_t)c.tn;
  a.steps = c.steps;
  a.per = c.per;
  a.parts = (uint32_t)c.parts;
  if (c.parts == 1) {
    a.c = j.c.p;
    a.ldc = j.c.ld;
    a.bias = j.bias;
    a.relu = j.relu;
    return product<TL, T>(a, st);
  }
  a.c = j.part;
  a.ldc = part_ld(j.n);
  const hipError_t e = product<TL, float>(a, st);
  return e != hipSuccess ? e : join<T>(j.part, c.parts, j.m, j.n, j.bias, j.relu, j.c, st);
}

template <Type TY, int MT, typename T>
hipError_t rows8(const Matmul8Job& j, const Cut& c, hipStream_t st) {
  const RowsArgs a{operand(j.a, j.m), operand(j.b, j.n), j.c.p, j.c.ld, j.bias, (int)j.m, (int)j.n, c.steps, j.relu};
  return enqueue(k_rows<TY, MT, T>, dim3((unsigned)tiles_of(j.n, 16), (unsigned)tiles_of(j.m, 16 * MT)),
                 dim3(64 * kRowWaves), 0, st, a);
}

template <Type TY, class SMALL, typename T>
hipError_t matmul8(const Matmul8Job& j, const Choice& c, hipStream_t st) {
  switch (c.kind) {
    case kRowsOne: return rows8<TY, 1, T>(j, c, st);
    case kRowsTwo: return rows8<TY, 2, T>(j, c, st);
    case kRowsFour: return rows8<TY, 4, T>(j, c, st);
    case kLargeTile:
      if constexpr (TY == kE4m3) return tiles8<Large, T>(j, c, st);
      [[fallthrough]];
    default: return tiles8<SMALL, T>(j, c, st);
  }
}

}  // namespace

size_t matmul8_workspace(int64_t m, int64_t n, int64_t k) {
  size_t most = 0;
  for (Elt e : {F32, BF16}) {
    const Cut c = choose(e, m, n, k);
    if (c.parts > 1) most = std::max(most, (size_t)c.parts * (size_t)m * (size_t)part_ld(n) * sizeof(float));
  }
  return most;
}

hipError_t launch_matmul8(Elt e, const Matmul8Job& j, hipStream_t st) {
  const Choice c = choose(e, j.m, j.n, j.k);
  return e == F32 ? matmul8<kE4m3Wide, Wide, float>(j, c, st) : matmul8<kE4m3, Small, uint16_t>(j, c, st);
}

}  // namespace vfl
