// Kernels of a matrix product over the core of gemm.h: a tile a workgroup, the
// sum cut into parts where there are few tiles, the parts joined in order.
#pragma once
#include <algorithm>

#include "gemm.h"
#include "rowchunk.h"

namespace vfl {
namespace {

using namespace dev;
using namespace gemm;

struct ProductArgs {
  Operand a, b;
  void* c;
  int64_t ldc;
  const float* bias;
  uint32_t tm, tn, parts;
  int n, steps, per;                   // per: steps of a part
  int64_t m;
  int relu;
};

__device__ __forceinline__ f32x4 finish(f32x4 v, const f32x4& bias, int relu) {
  v += bias;
  // a NaN passes, as through a comparison
  if (relu) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];
  }
  return v;
}

__device__ __forceinline__ f32x4 bias4(const float* bias, int col, int n) {
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (bias) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (col + i < n) v[i] = bias[col + i];
  }
  return v;
}

// the first `left` of four values (all: at once)
template <typename T>
__device__ __forceinline__ void store_to(T* p, const f32x4& v, int left) {
  if (left >= 4) {
    const float w[4] = {v[0], v[1], v[2], v[3]};
    store4(p, w);
    return;
  }
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (i < left) st1<T>(p + i, v[i]);
}

// One tile of the product, or (parts > 1) of a part of its sum, as float32 partial
// sums [part][m][n].  A lane stores four columns of a row at once, 16 lanes 128 bytes of
// bf16.  The matrix cores bound long sums (8192 x 8192 x 4096 in 8 bits: 240 us, 2.3
// PFLOP/s); where the sum is short a workgroup's first copies and its stores have
// nothing beside them (32768 x 512 x 1024: 22 us, of which the products are 14).
template <class TL, typename T>
__global__ __launch_bounds__(TL::kThreads) void k_product(ProductArgs j) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const Place at = place_of(blockIdx.x, j.tm, j.tn, j.parts);
  static_assert(TL::DN == 4, "a lane stores four columns at once");
  const TL tile;
  typename TL::Acc acc;
#pragma unroll
  for (int f = 0; f < TL::MF; ++f)
#pragma unroll
    for (int c = 0; c < TL::NF; ++c) acc[f][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int s0 = (int)at.part * j.per, s1 = min(s0 + j.per, j.steps);
  const int64_t m0 = (int64_t)at.m * TL::BM;
  const int n0 = (int)at.n * TL::BN;
  tile.run(j.a, j.b, m0, n0, s0, s1, smem, acc);
#pragma unroll
  for (int q = 0; q < TL::NF / 4; ++q) {
    const int col = n0 + tile.col(q), left = j.n - col;
    const f32x4 bias = bias4(j.bias, col, j.n);
#pragma unroll
    for (int f = 0; f < TL::MF; ++f)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int64_t row = m0 + tile.row(f, r);
        if (row >= j.m || left <= 0) continue;
        T* p = (T*)j.c + ((int64_t)at.part * j.m + row) * j.ldc + col;
        f32x4 v;
#pragma unroll
        for (int c = 0; c < 4; ++c) v[c] = acc[f][4 * q + c][r];
        store_to(p, finish(v, bias, j.relu), left);
      }
  }
}

// What a row's sum gets on top where its label's term was rounded: `rest` [rows], times
// `factor` and the label's row of w (null: nothing).
struct LabelTerm {
  const float* rest;
  const int32_t* labels;
  const uint16_t* w;
  int64_t ld, classes;                 // elements from row to row
  float factor;
};
template <int N>
__device__ __forceinline__ void add_label_term(const LabelTerm& j, int64_t row, int col, float* v) {
  const int label = j.labels[row];
  if (label < 0 || label >= j.classes) return;
  const float rest = j.rest[row] * j.factor;
  const uint16_t* const p = j.w + label * j.ld + col;
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const u32x2 w = *(const u32x2*)(p + i);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      v[i + k] = fmaf(rest, __uint_as_float(k & 1 ? w[k / 2] & 0xffff0000u : w[k / 2] << 16), v[i + k]);
  }
}

// A tile of C^T, C [n x m]: results of sum-major operands (gemm.h), or partial sums
// of them [part][n][m].  Each operand is read as it lies in memory, so neither G nor
// the weights are ever transposed there; a lane stores 4 D consecutive columns of C.
// bf16 over 50176 classes: dx of 8192 x 256 rows at 810 to 850 TFLOP/s, dw at 840 to 910,
// G coming from HBM once for each; float32, 1537 x 333 rows over 5003 classes: both 144 us,
// 71 TFLOP/s of 154 (333 columns fill 384 of tiles; two library products take 122).
struct SumArgs {
  SumMajor a, bs;
  Operand b;
  void* c;
  int64_t ldc, n;
  uint32_t tm, tn, parts;
  int m, steps, per, add, wide;        // wide: results in float32 whatever T
  float factor;                        // of the sums
  LabelTerm label;
};
// add: on top of what is there (sums of an earlier piece, which are float32)
template <typename T>
__device__ __forceinline__ void store_sums(T* out, float (&v)[8], int left, int add) {
  if (left >= 8) {
    if (add) {
      float o[8];
      unpack(load_at(out), o);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += o[i];
    }
    store8<false>(out, v);
  } else {
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (i < left) st1<T>(out + i, add ? v[i] + ld1<T>(out + i) : v[i]);
  }
}
template <class TL, typename T>
__device__ __forceinline__ void sum_tile(const SumArgs& j, uint32_t block, char* smem) {
  const Place at = place_of(block, j.tm, j.tn, j.parts);
  const TL tile;
  typename TL::Acc acc;
#pragma unroll
  for (int f = 0; f < TL::MF; ++f)
#pragma unroll
    for (int c = 0; c < TL::NF; ++c) acc[f][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int s0 = (int)at.part * j.per, s1 = min(s0 + j.per, j.steps);
  const int m0 = (int)at.m * TL::BM;
  const int64_t n0 = (int64_t)at.n * TL::BN;
  tile.run(j.a, j.bs, j.b, m0, n0, s0, s1, smem, acc);
#pragma unroll
  for (int f = 0; f < TL::NF; ++f) {
    const int64_t row = n0 + tile.b_col(f);
    if (row >= j.n) continue;
    const int64_t out = ((int64_t)at.part * j.n + row) * j.ldc;
#pragma unroll
    for (int q = 0; q < TL::MF / TL::D; ++q)
#pragma unroll
      for (int d = 0; d < TL::D; d += 2) {
        const int col = m0 + tile.a_col(q) + 4 * d;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = acc[q * TL::D + d + i / 4][f][i % 4] * j.factor;
        if (sizeof(T) == 2 && j.label.rest && col < j.m) add_label_term<8>(j.label, row, col, v);
        if (sizeof(T) == 4 || j.wide) store_sums((float*)j.c + out + col, v, j.m - col, j.add);
        else store_sums((T*)j.c + out + col, v, j.m - col, 0);
      }
  }
}
template <class TL, typename T>
__global__ __launch_bounds__(TL::kThreads) void k_sum_product(SumArgs j) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  sum_tile<TL, T>(j, blockIdx.x, smem);
}
// Two products in one launch: the first `split` workgroups take the first one.  Neither
// fills the card alone where there are few results (8192 x 256 rows over 1000 classes: a
// step 86 us in two launches, 64 in one); where both do, one launch takes what two take.
template <class TA, class TB, typename T>
__global__ __launch_bounds__(TA::kThreads) void k_sum_pair(SumArgs a, SumArgs b, uint32_t split) {
  static_assert(TA::kThreads == TB::kThreads && TA::kLds == TB::kLds);
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  if (blockIdx.x < split) sum_tile<TA, T>(a, blockIdx.x, smem);
  else sum_tile<TB, T>(b, blockIdx.x - split, smem);
}

constexpr int kJoinThreads = 256;
struct JoinArgs {
  const float* part;
  const float* bias;
  void* c;
  int64_t ldc, m, items, ld;           // ld: of the partial sums
  int n, quads, parts, relu;
  LabelTerm label;
};

// The parts of a split product, summed in a fixed order: SL threads take every SL-th
// part of the same four columns each and meet in LDS (many parts of few results: one
// row of 256 columns in 512 parts 15 us with a thread for all parts).
constexpr int64_t kJoinGrid = 1 << 20;
template <typename T, int SL>
__device__ __forceinline__ void join_block(const JoinArgs& j, uint32_t block) {
  constexpr int Q = kJoinThreads / SL;
  __shared__ f32x4 sums[SL > 1 ? SL : 1][Q];
  const int q = threadIdx.x % Q, slice = threadIdx.x / Q;
  const int64_t pitch = j.m * j.ld;
  int64_t at = (int64_t)block * Q + q;
  do {
    const bool live = at < j.items;
    const int64_t row = live ? at / j.quads : 0;
    const int col = live ? 4 * (int)(at - row * j.quads) : 0;
    const float* p = j.part + row * j.ld + col;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int i = slice; i < j.parts; i += 8 * SL) {  // eight loads in flight
      f32x4 o[8];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        o[u] = i + u * SL < j.parts ? *(const f32x4*)(p + (i + u * SL) * pitch) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < 8; ++u) v += o[u];
    }
    if constexpr (SL > 1) {
      sums[slice][q] = v;
      __syncthreads();
      if (slice > 0) return;
#pragma unroll
      for (int i = 1; i < SL; ++i) v += sums[i][q];
    }
    if (j.label.rest && live) {
      float w[4] = {v[0], v[1], v[2], v[3]};
      add_label_term<4>(j.label, row, col, w);
      v = f32x4{w[0], w[1], w[2], w[3]};
    }
    if (live) store_to((T*)j.c + row * j.ldc + col, finish(v, bias4(j.bias, col, j.n), j.relu), j.n - col);
    at += kJoinGrid * Q;
  } while (SL == 1 && at < j.items);   // in slices there are few results
}

template <typename T, int SL>
__global__ __launch_bounds__(kJoinThreads) void k_product_join(JoinArgs j) {
  join_block<T, SL>(j, blockIdx.x);
}

int64_t tiles_of(int64_t v, int by) { return (v + by - 1) / by; }
// elements of a row of partial sums over n columns
int64_t part_ld(int64_t n) { return (n + 3) & ~(int64_t)3; }

// What the steps of a kind of tile take, us: a step's share of a CU that is full, a
// step of a workgroup that has a CU to itself, and the workgroups that a CU holds.
struct StepTime { double share, alone; int room; };

// How a product is cut up: its tiles, the parts of its sum, and what that should take.
struct Cut {
  int64_t tm, tn;
  int steps, parts, per;
  double us;
};

// A product of m x n results over `steps` steps in tiles of bm x bn: the number of parts
// (of four steps or more) that should take the least time, full rounds of workgroups
// and a last one, 2 us to start and end each, and for more than one part the partial
// sums that are written and read, at a copy's rate, and a launch.
inline Cut cut_up(int64_t m, int64_t n, int bm, int bn, int steps, const StepTime& t) {
  Cut c{tiles_of(m, bm), tiles_of(n, bn), steps, 1, steps, 0.0};
  const int64_t tiles = c.tm * c.tn, round = 256 * t.room;
  const int most = (int)std::min<int64_t>(std::max<int64_t>(1, 4 * round / tiles), std::max(1, steps / 4));
  for (int parts = 1; parts <= most; parts += parts < 16 ? 1 : parts / 8) {
    const int64_t full = tiles * parts / round, rest = tiles * parts % round;
    const double step = (double)full * std::max(t.room * t.share, t.alone) +
                        (rest ? std::max((double)tiles_of(rest, 256) * t.share, t.alone) : 0.0);
    const double us = (double)tiles_of(steps, parts) * step + 2.0 * (double)(full + (rest > 0)) +
                      (parts > 1 ? 4.0 + (double)parts * (double)m * (double)n * (8.0 / 5e6) : 0.0);
    if (parts == 1 || us < c.us) c.us = us, c.parts = parts;
  }
  c.per = (int)tiles_of(steps, c.parts);
  c.parts = (int)tiles_of(steps, c.per);
  return c;
}

template <class TL, typename T>
hipError_t sum_product(const SumArgs& a, hipStream_t st) {
  return enqueue(k_sum_product<TL, T>, dim3(a.tm * a.tn * a.parts), dim3(TL::kThreads), TL::kLds, st, a);
}

template <class TL, typename T>
hipError_t product(const ProductArgs& a, hipStream_t st) {
  return enqueue(k_product<TL, T>, dim3(a.tm * a.tn * a.parts), dim3(TL::kThreads), TL::kLds, st, a);
}

// parts [parts][m][part_ld(n)] -> c
JoinArgs join_args(const float* part, int parts, int64_t m, int64_t n, const float* bias, int relu, const Mat& c) {
  const int64_t ld = part_ld(n), items = m * (ld / 4);
  return {part, bias, c.p, c.ld, m, items, ld, (int)n, (int)(ld / 4), parts, relu, LabelTerm{}};
}
bool joins_in_slices(const JoinArgs& a) { return a.parts >= 16 && a.items <= 65536; }
int64_t join_blocks(const JoinArgs& a) {
  return std::min(tiles_of(a.items, joins_in_slices(a) ? kJoinThreads / 16 : kJoinThreads), kJoinGrid);
}
template <typename T>
hipError_t join(const float* part, int parts, int64_t m, int64_t n, const float* bias, int relu, const Mat& c,
                hipStream_t st) {
  const JoinArgs a = join_args(part, parts, m, n, bias, relu, c);
  return enqueue(joins_in_slices(a) ? k_product_join<T, 16> : k_product_join<T, 1>, dim3((unsigned)join_blocks(a)),
                 dim3(kJoinThreads), 0, st, a);
}

}  // namespace
}  // namespace vfl
