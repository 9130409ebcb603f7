// Row operators of residual towers on gfx950: dropout, layer norm and the
// residual join of the two, forward and backward.
//
// The unit of work is a chunk: eight consecutive columns of a row, which share
// one Philox block of the dropout's numbers and are 16 bytes of bf16 or 32 of
// float32.  All of these operators move a few bytes per operation, so HBM
// bounds them; every matrix is read once and written once, and a row stays in
// registers between the passes over it.  All sums are float32; a value is
// rounded to the storage type where it is stored.
#include <algorithm>

#include "device.h"
#include "kernels.h"

namespace vfl {
namespace {

using namespace dev;

constexpr int kThreads = 256;

// ------------------------------------------------------------------- chunks
// Vectors at element alignment: gfx950 loads and stores 16 bytes at any
// address, so rows of an odd stride take the same path as aligned ones.
typedef u32x4 __attribute__((aligned(2))) u32x4_a2;
typedef u32x2 __attribute__((aligned(2))) u32x2_a2;
typedef uint32_t __attribute__((aligned(2))) u32_a2;
typedef f32x4 __attribute__((aligned(4))) f32x4_a4;
typedef f32x2 __attribute__((aligned(4))) f32x2_a4;

template <typename T> struct Raw;                 // a chunk as it is stored
template <> struct Raw<uint16_t> { u32x4 a; };
template <> struct Raw<float> { f32x4 a, b; };

__device__ __forceinline__ Raw<uint16_t> load_at(const uint16_t* p) { return {*(const u32x4_a2*)p}; }
__device__ __forceinline__ Raw<float> load_at(const float* p) {
  return {*(const f32x4_a4*)p, *(const f32x4_a4*)(p + 4)};
}
__device__ __forceinline__ void unpack(const Raw<uint16_t>& r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(r.a[i] << 16);
    v[2 * i + 1] = __uint_as_float(r.a[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack(const Raw<float>& r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = r.a[i];
    v[4 + i] = r.b[i];
  }
}

// The columns of a row (kernel-uniform): n of them in `per` chunks, the last
// one `part` columns wide when that is not 0.
struct Cols {
  int n, per, part;
  __device__ explicit Cols(int cols) : n(cols), per((cols + 7) >> 3), part(cols & 7) {}
};

// How the columns of a kernel's rows lie: kExact: each lane's chunks are all
// whole; kRagged: a row may end inside a chunk, and lanes may have none of it
// (rows of eight columns and more); kSmall: rows of one chunk of any width.
enum Form { kExact, kRagged, kSmall };

// Chunk q of a row, loaded without a branch: the last chunk of a row that ends
// inside it, and chunks past the row's end, are read from the row's last eight
// columns, so that no access leaves the row (rows of fewer than eight columns
// are gathered).
template <Form F, typename T>
__device__ __forceinline__ Raw<T> load_chunk(const T* row, int q, const Cols& k) {
  if constexpr (F == kExact) return load_at(row + 8 * q);
  if constexpr (F == kSmall) {
    if (k.n < 8) {
      T e[8] = {};
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if (i < k.n) e[i] = row[i];
      return __builtin_bit_cast(Raw<T>, e);
    }
  }
  return load_at(row + min(8 * q, k.n - 8));
}

// Its values: those of a partial chunk moved to their places, zero at and past
// the row's end.
template <Form F, typename T>
__device__ __forceinline__ void chunk_values(const Raw<T>& r, int q, const Cols& k, float (&v)[8]) {
  unpack(r, v);
  if constexpr (F == kExact) return;
  if (F == kSmall && k.n < 8) return;
  if (k.part && q == k.per - 1) {
    const int by = 8 - k.part;                       // uniform
    if (by & 4) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i + 4 < 8 ? v[(i + 4) & 7] : 0.f;
    }
    if (by & 2) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i + 2 < 8 ? v[(i + 2) & 7] : 0.f;
    }
    if (by & 1) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i + 1 < 8 ? v[(i + 1) & 7] : 0.f;
    }
  }
  if (q >= k.per) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
  }
}

__device__ __forceinline__ void store4(uint16_t* p, const float* v) {
  *(u32x2_a2*)p = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
}
__device__ __forceinline__ void store4(float* p, const float* v) { *(f32x4_a4*)p = f32x4{v[0], v[1], v[2], v[3]}; }
__device__ __forceinline__ void store2(uint16_t* p, const float* v) { *(u32_a2*)p = pack_bf16(v[0], v[1]); }
__device__ __forceinline__ void store2(float* p, const float* v) { *(f32x2_a4*)p = f32x2{v[0], v[1]}; }
__device__ __forceinline__ void store8(uint16_t* p, const float* v) {
  *(u32x4_a2*)p = u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
}
__device__ __forceinline__ void store8(float* p, const float* v) {
  store4(p, v);
  store4(p + 4, v + 4);
}

// Stores chunk q of a row: whole, or the columns that the row has of it, in
// pieces of four, two and one.
template <Form F, typename T>
__device__ __forceinline__ void store_chunk(T* row, int q, const Cols& k, const float (&v)[8]) {
  T* p = row + 8 * q;
  if (F == kExact || 8 * q + 8 <= k.n) {
    store8(p, v);
  } else if (q < k.per) {
    const int m = k.part;                          // uniform
    if (m & 4) {
      store4(p, v);
      if (m & 2) {
        store2(p + 4, v + 4);
        if (m & 1) st1<T>(p + 6, v[6]);
      } else if (m & 1) {
        st1<T>(p + 4, v[4]);
      }
    } else if (m & 2) {
      store2(p, v);
      if (m & 1) st1<T>(p + 2, v[2]);
    } else {
      st1<T>(p, v[0]);
    }
  }
}

// ------------------------------------------------------------------ dropout
__device__ __forceinline__ uint32_t step_of(const DropKey& d) {
  return d.step + (d.step_dev ? *d.step_dev : 0u);
}

// The numbers of chunk q of global row id `row`: one Philox block of 16-bit
// numbers per chunk (32-bit numbers would take two blocks).
struct Numbers { uint32_t w[4]; };
__device__ __forceinline__ Numbers chunk_numbers(const DropKey& d, uint32_t step, int64_t row, int q) {
  const uint64_t id = (uint64_t)row;
  Numbers n{{step, (uint32_t)id, (uint32_t)q, 0x80000000u | ((uint32_t)(id >> 32) << 16) | d.tag}};
  philox4x32_10(n.w, d.k0, d.k1);
  return n;
}

// v = dropout(v).  A number u is at least thr where it exceeds thr - 1, and a
// word's high half does where the word exceeds (thr - 1) * 2^16 + 65535: neither
// half is moved to be compared.
__device__ __forceinline__ void drop_values(const DropKey& d, const Numbers& n, float (&v)[8]) {
  const uint32_t last = (d.thr << 16) - 1u;        // thr in 1 .. 65536
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = (uint16_t)n.w[i] > (uint16_t)(d.thr - 1u) ? v[2 * i] * d.scale : 0.f;
    v[2 * i + 1] = n.w[i] > last ? v[2 * i + 1] * d.scale : 0.f;
  }
}

template <typename T>
__device__ __forceinline__ const T* row_of(const Mat& m, int64_t r) { return (const T*)m.p + r * m.ld; }
template <typename T>
__device__ __forceinline__ T* out_row(const Mat& m, int64_t r) { return (T*)m.p + r * m.ld; }

// The matrix's chunks dealt to the threads in order, so that a wavefront's are
// consecutive whatever the width; a thread steps its (row, chunk) pair by
// (drow, dq), a whole grid, without a division.
template <typename T, Form F>
__global__ __launch_bounds__(kThreads) void k_dropout(DropJob j, int64_t drow, int dq) {
  const Cols k(j.cols);
  const uint32_t step = step_of(j.d);
  const uint32_t first = blockIdx.x * kThreads + threadIdx.x;
  int64_t r = first / (uint32_t)k.per;
  int q = (int)(first % (uint32_t)k.per);
  while (r < j.rows) {
    const Raw<T> raw = load_chunk<F>(row_of<T>(j.x, r), q, k);
    Numbers n;
    if (j.d.thr) n = chunk_numbers(j.d, step, j.d.row0 + r, q);
    float v[8];
    chunk_values<F>(raw, q, k, v);
    if (j.d.thr) drop_values(j.d, n, v);
    store_chunk<F>(out_row<T>(j.y, r), q, k, v);
    r += drow;
    q += dq;
    if (q >= k.per) {
      q -= k.per;
      ++r;
    }
  }
}

// --------------------------------------------------------------------- sums
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, true));
}

// The sum over each group of G lanes, in every lane of it (the same bits: each
// step adds the same two values, in either order).
template <int G>
__device__ __forceinline__ float group_sum(float v) {
  if constexpr (G >= 2) v += dpp<0xB1>(v);          // lane ^ 1
  if constexpr (G >= 4) v += dpp<0x4E>(v);          // lane ^ 2
  if constexpr (G >= 8) v += dpp<0x141>(v);         // mirrored in 8 lanes
  if constexpr (G >= 16) v += dpp<0x140>(v);        // mirrored in 16 lanes
  if constexpr (G >= 32) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
  if constexpr (G >= 64) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
  return v;
}

// The row group of a thread: a scalar where a wavefront holds one row only.
template <int G>
__device__ __forceinline__ int group_of_thread() {
  const int g = threadIdx.x / G;
  return G >= 64 ? __builtin_amdgcn_readfirstlane(g) : g;
}

// ------------------------------------------------------------------ forward
// G lanes hold a row, CH chunks each (chunk c * G + lane); a workgroup of
// max(kThreads, G) threads holds kThreads / G rows, or one.  The next row's
// loads are in flight while a row is worked on.  Mean and variance in two sums
// over the registers.  Where a row spans W = G / 64 wavefronts, each forms its
// own mean and sum of squares, and these meet in LDS: with n_w, m_w, M_w of
// wavefront w, the row's sum of squares is the sum of M_w + n_w (m_w -
// mean)^2, which takes one barrier a row (the slots alternate) and loses
// nothing to cancellation.  HOIST: a thread's gamma and beta are loaded before
// its first row and kept.
template <typename T, bool RES, int G, int CH, Form F, bool HOIST>
__global__ __launch_bounds__(G > kThreads ? G : kThreads) void k_norm_forward(NormJob j) {
  constexpr int W = G > 64 ? G / 64 : 1;
  constexpr int RPB = G > 64 ? 1 : kThreads / G;
  constexpr int GL = G < 64 ? G : 64;
  constexpr bool AHEAD = G < 1024;                 // the next row is loaded early
  static_assert(G <= 64 || G >= kThreads, "a workgroup holds whole rows");
  __shared__ f32x2 slots[2][W];                    // a wavefront's mean and sum of squares
  __shared__ float columns[W];                     // and its columns of a row
  const Cols k(j.cols);
  const int lane = threadIdx.x % G, wave = threadIdx.x / 64;
  const float inv = 1.f / (float)k.n;

  Raw<T> x[CH], res[CH];
  auto fetch = [&](int64_t r) {
    const T* px = row_of<T>(j.x, r);
    const T* pr = RES ? row_of<T>(j.r, r) : nullptr;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      x[c] = load_chunk<F>(px, c * G + lane, k);
      if constexpr (RES) res[c] = load_chunk<F>(pr, c * G + lane, k);
    }
  };
  const int64_t stride = (int64_t)gridDim.x * RPB;
  int64_t r = (int64_t)blockIdx.x * RPB + group_of_thread<G>();
  if (AHEAD && r < j.rows) fetch(r);
  uint32_t step = 0;
  if constexpr (RES) step = step_of(j.d);

  float g[HOIST ? CH : 1][8], b[HOIST ? CH : 1][8];
  auto weights = [&](int c, int slot) {
    const int q = c * G + lane;
#pragma unroll
    for (int i = 0; i < 8; ++i) g[slot][i] = 1.f, b[slot][i] = 0.f;
    if (j.gamma) chunk_values<F>(load_chunk<F>(j.gamma, q, k), q, k, g[slot]);
    if (j.beta) chunk_values<F>(load_chunk<F>(j.beta, q, k), q, k, b[slot]);
  };
  if constexpr (HOIST)
    for (int c = 0; c < CH; ++c) weights(c, c);
  float nw = 0.f;
  if constexpr (W > 1) {
#pragma unroll
    for (int c = 0; c < CH; ++c) nw += (float)min(max(k.n - 8 * (c * G + 64 * wave), 0), 512);
    if (threadIdx.x % 64 == 0) columns[wave] = nw;   // read past the first row's barrier
  }
  const float inv_nw = nw > 0.f ? 1.f / nw : 0.f;

  int flip = 0;
  for (; r < j.rows; r += stride) {
    if constexpr (!AHEAD) fetch(r);
    float v[CH][8];
    float sum = 0.f;
    if constexpr (RES) {
      Numbers n[CH];
      if (AHEAD && j.d.thr) {                        // beside the row's loads
#pragma unroll
        for (int c = 0; c < CH; ++c) n[c] = chunk_numbers(j.d, step, j.d.row0 + r, c * G + lane);
      }
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int q = c * G + lane;
        chunk_values<F>(x[c], q, k, v[c]);
        if (!AHEAD && j.d.thr) n[c] = chunk_numbers(j.d, step, j.d.row0 + r, q);
        if (j.d.thr) drop_values(j.d, n[c], v[c]);
        float t[8];
        chunk_values<F>(res[c], q, k, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] += t[i];
      }
    } else {
#pragma unroll
      for (int c = 0; c < CH; ++c) chunk_values<F>(x[c], c * G + lane, k, v[c]);
    }
    if (AHEAD && r + stride < j.rows) fetch(r + stride);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if constexpr (RES)
        if (j.s.p) store_chunk<F>(out_row<T>(j.s, r), c * G + lane, k, v[c]);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += v[c][i];
    }
    sum = group_sum<GL>(sum);
    float mean = sum * (W > 1 ? inv_nw : inv);
    float sq = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int left = k.n - 8 * (c * G + lane);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float d = F == kExact || i < left ? v[c][i] - mean : 0.f;
        sq = fmaf(d, d, sq);
      }
    }
    sq = group_sum<GL>(sq);
    if constexpr (W > 1) {
      if (threadIdx.x % 64 == 0) slots[flip][wave] = f32x2{mean, sq};
      __syncthreads();
      sum = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) sum = fmaf(columns[w], slots[flip][w][0], sum);
      mean = sum * inv;
      sq = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const f32x2 s = slots[flip][w];
        const float d = s[0] - mean;
        sq += fmaf(columns[w] * d, d, s[1]);
      }
      flip ^= 1;
    }
    const float rs = 1.f / sqrtf(fmaf(sq, inv, j.eps));
    if (j.stats && lane == 0) *(f32x2*)(j.stats + 2 * r) = f32x2{mean, rs};
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int at = HOIST ? c : 0;
      if constexpr (!HOIST) weights(c, 0);
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = fmaf((v[c][i] - mean) * rs, g[at][i], b[at][i]);
      store_chunk<F>(out_row<T>(j.y, r), c * G + lane, k, y);
    }
  }
}

// ----------------------------------------------------------------- backward
// The sum over the lanes of a wavefront that share lane % G, in lanes 0 .. G-1.
template <int G>
__device__ __forceinline__ float stride_sum(float v) {
  if constexpr (G <= 8) v += dpp<0x128>(v);          // rotated by 8 in 16 lanes
  if constexpr (G <= 4) v += dpp<0x124>(v);          // by 4
  if constexpr (G <= 2) v += dpp<0x122>(v);          // by 2
  if constexpr (G <= 1) v += dpp<0x121>(v);          // by 1
  if constexpr (G <= 16) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
  if constexpr (G <= 32) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
  return v;
}

// Rows as in the forward, one pass: both row sums and the weights' gradients
// come from the same registers.  A thread keeps its columns' two sums over all
// of its rows; at the end the workgroup's rows of threads meet in LDS and leave
// one partial pair of float32 rows (2 x cols at j.part), or the result itself
// where the grid is one workgroup.
template <typename T, bool RES, int G, int CH, int NT, Form F>
__global__ __launch_bounds__(NT) void k_norm_backward(NormJob j) {
  constexpr int W = G > 64 ? G / 64 : 1;
  constexpr int NW = NT / 64;
  constexpr int RPB = NT / G;
  constexpr int GL = G < 64 ? G : 64;
  constexpr bool HOIST = G <= 64;
  static_assert(G <= 64 || G == NT, "a workgroup holds whole rows");
  __shared__ f32x2 slots[2][W];
  __shared__ float sums[W > 1 ? 1 : NW][W > 1 ? 1 : GL * 8];
  const Cols k(j.cols);
  const int lane = threadIdx.x % G, wave = threadIdx.x / 64;
  const float inv = 1.f / (float)k.n;
  uint32_t step = 0;
  if constexpr (RES) step = step_of(j.d);

  float gm[HOIST ? CH : 1][8];
  auto weights = [&](int c, int slot) {
    const int q = c * G + lane;
#pragma unroll
    for (int i = 0; i < 8; ++i) gm[slot][i] = 1.f;
    if (j.gamma) chunk_values<F>(load_chunk<F>(j.gamma, q, k), q, k, gm[slot]);
  };
  if constexpr (HOIST)
    for (int c = 0; c < CH; ++c) weights(c, c);
  float ag[CH][8] = {}, ab[CH][8] = {};

  int flip = 0;
  for (int64_t r = (int64_t)blockIdx.x * RPB + group_of_thread<G>(); r < j.rows; r += (int64_t)gridDim.x * RPB) {
    Raw<T> xr[CH], yr[CH], sr[CH];
    const f32x2 st = *(const f32x2*)(j.stats + 2 * r);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int q = c * G + lane;
      xr[c] = load_chunk<F>(row_of<T>(j.v, r), q, k);
      yr[c] = load_chunk<F>(row_of<T>(j.dy, r), q, k);
      if constexpr (RES)
        if (j.ds.p) sr[c] = load_chunk<F>(row_of<T>(j.ds, r), q, k);
    }
    float h[CH][8], g[CH][8];
    float sg = 0.f, sgh = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int q = c * G + lane, at = HOIST ? c : 0;
      if constexpr (!HOIST) weights(c, 0);
      chunk_values<F>(xr[c], q, k, h[c]);
      chunk_values<F>(yr[c], q, k, g[c]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        h[c][i] = (h[c][i] - st[0]) * st[1];
        ag[c][i] = fmaf(g[c][i], h[c][i], ag[c][i]);
        ab[c][i] += g[c][i];
        g[c][i] *= gm[at][i];
        sg += g[c][i];
        sgh = fmaf(g[c][i], h[c][i], sgh);
      }
    }
    sg = group_sum<GL>(sg);
    sgh = group_sum<GL>(sgh);
    if constexpr (W > 1) {
      if (threadIdx.x % 64 == 0) slots[flip][wave] = f32x2{sg, sgh};
      __syncthreads();
      sg = sgh = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        sg += slots[flip][w][0];
        sgh += slots[flip][w][1];
      }
      flip ^= 1;
    }
    const float mg = sg * inv, mgh = sgh * inv;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int q = c * G + lane;
      float d[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) d[i] = st[1] * (g[c][i] - mg - h[c][i] * mgh);
      if constexpr (RES) {
        if (j.ds.p) {
          float t[8];
          chunk_values<F>(sr[c], q, k, t);
#pragma unroll
          for (int i = 0; i < 8; ++i) d[i] += t[i];
        }
      }
      if (j.dr.p) store_chunk<F>(out_row<T>(j.dr, r), q, k, d);
      if constexpr (RES) {
        if (j.dx.p) {
          if (j.d.thr) drop_values(j.d, chunk_numbers(j.d, step, j.d.row0 + r, q), d);
          store_chunk<F>(out_row<T>(j.dx, r), q, k, d);
        }
      }
    }
  }

  if (!j.dgamma && !j.dbeta) return;
  float* const out[2] = {gridDim.x == 1 ? j.dgamma : j.part + (int64_t)(2 * blockIdx.x) * k.n,
                         gridDim.x == 1 ? j.dbeta : j.part + (int64_t)(2 * blockIdx.x + 1) * k.n};
#pragma unroll
  for (int c = 0; c < CH; ++c) {
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      float* const dst = out[a];
      float(&acc)[8] = a == 0 ? ag[c] : ab[c];
      if constexpr (W > 1) {
        if (dst) store_chunk<F>(dst, c * G + lane, k, acc);
      } else {
        if constexpr (GL < 64)
          for (int i = 0; i < 8; ++i) acc[i] = stride_sum<GL>(acc[i]);
        __syncthreads();                             // the previous sums have been read
        if (threadIdx.x % 64 < GL) {
          *(f32x4*)&sums[wave][lane * 8] = f32x4{acc[0], acc[1], acc[2], acc[3]};
          *(f32x4*)&sums[wave][lane * 8 + 4] = f32x4{acc[4], acc[5], acc[6], acc[7]};
        }
        __syncthreads();
        for (int i = threadIdx.x; i < GL * 8; i += NT) {
          const int col = c * G * 8 + i;
          if (dst && col < k.n) {
            float t = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) t += sums[w][i];
            dst[col] = t;
          }
        }
      }
    }
  }
}

// The partial pairs summed: a workgroup takes 64 of the 2 x cols columns, each
// of its wavefronts every kSlices-th part; the wavefronts' sums meet in LDS.
constexpr int kSlices = 16;
__global__ __launch_bounds__(64 * kSlices) void k_norm_reduce(NormJob j, int parts) {
  __shared__ float sums[kSlices][64];
  const int lane = threadIdx.x % 64, slice = threadIdx.x / 64;
  const int64_t pitch = 2 * (int64_t)j.cols;
  const int64_t c = (int64_t)blockIdx.x * 64 + lane;
  float t = 0.f;
  if (c < pitch) {
    const float* p = j.part + c;
#pragma unroll 8
    for (int i = slice; i < parts; i += kSlices) t += p[i * pitch];
  }
  sums[slice][lane] = t;
  __syncthreads();
  if (slice == 0 && c < pitch) {
    t = 0.f;
#pragma unroll
    for (int s = 0; s < kSlices; ++s) t += sums[s][lane];
    float* const dst = c < j.cols ? j.dgamma : j.dbeta;
    if (dst) dst[c < j.cols ? c : c - j.cols] = t;
  }
}

// The forward's workgroups (in units of 256 threads).  Rows of one chunk a lane
// take one round of resident workgroups (two for the residual join, whose rows
// differ more in time), so that a thread's gamma and beta serve several rows
// and the next row's loads run beside a row's work: 120291 x 49 bf16 takes 7.8
// us, 9.3 in two rounds; residual 118955 x 175 bf16 48.5 in two, 52.5 in one.
// Wider rows are dealt out by the hardware: residual 32768 x 1024 bf16 46.6 us,
// 48.5 in two rounds.
constexpr int kResident = 2048, kMany = 16384;

template <typename T, bool RES, int G, int CH, bool HOIST = G <= 64>
hipError_t forward_with(const NormJob& j, hipStream_t st) {
  constexpr int nt = G > kThreads ? G : kThreads;
  constexpr int rpb = nt / G;
  constexpr int most = G <= 64 && CH == 1 ? (RES ? 2 * kResident : kResident) : kMany;
  const int64_t blocks = (j.rows + rpb - 1) / rpb;
  const int grid = (int)std::min<int64_t>(blocks, most * kThreads / nt);
  constexpr Form other = G == 1 ? kSmall : kRagged;
  if (j.cols == 8 * G * CH)
    hipLaunchKernelGGL((k_norm_forward<T, RES, G, CH, kExact, HOIST>), dim3(grid), dim3(nt), 0, st, j);
  else
    hipLaunchKernelGGL((k_norm_forward<T, RES, G, CH, other, HOIST>), dim3(grid), dim3(nt), 0, st, j);
  return hipGetLastError();
}

// Rows of several wavefronts: up to about a round of workgroups, gamma and beta
// are fetched beside the row (378 x 5578 bf16: 8.2 us, 8.5 after it); beyond
// that, reading them after the row's sums leaves the registers to more
// wavefronts (7311 x 4040 bf16: 47.4 us, 50.3 before).
template <typename T, bool RES, int G, int CH>
hipError_t forward_wide(const NormJob& j, hipStream_t st) {
  return j.rows <= 1024 ? forward_with<T, RES, G, CH, true>(j, st) : forward_with<T, RES, G, CH, false>(j, st);
}

// threads of a workgroup of the backward, and its rows at a time
constexpr int backward_threads(int G) { return G > 512 ? G : 512; }

// Lanes per row of a width (G of the kernels).
int lanes_for(int cols) {
  const int per = (cols + 7) / 8;
  for (int g = 1; g <= 64; g *= 2)
    if (per <= g) return g;
  if (per <= 128) return 64;
  return per <= 1024 ? 512 : 1024;
}

template <typename T, bool RES, int G, int CH>
hipError_t backward_with(const NormJob& j, int parts, hipStream_t st) {
  constexpr int nt = backward_threads(G);
  constexpr Form other = G == 1 ? kSmall : kRagged;
  if (j.cols == 8 * G * CH) hipLaunchKernelGGL((k_norm_backward<T, RES, G, CH, nt, kExact>), dim3(parts), dim3(nt), 0, st, j);
  else hipLaunchKernelGGL((k_norm_backward<T, RES, G, CH, nt, other>), dim3(parts), dim3(nt), 0, st, j);
  return hipGetLastError();
}

template <typename T, bool RES>
hipError_t backward(const NormJob& j, int parts, hipStream_t st) {
  const int per = (j.cols + 7) / 8;
  switch (lanes_for(j.cols)) {
    case 1: return backward_with<T, RES, 1, 1>(j, parts, st);
    case 2: return backward_with<T, RES, 2, 1>(j, parts, st);
    case 4: return backward_with<T, RES, 4, 1>(j, parts, st);
    case 8: return backward_with<T, RES, 8, 1>(j, parts, st);
    case 16: return backward_with<T, RES, 16, 1>(j, parts, st);
    case 32: return backward_with<T, RES, 32, 1>(j, parts, st);
    case 64: return per <= 64 ? backward_with<T, RES, 64, 1>(j, parts, st) : backward_with<T, RES, 64, 2>(j, parts, st);
    case 512: return per <= 512 ? backward_with<T, RES, 512, 1>(j, parts, st) : backward_with<T, RES, 512, 2>(j, parts, st);
    default: return per <= 2048 ? backward_with<T, RES, 1024, 2>(j, parts, st) : backward_with<T, RES, 1024, 4>(j, parts, st);
  }
}

template <typename T, bool RES>
hipError_t forward(const NormJob& j, hipStream_t st) {
  const int per = (j.cols + 7) / 8;
  if (per <= 1) return forward_with<T, RES, 1, 1>(j, st);
  if (per <= 2) return forward_with<T, RES, 2, 1>(j, st);
  if (per <= 4) return forward_with<T, RES, 4, 1>(j, st);
  if (per <= 8) return forward_with<T, RES, 8, 1>(j, st);
  if (per <= 16) return forward_with<T, RES, 16, 1>(j, st);
  if (per <= 32) return forward_with<T, RES, 32, 1>(j, st);
  if (per <= 64) return forward_with<T, RES, 64, 1>(j, st);
  if (per <= 128) return forward_with<T, RES, 64, 2>(j, st);
  if (per <= 256) return forward_wide<T, RES, 256, 1>(j, st);
  if (per <= 512) return forward_wide<T, RES, 256, 2>(j, st);
  if (per <= 1024) return forward_wide<T, RES, 512, 2>(j, st);
  if (per <= 2048) return forward_with<T, RES, 1024, 2, true>(j, st);
  return forward_with<T, RES, 1024, 4, false>(j, st);   // registers: none left for gamma and beta
}

}  // namespace

// One round of resident workgroups (two of 512 threads a CU, or one of 1024),
// the rows dealt out evenly.
int norm_parts(int64_t rows, int cols) {
  const int g = lanes_for(cols), nt = backward_threads(g), rpb = nt / g;
  const int64_t blocks = (rows + rpb - 1) / rpb, resident = 256 * (1024 / nt);
  const int64_t rounds = (blocks + resident - 1) / resident;
  return rounds ? (int)((blocks + rounds - 1) / rounds) : 0;
}

template <typename T>
hipError_t dropout(const DropJob& j, hipStream_t st) {
  const int64_t per = ((int64_t)j.cols + 7) / 8;
  const int64_t chunks = j.rows > (INT64_MAX >> 2) / per ? INT64_MAX >> 2 : j.rows * per;
  const int grid = (int)std::min<int64_t>((chunks + kThreads - 1) / kThreads, kMany);
  const int64_t stride = (int64_t)grid * kThreads, drow = stride / per;
  const int dq = (int)(stride % per);
  if (j.cols % 8 == 0) hipLaunchKernelGGL((k_dropout<T, kExact>), dim3(grid), dim3(kThreads), 0, st, j, drow, dq);
  else if (j.cols > 8) hipLaunchKernelGGL((k_dropout<T, kRagged>), dim3(grid), dim3(kThreads), 0, st, j, drow, dq);
  else hipLaunchKernelGGL((k_dropout<T, kSmall>), dim3(grid), dim3(kThreads), 0, st, j, drow, dq);
  return hipGetLastError();
}

hipError_t launch_dropout(Elt e, const DropJob& j, hipStream_t st) {
  return e == BF16 ? dropout<uint16_t>(j, st) : dropout<float>(j, st);
}

hipError_t launch_norm_forward(Elt e, const NormJob& j, hipStream_t st) {
  if (e == BF16) return j.r.p ? forward<uint16_t, true>(j, st) : forward<uint16_t, false>(j, st);
  return j.r.p ? forward<float, true>(j, st) : forward<float, false>(j, st);
}

hipError_t launch_norm_backward(Elt e, const NormJob& j, hipStream_t st) {
  const int parts = norm_parts(j.rows, j.cols);
  const bool residual = j.ds.p || j.dx.p || j.d.thr;
  hipError_t err = hipSuccess;
  if (parts > 0) {
    if (e == BF16) err = residual ? backward<uint16_t, true>(j, parts, st) : backward<uint16_t, false>(j, parts, st);
    else err = residual ? backward<float, true>(j, parts, st) : backward<float, false>(j, parts, st);
  }
  if (err == hipSuccess && parts != 1 && (j.dgamma || j.dbeta)) {
    hipLaunchKernelGGL(k_norm_reduce, dim3((j.cols + 31) / 32), dim3(64 * kSlices), 0, st, j, parts);
    err = hipGetLastError();
  }
  return err;
}

}  // namespace vfl
