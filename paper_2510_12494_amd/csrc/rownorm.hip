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
#include <type_traits>

#include "device.h"
#include "rowops.h"

namespace vfl {
namespace {

using namespace dev;

constexpr int kThreads = 256;

// Kernel arguments: what a kernel reads and no more, the sizes of its grid and
// workgroups among them (asking for those would add 256 bytes of hidden
// arguments).  The host writes them for every launch: a layer norm's 72 bytes
// instead of the whole job and the hidden ones take 0.5 us off a call of 3.7.
struct DropArgs {
  DropKey d;
  Mat x, y;
  int64_t rows, drow;
  int cols, dq;
};
struct NoResidual {};
struct ForwardResidual { DropKey d; Mat r, s; };
template <bool RES>
struct ForwardArgs : std::conditional_t<RES, ForwardResidual, NoResidual> {
  Mat x, y;
  const float *gamma, *beta;
  float* stats;
  int64_t rows;
  int cols, grid, threads;
  float eps;
};
struct BackwardResidual { DropKey d; Mat ds, dx; int add; };
template <bool RES>
struct BackwardArgs : std::conditional_t<RES, BackwardResidual, NoResidual> {
  Mat v, dy, dr;
  const float *gamma, *stats;
  float *dgamma, *dbeta, *part;
  int64_t rows;
  int cols, grid, lanes, groups, col_blocks;       // lanes: threads of a wide row
};
struct ReduceArgs {
  const float* part;
  float *dgamma, *dbeta;
  int cols, parts;
};

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
// one `part` columns wide when that is not 0.  Rows from `edge` on are so near
// the matrix's end that a whole last chunk would pass it.
struct Cols {
  int n, per, part;
  int64_t edge;
  __device__ explicit Cols(int cols, int64_t rows) : n(cols), per((cols + 7) >> 3), part(cols & 7) {
    const int past = 8 * per - n;                    // rows of n columns and more hold these
    edge = past ? rows - (past + n - 1) / n : INT64_MAX;
  }
};

// How the columns of a kernel's rows lie: kExact: each lane's chunks are all
// whole; kRagged: a row may end inside a chunk, and lanes may have none of it
// (rows of eight columns and more); kSmall: rows of one chunk of any width.
// `whole`: this chunk is whole whatever the form.
enum Form { kExact, kRagged, kSmall };

// Chunk q of a row, loaded without a branch.  A row's last chunk is read whole:
// past the row's end lie the next row or what is between the two.  Lanes
// without a chunk read the last one.  On the matrix's edge rows the last eight
// columns are read instead (rows of fewer are gathered), so that no access
// passes the matrix.
template <Form F, typename T>
__device__ __forceinline__ Raw<T> load_chunk(const T* row, int q, const Cols& k, bool edge, bool whole = false) {
  if (F == kExact || whole) return load_at(row + 8 * q);
  if constexpr (F == kSmall) {
    if (k.n < 8) {
      if (!edge) return load_at(row);
      T e[8] = {};
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if (i < k.n) e[i] = row[i];
      return __builtin_bit_cast(Raw<T>, e);
    }
  }
  return load_at(row + min(8 * q, edge ? k.n - 8 : 8 * k.per - 8));
}

// Its values: `past` at and past the row's end (on an edge row, those of a
// partial chunk moved to their places).
template <Form F, typename T>
__device__ __forceinline__ void chunk_values(const Raw<T>& r, int q, const Cols& k, bool edge, float (&v)[8],
                                             bool whole = false, float past = 0.f) {
  unpack(r, v);
  if (F == kExact || whole) return;
  if (edge && k.n >= 8 && q == k.per - 1) {
    const int by = 8 - k.part;                       // uniform
    if (by & 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = v[i + 4];
    }
    if (by & 2) {
#pragma unroll
      for (int i = 0; i < 6; ++i) v[i] = v[i + 2];
    }
    if (by & 1) {
#pragma unroll
      for (int i = 0; i < 7; ++i) v[i] = v[i + 1];
    }
  }
  const int left = k.n - 8 * q;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = i < left ? v[i] : past;
}

// Those of a row of its own (gamma, beta).
template <Form F>
__device__ __forceinline__ void vector_values(const float* p, int q, const Cols& k, float (&v)[8], bool whole) {
  chunk_values<F>(load_chunk<F>(p, q, k, true, whole), q, k, true, v, whole);
}

__device__ __forceinline__ void store4(uint16_t* p, const float* v) {
  *(u32x2_a2*)p = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
}
__device__ __forceinline__ void store4(float* p, const float* v) { *(f32x4_a4*)p = f32x4{v[0], v[1], v[2], v[3]}; }
__device__ __forceinline__ void store2(uint16_t* p, const float* v) { *(u32_a2*)p = pack_bf16(v[0], v[1]); }
__device__ __forceinline__ void store2(float* p, const float* v) { *(f32x2_a4*)p = f32x2{v[0], v[1]}; }
// EARLY: the lines leave the L2 as they are written (a non-temporal store)
// instead of all at the kernel's end.
template <bool EARLY>
__device__ __forceinline__ void store8(uint16_t* p, const float* v) {
  const u32x4_a2 w{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
  if constexpr (EARLY) __builtin_nontemporal_store(w, (u32x4_a2*)p);
  else *(u32x4_a2*)p = w;
}
template <bool EARLY>
__device__ __forceinline__ void store8(float* p, const float* v) {
  if constexpr (EARLY) {
    __builtin_nontemporal_store(f32x4_a4{v[0], v[1], v[2], v[3]}, (f32x4_a4*)p);
    __builtin_nontemporal_store(f32x4_a4{v[4], v[5], v[6], v[7]}, (f32x4_a4*)(p + 4));
  } else {
    store4(p, v);
    store4(p + 4, v + 4);
  }
}

// Stores chunk q of a row: whole, or the columns that the row has of it, in
// pieces of four, two and one.
template <Form F, bool EARLY = false, typename T>
__device__ __forceinline__ void store_chunk(T* row, int q, const Cols& k, const float (&v)[8], bool whole = false) {
  T* p = row + 8 * q;
  if (F == kExact || whole || 8 * q + 8 <= k.n) {
    store8<EARLY>(p, v);
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
// (drow, dq), a whole grid, without a division.  HBM bounds it (32768 x 1024
// bf16: 23.6 us, 5.7 TB/s; the Philox block of a chunk costs 10 rounds of two
// multiplications beside 32 bytes moved), and the launch below about 10 MB
// (4099 x 333 float32: 4.2 us).
template <typename T, Form F>
__global__ __launch_bounds__(kThreads) void k_dropout(DropArgs j) {
  const Cols k(j.cols, j.rows);
  const uint32_t step = step_of(j.d);
  const uint32_t first = blockIdx.x * kThreads + threadIdx.x;
  int64_t r = first / (uint32_t)k.per;
  int q = (int)(first % (uint32_t)k.per);
  while (r < j.rows) {
    const bool edge = r >= k.edge;
    const Raw<T> raw = load_chunk<F>(row_of<T>(j.x, r), q, k, edge);
    Numbers n;
    if (j.d.thr) n = chunk_numbers(j.d, step, j.d.row0 + r, q);
    float v[8];
    chunk_values<F>(raw, q, k, edge, v);
    if (j.d.thr) drop_values(j.d, n, v);
    store_chunk<F>(out_row<T>(j.y, r), q, k, v);
    r += j.drow;
    q += j.dq;
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

// That of a wavefront where `lanes` threads hold a row.
__device__ __forceinline__ int group_of_wave(int lanes) {
  return __builtin_amdgcn_readfirstlane(threadIdx.x / 64) / (lanes / 64);
}

// ------------------------------------------------------------------ forward
// Up to G = 64 lanes hold a row, CH chunks each (chunk c * G + lane), and a
// workgroup kThreads / G rows; wider rows (G = 512 or 1024) take a workgroup of
// as many wavefronts as they fill, G threads at most.  The next row's loads are
// in flight while a row is worked on.  Mean and variance in two sums over the
// registers.  Where a row spans several wavefronts, each forms its own mean and
// sum of squares, and these meet in LDS: with n_w, m_w, M_w of wavefront w, the
// row's sum of squares is the sum of M_w + n_w (m_w - mean)^2, which takes one
// barrier a row (the slots alternate) and loses nothing to cancellation.  HOIST:
// a thread's gamma and beta are loaded before its first row and kept.  HBM
// bounds it: residual 32768 x 1024 bf16 45.9 us (5.8 TB/s), layer norm 32768 x
// 512 bf16 11.1 us (6.1 TB/s, partly from the last-level cache); one row takes
// 2.1 us, a kernel's launch.
template <typename T, bool RES, int G, int CH, Form F, bool HOIST, bool EARLY>
__global__ __launch_bounds__(G > kThreads ? G : kThreads) void k_norm_forward(ForwardArgs<RES> j) {
  constexpr bool WIDE = G > 64;
  constexpr int RPB = WIDE ? 1 : kThreads / G;
  constexpr int GL = G < 64 ? G : 64;
  constexpr bool AHEAD = G < 1024;                 // the next row is loaded early
  __shared__ f32x2 slots[2][WIDE ? 16 : 1];        // a wavefront's mean and sum of squares
  __shared__ float columns[WIDE ? 16 : 1];         // and its columns of a row
  const Cols k(j.cols, j.rows);
  const int lanes = WIDE ? j.threads : G;
  const int lane = WIDE ? (int)threadIdx.x : threadIdx.x % G, wave = threadIdx.x / 64;
  const float inv = 1.f / (float)k.n;

  Raw<T> x[CH], res[CH];
  auto fetch = [&](int64_t r) {
    const T* px = row_of<T>(j.x, r);
    const T* pr = nullptr;
    if constexpr (RES) pr = row_of<T>(j.r, r);
    const bool edge = r >= k.edge;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      x[c] = load_chunk<F>(px, c * lanes + lane, k, edge, c < CH / 2);
      if constexpr (RES) res[c] = load_chunk<F>(pr, c * lanes + lane, k, edge, c < CH / 2);
    }
  };
  const int64_t stride = (int64_t)j.grid * RPB;
  int64_t r = (int64_t)blockIdx.x * RPB + group_of_thread<G>();
  if (AHEAD && r < j.rows) fetch(r);
  uint32_t step = 0;
  if constexpr (RES) step = step_of(j.d);

  float g[HOIST ? CH : 1][8], b[HOIST ? CH : 1][8];
  auto weights = [&](int c, int slot) {
    const int q = c * lanes + lane;
#pragma unroll
    for (int i = 0; i < 8; ++i) g[slot][i] = 1.f, b[slot][i] = 0.f;
    if (j.gamma) vector_values<F>(j.gamma, q, k, g[slot], c < CH / 2);
    if (j.beta) vector_values<F>(j.beta, q, k, b[slot], c < CH / 2);
  };
  if constexpr (HOIST)
    for (int c = 0; c < CH; ++c) weights(c, c);
  float nw = 0.f;
  if constexpr (WIDE) {
#pragma unroll
    for (int c = 0; c < CH; ++c) nw += (float)min(max(k.n - 8 * (c * lanes + 64 * wave), 0), 512);
    if (threadIdx.x % 64 == 0) columns[wave] = nw;   // read past the first row's barrier
  }
  const float inv_nw = nw > 0.f ? 1.f / nw : 0.f;

  int flip = 0;
  for (; r < j.rows; r += stride) {
    if constexpr (!AHEAD) fetch(r);
    const bool edge = r >= k.edge;
    float v[CH][8];
    float sum = 0.f;
    if constexpr (RES) {
      Numbers n[CH];
      if (AHEAD && j.d.thr) {                        // beside the row's loads
#pragma unroll
        for (int c = 0; c < CH; ++c) n[c] = chunk_numbers(j.d, step, j.d.row0 + r, c * lanes + lane);
      }
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int q = c * lanes + lane;
        chunk_values<F>(x[c], q, k, edge, v[c], c < CH / 2);
        if (!AHEAD && j.d.thr) n[c] = chunk_numbers(j.d, step, j.d.row0 + r, q);
        if (j.d.thr) drop_values(j.d, n[c], v[c]);
        float t[8];
        chunk_values<F>(res[c], q, k, edge, t, c < CH / 2);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] += t[i];
      }
    } else {
#pragma unroll
      for (int c = 0; c < CH; ++c) chunk_values<F>(x[c], c * lanes + lane, k, edge, v[c], c < CH / 2);
    }
    if (AHEAD && r + stride < j.rows) fetch(r + stride);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if constexpr (RES)
        if (j.s.p) store_chunk<F, EARLY>(out_row<T>(j.s, r), c * lanes + lane, k, v[c], c < CH / 2);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += v[c][i];
    }
    sum = group_sum<GL>(sum);
    float mean = sum * (WIDE ? inv_nw : inv);
    float sq = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int left = k.n - 8 * (c * lanes + lane);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float d = F == kExact || c < CH / 2 || i < left ? v[c][i] - mean : 0.f;
        sq = fmaf(d, d, sq);
      }
    }
    sq = group_sum<GL>(sq);
    if constexpr (WIDE) {
      if (threadIdx.x % 64 == 0) slots[flip][wave] = f32x2{mean, sq};
      __syncthreads();
      // every 16 lanes add the wavefronts' values, a lane each
      const int w = threadIdx.x % 16;
      const bool has = 64 * w < lanes;
      const f32x2 s = has ? slots[flip][w] : f32x2{0.f, 0.f};
      const float n = has ? columns[w] : 0.f;
      mean = group_sum<16>(n * s[0]) * inv;
      const float d = s[0] - mean;
      sq = group_sum<16>(fmaf(n * d, d, s[1]));
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
      store_chunk<F, EARLY>(out_row<T>(j.y, r), c * lanes + lane, k, y, c < CH / 2);
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

// Rows first, first + stride, ... as in the forward, one pass.  G = 256: a
// workgroup's groups of wavefronts take a row each, with barriers in common;
// those without a row left go along.  ACC: a thread also adds its columns' terms
// of the weights' gradients to ag and ab (not with four chunks a lane, which
// leave no registers for those).
template <typename T, bool RES, int G, int CH, Form F, bool ACC, bool OUT, bool EARLY>
__device__ __forceinline__ void backward_rows(const BackwardArgs<RES>& j, int64_t r, int64_t stride, float (&ag)[CH][8],
                                              float (&ab)[CH][8]) {
  constexpr bool WIDE = G > 64;
  constexpr int GL = G < 64 ? G : 64;
  constexpr bool GROUPS = G == 256;
  constexpr bool AHEAD = G < 1024 || CH == 1, HOIST = CH <= 2;
  static_assert(!(ACC && CH > 2), "registers");
  __shared__ f32x2 slots[2][WIDE ? 16 : 1];
  const Cols k(j.cols, j.rows);
  const int lanes = WIDE ? j.lanes : G;
  const int group = GROUPS ? group_of_wave(lanes) : 0;
  const int lane = WIDE ? (int)threadIdx.x - group * lanes : threadIdx.x % G;
  const float inv = 1.f / (float)k.n;
  bool add = false, drop = false;
  if constexpr (RES) {
    add = j.add;
    drop = j.d.thr;
  }

  Raw<T> xr[CH], yr[CH], sr[CH];
  f32x2 st = {0.f, 0.f};
  auto fetch = [&](int64_t r) {
    st = *(const f32x2*)(j.stats + 2 * r);
    const bool edge = r >= k.edge;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int q = c * lanes + lane;
      xr[c] = load_chunk<F>(row_of<T>(j.v, r), q, k, edge, c < CH / 2);
      yr[c] = load_chunk<F>(row_of<T>(j.dy, r), q, k, edge, c < CH / 2);
      if constexpr (RES && OUT) sr[c] = load_chunk<F>(row_of<T>(j.ds, r), q, k, edge, c < CH / 2);
    }
  };
  if constexpr (GROUPS) fetch(min(r, j.rows - 1));
  else if (AHEAD && r < j.rows) fetch(r);
  uint32_t step = 0;
  if constexpr (RES) step = step_of(j.d);

  float gm[HOIST ? CH : 1][8];
  auto weights = [&](int c, int slot) {
    const int q = c * lanes + lane;
#pragma unroll
    for (int i = 0; i < 8; ++i) gm[slot][i] = 1.f;
    if (j.gamma) vector_values<F>(j.gamma, q, k, gm[slot], c < CH / 2);
  };
  if constexpr (HOIST)
    for (int c = 0; c < CH; ++c) weights(c, c);

  int flip = 0;
  for (; r - group < j.rows; r += stride) {          // as often for every group
    const bool live = !GROUPS || r < j.rows;
    if constexpr (!AHEAD) fetch(r);
    Numbers n[CH];
    if constexpr (RES && AHEAD && OUT) {
      if (drop) {                                    // beside the row's loads
#pragma unroll
        for (int c = 0; c < CH; ++c) n[c] = chunk_numbers(j.d, step, j.d.row0 + r, c * lanes + lane);
      }
    }
    const float mean = st[0], rs = st[1];
    const bool edge = r >= k.edge;
    Raw<T> sc[CH];
    float h[CH][8], g[CH][8];
    float sg = 0.f, sgh = 0.f;
    if (live) {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int q = c * lanes + lane;
        if constexpr (!HOIST) weights(c, 0);
        // past the row's end x is its mean: h is 0 there, and not mean * rs,
        // which may be infinite and would make the sums of g * h NaN
        chunk_values<F>(xr[c], q, k, edge, h[c], c < CH / 2, mean);
        chunk_values<F>(yr[c], q, k, edge, g[c], c < CH / 2);
        if constexpr (RES && OUT) sc[c] = sr[c];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          h[c][i] = (h[c][i] - mean) * rs;
          if constexpr (ACC) {
            ag[c][i] = fmaf(g[c][i], h[c][i], ag[c][i]);
            ab[c][i] += g[c][i];
          }
          g[c][i] *= gm[HOIST ? c : 0][i];
          sg += g[c][i];
          sgh = fmaf(g[c][i], h[c][i], sgh);
        }
      }
    }
    if (AHEAD) fetch(r + stride < j.rows ? r + stride : GROUPS ? min(r, j.rows - 1) : r);
    if constexpr (!OUT) continue;
    sg = group_sum<GL>(sg);
    sgh = group_sum<GL>(sgh);
    if constexpr (WIDE) {
      if (threadIdx.x % 64 == 0) slots[flip][threadIdx.x / 64] = f32x2{sg, sgh};
      __syncthreads();
      const int w = threadIdx.x % 16;
      const f32x2 s = 64 * w < lanes ? slots[flip][group * (lanes / 64) + w] : f32x2{0.f, 0.f};
      sg = group_sum<16>(s[0]);
      sgh = group_sum<16>(s[1]);
      flip ^= 1;
    }
    if (!live) continue;
    const float mg = sg * inv, mgh = sgh * inv;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int q = c * lanes + lane;
      float d[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) d[i] = rs * (g[c][i] - mg - h[c][i] * mgh);
      if constexpr (RES) {
        if (add) {
          float t[8];
          chunk_values<F>(sc[c], q, k, edge, t, c < CH / 2);
#pragma unroll
          for (int i = 0; i < 8; ++i) d[i] += t[i];
        }
      }
      store_chunk<F, EARLY>(out_row<T>(j.dr, r), q, k, d, c < CH / 2);
      if constexpr (RES) {
        if (!AHEAD && drop) n[c] = chunk_numbers(j.d, step, j.d.row0 + r, q);
        if (drop) drop_values(j.d, n[c], d);
        store_chunk<F, EARLY>(out_row<T>(j.dx, r), q, k, d, c < CH / 2);
      }
    }
  }
}

// Many rows: rows and weights' gradients from the same registers, so that every
// matrix is read once.  At the end the workgroup's rows of threads meet in LDS
// and leave one partial pair of float32 rows (2 x cols at j.part), or the result
// itself where the grid is one workgroup.  A workgroup a CU keeps the partial
// pairs few; HBM bounds it, and beside that the start, the end and the second
// launch, about 8 us in all: residual 32768 x 1024 bf16 66.8 us (5.0 TB/s),
// 1537 x 5001 float32 38.5 (4.0 TB/s), layer norm 262144 x 64 bf16 22.7 (4.5
// TB/s; 24.2 with two workgroups a CU).
template <typename T, bool RES, int G, int CH, int NT, Form F, bool EARLY>
__global__ __launch_bounds__(NT) void k_norm_backward(BackwardArgs<RES> j) {
  constexpr int NW = NT / 64;
  constexpr int GL = G < 64 ? G : 64;
  constexpr bool GROUPS = G == 256;
  __shared__ float sums[G > 256 ? 1 : NW][G > 256 ? 1 : GL * 8];
  float ag[CH][8] = {}, ab[CH][8] = {};
  const int group = GROUPS ? group_of_wave(j.lanes) : G > 64 ? 0 : group_of_thread<G>();
  const int rpb = GROUPS ? j.groups : G > 64 ? 1 : NT / G;
  const int64_t first = (int64_t)blockIdx.x * rpb + group, stride = (int64_t)j.grid * rpb;
  if (j.dr.p) backward_rows<T, RES, G, CH, F, true, true, EARLY>(j, first, stride, ag, ab);
  else backward_rows<T, RES, G, CH, F, true, false, false>(j, first, stride, ag, ab);
  const Cols k(j.cols, j.rows);
  const int lane = G > 64 ? (int)threadIdx.x - group * j.lanes : threadIdx.x % G, wave = threadIdx.x / 64;
  float* const out[2] = {j.grid == 1 ? j.dgamma : j.part + (int64_t)(2 * blockIdx.x) * k.n,
                         j.grid == 1 ? j.dbeta : j.part + (int64_t)(2 * blockIdx.x + 1) * k.n};
#pragma unroll
  for (int c = 0; c < CH; ++c) {
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      float* const dst = out[a];
      float(&acc)[8] = a == 0 ? ag[c] : ab[c];
      if constexpr (G > 64) {
        if (GROUPS && j.groups > 1) {
          f32x4* const mine = (f32x4*)&sums[0][8 * threadIdx.x];
          __syncthreads();                           // the previous sums have been read
          if (group > 0) {
            mine[0] = f32x4{acc[0], acc[1], acc[2], acc[3]};
            mine[1] = f32x4{acc[4], acc[5], acc[6], acc[7]};
          }
          __syncthreads();
          if (group > 0) continue;
          for (int g = 1; g < j.groups; ++g) {
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] += (&sums[0][0])[8 * (g * j.lanes + lane) + i];
          }
        }
        if (dst) store_chunk<F>(dst, c * j.lanes + lane, k, acc, c < CH / 2);
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

// Chunks of the columns that a workgroup of backward_columns takes.
constexpr int column_lanes(int G) { return G > 64 ? 8 : 4; }

// Few rows (and any number of more than 16384 columns): the first workgroups take
// 32 columns of the weights' gradients each over all rows (64 of wide rows), the
// others the rows; x and dy are read twice (few rows the second time from a
// cache), but nothing has to meet between workgroups.  The columns' chain of loads
// bounds it: layer norm 512 x 16 float32 3.6 us, 1024 x 2048 bf16 10.2.
template <typename T, bool RES, int NT, int LC, Form F>
__device__ __forceinline__ void backward_columns(const BackwardArgs<RES>& j, int block) {
  constexpr int NW = NT / 64, SL = NT / LC, U = sizeof(T) == 2 && LC == 4 ? 8 : 4;
  __shared__ float sums[NW][2][8 * LC];
  const Cols k(j.cols, j.rows);
  const int lane = threadIdx.x % LC, q = block * LC + lane;
  float acc[2][8] = {};
  for (int64_t r = threadIdx.x / LC; r < j.rows; r += U * SL) {
    Raw<T> x[U], y[U];
    f32x2 st[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t ru = r + u * SL;
      if (ru < j.rows) {
        st[u] = *(const f32x2*)(j.stats + 2 * ru);
        x[u] = load_chunk<F>(row_of<T>(j.v, ru), q, k, ru >= k.edge);
        y[u] = load_chunk<F>(row_of<T>(j.dy, ru), q, k, ru >= k.edge);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t ru = r + u * SL;
      if (ru < j.rows) {
        float h[8], d[8];
        chunk_values<F>(x[u], q, k, ru >= k.edge, h);
        chunk_values<F>(y[u], q, k, ru >= k.edge, d);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          acc[0][i] = fmaf(d[i], (h[i] - st[u][0]) * st[u][1], acc[0][i]);
          acc[1][i] += d[i];
        }
      }
    }
  }
#pragma unroll
  for (int a = 0; a < 2; ++a) {
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[a][i] = stride_sum<LC>(acc[a][i]);
    if (threadIdx.x % 64 < LC) {
      *(f32x4*)&sums[threadIdx.x / 64][a][lane * 8] = f32x4{acc[a][0], acc[a][1], acc[a][2], acc[a][3]};
      *(f32x4*)&sums[threadIdx.x / 64][a][lane * 8 + 4] = f32x4{acc[a][4], acc[a][5], acc[a][6], acc[a][7]};
    }
  }
  __syncthreads();
  const int a = threadIdx.x / (8 * LC), i = threadIdx.x % (8 * LC), col = block * 8 * LC + i;
  if (a < 2 && col < k.n) {
    float* const dst = a == 0 ? j.dgamma : j.dbeta;
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) t += sums[w][a][i];
    if (dst) dst[col] = t;
  }
}

template <typename T, bool RES, int G, int CH, int NT, Form F>
__global__ __launch_bounds__(NT) void k_norm_backward_split(BackwardArgs<RES> j) {
  constexpr int RPB = G > 64 ? 1 : NT / G;
  constexpr int LC = column_lanes(G);
  constexpr Form FC = F == kExact && G * CH % LC != 0 ? (G == 1 ? kSmall : kRagged) : F;
  if ((int)blockIdx.x < j.col_blocks) {
    backward_columns<T, RES, NT, LC, FC>(j, blockIdx.x);
  } else {
    float none[CH][8];
    backward_rows<T, RES, G, CH, F, false, true, false>(j, (int64_t)(blockIdx.x - j.col_blocks) * RPB + group_of_thread<G>(),
                                           (int64_t)(j.grid - j.col_blocks) * RPB, none, none);
  }
}

// The partial pairs summed: a workgroup takes RC of the 2 x cols columns, each
// group of RC lanes every (kReduceThreads / RC)-th part; the groups meet in the
// wavefront, the wavefronts in LDS, always in the same order.  Latency bounds it
// (a launch, one round of loads that other XCDs wrote, two sums): 256 parts of 64
// columns 2.7 to 4.6 us, 220 of 5001 4.8.
constexpr int kReduceThreads = 1024;
template <int RC>
__global__ __launch_bounds__(kReduceThreads) void k_norm_reduce(ReduceArgs j) {
  constexpr int slices = kReduceThreads / RC, waves = kReduceThreads / 64;
  constexpr int U = 256 / slices;                  // the loads of 256 parts in flight
  __shared__ float sums[waves][RC];
  const int lane = threadIdx.x % RC, slice = threadIdx.x / RC;
  const int64_t pitch = 2 * (int64_t)j.cols;
  const int64_t c = (int64_t)blockIdx.x * RC + lane;
  float t = 0.f;
  if (c < pitch) {
    const float* p = j.part + c;
    for (int i = slice; i < j.parts; i += U * slices) {
      float v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = i + u * slices < j.parts ? p[(i + u * slices) * pitch] : 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u) t += v[u];
    }
  }
  if constexpr (RC < 64) t = stride_sum<RC>(t);
  if (threadIdx.x % 64 < RC) sums[threadIdx.x / 64][lane] = t;
  __syncthreads();
  if (slice == 0 && c < pitch) {
    t = 0.f;
#pragma unroll
    for (int w = 0; w < waves; ++w) t += sums[w][lane];
    float* const dst = c < j.cols ? j.dgamma : j.dbeta;
    if (dst) dst[c < j.cols ? c : c - j.cols] = t;
  }
}

// The forward's workgroups (in units of 256 threads).  Rows of one chunk a lane
// take one round of resident workgroups (two for the residual join, whose rows
// differ more in time), so that a thread's gamma and beta serve several rows
// and the next row's loads run beside a row's work: 120291 x 49 bf16 takes 7.8
// us, 9.3 in two rounds; residual 118955 x 175 bf16 48.5 in two, 52.5 in one.
// Wider rows are dealt out by the hardware (residual 32768 x 1024 bf16 46.6 us,
// 48.5 in two rounds) up to 8192 columns, beyond which gamma and beta are too
// many bytes to read for each row: 2000 x 16384 bf16 28.9 us with a workgroup a
// CU, 38 with one a row.
constexpr int kResident = 2048, kMany = 16384;

// threads for a row of `per` chunks, CH a thread, that takes several wavefronts
int wide_threads(int per, int CH) { return (per + 64 * CH - 1) / (64 * CH) * 64; }

// What a kernel of G lanes a row and CH chunks a lane takes for granted: the
// chunks fit, and the first half of a lane's are whole.
bool chunks_fit(int per, int lanes, int CH) { return per <= lanes * CH && (CH == 1 || per > lanes * (CH / 2)); }

// Whether the results of a call (of a backward pass: over many rows) leave the
// L2s early.  These hold up to 32 MB that a kernel's end has to write back;
// written early, that overlaps with the rows' work, but what reads a large result
// next no longer finds a part of it in a cache.  The time of the call, and of the
// call and a layer norm of its result, us, late and early: layer norm of 8 MB
// (4194 x 1000 bf16) 5.5, 4.8 and 10.2, 9.2; 16 MB (4096 x 1024 float32) 7.6, 6.2 and 15.7, 12.6; 32 MB 12.0,
// 11.2 and 25.8, 26.9; residual join of 12 MB each (6144 x 1024 bf16) 8.9, 6.2 and
// 14.5, 13.8; of 24 MB each (float32) 16.4, 19.1 and 27.3, 29.8; its backward of 8
// MB each (2048 x 1024 float32) 12.0, 10.2 and 18.3, 16.6, of 24 MB each 24.9, 26.6
// and 35.2, 37.7; a layer norm's backward of 16 MB (7813 x 500 float32) 12.0, 12.7.
// Rows of few bytes, whose stores end inside a line, take longer (layer norm
// 262144 x 13 float32 10.2, 11.8).
constexpr int64_t kEarlyNorm = 16 << 20, kEarlyJoin = 12 << 20, kEarlyBackward = 8 << 20;   // bytes of a result
constexpr int64_t kEarlyRow = 256;
template <typename T>
constexpr bool can_store_early(int chunks) { return chunks * 8 * (int)sizeof(T) >= kEarlyRow; }
template <typename T>
bool stores_early(int64_t rows, int cols, int64_t most) {
  const int64_t row = (int64_t)cols * (int64_t)sizeof(T);
  return row >= kEarlyRow && rows <= most / row;
}

template <typename T, bool RES, int G, int CH, bool HOIST = G <= 64>
hipError_t forward_with(const NormJob& j, hipStream_t st) {
  const int per = (j.cols + 7) / 8;
  const int nt = G > 64 ? wide_threads(per, CH) : kThreads, lanes = G > 64 ? nt : G;
  const int rpb = G > 64 ? 1 : nt / G;
  if (!chunks_fit(per, lanes, CH) || nt > std::max(G, kThreads)) return hipErrorInvalidConfiguration;
  const int64_t blocks = (j.rows + rpb - 1) / rpb;
  const int64_t most = G <= 64 && CH == 1 ? (RES ? 2 * kResident : kResident)
                                          : kMany;
  const int grid = (int)std::min<int64_t>(blocks, G == 1024 ? 256 : most * kThreads / nt);
  ForwardArgs<RES> a;
  if constexpr (RES) {
    a.d = j.d;
    a.r = j.r;
    a.s = j.s;
  }
  a.x = j.x;
  a.y = j.y;
  a.gamma = j.gamma;
  a.beta = j.beta;
  a.stats = j.stats;
  a.rows = j.rows;
  a.cols = j.cols;
  a.grid = grid;
  a.threads = nt;
  a.eps = j.eps;
  constexpr Form other = G == 1 ? kSmall : kRagged;
  const bool exact = j.cols == 8 * CH * lanes;
  if constexpr (can_store_early<T>(G * CH)) {
    if (stores_early<T>(j.rows, j.cols, RES && j.s.p ? kEarlyJoin : kEarlyNorm)) {
      return enqueue(exact ? k_norm_forward<T, RES, G, CH, kExact, HOIST, true>
                           : k_norm_forward<T, RES, G, CH, other, HOIST, true>, grid, nt, 0, st, a);
    }
  }
  return enqueue(exact ? k_norm_forward<T, RES, G, CH, kExact, HOIST, false>
                       : k_norm_forward<T, RES, G, CH, other, HOIST, false>, grid, nt, 0, st, a);
}

// Rows of several wavefronts: where a round of workgroups takes them all, gamma
// and beta are fetched beside the row (residual 1024 x 2048 float32: 8.1 us, 8.8
// after it); beyond that, reading them after the row's sums leaves the registers
// to more workgroups (residual 896 x 5001 bf16 11.2 us, 16.8 before; 7311 x 4040
// bf16 47.4, 50.3).  Eight wavefronts of two chunks a lane gain no workgroup by
// it (residual 1024 x 8192 bf16 13.7 after, 12.8 before).
template <typename T, bool RES, int G, int CH>
hipError_t forward_wide(const NormJob& j, hipStream_t st) {
  const int per = (j.cols + 7) / 8;
  const int64_t most = per <= 256 || per > 896 ? 1024 : 256;
  return j.rows <= most ? forward_with<T, RES, G, CH, true>(j, st) : forward_with<T, RES, G, CH, false>(j, st);
}

// threads of a workgroup of the backward
constexpr int backward_threads(int G) { return G > 512 ? G : 512; }

// Rows up to which (these included) a backward pass reads x and dy twice in one
// launch instead of leaving partial sums to a second one.  The columns' workgroups
// take a time that grows with the rows, and with their bytes once these no longer
// come from one cache; the second launch costs 2 to 4 us.  One launch against two,
// us: 1536 x 64 6.6, 7.9; bf16 layer norm 1024 x 500 7.9, 7.9, 1024 x 2048 9.9,
// 9.9; float32 layer norm 768 x 500 7.9, 7.9, residual 768 x 3000 17.5, 18.1,
// 1024 x 5001 34.4, 28.8.  One limit serves both operators, so it is too high for
// some layer norms that lie on it (1280 x 256 float32 8.1, 7.9; 768 x 5001 bf16
// 14.7, 13.8; 768 x 1500 float32 11.8, 9.8) and too low for others (2048 x 64
// 7.7, 8.0) and for some joins (1536 x 1500 bf16 13.8, 14.5).
int64_t few_rows(int per, Elt e) {
  if (per <= 16) return 1920;
  if (per <= 32) return 1280;
  return e == BF16 && per <= 512 ? 1152 : 768;
}

// How a backward pass over rows x cols runs.
struct BackwardPlan {
  int lanes, chunks;     // G and CH of the kernels
  int threads;           // of a row that takes several wavefronts, else of a workgroup
  int groups;            // rows that k_norm_backward's workgroup holds, where wide
  int parts;             // workgroups of k_norm_backward (0: k_norm_backward_split)
  int room;              // parts that these or fewer rows may take
  int col_blocks, row_blocks;   // of k_norm_backward_split
};

BackwardPlan backward_plan(int64_t rows, int cols, Elt e, bool weights) {
  const int per = (cols + 7) / 8;
  const bool wide = per > 128;
  // More than 16384 columns are four chunks a lane, which leave no registers for
  // the weights' gradients: one launch reads x and dy twice whatever the rows, and
  // a residual join keeps up to 54 registers a lane in scratch memory (its float32
  // pass over 8193 to 16384 columns up to 7).  1000 x 20000 layer norm float32 82
  // us, bf16 46 (47 and 23 for the bytes at a copy's rate), residual join 189 and
  // 123 (78 and 39).
  BackwardPlan p{};
  for (p.lanes = 1; p.lanes < 64 && p.lanes < per; p.lanes *= 2) {}
  if (wide) p.lanes = per <= 1024 ? 512 : 1024;
  p.chunks = per <= 64 ? 1 : per <= 128 ? 2 : per <= 512 ? 1 : per <= 2048 ? 2 : 4;
  p.threads = backward_threads(p.lanes);
  p.groups = 1;
  const int rpb = wide ? 1 : p.threads / p.lanes;
  int64_t blocks = (rows + rpb - 1) / rpb;
  if (weights && blocks == 1 && p.chunks <= 2) {
    p.parts = 1;
  } else if (weights && rows > few_rows(per, e) && p.chunks <= 2) {
    // bf16 rows of few wavefronts take two chunks a lane: twice the bytes in flight
    if (wide && per <= 384 && e == BF16) p.chunks = 2;
    // the workgroups of narrow wide rows hold as many of them as fill eight
    // wavefronts, so that fewer partial pairs are written and read: 2500 x 2048
    // bf16 12.4 us, 15.6 with a row each; residual 8000 x 1500 bf16 33.1, 35.6;
    // 8000 x 2048 float32 40.8, 42.1.  Not float32 rows of three wavefronts:
    // 8000 x 1032 26.9, 25.3 with a row each
    if (wide && per <= 256 && (e == BF16 || per > 192)) p.lanes = 256;
    // one chunk a lane in twice the wavefronts: their number then differs less
    // from SIMD to SIMD (1537 x 5001 residual, float32 40.7 -> 38.4 us, bf16
    // 29.0 -> 26.0; at 8192 columns, whole wavefronts either way, 59.1 -> 57.9
    // and 33.1 both)
    if (per > 512 && per <= 1024) p.lanes = 1024, p.chunks = 1;
    if (wide) p.threads = wide_threads(per, p.chunks);
    if (p.lanes == 256) {
      p.groups = 512 / p.threads;
      blocks = (rows + p.groups - 1) / p.groups;
    }
    // the rows dealt out evenly to workgroups of eight wavefronts in all a CU
    const int64_t most = 256 * std::max(1, 512 / (p.threads * p.groups));
    const int64_t rounds = (blocks + most - 1) / most;
    p.parts = (int)((blocks + rounds - 1) / rounds);
    p.room = (int)std::min(blocks, most);
  } else {
    p.col_blocks = weights ? (per + column_lanes(p.lanes) - 1) / column_lanes(p.lanes) : 0;
    p.row_blocks = (int)std::min<int64_t>(blocks, kMany);
  }
  return p;
}

template <typename T, bool RES, int G, int CH>
hipError_t backward_with(const NormJob& j, const BackwardPlan& p, hipStream_t st) {
  constexpr int nt = backward_threads(G);
  constexpr Form other = G == 1 ? kSmall : kRagged;
  const int lanes = G > 64 ? p.threads : G;
  const bool exact = j.cols == 8 * CH * lanes;
  if (!chunks_fit((j.cols + 7) / 8, lanes, CH)) return hipErrorInvalidConfiguration;
  BackwardArgs<RES> a;
  if constexpr (RES) {
    // an absent operand becomes one that changes nothing, at the price of a load
    // that is not used or of a second store to the same place: ds is read from v
    // and not added, dr goes where dx is written after it, dx where dr is, undropped
    a.d = j.d;
    a.add = j.ds.p != nullptr;
    a.ds = j.ds.p ? j.ds : j.v;
    a.dx = j.dx.p ? j.dx : j.dr;
    if (!j.dx.p) a.d.thr = 0;
  }
  a.v = j.v;
  a.dy = j.dy;
  a.dr = j.dr.p ? j.dr : j.dx;
  a.gamma = j.gamma;
  a.stats = j.stats;
  a.dgamma = j.dgamma;
  a.dbeta = j.dbeta;
  a.part = j.part;
  a.rows = j.rows;
  a.cols = j.cols;
  a.lanes = p.threads;
  a.groups = p.groups;
  a.col_blocks = 0;
  if constexpr (CH <= 2) {
    if (p.parts > 0) {
      a.grid = p.parts;
      const int threads = p.threads * p.groups;
      if constexpr (can_store_early<T>(G * CH)) {
        if (stores_early<T>(j.rows, j.cols, kEarlyBackward)) {
          return enqueue(exact ? k_norm_backward<T, RES, G, CH, nt, kExact, true>
                               : k_norm_backward<T, RES, G, CH, nt, other, true>, p.parts, threads, 0, st, a);
        }
      }
      return enqueue(exact ? k_norm_backward<T, RES, G, CH, nt, kExact, false>
                           : k_norm_backward<T, RES, G, CH, nt, other, false>, p.parts, threads, 0, st, a);
    }
  }
  if constexpr (G == 256 || (G == 1024 && CH == 1)) {   // many rows only
    return hipErrorInvalidConfiguration;
  } else {
    auto run = [&](int col_blocks, int row_blocks) {
      a.col_blocks = col_blocks;
      a.grid = col_blocks + row_blocks;
      if (a.grid == 0) return hipSuccess;
      return enqueue(exact ? k_norm_backward_split<T, RES, G, CH, nt, kExact>
                           : k_norm_backward_split<T, RES, G, CH, nt, other>, a.grid, nt, 0, st, a);
    };
    const int row_blocks = j.dr.p || j.dx.p ? p.row_blocks : 0;
    auto over = [&](const Mat& m) { return m.p && (m.p == j.dy.p || m.p == j.v.p); };
    if (row_blocks > 0 && (over(j.dr) || over(j.dx))) {   // in place: the columns first
      const hipError_t e = run(p.col_blocks, 0);
      return e == hipSuccess ? run(0, row_blocks) : e;
    }
    return run(p.col_blocks, row_blocks);
  }
}

template <typename T, bool RES>
hipError_t backward(const NormJob& j, const BackwardPlan& p, hipStream_t st) {
  switch (p.lanes) {
    case 1: return backward_with<T, RES, 1, 1>(j, p, st);
    case 2: return backward_with<T, RES, 2, 1>(j, p, st);
    case 4: return backward_with<T, RES, 4, 1>(j, p, st);
    case 8: return backward_with<T, RES, 8, 1>(j, p, st);
    case 16: return backward_with<T, RES, 16, 1>(j, p, st);
    case 32: return backward_with<T, RES, 32, 1>(j, p, st);
    case 64: return p.chunks == 1 ? backward_with<T, RES, 64, 1>(j, p, st) : backward_with<T, RES, 64, 2>(j, p, st);
    case 256: return backward_with<T, RES, 256, sizeof(T) == 2 ? 2 : 1>(j, p, st);
    case 512: return p.chunks == 1 ? backward_with<T, RES, 512, 1>(j, p, st) : backward_with<T, RES, 512, 2>(j, p, st);
    default:
      if (p.chunks == 1) return backward_with<T, RES, 1024, 1>(j, p, st);
      return p.chunks == 2 ? backward_with<T, RES, 1024, 2>(j, p, st) : backward_with<T, RES, 1024, 4>(j, p, st);
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
  // bf16 rows take two chunks a lane for as many bytes in flight as float32
  // rows have with one: 20000 x 1200 bf16 29.3 us, 31.9 with one
  if (per <= 512 && sizeof(T) == 4) return forward_wide<T, RES, 512, 1>(j, st);
  if (per <= 1024) return forward_wide<T, RES, 512, 2>(j, st);
  if (per <= 2048) return forward_with<T, RES, 1024, 2, true>(j, st);
  return forward_with<T, RES, 1024, 4, false>(j, st);   // registers: none left for gamma and beta
}

}  // namespace

int norm_parts(int64_t rows, int cols) {
  return std::max({1, backward_plan(rows, cols, F32, true).room, backward_plan(rows, cols, BF16, true).room});
}

template <typename T>
hipError_t dropout(const DropJob& j, hipStream_t st) {
  const int64_t per = ((int64_t)j.cols + 7) / 8;
  const int64_t chunks = j.rows > (INT64_MAX >> 2) / per ? INT64_MAX >> 2 : j.rows * per;
  const int grid = (int)std::min<int64_t>((chunks + kThreads - 1) / kThreads, kMany);
  const int64_t stride = (int64_t)grid * kThreads;
  const DropArgs a{j.d, j.x, j.y, j.rows, stride / per, j.cols, (int)(stride % per)};
  return enqueue(j.cols % 8 == 0 ? k_dropout<T, kExact> : j.cols > 8 ? k_dropout<T, kRagged> : k_dropout<T, kSmall>,
                 grid, kThreads, 0, st, a);
}

hipError_t launch_dropout(Elt e, const DropJob& j, hipStream_t st) {
  return e == BF16 ? dropout<uint16_t>(j, st) : dropout<float>(j, st);
}

hipError_t launch_norm_forward(Elt e, const NormJob& j, hipStream_t st) {
  if (e == BF16) return j.r.p ? forward<uint16_t, true>(j, st) : forward<uint16_t, false>(j, st);
  return j.r.p ? forward<float, true>(j, st) : forward<float, false>(j, st);
}

hipError_t launch_norm_backward(Elt e, const NormJob& j, hipStream_t st) {
  const bool weights = j.dgamma || j.dbeta, residual = j.ds.p || j.dx.p;
  const BackwardPlan p = backward_plan(j.rows, j.cols, e, weights);
  hipError_t err;
  if (e == BF16) err = residual ? backward<uint16_t, true>(j, p, st) : backward<uint16_t, false>(j, p, st);
  else err = residual ? backward<float, true>(j, p, st) : backward<float, false>(j, p, st);
  if (err != hipSuccess || p.parts <= 1) return err;
  const ReduceArgs a{j.part, j.dgamma, j.dbeta, j.cols, p.parts};
  // 64 columns a workgroup once they fill the CUs, else 16
  if (2 * j.cols > 256 * 16) return enqueue(k_norm_reduce<64>, (2 * j.cols + 63) / 64, kReduceThreads, 0, st, a);
  return enqueue(k_norm_reduce<16>, (2 * j.cols + 15) / 16, kReduceThreads, 0, st, a);
}

}  // namespace vfl
