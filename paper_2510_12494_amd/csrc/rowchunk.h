// Device helpers of the row operators (dropout, norms, joins, matrices in 8
// bits): chunks of eight columns, loaded and stored at element alignment, and sums
// over groups of lanes.
#pragma once
#include "device.h"
#include "rowops.h"

namespace vfl {
namespace dev {

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

template <typename T>
__device__ __forceinline__ const T* row_of(const Mat& m, int64_t r) { return (const T*)m.p + r * m.ld; }
template <typename T>
__device__ __forceinline__ T* out_row(const Mat& m, int64_t r) { return (T*)m.p + r * m.ld; }

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

}  // namespace dev
}  // namespace vfl
