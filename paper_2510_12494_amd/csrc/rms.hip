// The root-mean-square norm of a residual join, with results in the storage type,
// in 8 bits, or both, and the conversion of a matrix (and its transpose) to 8
// bits, on gfx950.  Both move a few bytes per operation, so HBM bounds them.
#include <algorithm>

#include "eight.h"
#include "ops8.h"

namespace vfl {
namespace {

using namespace dev;

constexpr int kThreads = 256;

struct RmsArgs {
  Mat x, r, s, y;
  Mat8 q;
  const float* gamma;
  float* stats;
  int64_t rows;
  int cols, grid, threads;
  double eps;
};
struct QuantArgs {
  Mat x;
  Mat8 q, qt;
  int64_t rows, tiles;
  int cols, tn, grid;
};

// The sum over each group of G lanes, in every lane of it, in 64 bits.
__device__ __forceinline__ double halves(uint32_t lo, uint32_t hi) {
  return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
template <int CTRL>
__device__ __forceinline__ double dpp64(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  return halves((uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, 0xf, 0xf, true),
                (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, 0xf, 0xf, true));
}
template <int G>
__device__ __forceinline__ double group_sum64(double v) {
  v += dpp64<0xB1>(v);
  v += dpp64<0x4E>(v);
  v += dpp64<0x141>(v);
  v += dpp64<0x140>(v);
  if constexpr (G >= 32) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)u, (uint32_t)u, false, false);
    const auto hi = __builtin_amdgcn_permlane16_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
    v = halves(lo[0], hi[0]) + halves(lo[1], hi[1]);
  }
  if constexpr (G >= 64) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const auto lo = __builtin_amdgcn_permlane32_swap((uint32_t)u, (uint32_t)u, false, false);
    const auto hi = __builtin_amdgcn_permlane32_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
    v = halves(lo[0], hi[0]) + halves(lo[1], hi[1]);
  }
  return v;
}

// 1 / sqrt(v) in 64 bits: the instruction's estimate and two Newton steps
__device__ __forceinline__ double inverse_root(double v) {
  double k = __builtin_amdgcn_rsq(v);
  const double half = 0.5 * v;
  double n = k * fma(-half * k, k, 1.5);
  n = n * fma(-half * n, n, 1.5);
  return v < __builtin_inf() ? n : k;                 // of an infinity 0, of a NaN NaN
}

// Lanes hold rows as in the layer norm's forward: G = 16 to 64 lanes and CH chunks
// of eight columns each, or (G > 64) a workgroup's wavefronts.  16 lanes hold a
// block of 128 columns, so a block's largest magnitude is four exchanges away.
// The sum of squares is taken in 64 bits: products of float32 values are exact
// there, so k does not depend on the order of the sum and the same row gives the
// same 8-bit values whatever the batch, the width's layout or the machine.  HBM bounds
// it: 32768 x 1024 bf16, x and r in, s, 8 bits and k out, 235 MB: 35 us beside the
// last-level cache, 42 from memory (5.6 TB/s); one row 2.6 us, latency.
template <typename T, int G, int CH, Form F>
__global__ __launch_bounds__(G > kThreads ? G : kThreads) void k_rms_forward(RmsArgs j) {
  constexpr bool WIDE = G > 64;
  constexpr int RPB = WIDE ? 1 : kThreads / G;
  constexpr int GL = G < 64 ? G : 64;
  constexpr bool AHEAD = G < 1024, HOIST = CH <= 2;
  __shared__ double slots[2][WIDE ? 16 : 1];
  const Cols k(j.cols, j.rows);
  const int lanes = WIDE ? j.threads : G;
  const int lane = WIDE ? (int)threadIdx.x : threadIdx.x % G;
  const int blocks = (j.cols + kBlock8 - 1) / kBlock8;
  const double inv = 1.0 / (double)k.n;

  Raw<T> x[CH], res[CH];
  auto fetch = [&](int64_t r) {
    const bool edge = r >= k.edge;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      x[c] = load_chunk<F>(row_of<T>(j.x, r), c * lanes + lane, k, edge, c < CH / 2);
      if (j.r.p) res[c] = load_chunk<F>(row_of<T>(j.r, r), c * lanes + lane, k, edge, c < CH / 2);
    }
  };
  const int64_t stride = (int64_t)j.grid * RPB;
  int64_t r = (int64_t)blockIdx.x * RPB + group_of_thread<G>();
  if (AHEAD && r < j.rows) fetch(r);

  float gm[HOIST ? CH : 1][8];
  auto weights = [&](int c, int slot) {
#pragma unroll
    for (int i = 0; i < 8; ++i) gm[slot][i] = 1.f;
    if (j.gamma) vector_values<F>(j.gamma, c * lanes + lane, k, gm[slot], c < CH / 2);
  };
  if constexpr (HOIST)
    for (int c = 0; c < CH; ++c) weights(c, c);

  int flip = 0;
  for (; r < j.rows; r += stride) {
    if constexpr (!AHEAD) fetch(r);
    const bool edge = r >= k.edge;
    float v[CH][8];
    double sum = 0.0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int q = c * lanes + lane;
      chunk_values<F>(x[c], q, k, edge, v[c], c < CH / 2);
      if (j.r.p) {
        float t[8];
        chunk_values<F>(res[c], q, k, edge, t, c < CH / 2);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] += t[i];
      }
    }
    if (AHEAD && r + stride < j.rows) fetch(r + stride);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if (j.s.p) store_chunk<F>(out_row<T>(j.s, r), c * lanes + lane, k, v[c], c < CH / 2);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fma((double)v[c][i], (double)v[c][i], sum);
    }
    sum = group_sum64<GL>(sum);
    if constexpr (WIDE) {
      if (threadIdx.x % 64 == 0) slots[flip][threadIdx.x / 64] = sum;
      __syncthreads();
      const int w = threadIdx.x % 16;
      sum = group_sum64<16>(64 * w < lanes ? slots[flip][w] : 0.0);
      flip ^= 1;
    }
    const float rk = (float)inverse_root(fma(sum, inv, j.eps));
    if (j.stats && lane == 0) j.stats[r] = rk;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int q = c * lanes + lane;
      const int at = HOIST ? c : 0;
      if constexpr (!HOIST) weights(c, 0);
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = v[c][i] * rk * gm[at][i];
      if (j.y.p) store_chunk<F>(out_row<T>(j.y, r), q, k, y, c < CH / 2);
      if (j.q.p) {
        // past the row's end the values are 0, or NaN where k is infinite or NaN
        const int left = k.n - 8 * q;
        if (F != kExact) {
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = i < left ? y[i] : 0.f;
        }
        uint32_t m = block_max(chunk_max(y));
        if (m >= kInfinite) {
          m = 0;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            m = max(m, number_magnitude(y[i]));
            y[i] = number_or_nan(y[i]);
          }
          m = block_max(m);
        }
        const uint32_t b = scale_byte(m);
        if ((q >> 4) < blocks) {
          *(u32x2*)(j.q.p + r * j.q.ld + 8 * (int64_t)q) = pack_e4m3(y, inverse_scale(b));
          if ((q & 15) == 0) j.q.scale[(int64_t)(q >> 4) * j.q.scale_ld + r] = (uint8_t)b;
        }
      }
    }
  }
}

// The largest over the four lanes of a wavefront that share lane % 16.
__device__ __forceinline__ uint32_t quarters_max(uint32_t v) {
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max((uint32_t)a[0], (uint32_t)a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max((uint32_t)b[0], (uint32_t)b[1]);
}

// Chunks as they are stored: value i, and a chunk of values of the storage type.
__device__ __forceinline__ float value(const Raw<uint16_t>& r, int i) {
  return __uint_as_float(i & 1 ? r.a[i / 2] & 0xffff0000u : r.a[i / 2] << 16);
}
__device__ __forceinline__ float value(const Raw<float>& r, int i) { return i < 4 ? r.a[i] : r.b[i - 4]; }
__device__ __forceinline__ void hold(Raw<uint16_t>& r, const float (&v)[8]) {
  r.a = u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
}
__device__ __forceinline__ void hold(Raw<float>& r, const float (&v)[8]) {
  r.a = f32x4{v[0], v[1], v[2], v[3]};
  r.b = f32x4{v[4], v[5], v[6], v[7]};
}
// What follows unpacks the chunk again instead of holding its values.
__device__ __forceinline__ void again(Raw<uint16_t>& r) { asm volatile("" : "+v"(r.a)); }
__device__ __forceinline__ void again(Raw<float>&) {}

// A workgroup takes 128 x 128 values, a thread eight rows of a chunk of eight
// columns: its rows' blocks are 16 lanes wide, its columns' blocks the workgroup's
// 16 groups of them, which meet in LDS.  A thread's eight rows of a column are
// eight consecutive bytes of the transpose.  HBM bounds it, and what keeps it busy is
// the number of tiles in flight: a thread holds its values as they are stored and
// unpacks them for each pass (four wavefronts a SIMD in bf16; two with 64 floats
// held).  32768 x 1024 bf16, 64 MB in and 67 out, from memory: 33 us, 38 with floats
// held (131072 x 200: 33, 47); without the transpose 22, 27.
template <typename T, Form F>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 4 : 3) void k_quantize(QuantArgs j) {
  __shared__ uint32_t tops[2][4][128];
  const Cols k(j.cols, j.rows);
  const int lane = threadIdx.x & 15, group = threadIdx.x >> 4, wave = threadIdx.x >> 6;
  int flip = 0;
  for (int64_t t = blockIdx.x; t < j.tiles; t += j.grid, flip ^= 1) {
    const int64_t tm = t / j.tn;
    const int tn = (int)(t - tm * j.tn);
    const int64_t r0 = 128 * tm + 8 * group;
    const int q = 16 * tn + lane;
    Raw<T> x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t r = min(r0 + i, j.rows - 1);
      x[i] = load_chunk<F>(row_of<T>(j.x, r), q, k, r >= k.edge);
    }
    // the rows' and the thread's largest magnitudes; what is no number shows in them
    uint32_t top[8], most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t r = min(r0 + i, j.rows - 1);
      float v[8];
      chunk_values<F>(x[i], q, k, r >= k.edge, v);
      if (F != kExact) hold(x[i], v);
      top[i] = chunk_max(v);
      if (r0 + i >= j.rows) {
        x[i] = Raw<T>{};
        top[i] = 0;
      }
      most = max(most, top[i]);
      again(x[i]);
    }
    if (__any(most >= kInfinite)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float v[8];
        unpack(x[i], v);
        top[i] = 0;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          top[i] = max(top[i], number_magnitude(v[c]));
          v[c] = number_or_nan(v[c]);
        }
        hold(x[i], v);
      }
    }
    if (j.q.p) {
      u32x2 bytes = {0u, 0u};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float v[8];
        unpack(x[i], v);
        const uint32_t b = scale_byte(block_max(top[i]));
        bytes[i / 4] |= b << (8 * (i % 4));
        if (r0 + i < j.rows) *(u32x2*)(j.q.p + (r0 + i) * j.q.ld + 8 * (int64_t)q) = pack_e4m3(v, inverse_scale(b));
        again(x[i]);
      }
      if (lane == 0 && r0 < j.rows) *(u32x2*)(j.q.scale + tn * j.q.scale_ld + r0) = bytes;
    }
    if (j.qt.p) {
      uint32_t m[8];
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        m[c] = 0;
        if (most < kInfinite) {
#pragma unroll
          for (int i = 0; i < 8; ++i) m[c] = max(m[c], magnitude(value(x[i], c)));
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) m[c] = max(m[c], number_magnitude(value(x[i], c)));
        }
        m[c] = quarters_max(m[c]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) again(x[i]);
      if ((threadIdx.x & 63) < 16) {
        *(u32x4*)&tops[flip][wave][8 * lane] = u32x4{m[0], m[1], m[2], m[3]};
        *(u32x4*)&tops[flip][wave][8 * lane + 4] = u32x4{m[4], m[5], m[6], m[7]};
      }
      __syncthreads();
      u32x2 bytes = {0u, 0u};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4 top = *(const u32x4*)&tops[flip][0][8 * lane + 4 * h];
#pragma unroll
        for (int w = 1; w < 4; ++w) {
          const u32x4 o = *(const u32x4*)&tops[flip][w][8 * lane + 4 * h];
#pragma unroll
          for (int c = 0; c < 4; ++c) top[c] = max(top[c], o[c]);
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) bytes[h] |= scale_byte(top[c]) << (8 * c);
      }
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        float w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = value(x[i], c);
        const uint32_t b = (bytes[c / 4] >> (8 * (c % 4))) & 255u;
        const int64_t col = 8 * (int64_t)q + c;
        if (col < j.cols) *(u32x2*)(j.qt.p + col * j.qt.ld + r0) = pack_e4m3(w, inverse_scale(b));
      }
      if (group == 0 && 8 * (int64_t)q < j.cols) *(u32x2*)(j.qt.scale + tm * j.qt.scale_ld + 8 * (int64_t)q) = bytes;
    }
  }
}

constexpr int kResident = 4096, kMany = 16384;   // workgroups of 256 threads

template <typename T, int G, int CH>
hipError_t forward_with(const RmsJob& j, hipStream_t st) {
  const int per = (j.cols + 7) / 8;
  const int nt = G > 64 ? (per + 64 * CH - 1) / (64 * CH) * 64 : kThreads, lanes = G > 64 ? nt : G;
  const int rpb = G > 64 ? 1 : nt / G;
  if (per > lanes * CH || (CH > 1 && per <= lanes * (CH / 2)) || nt > std::max(G, kThreads))
    return hipErrorInvalidConfiguration;
  const int64_t blocks = (j.rows + rpb - 1) / rpb;
  const int64_t most = G <= 64 && CH == 1 ? kResident : kMany;
  RmsArgs a{j.x, j.r, j.s, j.y, j.q, j.gamma, j.stats, j.rows, j.cols, 0, nt, (double)j.eps};
  a.grid = (int)std::min<int64_t>(blocks, G == 1024 ? 256 : most * kThreads / nt);
  const bool exact = j.cols == 8 * CH * lanes;
  if constexpr (G == 16)
    if (j.cols < 8) return enqueue(k_rms_forward<T, G, CH, kSmall>, a.grid, nt, 0, st, a);
  return enqueue(exact ? k_rms_forward<T, G, CH, kExact> : k_rms_forward<T, G, CH, kRagged>, a.grid, nt, 0, st, a);
}

template <typename T>
hipError_t forward(const RmsJob& j, hipStream_t st) {
  const int per = (j.cols + 7) / 8;
  if (per <= 16) return forward_with<T, 16, 1>(j, st);
  if (per <= 32) return forward_with<T, 32, 1>(j, st);
  if (per <= 64) return forward_with<T, 64, 1>(j, st);
  if (per <= 128) return forward_with<T, 64, 2>(j, st);
  if (per <= 512 && sizeof(T) == 4) return forward_with<T, 512, 1>(j, st);
  if (per <= 1024) return forward_with<T, 512, 2>(j, st);
  if (per <= 2048) return forward_with<T, 1024, 2>(j, st);
  return forward_with<T, 1024, 4>(j, st);
}

template <typename T>
hipError_t quantize(const QuantJob& j, hipStream_t st) {
  QuantArgs a{j.x, j.q, j.qt, j.rows, 0, (int)j.cols, (int)((j.cols + 127) / 128), 0};
  a.tiles = (j.rows + 127) / 128 * a.tn;
  a.grid = (int)std::min<int64_t>(a.tiles, kMany);
  return enqueue(j.cols % 128 == 0 ? k_quantize<T, kExact> : j.cols >= 8 ? k_quantize<T, kRagged> : k_quantize<T, kSmall>,
                 a.grid, kThreads, 0, st, a);
}

}  // namespace

hipError_t launch_rms_forward(Elt e, const RmsJob& j, hipStream_t st) {
  return e == BF16 ? forward<uint16_t>(j, st) : forward<float>(j, st);
}

hipError_t launch_quantize(Elt e, const QuantJob& j, hipStream_t st) {
  return e == BF16 ? quantize<uint16_t>(j, st) : quantize<float>(j, st);
}

}  // namespace vfl
