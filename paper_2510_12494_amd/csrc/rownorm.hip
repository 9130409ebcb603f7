// Row operators of residual towers on gfx950: dropout, layer norm and the
// residual join of the two, forward and backward.
//
// A workgroup of 256 threads takes a row at a time; a thread takes chunks of
// eight columns, which share one Philox block of the dropout's numbers.  All
// sums are float32.
#include <algorithm>

#include "device.h"
#include "kernels.h"

namespace vfl {
namespace {

using namespace dev;

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMaxParts = 256;

// bit i: column 8q + i of the row is kept
__device__ __forceinline__ uint32_t keep_bits(const DropKey& d, uint32_t step, int64_t row, uint32_t q) {
  const uint64_t id = (uint64_t)row;
  uint32_t c[4] = {step, (uint32_t)id, q, 0x80000000u | ((uint32_t)(id >> 32) << 16) | d.tag};
  philox4x32_10(c, d.k0, d.k1);
  uint32_t bits = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    bits |= ((c[i] & 0xffffu) >= d.thr ? 1u : 0u) << (2 * i);
    bits |= ((c[i] >> 16) >= d.thr ? 1u : 0u) << (2 * i + 1);
  }
  return bits;
}

__device__ __forceinline__ uint32_t step_of(const DropKey& d) {
  return d.step + (d.step_dev ? *d.step_dev : 0u);
}

template <typename T>
__device__ __forceinline__ const T* row_of(const Mat& m, int64_t r) { return (const T*)m.p + r * m.ld; }
template <typename T>
__device__ __forceinline__ T* out_row(const Mat& m, int64_t r) { return (T*)m.p + r * m.ld; }

// the sum over the workgroup's threads, in every thread
__device__ __forceinline__ float block_sum(float v, float* lds) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  __syncthreads();                               // the previous sum has been read
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) s += lds[w];
  return s;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_dropout(DropJob j) {
  const uint32_t step = step_of(j.d);
  for (int64_t r = blockIdx.x; r < j.rows; r += gridDim.x)
    for (int q = threadIdx.x; q * 8 < j.cols; q += kThreads) {
      const uint32_t keep = j.d.thr ? keep_bits(j.d, step, j.d.row0 + r, q) : 0xffu;
      for (int i = 0; i < 8 && q * 8 + i < j.cols; ++i) {
        const float v = ld1<T>(row_of<T>(j.x, r) + q * 8 + i);
        st1<T>(out_row<T>(j.y, r) + q * 8 + i, (keep >> i & 1u) ? v * j.d.scale : 0.f);
      }
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_norm_forward(NormJob j) {
  __shared__ float lds[kWaves];
  const uint32_t step = step_of(j.d);
  const float inv = 1.f / (float)j.cols;
  for (int64_t r = blockIdx.x; r < j.rows; r += gridDim.x) {
    const T* x = row_of<T>(j.x, r);
    const T* res = j.r.p ? row_of<T>(j.r, r) : nullptr;
    auto visit = [&](auto&& f) {
      for (int q = threadIdx.x; q * 8 < j.cols; q += kThreads) {
        const uint32_t keep = j.d.thr ? keep_bits(j.d, step, j.d.row0 + r, q) : 0xffu;
        for (int i = 0; i < 8 && q * 8 + i < j.cols; ++i) {
          const int c = q * 8 + i;
          float v = (keep >> i & 1u) ? ld1<T>(x + c) * j.d.scale : 0.f;
          if (res) v += ld1<T>(res + c);
          f(c, v);
        }
      }
    };
    float sum = 0.f, sq = 0.f;
    visit([&](int, float v) { sum += v; });
    const float mean = block_sum(sum, lds) * inv;
    visit([&](int, float v) { sq += (v - mean) * (v - mean); });
    const float k = 1.f / sqrtf(block_sum(sq, lds) * inv + j.eps);
    visit([&](int c, float v) {
      const float g = j.gamma ? j.gamma[c] : 1.f, b = j.beta ? j.beta[c] : 0.f;
      if (j.s.p) st1<T>(out_row<T>(j.s, r) + c, v);
      st1<T>(out_row<T>(j.y, r) + c, (v - mean) * k * g + b);
    });
    if (j.stats && threadIdx.x == 0) {
      j.stats[2 * r] = mean;
      j.stats[2 * r + 1] = k;
    }
  }
}

// Partial weight gradients: block (x, y) sums the rows of part y in columns
// 256 x ..  It runs before k_norm_dx, which may write over dy.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_norm_part(NormJob j, int parts) {
  const int c = blockIdx.x * kThreads + threadIdx.x;
  if (c >= j.cols) return;
  float dg = 0.f, db = 0.f;
  for (int64_t r = blockIdx.y; r < j.rows; r += parts) {
    const float dy = ld1<T>(row_of<T>(j.dy, r) + c);
    dg += dy * ((ld1<T>(row_of<T>(j.v, r) + c) - j.stats[2 * r]) * j.stats[2 * r + 1]);
    db += dy;
  }
  j.part[(int64_t)(2 * blockIdx.y) * j.cols + c] = dg;
  j.part[(int64_t)(2 * blockIdx.y + 1) * j.cols + c] = db;
}

__global__ __launch_bounds__(kThreads) void k_norm_reduce(NormJob j, int parts) {
  const int c = blockIdx.x * kThreads + threadIdx.x;
  if (c >= j.cols) return;
  float dg = 0.f, db = 0.f;
  for (int p = 0; p < parts; ++p) {
    dg += j.part[(int64_t)(2 * p) * j.cols + c];
    db += j.part[(int64_t)(2 * p + 1) * j.cols + c];
  }
  if (j.dgamma) j.dgamma[c] = dg;
  if (j.dbeta) j.dbeta[c] = db;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_norm_dx(NormJob j) {
  __shared__ float lds[kWaves];
  const uint32_t step = step_of(j.d);
  const float inv = 1.f / (float)j.cols;
  for (int64_t r = blockIdx.x; r < j.rows; r += gridDim.x) {
    const T *v = row_of<T>(j.v, r), *dy = row_of<T>(j.dy, r);
    const float mean = j.stats[2 * r], k = j.stats[2 * r + 1];
    float sg = 0.f, sgh = 0.f;
    for (int c = threadIdx.x; c < j.cols; c += kThreads) {
      const float g = ld1<T>(dy + c) * (j.gamma ? j.gamma[c] : 1.f);
      sg += g;
      sgh += g * ((ld1<T>(v + c) - mean) * k);
    }
    const float mg = block_sum(sg, lds) * inv, mgh = block_sum(sgh, lds) * inv;
    for (int q = threadIdx.x; q * 8 < j.cols; q += kThreads) {
      const uint32_t keep = j.d.thr && j.dx.p ? keep_bits(j.d, step, j.d.row0 + r, q) : 0xffu;
      for (int i = 0; i < 8 && q * 8 + i < j.cols; ++i) {
        const int c = q * 8 + i;
        const float g = ld1<T>(dy + c) * (j.gamma ? j.gamma[c] : 1.f);
        float d = k * (g - mg - (ld1<T>(v + c) - mean) * k * mgh);
        if (j.ds.p) d += ld1<T>(row_of<T>(j.ds, r) + c);
        if (j.dr.p) st1<T>(out_row<T>(j.dr, r) + c, d);
        if (j.dx.p) st1<T>(out_row<T>(j.dx, r) + c, (keep >> i & 1u) ? d * j.d.scale : 0.f);
      }
    }
  }
}

int row_grid(int64_t rows) { return (int)std::min<int64_t>(rows, 1 << 16); }

}  // namespace

int norm_parts(int64_t rows, int) { return (int)std::min<int64_t>(rows, kMaxParts); }

hipError_t launch_dropout(Elt e, const DropJob& j, hipStream_t st) {
  const dim3 g(row_grid(j.rows));
  if (e == BF16) hipLaunchKernelGGL(k_dropout<uint16_t>, g, dim3(kThreads), 0, st, j);
  else hipLaunchKernelGGL(k_dropout<float>, g, dim3(kThreads), 0, st, j);
  return hipGetLastError();
}

hipError_t launch_norm_forward(Elt e, const NormJob& j, hipStream_t st) {
  const dim3 g(row_grid(j.rows));
  if (e == BF16) hipLaunchKernelGGL(k_norm_forward<uint16_t>, g, dim3(kThreads), 0, st, j);
  else hipLaunchKernelGGL(k_norm_forward<float>, g, dim3(kThreads), 0, st, j);
  return hipGetLastError();
}

hipError_t launch_norm_backward(Elt e, const NormJob& j, hipStream_t st) {
  const int cb = (j.cols + kThreads - 1) / kThreads;
  if (j.dgamma || j.dbeta) {
    const int parts = norm_parts(j.rows, j.cols);
    if (parts > 0) {
      if (e == BF16) hipLaunchKernelGGL(k_norm_part<uint16_t>, dim3(cb, parts), dim3(kThreads), 0, st, j, parts);
      else hipLaunchKernelGGL(k_norm_part<float>, dim3(cb, parts), dim3(kThreads), 0, st, j, parts);
    }
    hipLaunchKernelGGL(k_norm_reduce, dim3(cb), dim3(kThreads), 0, st, j, parts);
  }
  if (j.rows > 0 && (j.dr.p || j.dx.p)) {
    const dim3 g(row_grid(j.rows));
    if (e == BF16) hipLaunchKernelGGL(k_norm_dx<uint16_t>, g, dim3(kThreads), 0, st, j);
    else hipLaunchKernelGGL(k_norm_dx<float>, g, dim3(kThreads), 0, st, j);
  }
  return hipGetLastError();
}

}  // namespace vfl
