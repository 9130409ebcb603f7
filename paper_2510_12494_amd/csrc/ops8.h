// Internal launch interface of the operators of towers in 8 bits and of a head
// with many classes (not part of the C ABI): vfl_rmsnorm_*, vfl_quantize,
// vfl_matmul8, vfl_softmax_loss_*.
#pragma once
#include "rowops.h"

namespace vfl {

constexpr int kBlock8 = 128;           // columns that share a power of two

// A matrix in 8 bits (vfl_q8); a null p: absent.
struct Mat8 {
  uint8_t* p = nullptr;
  int64_t ld = 0;
  uint8_t* scale = nullptr;
  int64_t scale_ld = 0;
};

// v = r + x (r null: x), s = v, y = v * k * gamma in the storage type and / or in
// 8 bits, stats = k, each where not null.
struct RmsJob {
  Mat x, r, s, y;
  Mat8 q;
  const float* gamma;
  float* stats;
  float eps;
  int cols;
  int64_t rows;
};

struct QuantJob {
  Mat x;
  Mat8 q, qt;
  int64_t rows, cols;
};

// c = a b^T + bias, ReLU; part: the partial sums of a split product
struct Matmul8Job {
  Mat8 a, b;
  Mat c;
  const float* bias;
  float* part;
  int relu;
  int64_t m, n, k;
};

// The softmax loss of a linear head: z = x w^T + bias over `classes` columns.
// forward: lse and loss of each row; backward: dx, dw, dbias, each where not null.
struct LossJob {
  Mat x, w, dx, dw;
  const float* bias;
  const int32_t* labels;
  float *loss, *lse;
  const float* dloss;                  // of each row (null: `scale` for all)
  float scale;
  float* dbias;
  char* workspace;
  int dim;
  int64_t rows, classes;
};

hipError_t launch_rms_forward(Elt e, const RmsJob& j, hipStream_t st);
hipError_t launch_quantize(Elt e, const QuantJob& j, hipStream_t st);
size_t matmul8_workspace(int64_t m, int64_t n, int64_t k);
hipError_t launch_matmul8(Elt e, const Matmul8Job& j, hipStream_t st);

// bytes that the forward and the backward pass of these sizes need
size_t loss_workspace(Elt e, int64_t rows, int dim, int64_t classes);
hipError_t launch_loss_forward(Elt e, const LossJob& j, hipStream_t st);
hipError_t launch_loss_backward(Elt e, const LossJob& j, hipStream_t st);

}  // namespace vfl
