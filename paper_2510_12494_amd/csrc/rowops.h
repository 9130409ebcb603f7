// Internal launch interface of the row operators (not part of the C ABI):
// dropout, layer norm and the residual join of the two (vfl_dropout,
// vfl_layernorm_*, vfl_residual_*).
#pragma once
#include "kernels.h"

namespace vfl {

// A row-major matrix of elements of the call's type with its own ld; a null p:
// absent.
struct Mat { void* p = nullptr; int64_t ld = 0; };

// thr: elements whose 16-bit number is below it are dropped (0: no dropout,
// 65536: all); scale = 65536 / (65536 - thr) (0 where all are dropped).
struct DropKey {
  uint32_t thr = 0, k0 = 0, k1 = 0, step = 0, tag = 0;
  float scale = 1.f;
  const uint32_t* step_dev = nullptr;
  int64_t row0 = 0;
};

struct DropJob { DropKey d; Mat x, y; int64_t rows; int cols; };

// forward: v = r + dropout(x) (r null: v = x), s = v (where not null), y =
// layer norm of v, stats (where not null).  backward: v as stored (a layer
// norm's x, a residual join's s), dr = ds + dx of the layer norm, dx =
// dropout(dr), dgamma, dbeta, each where not null.
struct NormJob {
  DropKey d;
  Mat x, r, s, y;
  Mat v, dy, ds, dr, dx;
  const float *gamma, *beta;
  float *stats, *dgamma, *dbeta, *part;
  float eps;
  int cols;
  int64_t rows;
};

// the most partial pairs (2 x cols floats each) of weights' gradients that a
// backward pass over rows x cols, or fewer rows, leaves in its workspace,
// whatever its element type (1: none, the result is written at once)
int norm_parts(int64_t rows, int cols);
hipError_t launch_dropout(Elt e, const DropJob& j, hipStream_t st);
hipError_t launch_norm_forward(Elt e, const NormJob& j, hipStream_t st);
hipError_t launch_norm_backward(Elt e, const NormJob& j, hipStream_t st);
// the root-mean-square norm's: of v, dy, ds, stats (k of each row) into dr and dgamma
hipError_t launch_rms_backward(Elt e, const NormJob& j, hipStream_t st);
// text that vfl_last_error(NULL) returns on the calling thread
void set_call_error(const char* why) noexcept;

}  // namespace vfl
