// Host side of the row operators (dropout, layer norm, residual join): the
// argument checks of the C entry points and their launch jobs.  Every refusal
// comes before the first launch, and no call allocates, synchronises or throws.
#include "checks.h"

using namespace vfl;

namespace {

template <typename Args>
NormJob norm_job(Checks& c, const Args& a) {
  NormJob j{};
  c.need((uintptr_t)a.gamma % 4 == 0 && (uintptr_t)a.beta % 4 == 0, "gamma and beta must be 4-byte aligned");
  c.need((uintptr_t)a.stats % 8 == 0, "stats must be 8-byte aligned");
  j.gamma = a.gamma;
  j.beta = a.beta;
  j.stats = a.stats;
  j.cols = a.cols;
  j.rows = a.rows;
  j.eps = a.eps;
  return j;
}

size_t workspace_bytes(int64_t rows, int32_t cols) {
  const int parts = norm_parts(rows, cols);
  return parts > 1 ? (size_t)parts * 2 * (size_t)cols * sizeof(float) : 0;
}

// what every backward pass checks: the statistics, the weights' gradients and
// the workspace that they need (*nomem: it is too small)
template <typename Args>
void norm_grads(Checks& c, const Args& a, NormJob& j, bool* nomem) {
  c.need(a.stats || a.rows == 0, "stats must not be NULL");
  c.need((uintptr_t)a.dgamma % 4 == 0 && (uintptr_t)a.dbeta % 4 == 0, "dgamma and dbeta must be 4-byte aligned");
  if (c.why || (!a.dgamma && !a.dbeta)) return;
  j.dgamma = a.dgamma;
  j.dbeta = a.dbeta;
  c.need((uintptr_t)a.workspace % 16 == 0, "workspace must be 16-byte aligned");
  if (c.why) return;
  const size_t bytes = workspace_bytes(a.rows, a.cols);
  if (bytes == 0) return;
  if (!a.workspace || a.workspace_bytes < bytes) {
    c.why = "workspace smaller than vfl_norm_workspace_size()";
    *nomem = true;
  }
  j.part = (float*)a.workspace;
}

}  // namespace

extern "C" {

vfl_status vfl_dropout(const vfl_dropout_args* a, void* stream) {
  const char* call = "vfl_dropout";
  if (!a) return refuse(call, "args must not be NULL");
  Checks c = begin(call, dtype_of(a->dtype), a->rows, a->cols, INT32_MAX - 64);
  DropJob j;
  j.d = c.drop(a->drop);
  j.x = c.mat(a->x, true, "x: bad data or ld");
  j.y = c.mat(a->y, true, "y: bad data or ld");
  j.rows = a->rows;
  j.cols = a->cols;
  if (c.why) return refuse(call, c.why);
  if (j.rows == 0) return enqueued(call, hipSuccess);
  return enqueued(call, launch_dropout(elt(c.dtype), j, (hipStream_t)stream));
}

vfl_status vfl_norm_workspace_size(int64_t rows, int32_t cols, size_t* bytes) {
  const char* call = "vfl_norm_workspace_size";
  Checks c = begin(call, VFL_F32, rows, cols, VFL_NORM_MAX_COLS);
  c.need(bytes != nullptr, "bytes must not be NULL");
  if (c.why) return refuse(call, c.why);
  *bytes = workspace_bytes(rows, cols);
  return enqueued(call, hipSuccess);
}

vfl_status vfl_layernorm_forward(const vfl_layernorm_args* a, void* stream) {
  const char* call = "vfl_layernorm_forward";
  if (!a) return refuse(call, "args must not be NULL");
  Checks c = begin(call, dtype_of(a->dtype), a->rows, a->cols, VFL_NORM_MAX_COLS);
  NormJob j = norm_job(c, *a);
  c.need(a->eps > 0.f && std::isfinite(a->eps), "eps must be positive and finite");
  j.x = c.mat(a->x, true, "x: bad data or ld");
  j.y = c.mat(a->y, true, "y: bad data or ld");
  if (c.why) return refuse(call, c.why);
  if (j.rows == 0) return enqueued(call, hipSuccess);
  return enqueued(call, launch_norm_forward(elt(c.dtype), j, (hipStream_t)stream));
}

vfl_status vfl_layernorm_backward(const vfl_layernorm_args* a, void* stream) {
  const char* call = "vfl_layernorm_backward";
  if (!a) return refuse(call, "args must not be NULL");
  Checks c = begin(call, dtype_of(a->dtype), a->rows, a->cols, VFL_NORM_MAX_COLS);
  NormJob j = norm_job(c, *a);
  bool nomem = false;
  norm_grads(c, *a, j, &nomem);
  j.v = c.mat(a->x, true, "x: bad data or ld");
  j.dy = c.mat(a->dy, true, "dy: bad data or ld");
  j.dr = c.mat(a->dx, false, "dx: bad data or ld");
  c.need(a->dx.data || a->dgamma || a->dbeta, "no output");
  if (c.why) return refuse(call, c.why, nomem ? VFL_E_NOMEM : VFL_E_INVALID);
  return enqueued(call, launch_norm_backward(elt(c.dtype), j, (hipStream_t)stream));
}

vfl_status vfl_residual_forward(const vfl_residual_args* a, void* stream) {
  const char* call = "vfl_residual_forward";
  if (!a) return refuse(call, "args must not be NULL");
  Checks c = begin(call, dtype_of(a->dtype), a->rows, a->cols, VFL_NORM_MAX_COLS);
  NormJob j = norm_job(c, *a);
  c.need(a->eps > 0.f && std::isfinite(a->eps), "eps must be positive and finite");
  j.d = c.drop(a->drop);
  j.x = c.mat(a->x, true, "x: bad data or ld");
  j.r = c.mat(a->r, true, "r: bad data or ld");
  j.s = c.mat(a->s, false, "s: bad data or ld");
  j.y = c.mat(a->y, true, "y: bad data or ld");
  if (c.why) return refuse(call, c.why);
  if (j.rows == 0) return enqueued(call, hipSuccess);
  return enqueued(call, launch_norm_forward(elt(c.dtype), j, (hipStream_t)stream));
}

vfl_status vfl_residual_backward(const vfl_residual_args* a, void* stream) {
  const char* call = "vfl_residual_backward";
  if (!a) return refuse(call, "args must not be NULL");
  Checks c = begin(call, dtype_of(a->dtype), a->rows, a->cols, VFL_NORM_MAX_COLS);
  NormJob j = norm_job(c, *a);
  bool nomem = false;
  norm_grads(c, *a, j, &nomem);
  j.d = c.drop(a->drop);
  j.v = c.mat(a->s, true, "s: bad data or ld");
  j.dy = c.mat(a->dy, true, "dy: bad data or ld");
  j.ds = c.mat(a->ds, false, "ds: bad data or ld");
  j.dr = c.mat(a->dr, false, "dr: bad data or ld");
  j.dx = c.mat(a->dx, false, "dx: bad data or ld");
  c.need(a->dr.data || a->dx.data || a->dgamma || a->dbeta, "no output");
  if (c.why) return refuse(call, c.why, nomem ? VFL_E_NOMEM : VFL_E_INVALID);
  return enqueued(call, launch_norm_backward(elt(c.dtype), j, (hipStream_t)stream));
}

}  // extern "C"
