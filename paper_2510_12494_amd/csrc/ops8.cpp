// Host side of the root-mean-square norm, of matrices in 8 bits and of the softmax
// loss: the argument checks of the C entry points and their launch jobs.  Every refusal comes before
// the first launch, and no call allocates, synchronises or throws.
#include <algorithm>

#include "checks.h"
#include "ops8.h"

using namespace vfl;

namespace {

constexpr int64_t kMaxSide8 = (int64_t)1 << 30;      // rows of an operand of a product, results' columns
constexpr int64_t kMaxResults = (int64_t)1 << 36;    // of a product: its grid is below 2^32 threads
constexpr int64_t kMaxLogits = (int64_t)1 << 37;
constexpr int64_t kMaxDepth = VFL_MATMUL8_MAX_DEPTH;

int64_t round_up(int64_t v, int64_t by) { return (v + by - 1) / by * by; }

// a matrix of a shape of its own
Mat shaped(Checks& c, const vfl_matrix& m, int64_t rows, int64_t cols, bool required, const char* what) {
  Checks k = c;
  k.rows = rows;
  k.cols = (int)cols;
  const Mat out = k.mat(m, required, what);
  c.why = k.why;
  return out;
}

// a matrix in 8 bits: present (or optional and absent), its rows and its exponents'
// aligned, padded to whole blocks, not overlapping and addressable
Mat8 eight(Checks& c, const vfl_q8& m, int64_t rows, int64_t cols, bool required, const char* what) {
  Mat8 out;
  if (c.why) return out;
  if (!m.data) {
    if (required && rows > 0) c.why = what;
    return out;
  }
  const int64_t wide = round_up(cols, kBlock8), ld = m.ld == 0 ? wide : m.ld;
  const int64_t long_ = round_up(rows, 16), sld = m.scale_ld == 0 ? long_ : m.scale_ld;
  if ((uintptr_t)m.data % 16 != 0 || ld % kBlock8 != 0 || ld < wide || ld > kMaxExtent / std::max<int64_t>(rows, 1) ||
      !m.scale || (uintptr_t)m.scale % 16 != 0 || sld % 16 != 0 || sld < long_ ||
      sld > kMaxExtent / std::max<int64_t>(wide / kBlock8, 1)) {
    c.why = what;
    return out;
  }
  out.p = (uint8_t*)m.data;
  out.ld = ld;
  out.scale = m.scale;
  out.scale_ld = sld;
  return out;
}

Checks loss_checks(const char* call, const vfl_softmax_loss_args& a) {
  Checks c = begin(call, dtype_of(a.dtype), a.rows, a.dim, VFL_LOSS_MAX_DIM);
  c.need(a.rows <= VFL_LOSS_MAX_ROWS, "rows above the operator's limit");
  c.need(a.classes >= 1 && a.classes <= VFL_LOSS_MAX_CLASSES, "classes out of range");
  c.need(c.why || a.rows <= kMaxLogits / a.classes, "rows x classes out of range");
  return c;
}

// what both directions read
void loss_job(Checks& c, const vfl_softmax_loss_args& a, LossJob& j) {
  c.need((uintptr_t)a.bias % 4 == 0 && (uintptr_t)a.labels % 4 == 0, "bias and labels must be 4-byte aligned");
  c.need((uintptr_t)a.loss % 4 == 0 && (uintptr_t)a.lse % 4 == 0, "loss and lse must be 4-byte aligned");
  c.need((uintptr_t)a.workspace % 16 == 0, "workspace must be 16-byte aligned");
  j = LossJob{};
  j.x = shaped(c, a.x, a.rows, a.dim, true, "x: bad data or ld");
  j.w = shaped(c, a.w, a.classes, a.dim, true, "w: bad data or ld");
  j.bias = a.bias;
  j.labels = a.labels;
  j.loss = a.loss;
  j.lse = a.lse;
  j.workspace = (char*)a.workspace;
  j.dim = a.dim;
  j.rows = a.rows;
  j.classes = a.classes;
}

const char* loss_workspace_why(const Checks& c, const vfl_softmax_loss_args& a) {
  const size_t need = a.rows == 0 ? 0 : loss_workspace(elt(c.dtype), a.rows, a.dim, a.classes);
  return need && (!a.workspace || a.workspace_bytes < need) ? "workspace smaller than vfl_softmax_loss_workspace_size()"
                                                            : nullptr;
}

}  // namespace

extern "C" {

vfl_status vfl_rmsnorm_forward(const vfl_rmsnorm_args* a, void* stream) {
  const char* call = "vfl_rmsnorm_forward";
  if (!a) return refuse(call, "args must not be NULL");
  Checks c = begin(call, dtype_of(a->dtype), a->rows, a->cols, VFL_NORM_MAX_COLS);
  c.need((uintptr_t)a->gamma % 4 == 0, "gamma must be 4-byte aligned");
  c.need((uintptr_t)a->stats % 4 == 0, "stats must be 4-byte aligned");
  c.need(a->eps > 0.f && std::isfinite(a->eps), "eps must be positive and finite");
  RmsJob j;
  j.x = c.mat(a->x, true, "x: bad data or ld");
  j.r = c.mat(a->r, false, "r: bad data or ld");
  j.s = c.mat(a->s, false, "s: bad data or ld");
  j.y = c.mat(a->y, false, "y: bad data or ld");
  j.q = eight(c, a->q, a->rows, a->cols, false, "q: bad data, scale or ld");
  c.need(a->rows == 0 || a->s.data || a->y.data || a->q.data || a->stats, "no output");
  if (c.why) return refuse(call, c.why);
  j.gamma = a->gamma;
  j.stats = a->stats;
  j.eps = a->eps;
  j.cols = a->cols;
  j.rows = a->rows;
  if (j.rows == 0) return enqueued(call, hipSuccess);
  return enqueued(call, launch_rms_forward(elt(c.dtype), j, (hipStream_t)stream));
}

vfl_status vfl_rmsnorm_backward(const vfl_rmsnorm_args* a, void* stream) {
  const char* call = "vfl_rmsnorm_backward";
  if (!a) return refuse(call, "args must not be NULL");
  Checks c = begin(call, dtype_of(a->dtype), a->rows, a->cols, VFL_NORM_MAX_COLS);
  c.need((uintptr_t)a->gamma % 4 == 0 && (uintptr_t)a->dgamma % 4 == 0, "gamma and dgamma must be 4-byte aligned");
  c.need(a->rows == 0 || (a->stats && (uintptr_t)a->stats % 4 == 0), "stats must not be NULL, and be 4-byte aligned");
  NormJob j{};
  j.v = c.mat(a->s, true, "s: bad data or ld");
  j.dy = c.mat(a->dy, true, "dy: bad data or ld");
  j.ds = c.mat(a->ds, false, "ds: bad data or ld");
  j.dr = c.mat(a->dx, false, "dx: bad data or ld");
  c.need(a->dx.data || a->dgamma, "no output");
  c.need((uintptr_t)a->workspace % 16 == 0, "workspace must be 16-byte aligned");
  if (c.why) return refuse(call, c.why);
  j.gamma = a->gamma;
  j.stats = a->stats;
  j.dgamma = a->dgamma;
  j.cols = a->cols;
  j.rows = a->rows;
  const int parts = norm_parts(a->rows, a->cols);
  if (a->dgamma && parts > 1) {
    if (!a->workspace || a->workspace_bytes < (size_t)parts * 2 * (size_t)a->cols * sizeof(float))
      return refuse(call, "workspace smaller than vfl_norm_workspace_size()", VFL_E_NOMEM);
    j.part = (float*)a->workspace;
  }
  return enqueued(call, launch_rms_backward(elt(c.dtype), j, (hipStream_t)stream));
}

vfl_status vfl_quantize(const vfl_quantize_args* a, void* stream) {
  const char* call = "vfl_quantize";
  if (!a) return refuse(call, "args must not be NULL");
  Checks c = begin(call, dtype_of(a->dtype), a->rows, a->cols, INT32_MAX - 256);
  QuantJob j;
  j.x = c.mat(a->x, true, "x: bad data or ld");
  j.q = eight(c, a->q, a->rows, a->cols, false, "q: bad data, scale or ld");
  j.qt = eight(c, a->qt, a->cols, a->rows, false, "qt: bad data, scale or ld");
  c.need(a->rows == 0 || a->q.data || a->qt.data, "no output");
  if (c.why) return refuse(call, c.why);
  j.rows = a->rows;
  j.cols = a->cols;
  if (j.rows == 0) return enqueued(call, hipSuccess);
  return enqueued(call, launch_quantize(elt(c.dtype), j, (hipStream_t)stream));
}

vfl_status vfl_matmul8_workspace_size(int64_t m, int64_t n, int64_t k, size_t* bytes) {
  const char* call = "vfl_matmul8_workspace_size";
  if (m < 0 || m > kMaxSide8 || n < 0 || n > kMaxSide8) return refuse(call, "m or n out of range");
  if (n > 0 && m > kMaxResults / n) return refuse(call, "m x n out of range");
  if (k < 1 || k > kMaxDepth) return refuse(call, "k out of range");
  if (!bytes) return refuse(call, "bytes must not be NULL");
  *bytes = m == 0 || n == 0 ? 0 : matmul8_workspace(m, n, k);
  return enqueued(call, hipSuccess);
}

vfl_status vfl_matmul8(const vfl_matmul8_args* a, void* stream) {
  const char* call = "vfl_matmul8";
  if (!a) return refuse(call, "args must not be NULL");
  Checks c = begin(call, dtype_of(a->dtype), a->m, 1, 1);
  c.need(a->m <= kMaxSide8 && a->n >= 0 && a->n <= kMaxSide8, "m or n out of range");
  c.need(c.why || a->n == 0 || a->m <= kMaxResults / a->n, "m x n out of range");
  c.need(a->k >= 1 && a->k <= kMaxDepth, "k out of range");
  c.need((uintptr_t)a->bias % 4 == 0, "bias must be 4-byte aligned");
  c.need((uintptr_t)a->workspace % 16 == 0, "workspace must be 16-byte aligned");
  if (c.why) return refuse(call, c.why);
  if (a->m == 0 || a->n == 0) return enqueued(call, hipSuccess);
  Matmul8Job j;
  j.a = eight(c, a->a, a->m, a->k, true, "a: bad data, scale or ld");
  j.b = eight(c, a->b, a->n, a->k, true, "b: bad data, scale or ld");
  c.need(j.a.ld < (int64_t)1 << 24, "a: ld above the operator's limit");
  c.need(j.b.ld < (int64_t)1 << 24, "b: ld above the operator's limit");
  j.c = shaped(c, a->c, a->m, a->n, true, "c: bad data or ld");
  if (c.why) return refuse(call, c.why);
  j.bias = a->bias;
  j.relu = a->relu != 0;
  j.m = a->m;
  j.n = a->n;
  j.k = a->k;
  const size_t need = matmul8_workspace(a->m, a->n, a->k);
  if (need && (!a->workspace || a->workspace_bytes < need))
    return refuse(call, "workspace smaller than vfl_matmul8_workspace_size()", VFL_E_NOMEM);
  j.part = (float*)a->workspace;
  return enqueued(call, launch_matmul8(elt(c.dtype), j, (hipStream_t)stream));
}

vfl_status vfl_softmax_loss_workspace_size(vfl_dtype dtype, int64_t rows, int32_t dim, int64_t classes, size_t* bytes) {
  const char* call = "vfl_softmax_loss_workspace_size";
  Checks c = begin(call, dtype_of(dtype), rows, dim, VFL_LOSS_MAX_DIM);
  c.need(rows <= VFL_LOSS_MAX_ROWS, "rows above the operator's limit");
  c.need(classes >= 1 && classes <= VFL_LOSS_MAX_CLASSES, "classes out of range");
  c.need(c.why || rows <= kMaxLogits / classes, "rows x classes out of range");
  c.need(bytes != nullptr, "bytes must not be NULL");
  if (c.why) return refuse(call, c.why);
  *bytes = rows == 0 ? 0 : loss_workspace(elt(c.dtype), rows, dim, classes);
  return enqueued(call, hipSuccess);
}

vfl_status vfl_softmax_loss_forward(const vfl_softmax_loss_args* a, void* stream) {
  const char* call = "vfl_softmax_loss_forward";
  if (!a) return refuse(call, "args must not be NULL");
  Checks c = loss_checks(call, *a);
  LossJob j;
  loss_job(c, *a, j);
  c.need(a->rows == 0 || a->loss || a->lse, "no output");
  c.need(a->rows == 0 || !a->loss || a->labels, "labels must not be NULL");
  if (c.why) return refuse(call, c.why);
  if (j.rows == 0) return enqueued(call, hipSuccess);
  if (const char* why = loss_workspace_why(c, *a)) return refuse(call, why, VFL_E_NOMEM);
  return enqueued(call, launch_loss_forward(elt(c.dtype), j, (hipStream_t)stream));
}

vfl_status vfl_softmax_loss_backward(const vfl_softmax_loss_args* a, void* stream) {
  const char* call = "vfl_softmax_loss_backward";
  if (!a) return refuse(call, "args must not be NULL");
  Checks c = loss_checks(call, *a);
  LossJob j;
  loss_job(c, *a, j);
  j.dx = shaped(c, a->dx, a->rows, a->dim, false, "dx: bad data or ld");
  j.dw = shaped(c, a->dw, a->classes, a->dim, false, "dw: bad data or ld");
  c.need(a->dx.data || a->dw.data || a->dbias, "no output");
  c.need(a->rows == 0 || a->labels, "labels must not be NULL");
  c.need(a->rows == 0 || a->lse, "lse must not be NULL");
  c.need((uintptr_t)a->dloss % 4 == 0 && (uintptr_t)a->dbias % 4 == 0, "dloss and dbias must be 4-byte aligned");
  if (c.why) return refuse(call, c.why);
  if (const char* why = loss_workspace_why(c, *a)) return refuse(call, why, VFL_E_NOMEM);
  j.dloss = a->dloss;
  j.scale = a->scale;
  j.dbias = a->dbias;
  return enqueued(call, launch_loss_backward(elt(c.dtype), j, (hipStream_t)stream));
}

}  // extern "C"
