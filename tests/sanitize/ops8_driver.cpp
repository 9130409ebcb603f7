// Test infrastructure: drives the argument checks of the root-mean-square norm,
// of matrices in 8 bits and of the softmax loss (ops8.cpp) under the host address
// and undefined-behaviour sanitizers, with random and extreme descriptors.  The
// launches are stand-ins that check what the kernels rely on.  Exits 0 after
// printing "operator checks passed".
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <limits>
#include <random>

#include "../../include/vfl.h"
#include "../../paper_2510_12494_amd/csrc/ops8.h"

namespace {
int launched = 0, fails = 0;
size_t ws_bytes = 0;
char last_text[256];

void expect(bool ok, const char* what) {
  if (!ok) {
    std::printf("FAILED: %s\n", what);
    ++fails;
  }
}
}  // namespace

namespace vfl {
void set_call_error(const char* why) noexcept { std::snprintf(last_text, sizeof(last_text), "%s", why); }
int norm_parts(int64_t rows, int) { return rows < 64 ? (int)rows : 64; }
size_t matmul8_workspace(int64_t m, int64_t n, int64_t k) { return (size_t)((m + n + k) % 4096); }
size_t loss_workspace(Elt e, int64_t rows, int dim, int64_t classes) {
  return (size_t)((rows + dim + classes) % 4096) + (e == F32 ? 1 : 2);
}

static void check_mat(const Mat& m, int64_t rows, int64_t cols, int64_t esz, bool required) {
  expect(!required || m.p || rows == 0, "a required matrix is present");
  if (!m.p) return;
  expect(m.ld >= cols, "ld covers the columns");
  expect(rows == 0 || (m.ld <= ((int64_t)1 << 60) / esz / (rows > 1 ? rows : 1)), "the extent is addressable");
  expect((uintptr_t)m.p % (uintptr_t)esz == 0, "element-aligned");
}
static void check_8(const Mat8& m, int64_t rows, int64_t cols, bool required) {
  expect(!required || m.p || rows == 0, "a required matrix in 8 bits is present");
  if (!m.p) return;
  const int64_t blocks = (cols + 127) / 128;
  expect((uintptr_t)m.p % 16 == 0 && m.ld % 128 == 0 && m.ld >= 128 * blocks, "rows of whole blocks");
  expect(m.scale && (uintptr_t)m.scale % 16 == 0 && m.scale_ld % 16 == 0 && m.scale_ld >= rows, "exponents");
  expect(rows == 0 || m.ld <= ((int64_t)1 << 60) / rows, "the extent is addressable");
}
hipError_t launch_rms_forward(Elt e, const RmsJob& j, hipStream_t) {
  ++launched;
  check_mat(j.x, j.rows, j.cols, elt_size(e), true);
  for (const Mat* m : {&j.r, &j.s, &j.y}) check_mat(*m, j.rows, j.cols, elt_size(e), false);
  check_8(j.q, j.rows, j.cols, false);
  expect(j.s.p || j.y.p || j.q.p || j.stats, "an output");
  expect(j.eps > 0.f && std::isfinite(j.eps) && j.cols >= 1 && j.cols <= VFL_NORM_MAX_COLS && j.rows > 0, "sizes and eps");
  return hipSuccess;
}
hipError_t launch_rms_backward(Elt e, const NormJob& j, hipStream_t) {
  ++launched;
  check_mat(j.v, j.rows, j.cols, elt_size(e), true);
  check_mat(j.dy, j.rows, j.cols, elt_size(e), true);
  for (const Mat* m : {&j.ds, &j.dr}) check_mat(*m, j.rows, j.cols, elt_size(e), false);
  expect(!j.dx.p && !j.dbeta, "one gradient of the join");
  expect(j.stats || j.rows == 0, "statistics");
  expect(j.dr.p || j.dgamma, "an output");
  if (j.dgamma && norm_parts(j.rows, j.cols) > 1)
    expect(j.part && (size_t)norm_parts(j.rows, j.cols) * 8 * j.cols <= ws_bytes, "the workspace holds the partial sums");
  return hipSuccess;
}
hipError_t launch_quantize(Elt e, const QuantJob& j, hipStream_t) {
  ++launched;
  check_mat(j.x, j.rows, j.cols, elt_size(e), true);
  check_8(j.q, j.rows, j.cols, false);
  check_8(j.qt, j.cols, j.rows, false);
  expect((j.q.p || j.qt.p) && j.rows > 0 && j.cols > 0, "an output and sizes");
  return hipSuccess;
}
hipError_t launch_matmul8(Elt e, const Matmul8Job& j, hipStream_t) {
  ++launched;
  check_8(j.a, j.m, j.k, true);
  check_8(j.b, j.n, j.k, true);
  check_mat(j.c, j.m, j.n, elt_size(e), true);
  expect(j.a.ld < (1 << 24) && j.b.ld < (1 << 24), "a tile's offsets fit 32 bits");
  expect(j.m > 0 && j.n > 0 && j.k > 0 && j.m <= ((int64_t)1 << 36) / j.n && j.k <= VFL_MATMUL8_MAX_DEPTH, "sizes");
  const size_t need = matmul8_workspace(j.m, j.n, j.k);
  expect(need == 0 || (j.part && need <= ws_bytes), "the workspace holds the partial sums");
  return hipSuccess;
}
static void check_loss(Elt e, const LossJob& j) {
  check_mat(j.x, j.rows, j.dim, elt_size(e), true);
  check_mat(j.w, j.classes, j.dim, elt_size(e), true);
  expect(j.rows <= VFL_LOSS_MAX_ROWS && j.classes >= 1 && j.classes <= VFL_LOSS_MAX_CLASSES && j.dim >= 1 &&
             j.dim <= VFL_LOSS_MAX_DIM && j.rows <= ((int64_t)1 << 37) / j.classes, "sizes");
  expect(j.rows == 0 || (j.workspace && loss_workspace(e, j.rows, j.dim, j.classes) <= ws_bytes), "the workspace");
}
hipError_t launch_loss_forward(Elt e, const LossJob& j, hipStream_t) {
  ++launched;
  check_loss(e, j);
  expect((j.loss || j.lse) && (!j.loss || j.labels), "outputs and labels");
  return hipSuccess;
}
hipError_t launch_loss_backward(Elt e, const LossJob& j, hipStream_t) {
  ++launched;
  check_loss(e, j);
  check_mat(j.dx, j.rows, j.dim, elt_size(e), false);
  check_mat(j.dw, j.classes, j.dim, elt_size(e), false);
  expect((j.dx.p || j.dw.p || j.dbias) && (j.rows == 0 || (j.lse && j.labels)), "outputs, lse and labels");
  return hipSuccess;
}
}  // namespace vfl

namespace {
std::mt19937_64 rng(78);
int uni(int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); }
alignas(256) char buf[4096];

int64_t size_value() {
  static const int64_t odd[] = {0, 1, -1, 7, 64, 4099, 1 << 20, 1 << 24, (int64_t)1 << 30, (int64_t)1 << 40, ((int64_t)1 << 40) + 1,
                                (int64_t)1 << 59, std::numeric_limits<int64_t>::max(), std::numeric_limits<int64_t>::min()};
  return uni(0, 3) ? uni(1, 5000) : odd[uni(0, 13)];
}
int32_t cols_value() {
  static const int32_t odd[] = {0, -1, 1, 32768, 32769, std::numeric_limits<int32_t>::max(), std::numeric_limits<int32_t>::min()};
  return uni(0, 3) ? uni(1, 300) : odd[uni(0, 6)];
}
void* pointer() { return uni(0, 11) ? buf + 16 * uni(0, 7) + (!uni(0, 9) ? uni(1, 15) : 0) : nullptr; }
vfl_matrix matrix() { return {pointer(), uni(0, 2) ? 0 : size_value()}; }
vfl_q8 eight() {
  return {pointer(), uni(0, 2) ? 0 : (uni(0, 2) ? 128 * (int64_t)uni(0, 300) : size_value()), (uint8_t*)pointer(),
          uni(0, 2) ? 0 : (uni(0, 2) ? 16 * (int64_t)uni(0, 400) : size_value())};
}
float real() {
  static const float odd[] = {0.f, 1.f, -1.f, std::numeric_limits<float>::quiet_NaN(), std::numeric_limits<float>::infinity(), 1e-30f};
  return uni(0, 3) ? 1e-5f : odd[uni(0, 5)];
}
// any integer a caller might pass, written without loading it as the enum
void set_dtype(vfl_dtype& d) {
  const int v = uni(0, 9) ? uni(0, 1) : uni(-2, 9);
  std::memcpy(&d, &v, sizeof(d));
}
size_t room() { return uni(0, 2) ? (size_t)1 << 40 : (size_t)uni(0, 100000); }
}  // namespace

int main() {
  int ok = 0, refused = 0;
  auto result = [&](vfl_status st, int before) {
    expect((st == VFL_OK) == (last_text[0] == 0), "a refusal has a reason, a success none");
    if (st == VFL_OK) ++ok;
    else {
      ++refused;
      expect(launched == before, "a refused call launches nothing");
    }
  };
  for (int it = 0; it < 60000; ++it) {
    vfl_rmsnorm_args n{};
    set_dtype(n.dtype);
    n.cols = cols_value();
    n.rows = size_value();
    n.eps = real();
    n.gamma = (const float*)pointer();
    for (vfl_matrix* m : {&n.x, &n.r, &n.s, &n.y, &n.dy, &n.ds, &n.dx}) *m = matrix();
    n.q = eight();
    n.stats = (float*)pointer();
    n.dgamma = (float*)pointer();
    n.workspace = pointer();
    ws_bytes = n.workspace_bytes = room();
    result(vfl_rmsnorm_forward(&n, nullptr), launched);
    result(vfl_rmsnorm_backward(&n, nullptr), launched);
    vfl_quantize_args q{};
    set_dtype(q.dtype);
    q.cols = cols_value();
    q.rows = size_value();
    q.x = matrix();
    q.q = eight();
    q.qt = eight();
    result(vfl_quantize(&q, nullptr), launched);
    vfl_matmul8_args p{};
    set_dtype(p.dtype);
    p.relu = uni(-1, 1);
    p.m = size_value();
    p.n = size_value();
    p.k = size_value();
    p.a = eight();
    p.b = eight();
    p.bias = (const float*)pointer();
    p.c = matrix();
    p.workspace = pointer();
    ws_bytes = p.workspace_bytes = room();
    result(vfl_matmul8(&p, nullptr), launched);
    vfl_softmax_loss_args s{};
    set_dtype(s.dtype);
    s.dim = cols_value();
    s.rows = size_value();
    s.classes = size_value();
    for (vfl_matrix* m : {&s.x, &s.w, &s.dx, &s.dw}) *m = matrix();
    s.bias = (const float*)pointer();
    s.labels = (const int32_t*)pointer();
    s.loss = (float*)pointer();
    s.lse = (float*)pointer();
    s.dloss = (const float*)pointer();
    s.dbias = (float*)pointer();
    s.workspace = pointer();
    ws_bytes = s.workspace_bytes = room();
    result(vfl_softmax_loss_forward(&s, nullptr), launched);
    result(vfl_softmax_loss_backward(&s, nullptr), launched);
    size_t bytes = 0;
    result(vfl_matmul8_workspace_size(size_value(), size_value(), size_value(), uni(0, 9) ? &bytes : nullptr), launched);
    result(vfl_softmax_loss_workspace_size(uni(0, 1) ? VFL_F32 : VFL_BF16, size_value(), cols_value(), size_value(), uni(0, 9) ? &bytes : nullptr),
           launched);
  }
  expect(ok > 20000 && refused > 20000, "both accepted and refused calls were exercised");
  if (fails) {
    std::printf("%d checks failed\n", fails);
    return 1;
  }
  std::printf("operator checks passed (%d accepted, %d refused)\n", ok, refused);
  return 0;
}
