// Test infrastructure: drives the argument checks of the row operators
// (rowops.cpp) under the host address and undefined-behaviour sanitizers,
// with random and extreme descriptors.  The launches are stand-ins that check
// what the kernels rely on: present operands, row strides of at least the
// columns, and a workspace as large as the partial sums.  Exits 0 after
// printing "row operator checks passed".
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <limits>
#include <random>

#include "../../include/vfl.h"
#include "../../paper_2510_12494_amd/csrc/rowops.h"

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

static void check_mat(const Mat& m, int64_t rows, int cols, int64_t esz, bool required) {
  expect(!required || m.p || rows == 0, "a required matrix is present");
  if (!m.p) return;
  expect(m.ld >= cols, "ld covers the columns");
  expect(rows == 0 || (m.ld <= ((int64_t)1 << 60) / esz / (rows > 1 ? rows : 1)), "the extent is addressable");
  expect((uintptr_t)m.p % (uintptr_t)esz == 0, "element-aligned");
}
static void check_drop(const DropKey& d, int64_t rows) {
  expect(d.thr <= 65536 && d.tag < 65536 && d.row0 >= 0 && d.row0 + rows <= (int64_t)1 << 47, "dropout key in range");
  expect(d.thr == 65536 ? d.scale == 0.f : d.scale >= 1.f && std::isfinite(d.scale), "dropout scale");
}
hipError_t launch_dropout(Elt e, const DropJob& j, hipStream_t) {
  ++launched;
  check_drop(j.d, j.rows);
  check_mat(j.x, j.rows, j.cols, elt_size(e), true);
  check_mat(j.y, j.rows, j.cols, elt_size(e), true);
  return hipSuccess;
}
hipError_t launch_norm_forward(Elt e, const NormJob& j, hipStream_t) {
  ++launched;
  check_drop(j.d, j.rows);
  check_mat(j.x, j.rows, j.cols, elt_size(e), true);
  check_mat(j.y, j.rows, j.cols, elt_size(e), true);
  check_mat(j.r, j.rows, j.cols, elt_size(e), false);
  check_mat(j.s, j.rows, j.cols, elt_size(e), false);
  expect(j.eps > 0.f && j.cols <= VFL_NORM_MAX_COLS, "eps and width");
  return hipSuccess;
}
hipError_t launch_norm_backward(Elt e, const NormJob& j, hipStream_t) {
  ++launched;
  check_drop(j.d, j.rows);
  check_mat(j.v, j.rows, j.cols, elt_size(e), true);
  check_mat(j.dy, j.rows, j.cols, elt_size(e), true);
  for (const Mat* m : {&j.ds, &j.dr, &j.dx}) check_mat(*m, j.rows, j.cols, elt_size(e), false);
  expect(j.stats || j.rows == 0, "statistics");
  expect(j.dr.p || j.dx.p || j.dgamma || j.dbeta, "an output");
  if ((j.dgamma || j.dbeta) && norm_parts(j.rows, j.cols) > 1)
    expect(j.part && (size_t)norm_parts(j.rows, j.cols) * 8 * j.cols <= ws_bytes,
           "the workspace holds the partial sums");
  return hipSuccess;
}
}  // namespace vfl

namespace {
std::mt19937_64 rng(77);
int uni(int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); }
alignas(256) char buf[4096];

int64_t size_value() {
  static const int64_t odd[] = {0, 1, -1, 7, 64, 4099, 1 << 20, (int64_t)1 << 40, ((int64_t)1 << 40) + 1,
                                (int64_t)1 << 59, std::numeric_limits<int64_t>::max(), std::numeric_limits<int64_t>::min()};
  return uni(0, 2) ? uni(1, 5000) : odd[uni(0, 11)];
}
int32_t cols_value() {
  static const int32_t odd[] = {0, -1, 1, 32768, 32769, std::numeric_limits<int32_t>::max(), std::numeric_limits<int32_t>::min()};
  return uni(0, 2) ? uni(1, 300) : odd[uni(0, 6)];
}
void* pointer(bool odd) { return uni(0, 7) ? buf + 16 * uni(0, 7) + (odd && !uni(0, 5) ? uni(1, 7) : 0) : nullptr; }
vfl_matrix matrix() { return {pointer(true), uni(0, 2) ? 0 : size_value()}; }
float real() {
  static const float odd[] = {0.f, 1.f, -1.f, 2.f, std::numeric_limits<float>::quiet_NaN(),
                              std::numeric_limits<float>::infinity(), 1e-30f, 0.9999999f};
  return uni(0, 2) ? 0.25f : odd[uni(0, 7)];
}
vfl_dropout_spec drop() {
  return {real(), uni(0, 5) ? 3u : (uint32_t)rng(), rng(), (uint32_t)rng(), (const uint32_t*)(uni(0, 3) ? nullptr : pointer(true)),
          uni(0, 3) ? 5 : size_value()};
}
// any integer a caller might pass, written without loading it as the enum
void set_dtype(vfl_dtype& d) {
  const int v = uni(0, 9) ? uni(0, 1) : uni(-2, 9);
  std::memcpy(&d, &v, sizeof(d));
}
template <typename A>
void norm_fields(A& a) {
  set_dtype(a.dtype);
  a.cols = cols_value();
  a.rows = size_value();
  a.eps = uni(0, 4) ? 1e-5f : real();
  a.gamma = (const float*)pointer(true);
  a.beta = (const float*)pointer(true);
  a.stats = (float*)pointer(true);
  a.dgamma = (float*)pointer(true);
  a.dbeta = (float*)pointer(true);
  a.workspace = pointer(true);
  a.workspace_bytes = uni(0, 2) ? (size_t)1 << 40 : (size_t)uni(0, 100000);
}
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
    const int before = launched;
    vfl_dropout_args d{};
    set_dtype(d.dtype);
    d.cols = cols_value();
    d.rows = size_value();
    d.drop = drop();
    d.x = matrix();
    d.y = matrix();
    result(vfl_dropout(&d, nullptr), before);
    vfl_layernorm_args n{};
    norm_fields(n);
    n.x = matrix(); n.y = matrix(); n.dy = matrix(); n.dx = matrix();
    result(vfl_layernorm_forward(&n, nullptr), launched);
    ws_bytes = n.workspace_bytes;
    result(vfl_layernorm_backward(&n, nullptr), launched);
    vfl_residual_args r{};
    norm_fields(r);
    r.drop = drop();
    for (vfl_matrix* m : {&r.x, &r.r, &r.s, &r.y, &r.dy, &r.ds, &r.dr, &r.dx}) *m = matrix();
    result(vfl_residual_forward(&r, nullptr), launched);
    ws_bytes = r.workspace_bytes;
    result(vfl_residual_backward(&r, nullptr), launched);
    size_t bytes = 0;
    result(vfl_norm_workspace_size(size_value(), cols_value(), uni(0, 9) ? &bytes : nullptr), launched);
  }
  expect(ok > 5000 && refused > 5000, "both accepted and refused calls were exercised");
  if (fails) {
    std::printf("%d checks failed\n", fails);
    return 1;
  }
  std::printf("row operator checks passed (%d accepted, %d refused)\n", ok, refused);
  return 0;
}
