// Argument checks that the C entry points without a context share (host only).
#pragma once
#include <cmath>
#include <cstdio>
#include <cstring>

#include "../../include/vfl.h"
#include "rowops.h"

namespace vfl {

constexpr int64_t kMaxRows = (int64_t)1 << 40;
constexpr int64_t kMaxExtent = (int64_t)1 << 60;   // bytes from a matrix's first to its last element
constexpr int64_t kMaxSampleId = (int64_t)1 << 47;

inline vfl_status refuse(const char* call, const char* what, vfl_status st = VFL_E_INVALID) noexcept {
  char text[160];
  std::snprintf(text, sizeof(text), "%s: %s", call, what);
  set_call_error(text);
  return st;
}

inline vfl_status enqueued(const char* call, hipError_t e) noexcept {
  if (e != hipSuccess) return refuse(call, hipGetErrorString(e), VFL_E_HIP);
  set_call_error("");
  return VFL_OK;
}

// Collects the first failed check of a call.
struct Checks {
  const char* call;
  const char* why = nullptr;
  int dtype, cols;
  int64_t rows;

  void need(bool ok, const char* what) {
    if (!ok && !why) why = what;
  }
  // one matrix: present (or optional and absent), element-aligned, rows that
  // do not overlap and whose last byte is addressable
  Mat mat(const vfl_matrix& m, bool required, const char* what) {
    Mat out;
    if (why) return out;
    const int64_t esz = dtype == VFL_F32 ? 4 : 2;
    const int64_t ld = m.ld == 0 ? cols : m.ld;
    if (!m.data) {
      if (required && rows > 0) why = what;
      return out;
    }
    if ((uintptr_t)m.data % (uintptr_t)esz != 0) why = what;
    else if (ld < cols || ld > kMaxExtent / esz || (rows > 1 && ld > kMaxExtent / esz / rows)) why = what;
    out.p = m.data;
    out.ld = ld;
    return out;
  }
  DropKey drop(const vfl_dropout_spec& d) {
    DropKey k;
    if (why) return k;                               // rows is in range below
    need(d.p >= 0.f && d.p <= 1.f, "p must be in [0, 1]");      // a NaN fails too
    need(d.tag < 65536u, "tag must be below 65536");
    need(d.row0 >= 0 && d.row0 <= kMaxSampleId - rows, "sample ids must be in [0, 2^47)");
    need((uintptr_t)d.step_dev % 4 == 0, "step_dev must be 4-byte aligned");
    if (why) return k;
    k.thr = (uint32_t)std::floor((double)d.p * 65536.0 + 0.5);
    k.scale = k.thr < 65536u ? (float)(65536.0 / (65536.0 - k.thr)) : 0.f;
    k.k0 = (uint32_t)d.seed;
    k.k1 = (uint32_t)(d.seed >> 32);
    k.step = d.step;
    k.step_dev = d.step_dev;
    k.tag = d.tag;
    k.row0 = d.row0;
    return k;
  }
};

inline Checks begin(const char* call, int dtype, int64_t rows, int32_t cols, int32_t max_cols) {
  Checks c{call, nullptr, dtype, cols, rows};
  c.need(dtype == VFL_F32 || dtype == VFL_BF16, "dtype must be VFL_F32 or VFL_BF16");
  c.need(rows >= 0 && rows <= kMaxRows, "rows out of range");
  c.need(cols >= 1, "cols must be at least 1");
  c.need(cols <= max_cols, "cols above the operator's limit");
  return c;
}

// the enum as an integer: a caller's value need not be one of the enumerators
inline int dtype_of(const vfl_dtype& d) {
  int v;
  static_assert(sizeof(v) == sizeof(d), "vfl_dtype is an int");
  std::memcpy(&v, &d, sizeof(v));
  return v;
}

inline Elt elt(int dtype) { return dtype == VFL_F32 ? F32 : BF16; }

}  // namespace vfl
