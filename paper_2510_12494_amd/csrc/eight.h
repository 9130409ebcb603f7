// Device helpers of matrices in 8 bits: e4m3 values with one power of two for each
// block of 128, stored as the byte e + 127.
#pragma once
#include "rowchunk.h"

namespace vfl {
namespace dev {

// The magnitude of a value for a block's largest: its bits without the sign, in
// which NaN and infinity are above every number.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
constexpr uint32_t kInfinite = 0x7f800000u;

// The byte of the smallest power 2^e, e >= -127, that takes a magnitude to 448 =
// 1.75 * 2^8 or less: the exponent, one more where the fraction is past 1.75.
__device__ __forceinline__ uint32_t scale_byte(uint32_t magnitude_bits) {
  return (uint32_t)max((int)((magnitude_bits + 0x1fffffu) >> 23) - 8, 0);
}
// 2^-e of a byte (0 to 247)
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// Eight values times 2^-e, rounded to nearest even: an exact multiplication (what
// it flushes is far below e4m3's smallest value) and one rounding.
__device__ __forceinline__ u32x2 pack_e4m3(const float (&v)[8], float inv) {
  u32x2 w = {0u, 0u};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int x = 0;
    x = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i] * inv, v[4 * i + 1] * inv, x, false);
    x = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2] * inv, v[4 * i + 3] * inv, x, true);
    w[i] = (uint32_t)x;
  }
  return w;
}

// The largest over the 16 lanes that hold a block, in every one of them.
__device__ __forceinline__ uint32_t block_max(uint32_t v) {
  auto step = [&](uint32_t o) { v = max(v, o); };
  step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, true));
  step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, true));
  step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, true));
  step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, true));
  return v;
}

__device__ __forceinline__ uint32_t chunk_max(const float (&v)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, magnitude(v[i]));
  return m;
}

// Values that are no numbers stand for themselves as NaN (e4m3 has no infinity)
// and take no part in their block's power.
__device__ __forceinline__ float number_or_nan(float v) {
  return magnitude(v) >= kInfinite ? __uint_as_float(0x7fc00000u) : v;
}
__device__ __forceinline__ uint32_t number_magnitude(float v) {
  const uint32_t m = magnitude(v);
  return m >= kInfinite ? 0u : m;
}

}  // namespace dev
}  // namespace vfl
