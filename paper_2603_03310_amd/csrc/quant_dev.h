// 8-bit cache tiles: e4m3 codes with one float scale per (block, KV head) tile.
//
// A tile's scale is a power of two, the smallest 2^k with 448 2^k no less than
// the tile's largest magnitude (448 is e4m3's largest value), k at least
// kQ8MinExp.  e4m3 keeps 4 significant bits over its normal range of 2^-6 to
// 448 whatever the scale, so a power of two costs no precision against
// top / 448, and it makes scaling exact: when a later token needs a larger
// scale, the codes already there are rounded again by 2^-n, which changes only
// those that fall under 2^-6 of the new scale.
#pragma once

#include "ent_internal.h"

#if defined(__HIPCC__)
namespace ent {

constexpr float kQ8Top = 448.f;
constexpr int kQ8MinExp = -64;

typedef float q8_f32x2 __attribute__((ext_vector_type(2)));

// Magnitude of x for a tile's range: 0 for an infinity or a NaN (infinities
// saturate, NaN stay NaN).
__device__ __forceinline__ float q8_mag(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.f;
}

// The scale that a largest magnitude needs (top finite, >= 0).
__device__ __forceinline__ float q8_scale(float top) {
  const unsigned u = __float_as_uint(top);
  // top = m 2^x with m in [1, 2): 2^(x-8) where m <= 1.75 = 448 / 256, else twice that.
  int k = static_cast<int>(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  k = max(k, kQ8MinExp);
  return __uint_as_float(static_cast<unsigned>(k + 127) << 23);
}
// x clamped to +-448; a NaN passes.
__device__ __forceinline__ float q8_clamp(float x) {
  x = x > kQ8Top ? kQ8Top : x;
  return x < -kQ8Top ? -kQ8Top : x;
}
// Four codes, the first in the low byte, rounded to nearest even (464 and more, and
// infinities, become NaN: clamp first where they can occur).
__device__ __forceinline__ unsigned q8_pack4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  return static_cast<unsigned>(w);
}
__device__ __forceinline__ void q8_unpack4(unsigned w, float* x) {
  const q8_f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), false);
  const q8_f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), true);
  x[0] = lo.x;
  x[1] = lo.y;
  x[2] = hi.x;
  x[3] = hi.y;
}

}  // namespace ent
#endif
