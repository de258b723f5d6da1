// 8-bit elements of a cache: e4m3 codes (OCP: 3 bits behind the first one, down to 2^-9, up to 448, no infinities) times the scale of
// their block, the 16 tokens of a head that lie next to each other in a page.
#pragma once

#include "qcf_internal.h"

namespace qcf {
namespace {

constexpr int kBlock = QCF_PAGE8_BLOCK;
// Elements beyond this (infinities and NaN among them) are stored as NaN: what is left keeps products of codes and scales finite.
constexpr float kLargest = 0x1p100f;
// Least scale, 2^-100: a block of zeros has it.  (Smaller elements than 2^-110 become 0.)
constexpr uint32_t kLeastScale = 27u << 23;

typedef float pair_f32 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ bool storable(float x) { return __builtin_fabsf(x) <= kLargest; }

// The least power of two s with amax <= 448 s.  (448 = 1.75 * 2^8: one more than the exponent where the fraction is beyond 1.75.  A
// power of two keeps all bits of a code when a block's scale grows, but for codes that come beneath 2^-6, and costs nothing beside
// amax / 448: a floating-point code's relative step does not depend on its size.)
__device__ __forceinline__ float scale_for(float amax) {
  const uint32_t e = (__float_as_uint(amax) + 0x1fffffu) >> 23;
  return __uint_as_float(max(e > 8u ? (e - 8u) << 23 : 0u, kLeastScale));
}

// four elements (already divided by their scale) as codes, nearest, ties to even; NaN stays NaN
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}
__device__ __forceinline__ void values_of(uint32_t codes, float* f) {
  const pair_f32 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  f[0] = lo[0]; f[1] = lo[1]; f[2] = hi[0]; f[3] = hi[1];
}

// place of a block's scale: keys (which = 0) or values (1) of `slot`'s block
__device__ __forceinline__ int64_t scale_at(int64_t page, int Hkv, int g, int which, int slot, int log2_page) {
  return (((page * Hkv + g) * 2 + which) << (log2_page - 4)) + (slot >> 4);
}

}  // namespace
}  // namespace qcf
