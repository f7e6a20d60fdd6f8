// e4m3 numbers with a power of two per block: conversions that the 8-bit cache and the 8-bit rows and weights share.
#pragma once
#include "vvs_mfma.h"

namespace vvs {

constexpr int kQLeast = -110;               // smallest exponent of a block

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Eight e4m3 numbers times a power of two as bf16 (exact)
__device__ __forceinline__ bf16x8 e4m3_to_bf16(uint2 b, float scale) {
  uint4 r;
  r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b.x, scale, false));
  r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b.x, scale, true));
  r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b.y, scale, false));
  r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b.y, scale, true));
  return as_bf16x8(r);
}

// e4m3 byte <-> float.  The conversion rounds to nearest, ties to even; nothing above 448 is given to it but what is not finite, which becomes NaN.
template <int I>
__device__ __forceinline__ float e4m3_at(uint32_t w) { return __builtin_amdgcn_cvt_f32_fp8(w, I); }
__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
__device__ __forceinline__ uint2 to_e4m3x8(const float (&v)[8]) { return make_uint2(to_e4m3x4(v[0], v[1], v[2], v[3]), to_e4m3x4(v[4], v[5], v[6], v[7])); }
__device__ __forceinline__ void from_e4m3x8(uint2 b, float (&v)[8]) {
  v[0] = e4m3_at<0>(b.x); v[1] = e4m3_at<1>(b.x); v[2] = e4m3_at<2>(b.x); v[3] = e4m3_at<3>(b.x);
  v[4] = e4m3_at<0>(b.y); v[5] = e4m3_at<1>(b.y); v[6] = e4m3_at<2>(b.y); v[7] = e4m3_at<3>(b.y);
}

// Smallest E >= kQLeast with top <= 448 * 2^E = 0.875 * 2^(E + 9)
__device__ __forceinline__ int e4m3_exponent(float top) {
  int e;
  const float m = frexpf(top, &e);
  return top > 0.f ? max(e - 9 + (m > 0.875f), kQLeast) : kQLeast;
}
__device__ __forceinline__ int exponent_of(float scale) { return scale > 0.f ? ilogbf(scale) : kQLeast; }   // (a block never written holds 0)
__device__ __forceinline__ bool finite(float x) { return fabsf(x) < INFINITY; }

}  // namespace vvs
