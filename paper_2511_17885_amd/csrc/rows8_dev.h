// Rows in 8 bits: 32 neighbours share a power of two; four lanes with eight values each have a group.
#pragma once

#include "common.h"

#if defined(__HIPCC__)
namespace rows8 {

// Largest of the magnitudes' bits over four neighbouring lanes: finite values order as their bits do, infinities and NaN are above.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, false);   // lanes 1 0 3 2
  v = v > o ? v : o;
  o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, false);            // lanes 2 3 0 1
  return v > o ? v : o;
}

// The same over lanes 16 apart
__device__ __forceinline__ uint32_t column_max(uint32_t v) {
  auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = a[0] > a[1] ? a[0] : a[1];
  a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return a[0] > a[1] ? a[0] : a[1];
}

// Eight values of a lane: their e4m3 codes; `scale` becomes the group's scale byte; group_max: over the lanes of the group.  The scale is the least power of two with the
// largest magnitude at most 448 = 1.75 * 2^8 of it, at least 2^-126; 1 for zeros.  The instruction divides by it and rounds to
// the nearest code, ties to the even one.  An infinity or NaN in the group: codes 0, scale byte 255.
template <typename MAX>
__device__ __forceinline__ uint2 quantize(const float (&v)[8], uint32_t& scale, MAX&& group_max) {
  uint32_t big = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t m = __float_as_uint(v[e]) & 0x7fffffffu;
    big = big > m ? big : m;
  }
  big = group_max(big);
  int e8 = (int)(big >> 23) - 8 + ((big & 0x7fffffu) > 0x600000u ? 1 : 0);
  e8 = e8 < 1 ? 1 : e8;
  if (big == 0u) e8 = 127;
  const bool finite = big < 0x7f800000u;
  const float s = __uint_as_float((uint32_t)(finite ? e8 : 127) << 23);
  typedef short s16x2_t __attribute__((ext_vector_type(2)));
  s16x2_t c0 = {0, 0}, c1 = {0, 0};
  c0 = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c0, v[0], v[1], s, false);
  c0 = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c0, v[2], v[3], s, true);
  c1 = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c1, v[4], v[5], s, false);
  c1 = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c1, v[6], v[7], s, true);
  scale = finite ? (uint32_t)e8 : 255u;
  return finite ? uint2{__builtin_bit_cast(uint32_t, c0), __builtin_bit_cast(uint32_t, c1)} : uint2{0u, 0u};
}

}  // namespace rows8
#endif
