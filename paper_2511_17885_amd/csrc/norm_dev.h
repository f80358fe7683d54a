// Root-mean-square norm of a row that a wavefront, or four, hold in registers: shared by norm.hip and decode.hip.
//
// n = h * w * r, r = 1 / sqrt(mean h^2 + eps), is the fp32 number nearest to (all but) its exact value, or in 8 bits the code nearest to
// that value, so that it does not depend on who computes it: what decides experts or falls next to a border of two codes is the same
// everywhere.  bf16 is rounded from the fp32 number, as conversions from 64 bits do that go by way of it (the two roundings together
// are off by at most half a step and 2^-17 of one).  The sum of squares and r are taken in 64 bits, once a row.  An element needs no
// 64-bit instruction: r = 2^q (r_hi + r_lo) with r_hi in [1, 2), the products' errors come from fused multiply-adds (h is
// scaled by 2^q first, so that nothing overflows on the way), and the sum of what they leave decides the last rounding.  (From
// 2^-100 down the errors underflow: nearest but for that.)
#pragma once

#include "common.h"
#include "rows.h"

#if defined(__HIPCC__)
namespace rms {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

struct Scale {        // r = 2^q * (hi + lo)
  float hi, lo;
  int q;
};
// The root from the hardware's estimate (some 24 bits) by one step of third order: with e = 1 - m y^2 the error of
// y (1 + e/2 + 3 e^2/8) is of the order of e^3, far below the last bit of 64.
__device__ __forceinline__ Scale row_scale(double sum, double inv_d, float eps) {
  const double m = fma(sum, inv_d, (double)eps);
  double r = __builtin_amdgcn_rsq(m);
  Scale s{(float)r, 0.0f, 0};
  if (r > 0.0 && r < 1e300) {   // else 0 (a row with infinities), infinite (zeros without eps) or NaN as it is
    const double e = fma(-m * r, r, 1.0);
    r = fma(r * e, fma(0.375, e, 0.5), r);
    const int q = __builtin_amdgcn_frexp_exp(r) - 1;
    const double f = __builtin_amdgcn_ldexp(r, -q);
    s.hi = (float)f;
    s.lo = (float)(f - (double)s.hi);
    s.q = q;
  }
  return s;
}

__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }

// hi + lo, |lo| at most half a step of hi, as an fp32 number rounded to odd: from it a rounding to fewer bits (two fewer at
// least) is that of the sum.
__device__ __forceinline__ float odd(float hi, float lo) {
  uint32_t u = __float_as_uint(hi);
  if (lo != 0.0f && finite(hi) && hi != 0.0f) {
    u -= (u ^ __float_as_uint(lo)) >> 31;   // the other sign: the number below
    u |= 1u;
  }
  return __uint_as_float(u);
}
__device__ __forceinline__ bf16_t nearest_bf16(float v) { return __builtin_bit_cast(bf16_t, (__bf16)v); }   // ties to even, NaN stays one

// x + delta rounded to the type
template <typename T> __device__ __forceinline__ T add_rounded(float a, float b);
template <> __device__ __forceinline__ float add_rounded<float>(float a, float b) { return a + b; }
template <> __device__ __forceinline__ bf16_t add_rounded<bf16_t>(float a, float b) {
  const float s = a + b, t = s - a;
  return nearest_bf16(odd(s, (a - (s - t)) + (b - t)));
}

// The element's value as hi + lo, hi the nearest fp32 number
__device__ __forceinline__ void value(float h, float w, const Scale& r, float& hi, float& lo) {
  const float g = __builtin_amdgcn_ldexpf(h, r.q);
  const float t = g * w, te = fmaf(g, w, -t);
  const float p = t * r.hi;
  const float e = fmaf(te, r.hi, fmaf(t, r.lo, fmaf(t, r.hi, -p)));   // up to a step of p
  hi = p + e;
  lo = e - (hi - p);
  if (!finite(p)) {
    hi = p;
    lo = 0.0f;
  }
}
template <typename T> __device__ __forceinline__ T value_rounded(float h, float w, const Scale& r);
template <> __device__ __forceinline__ float value_rounded<float>(float h, float w, const Scale& r) {
  float hi, lo;
  value(h, w, r, hi, lo);
  return hi;
}
template <> __device__ __forceinline__ bf16_t value_rounded<bf16_t>(float h, float w, const Scale& r) {
  return nearest_bf16(value_rounded<float>(h, w, r));
}

// Eight neighbouring elements
template <typename T> struct Unit;
template <> struct Unit<bf16_t> {
  u32x4_t v;
  template <bool PASS = false>   // past the caches
  __device__ __forceinline__ void load(const bf16_t* p) {
    if constexpr (PASS) v = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
    else v = *reinterpret_cast<const u32x4_t*>(p);
  }
  template <bool PASS = false>
  __device__ __forceinline__ void store(bf16_t* p) const {
    if constexpr (PASS) __builtin_nontemporal_store(v, reinterpret_cast<u32x4_t*>(p));
    else *reinterpret_cast<u32x4_t*>(p) = v;
  }
  __device__ __forceinline__ void zero() { v = u32x4_t{0u, 0u, 0u, 0u}; }
  __device__ __forceinline__ float get(int i) const { return __uint_as_float((i & 1) ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16); }
  __device__ __forceinline__ void set2(int i, bf16_t a, bf16_t b) { v[i >> 1] = (uint32_t)a | ((uint32_t)b << 16); }   // i even
};
template <> struct Unit<float> {
  f32x4_t lo, hi;
  template <bool PASS = false>
  __device__ __forceinline__ void load(const float* p) {
    const f32x4_t* const q = reinterpret_cast<const f32x4_t*>(p);
    lo = PASS ? __builtin_nontemporal_load(q) : q[0];
    hi = PASS ? __builtin_nontemporal_load(q + 1) : q[1];
  }
  template <bool PASS = false>
  __device__ __forceinline__ void store(float* p) const {
    f32x4_t* const q = reinterpret_cast<f32x4_t*>(p);
    if constexpr (PASS) {
      __builtin_nontemporal_store(lo, q);
      __builtin_nontemporal_store(hi, q + 1);
    } else {
      q[0] = lo;
      q[1] = hi;
    }
  }
  __device__ __forceinline__ void zero() { lo = hi = f32x4_t{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ float get(int i) const { return i < 4 ? lo[i] : hi[i - 4]; }
  __device__ __forceinline__ void set2(int i, float a, float b) {
    if (i < 4) { lo[i] = a; lo[i + 1] = b; }
    else { hi[i - 4] = a; hi[i - 3] = b; }
  }
};

// v plus that of the lane 16, or 32, away
__device__ __forceinline__ double add_16_apart(double v) {
  const uint32_t lo = (uint32_t)__double2loint(v), hi = (uint32_t)__double2hiint(v);
  const auto l = __builtin_amdgcn_permlane16_swap(lo, lo, false, false), h = __builtin_amdgcn_permlane16_swap(hi, hi, false, false);
  return __hiloint2double((int)h[0], (int)l[0]) + __hiloint2double((int)h[1], (int)l[1]);
}
__device__ __forceinline__ double add_32_apart(double v) {
  const uint32_t lo = (uint32_t)__double2loint(v), hi = (uint32_t)__double2hiint(v);
  const auto l = __builtin_amdgcn_permlane32_swap(lo, lo, false, false), h = __builtin_amdgcn_permlane32_swap(hi, hi, false, false);
  return __hiloint2double((int)h[0], (int)l[0]) + __hiloint2double((int)h[1], (int)l[1]);
}
__device__ __forceinline__ double wave_sum(double v) {   // in every lane, a fixed order
  return add_32_apart(add_16_apart(row_sum_butterfly(v)));
}

// Eight weights of either type as floats
template <typename WT>
__device__ __forceinline__ void load_weights(const void* w, int k, float (&f)[8]) {
  Unit<WT> u;
  u.load(static_cast<const WT*>(w) + k);
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = u.get(i);
}

}  // namespace rms
#endif
