// Weights in 4 bits: groups of 32 values along a row share a power of two, a value is one of
// +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} times it.  Both directions are the conversion instructions of the hardware, which round
// to the nearest code, ties to the even one, and saturate (checked on the card against the definition: every code with
// every scale; every bf16 value, and fp32 values on and beside every middle of two codes).
//
// Bound: memory.  A lane has eight values (one or two 16-byte loads, four bytes of codes), four lanes a group.  The weights,
// which nobody asks for again soon, pass the caches by (non-temporal), both ways: 184.5 million bf16 weights to 4 bits and
// back 180 -> 148 us, 6.3 TB/s.

#include "common.h"

namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int GROUP = FMOE_QUANT_GROUP;

// Largest of the magnitudes' bits over the four lanes of a group: finite values order as their bits do, infinities and NaN
// are above them.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, false);   // lanes 1 0 3 2
  v = v > o ? v : o;
  o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, false);            // lanes 2 3 0 1
  return v > o ? v : o;
}

// Unit u of a row has values 8u .. 8u+7; units per row rounded up to whole groups (the rest are zeros and not stored).
template <typename WT>
__global__ __launch_bounds__(256) void quantize_kernel(const WT* __restrict__ w, long long rows, int K, int units,
                                                       int saturate, uint32_t* __restrict__ codes,
                                                       uint8_t* __restrict__ scales) {
  const long long total = rows * units;
  const long long step = (long long)gridDim.x * blockDim.x;   // a multiple of four
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < ((total + 63) & ~63ll); i += step) {
    const long long row = i / units;
    const int u = (int)(i - row * units);
    const bool in = i < total && u * 8 < K;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (in) {
      const WT* src = w + row * K + u * 8;
      if constexpr (sizeof(WT) == 2) {
        const u32x4_t b = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(src));
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          v[2 * p] = __uint_as_float(b[p] << 16);
          v[2 * p + 1] = __uint_as_float(b[p] & 0xffff0000u);
        }
      } else {
        const f32x4_t lo = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(src));
        const f32x4_t hi = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(src) + 1);
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          v[p] = lo[p];
          v[4 + p] = hi[p];
        }
      }
    }
    uint32_t big = 0;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const uint32_t m = __float_as_uint(v[p]) & 0x7fffffffu;
      big = big > m ? big : m;
    }
    big = quad_max(big);
    // exponent of the largest less two; one more where values past 6 scales are not to saturate (largest above 1.5 * 2^n)
    int e = (int)(big >> 23) - 2 + (!saturate && (big & 0x7fffffu) > 0x400000u ? 1 : 0);
    e = e < 1 ? 1 : e;
    if (big == 0u) e = 127;
    const bool finite = big < 0x7f800000u;
    const float scale = __uint_as_float((uint32_t)(finite ? e : 127) << 23);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], scale, 3);
    if (!in) continue;
    codes[(row * K >> 3) + u] = finite ? c : 0u;
    if ((u & 3) == 0) scales[row * (units >> 2) + (u >> 2)] = (uint8_t)(finite ? e : 255);
  }
}

template <typename WT>
__global__ __launch_bounds__(256) void dequantize_kernel(const uint32_t* __restrict__ codes,
                                                         const uint8_t* __restrict__ scales, long long rows, int K,
                                                         int units, WT* __restrict__ w) {
  const int per_row = K >> 3;
  const long long total = rows * per_row;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < total;
       i += (long long)gridDim.x * blockDim.x) {
    const long long row = i / per_row;
    const int u = (int)(i - row * per_row);
    const uint32_t c = codes[i];
    const float scale = __uint_as_float((uint32_t)scales[row * (units >> 2) + (u >> 2)] << 23);
    WT* dst = w + i * 8;
    if constexpr (sizeof(WT) == 2) {
      const u32x4_t v = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3))};
      __builtin_nontemporal_store(v, reinterpret_cast<u32x4_t*>(dst));
    } else {
      const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 1);
      const f32x2_t d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 3);
      __builtin_nontemporal_store(f32x4_t{a[0], a[1], b[0], b[1]}, reinterpret_cast<f32x4_t*>(dst));
      __builtin_nontemporal_store(f32x4_t{d[0], d[1], e[0], e[1]}, reinterpret_cast<f32x4_t*>(dst) + 1);
    }
  }
}

inline unsigned blocks_for(long long threads) {
  const long long b = (threads + 255) / 256;
  return (unsigned)(b < 65536 ? b : 65536);
}

}  // namespace

int launch_quantize(const void* w, int dtype, long long rows, int K, int saturate, void* codes, uint8_t* scales,
                    hipStream_t stream) {
  const int units = (K + GROUP - 1) / GROUP * (GROUP / 8);
  const dim3 grid(blocks_for(rows * units)), block(256);
  if (dtype == FMOE_BF16)
    hipLaunchKernelGGL(quantize_kernel<bf16_t>, grid, block, 0, stream, static_cast<const bf16_t*>(w), rows, K, units,
                       saturate, static_cast<uint32_t*>(codes), scales);
  else
    hipLaunchKernelGGL(quantize_kernel<float>, grid, block, 0, stream, static_cast<const float*>(w), rows, K, units,
                       saturate, static_cast<uint32_t*>(codes), scales);
  FMOE_HIP_CHECK(hipGetLastError());
  return FMOE_OK;
}

int launch_dequantize(const void* codes, const uint8_t* scales, long long rows, int K, int dtype, void* w,
                      hipStream_t stream) {
  const int units = (K + GROUP - 1) / GROUP * (GROUP / 8);
  const dim3 grid(blocks_for(rows * (K / 8))), block(256);
  if (dtype == FMOE_BF16)
    hipLaunchKernelGGL(dequantize_kernel<bf16_t>, grid, block, 0, stream, static_cast<const uint32_t*>(codes), scales,
                       rows, K, units, static_cast<bf16_t*>(w));
  else
    hipLaunchKernelGGL(dequantize_kernel<float>, grid, block, 0, stream, static_cast<const uint32_t*>(codes), scales,
                       rows, K, units, static_cast<float*>(w));
  FMOE_HIP_CHECK(hipGetLastError());
  return FMOE_OK;
}
