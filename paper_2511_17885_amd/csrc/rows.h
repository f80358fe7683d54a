// Reductions over the rows of 16 lanes of a wavefront, inside the vector unit.
#pragma once

#include "common.h"

#if defined(__HIPCC__)
// v of the lane `ROT` places on in the row of 16
template <int ROT>
__device__ __forceinline__ float row_rotate(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x120 + ROT, 0xf, 0xf, false));
}
template <int ROT>
__device__ __forceinline__ int row_rotate(int v) {
  return __builtin_amdgcn_update_dpp(0, v, 0x120 + ROT, 0xf, 0xf, false);
}
// Over the 16 lanes of a row, the result in every lane.  After the step by 8 all values repeat with period 8,
// so the step by 4 pairs what an exclusive-or by 4 would, and so on: the sum is the xor butterfly 8, 4, 2, 1.
__device__ __forceinline__ float row_sum_butterfly(float v) {
  v = v + row_rotate<8>(v);
  v = v + row_rotate<4>(v);
  v = v + row_rotate<2>(v);
  return v + row_rotate<1>(v);
}
__device__ __forceinline__ float larger(float v, float o) { return (o > v) ? o : v; }
__device__ __forceinline__ float row_max(float v) {
  v = larger(v, row_rotate<8>(v));
  v = larger(v, row_rotate<4>(v));
  v = larger(v, row_rotate<2>(v));
  return larger(v, row_rotate<1>(v));
}
__device__ __forceinline__ int row_min(int v) {
  v = min(v, row_rotate<8>(v));
  v = min(v, row_rotate<4>(v));
  v = min(v, row_rotate<2>(v));
  return min(v, row_rotate<1>(v));
}
// Largest over the row, in one instruction a step (all lanes of the wavefront are on).
__device__ __forceinline__ int row_max(int v) {
  v = max(v, __builtin_amdgcn_mov_dpp(v, 0x128, 0xf, 0xf, true));
  v = max(v, __builtin_amdgcn_mov_dpp(v, 0x124, 0xf, 0xf, true));
  v = max(v, __builtin_amdgcn_mov_dpp(v, 0x122, 0xf, 0xf, true));
  return max(v, __builtin_amdgcn_mov_dpp(v, 0x121, 0xf, 0xf, true));
}

// The same in 64 bits.
template <int ROT>
__device__ __forceinline__ double row_rotate(double v) {
  const int lo = row_rotate<ROT>(__double2loint(v)), hi = row_rotate<ROT>(__double2hiint(v));
  return __hiloint2double(hi, lo);
}
__device__ __forceinline__ double row_sum_butterfly(double v) {
  v = v + row_rotate<8>(v);
  v = v + row_rotate<4>(v);
  v = v + row_rotate<2>(v);
  return v + row_rotate<1>(v);
}
__device__ __forceinline__ double larger(double v, double o) { return (o > v) ? o : v; }
__device__ __forceinline__ double row_max(double v) {
  v = larger(v, row_rotate<8>(v));
  v = larger(v, row_rotate<4>(v));
  v = larger(v, row_rotate<2>(v));
  return larger(v, row_rotate<1>(v));
}
#endif
