// Expert products on 4-bit weights: codes to bf16 operands, work items found from the experts' offsets, shapes of the packed matrices.
#pragma once

#include "ffn_dev.h"

#if defined(__HIPCC__)
namespace {

// Eight codes times the scale in byte I of `scales`.  The instruction takes the exponent of its scale operand and nothing else
// (checked on the card for every exponent with thousands of other bits): the byte is only shifted there.
template <int I>
__device__ __forceinline__ u32x4_t dequantize(uint32_t codes, uint32_t scales) {
  const float s = __uint_as_float(I == 0 ? scales << 23 : I == 1 ? scales << 15 : I == 2 ? scales << 7 : scales >> 1);
  return u32x4_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3))};
}

struct QuantItem {
  int group, unit, row0, rows;     // group < 0: none
  bool shared;
};
// Row tiles of 1 << a.log2_bm rows.  Experts whose offsets are malformed are skipped as in fmoe_build_tiles.  Uniform.
// EVEN: an eighth of the shared groups' items and an eighth of the routed experts' for each XCD (workgroups: those of either, rounded
// up to eights); else an eighth of the sequence, which leaves the weights of the routed experts to some of them.
template <bool EVEN = false, typename ARGS>
__device__ __forceinline__ QuantItem find_tile(const ARGS& a, int block) {
  constexpr int Q = FMOE_MAX_EXPERTS / 64;
  const int lane = threadIdx.x & 63, bm = 1 << a.log2_bm;
  int r0[Q], cnt[Q], first[Q];   // of expert 64 q + lane: first row, rows, first tile
  int tiles = 0;
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int e = 64 * q + lane;
    r0[q] = cnt[q] = 0;
    if (64 * q < a.E && a.row_cap > 0) {   // uniform
      const int at = e < a.E ? e : a.E - 1;
      r0[q] = a.expert_offsets[at];
      cnt[q] = a.expert_offsets[at + 1];
    }
  }
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const bool good = 64 * q + lane < a.E && r0[q] >= 0 && cnt[q] > r0[q] && cnt[q] <= a.row_cap;
    cnt[q] = good ? cnt[q] - r0[q] : 0;
    const int nt = (cnt[q] + bm - 1) >> a.log2_bm;
    const int scan = wave_scan(nt);
    first[q] = tiles + scan - nt;
    tiles += __builtin_amdgcn_readlane(scan, 63);
  }
  const int n = resolve_count(a.n_cap, a.n_dev);
  const int shared_tiles = (n + bm - 1) >> a.log2_bm, per_group = shared_tiles * a.shared_cols;
  const int shared_items = per_group * a.shared_groups;
  QuantItem it{-1, 0, 0, 0, false};
  int g;
  if constexpr (EVEN) {
    const int s_share = (shared_items + 7) >> 3, r_items = tiles * a.cols, r_share = (r_items + 7) >> 3, xcd = block & 7;
    int place = block >> 3;
    if (place < s_share) {
      g = xcd * s_share + place;
      if (g >= shared_items) return it;
    } else {
      place -= s_share;
      g = xcd * r_share + place;
      if (place >= r_share || g >= r_items) return it;
      g += shared_items;
    }
  } else {
    const int items = shared_items + tiles * a.cols, share = (items + 7) >> 3, place = block >> 3;
    g = (block & 7) * share + place;
    if (place >= share || g >= items) return it;
  }
  if (g < shared_items) {
    it.shared = true;
    it.group = g / per_group;
    g -= it.group * per_group;
    it.unit = g / shared_tiles;
    it.row0 = (g - it.unit * shared_tiles) * bm;
    it.rows = n - it.row0 < bm ? n - it.row0 : bm;
    return it;
  }
  g -= shared_items;
  const int tile = g / a.cols;
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int nt = (cnt[q] + bm - 1) >> a.log2_bm;
    const unsigned long long mine = __ballot(first[q] <= tile && tile < first[q] + nt);
    if (mine != 0) {   // in one q only
      const int at = __ffsll((long long)mine) - 1;
      const int e_first = __builtin_amdgcn_readlane(first[q], at), e_tiles = __builtin_amdgcn_readlane(nt, at);
      const int e_rows = __builtin_amdgcn_readlane(cnt[q], at);
      g -= e_first * a.cols;
      it.group = 64 * q + at;
      it.unit = g / e_tiles;
      const int row = (g - it.unit * e_tiles) * bm;
      it.row0 = __builtin_amdgcn_readlane(r0[q], at) + row;
      it.rows = e_rows - row < bm ? e_rows - row : bm;
    }
  }
  return it;
}
// Matrices of a layer as they are packed: groups, column blocks, output features, reduction
struct PackedMatrix {
  int groups, nbw, N, K;
};
// 0 gate/up, 1 down, 2 shared gate/up, 3 shared down
inline PackedMatrix packed_matrix(const fmoe_config& c, int which) {
  const int Ft = c.n_shared * c.d_ffn_shared;
  switch (which) {
    case 0: return {c.n_experts, (c.d_ffn + 15) / 16, c.d_ffn, c.d_model};
    case 1: return {c.n_experts, (c.d_model + 31) / 32, c.d_model, c.d_ffn};
    case 2: return {Ft > 0 ? 1 : 0, (Ft + 15) / 16, Ft, c.d_model};
    default: return {Ft > 0 ? c.n_shared : 0, (c.d_model + 31) / 32, c.d_model, Ft > 0 ? c.d_ffn_shared : 8};
  }
}

}  // namespace
#endif
