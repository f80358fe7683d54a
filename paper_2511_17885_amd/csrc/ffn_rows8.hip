// The expert FFNs of Eq.4 on rows in 8 bits (e4m3, a power of two per 32 neighbours: rows8_dev.h) and weights in 4 bits
// (quant.hip), also the hidden rows h = silu(gate) * up between the two products, which are rounded to 8 bits on their way.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 takes both formats as they are, and the two scales of every 32 products: nothing is converted.
// It does in a step of 128 k what the bf16 instruction does in four of 32, in half the time.  Lane l has of a row (l % 16)
// the 16-byte pieces l / 16 and l / 16 + 4 of a k tile of 128, of a feature the 32 codes from 32 (l / 16) on; its scale operands
// have in one of their four bytes, which the instruction names, the power of two of the l / 16-th 32 of the row and the feature.
// The instruction cuts the products of eight neighbouring k at 2^-13 of the largest power of two among them and adds the eights up in
// fp32 (found on the card).  In tiles of 128 rows that stays: less is lost than the rounding of the rows to 8 bits has taken.  But gate
// and up decide on which code a hidden value becomes, and a thousandth of the values falls to another one by it; among a few
// rows one large value of those can be most of an output's error.  So tiles of 32 rows give the instruction the codes of 2 and more and
// the others one after the other: the products of either with 4-bit codes (multiples of 2^-3 with exponents up to 10, and of
// 2^-10 with exponents up to 2) have no digits to cut, and the sums are fp32's.  That is twice the matrix instructions where the weights' way from memory
// is the bound (400 tokens, d 2048, 128 experts of 768, 12 rows an expert, gate/up 43 us; 44 with one instruction and a ring of four).
//
// The weights are the first operand, so that a lane ends up with neighbouring features of one row: four of every fragment.  A column
// unit is four fragments, whose features are dealt so that the lane's are 8 neighbours in 32 hidden columns (gate and up of
// either half) or 16 neighbours in 64 output columns: rows are rounded to 8 bits and stored from registers.
// Packing (fmoe_set_weights_quant_rows): of a column unit, a k tile and a fragment lane l has one 16-byte unit, all units in one linear
// stream; of a column unit and a k tile the four fragments' scale bytes are a word.
//
// A workgroup has a tile of rows and a column unit per wavefront.  As in ffn.hip: rows global -> LDS directly, in a
// ring of k tiles (128 bytes a row, pieces exchanged so that operand reads meet no bank twice); weights into registers,
// as many tiles ahead; a barrier per k tile.  Work items are found from the experts' offsets (quant_items.h).

#include "ffn_dev.h"
#include "quant_items.h"
#include "rows8_dev.h"

namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));

#include "rows8_regs.inc"   // rows_acc<IDX>

constexpr int RBK = 128;       // k per tile
constexpr int FRAGS = 4;       // fragments of 16 features a column unit

struct RowsProblem {
  const uint8_t *A, *As;       // rows [*, lda] bytes and their scale bytes [*, ldas]
  uint32_t lda, ldas;
  const int32_t *map1, *map2;  // row -> index (perm_src) -> token (kept_idx), or null
  int map1_limit;
  const u32x4_t* Bp;
  const uint32_t* Sp;
  long long group_stride, scale_stride;   // units and words between groups
  int units, N, K;             // column units of a group
  uint8_t *H, *Hs;             // gate/up: the hidden rows
  uint32_t ldh, ldhs;
  int expert_groups;           // groups of 32 columns of one expert in H (shared experts stand side by side)
  bf16_t* C;                   // down
  int ldc;
  int a_group_off, as_group_off;          // of a shared expert's part of the rows
  long long c_group_off;
};

struct RowsArgs {
  RowsProblem p0, p1;              // routed experts; shared group
  const int32_t* expert_offsets;   // null without room for rows
  const int32_t* n_dev;            // or null
  int E, n_cap, row_cap;
  int cols;                        // column units of an expert
  int shared_groups, shared_cols;  // shared groups in this launch, column units of one
  int log2_bm;                     // rows of a row tile
};

__host__ __device__ inline int rows_tiles(int K) { return (K + RBK - 1) / RBK; }

// Operand of a row block from LDS: the lane's two pieces and its scale byte, see lds_issue_frags_at
template <int OFF, int OFF_S>
__device__ __forceinline__ void issue_rows(uint32_t a0, uint32_t a1, uint32_t as, u32x4_t& f0, u32x4_t& f1, uint32_t& s) {
  asm volatile("ds_read_b128 %0, %3 offset:%6\n\tds_read_b128 %1, %4 offset:%6\n\tds_read_u8 %2, %5 offset:%7"
               : "=&v"(f0), "=&v"(f1), "=&v"(s) : "v"(a0), "v"(a1), "v"(as), "n"(OFF), "n"(OFF_S) : "memory");
}
__device__ __forceinline__ void settle_rows(u32x4_t& f0, u32x4_t& f1, uint32_t& s) {
  asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(f0), "+v"(f1), "+v"(s) : : "memory");
}
__device__ __forceinline__ i32x8_t joined(u32x4_t a0, u32x4_t a1) {
  return i32x8_t{(int)a0[0], (int)a0[1], (int)a0[2], (int)a0[3], (int)a1[0], (int)a1[1], (int)a1[2], (int)a1[3]};
}
// Codes of 2 and more (bit 6 is set), 0 in the others' places
__device__ __forceinline__ i32x8_t large_codes(i32x8_t r) {
  i32x8_t large;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t c = (uint32_t)r[i];
    large[i] = (int)(c & __builtin_amdgcn_perm(c << 9, c << 1, 0x090b080au));   // selectors 8 to 11: eight times a byte's top bit
    __builtin_amdgcn_sched_barrier(0);   // one after the other: no registers for the steps between
  }
  return large;
}
// c += weights (byte I of sw) x rows (byte 0 of sr)
template <int I>
__device__ __forceinline__ f32x4_t mfma_rows(u32x4_t w, uint32_t sw, i32x8_t r, uint32_t sr, f32x4_t c) {
  typedef int i32x4_t __attribute__((ext_vector_type(4)));
  const i32x4_t w4 = __builtin_bit_cast(i32x4_t, w);
  const i32x8_t w8 = __builtin_shufflevector(w4, w4, 0, 1, 2, 3, -1, -1, -1, -1);   // 4-bit operands have four registers
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w8, r, c, 4, 0, I, (int)sw, 0, (int)sr);
}

// One work item: NRB row blocks of 16, LDS stages of ROWS rows; wavefront w has column unit cu0 + w.
template <bool SWIGLU, int NRB, int ROWS, int STAGES, bool NAMED>
__device__ __forceinline__ void rows_tile(const RowsProblem& P, int row0, int rows, int group, int cu0, char* smem) {
  constexpr int AHEAD = STAGES - 1;
  constexpr int NLA = (NRB + 1) / 2;                           // loads of eight rows a wavefront
  static_assert(32 * NLA <= ROWS, "the rows fit in a stage");
  constexpr int SROWS = ROWS > 64 ? ROWS : 64;                 // scale words a stage
  constexpr int PER_TILE = NLA + 1 + FRAGS + 1;                // loads of a k tile
  constexpr bool SPLIT = SWIGLU && !NAMED;                     // large and small codes apart, see above
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int K = P.K, NT = rows_tiles(K);
  char* const rows_lds = smem;
  char* const scales_lds = smem + STAGES * ROWS * RBK;

  const __amdgpu_buffer_rsrc_t b_rsrc = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<u32x4_t*>(P.Bp) + (size_t)group * P.group_stride, 0, 0xffffffff, 0x00020000);
  const __amdgpu_buffer_rsrc_t s_rsrc = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint32_t*>(P.Sp) + (size_t)group * P.scale_stride, 0, 0xffffffff, 0x00020000);
  const __amdgpu_buffer_rsrc_t a_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(P.A), 0, 0xffffffff, 0x00020000);
  const __amdgpu_buffer_rsrc_t as_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(P.As), 0, 0xffffffff, 0x00020000);
  const int cu = cu0 + wave < P.units ? cu0 + wave : P.units - 1;   // past the end the last one again, not stored
  const uint32_t bbase = (uint32_t)cu * (uint32_t)NT * (FRAGS * 1024u), sbase = (uint32_t)cu * (uint32_t)NT * 256u;   // scalar
  const uint32_t lane16 = (uint32_t)lane * 16u, lane4 = (uint32_t)lane * 4u;

  u32x4_t breg[STAGES][FRAGS];
  uint32_t sreg[STAGES];
  auto load_b = [&](int slot, int t, int i) {
    breg[slot][i] = __builtin_amdgcn_raw_buffer_load_b128(
        b_rsrc, lane16, bbase + (uint32_t)(t < NT ? t : NT - 1) * (FRAGS * 1024u) + (uint32_t)i * 1024u, 0);
  };
  auto load_s = [&](int slot, int t) {
    sreg[slot] = __builtin_amdgcn_raw_buffer_load_b32(s_rsrc, lane4, sbase + (uint32_t)(t < NT ? t : NT - 1) * 256u, 0);
  };
  // Rows this lane fetches: 32 it + 8 wave + lane / 8 of the tile; scale words of row 64 (wave % 2) + lane (or lane where the
  // stage has 64: the wavefronts then fetch the same).  Past the tile its last row.
  const uint32_t most = 0xffffffffu / P.lda - 1u;
  int src[NLA + 1];
#pragma unroll
  for (int it = 0; it <= NLA; ++it) {
    const int r = it < NLA ? 32 * it + 8 * wave + (lane >> 3) : (ROWS > 64 ? 64 * (wave & 1) : 0) + lane;
    src[it] = row0 + (r < rows ? r : rows - 1);
    if (P.map1) src[it] = P.map1[src[it]];
  }
  order_loads();
#pragma unroll
  for (int t = 0; t < AHEAD; ++t) {
    load_s(t, t);
#pragma unroll
    for (int i = 0; i < FRAGS; ++i) load_b(t, t, i);
  }
  order_loads();
  uint32_t a_src[NLA], a_last[NLA], as_src;   // of the lane's piece in k tile 0, and in the last one less its start
  const int k_last = (NT - 1) * RBK;
#pragma unroll
  for (int it = 0; it <= NLA; ++it) {
    int s = src[it];
    if (P.map1 && P.map1_limit > 0) s = s < 0 ? 0 : (s >= P.map1_limit ? P.map1_limit - 1 : s);
    if (P.map2) s = P.map2[s];
    const uint32_t at = (uint32_t)s < most ? (uint32_t)s : most;
    if (it < NLA) {   // row r keeps its 16-byte piece c at place c ^ (r / 2 % 8)
      const int piece = ((lane & 7) ^ ((4 * wave + (lane >> 4)) & 7)) * 16;
      a_last[it] = at * P.lda + (uint32_t)(k_last + piece < K ? piece : K - 16 - k_last);   // past K the row's end again
      a_src[it] = at * P.lda + (uint32_t)piece;
    } else {
      as_src = at * P.ldas;
    }
  }
  auto load_a = [&](int stage, int t, int it) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(a_rsrc, FMOE_LPTR(rows_lds + stage * (ROWS * RBK) + (32 * it + 8 * wave) * RBK), 16,
                                             t < NT - 1 ? a_src[it] : a_last[it], (uint32_t)(t < NT ? t : NT - 1) * RBK, 0, 0);
  };
  auto load_as = [&](int stage, int t) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(as_rsrc, FMOE_LPTR(scales_lds + stage * (SROWS * 4) + (ROWS > 64 ? (wave & 1) * 256 : 0)), 4,
                                             as_src, (uint32_t)(t < NT ? t : NT - 1) * 4u, 0, 0);
  };
#pragma unroll
  for (int t = 0; t < AHEAD; ++t) {
#pragma unroll
    for (int it = 0; it < NLA; ++it) load_a(t, t, it);
    load_as(t, t);
    order_loads();
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)FMOE_LPTR(rows_lds), lds1 = (uint32_t)(uintptr_t)FMOE_LPTR(scales_lds);
  const uint32_t frag_row = lds0 + (uint32_t)(lane & 15) * RBK;
  const uint32_t frag_a0 = frag_row + (uint32_t)(((lane >> 4)) ^ ((lane & 15) >> 1)) * 16;
  const uint32_t frag_a1 = frag_row + (uint32_t)(((lane >> 4) + 4) ^ ((lane & 15) >> 1)) * 16;
  const uint32_t frag_s = lds1 + (uint32_t)(lane & 15) * 4 + (uint32_t)(lane >> 4);

  // Accumulators: hand-placed ones (number FRAGS * rb + i) for tiles of 128 rows, where the compiler would put part of them into
  // scratch memory
  f32x4_t acc[NAMED ? 1 : NRB][FRAGS];
  if constexpr (NAMED) {
    dense_claim_acc();
  } else {
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
      for (int i = 0; i < FRAGS; ++i) acc[rb][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  // k tile t, U = t % STAGES: products, and the loads of tile t + AHEAD; of the LAST tiles, fewer than STAGES, products only
  u32x4_t fa[2][2];
  uint32_t fs[2];
  auto ktile = [&](auto uc, auto last, int t) {
    constexpr int U = decltype(uc)::value;
    constexpr bool LAST = decltype(last)::value;
    // loads newer than this tile's rows, see ffn_quant.hip
    constexpr int LATER = U < AHEAD ? AHEAD - 1 - U : 0;
    if constexpr (LAST) {
      if (t < AHEAD) FMOE_WAIT_VM(LATER * (NLA + 1));   // uniform
      else FMOE_WAIT_VM(LATER * PER_TILE);
    } else {
      if (t < AHEAD) FMOE_WAIT_VM(LATER * (NLA + 1) + U * PER_TILE);
      else FMOE_WAIT_VM((AHEAD - 1) * PER_TILE);
    }
    block_barrier();   // every wavefront's share of the tile is in LDS; all are done with the tile before
    constexpr int off = U * (ROWS * RBK), off_s = U * (SROWS * 4);
    issue_rows<off, off_s>(frag_a0, frag_a1, frag_s, fa[0][0], fa[0][1], fs[0]);
    static_for<0, NRB>([&](auto rc) {
      constexpr int rb = decltype(rc)::value, cur = rb & 1, nxt = cur ^ 1;
      settle_rows(fa[cur][0], fa[cur][1], fs[cur]);
      if constexpr (rb + 1 < NRB)
        issue_rows<off + (rb + 1) * 16 * RBK, off_s + (rb + 1) * 64>(frag_a0, frag_a1, frag_s, fa[nxt][0], fa[nxt][1], fs[nxt]);
      if constexpr (!LAST) {
#pragma unroll
        for (int i = 0; i < PER_TILE; ++i) {   // load i of the tile goes out with row block i * NRB / PER_TILE
          if ((i * NRB) / PER_TILE != rb) continue;
          if (i < NLA) load_a((U + AHEAD) % STAGES, t + AHEAD, i);
          else if (i == NLA) load_as((U + AHEAD) % STAGES, t + AHEAD);
          else if (i == NLA + 1) load_s((U + AHEAD) % STAGES, t + AHEAD);
          else load_b((U + AHEAD) % STAGES, t + AHEAD, i - NLA - 2);
        }
      }
      __builtin_amdgcn_sched_barrier(0);   // the next operand is on its way behind the products
      auto products = [&](i32x8_t r) {
        static_for<0, FRAGS>([&](auto ic) {
          constexpr int i = decltype(ic)::value;
          if constexpr (NAMED) rows_acc<FRAGS * rb + i>::template add<i>(breg[U][i], sreg[U], r, fs[cur]);
          else acc[rb][i] = mfma_rows<i>(breg[U][i], sreg[U], r, fs[cur], acc[rb][i]);
        });
      };
      const i32x8_t r = joined(fa[cur][0], fa[cur][1]);
      if constexpr (SPLIT) {
        const i32x8_t large = large_codes(r);
        products(large);
        __builtin_amdgcn_sched_barrier(0);
        products(r ^ large);
      } else {
        products(r);
      }
    });
  };
  int t0 = 0;
  for (; t0 + STAGES <= NT; t0 += STAGES)
    static_for<0, STAGES>([&](auto uc) { ktile(uc, std::false_type{}, t0 + decltype(uc)::value); });
  static_for<0, STAGES - 1>([&](auto uc) {
    if (t0 + decltype(uc)::value < NT) ktile(uc, std::true_type{}, t0 + decltype(uc)::value);   // uniform
  });
  FMOE_WAIT_VM(0);   // the loads issued past the end have landed before the workgroup's LDS is another's
  // the last matrix instructions have retired before hand-placed accumulators are read, see ffn.hip
  if constexpr (NAMED) asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 7" ::: "memory");
  if (cu0 + wave >= P.units) return;
  auto result = [&](auto rbc, auto ic) {
    if constexpr (NAMED) return read_acc<FRAGS * decltype(rbc)::value + decltype(ic)::value>();
    else return acc[decltype(rbc)::value][decltype(ic)::value];
  };
  static_for<0, NRB>([&](auto rbc) {
    constexpr int rb = decltype(rbc)::value;
    const f32x4_t c0 = result(rbc, std::integral_constant<int, 0>{}), c1 = result(rbc, std::integral_constant<int, 1>{});
    const f32x4_t c2 = result(rbc, std::integral_constant<int, 2>{}), c3 = result(rbc, std::integral_constant<int, 3>{});
    const int r = rb * 16 + (lane & 15), g = lane >> 4;
    const size_t at = (size_t)(row0 + r);
    if constexpr (SWIGLU) {   // eight neighbouring columns a lane, 32 of them in the four lanes of a row
      float v[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = silu_mul_bf16(c0[e], c1[e]);
        v[4 + e] = silu_mul_bf16(c2[e], c3[e]);
      }
      uint32_t scale;
      const uint2 c = rows8::quantize(v, scale, [](uint32_t m) { return rows8::column_max(m); });
      if (r < rows) {
        const int col = cu * 32 + 8 * g;
        *reinterpret_cast<uint2*>(P.H + at * P.ldh + col) = c;
        if (g == 0) {
          const int expert = cu / P.expert_groups, k = cu - expert * P.expert_groups;
          uint8_t* const s = P.Hs + at * P.ldhs + expert * ((P.expert_groups + 3) / 4 * 4) + k;
          s[0] = (uint8_t)scale;
          if (k == P.expert_groups - 1)
            for (int q = k + 1; q & 3; ++q) s[q - k] = 127;   // the word's unused bytes
        }
      }
    } else if (r < rows) {    // sixteen neighbouring columns a lane
      const int col = cu * 64 + 16 * g;
      if (col < P.N) {        // (a multiple of 32)
        auto pair = [](float a, float b) { return (uint32_t)f32_to_bf16(a) | ((uint32_t)f32_to_bf16(b) << 16); };
        u32x4_t* const to = reinterpret_cast<u32x4_t*>(P.C + at * P.ldc + col);
        // streaming stores: the next kernel reads the rows, this one never does
        __builtin_nontemporal_store(u32x4_t{pair(c0[0], c0[1]), pair(c0[2], c0[3]), pair(c1[0], c1[1]), pair(c1[2], c1[3])}, to);
        __builtin_nontemporal_store(u32x4_t{pair(c2[0], c2[1]), pair(c2[2], c2[3]), pair(c3[0], c3[1]), pair(c3[2], c3[3])}, to + 1);
      }
    }
  });
}

// field by field, so that the descriptors stay in scalar registers
__device__ __forceinline__ RowsProblem rows_problem(const RowsArgs& a, const QuantItem& it) {
  RowsProblem Q;
#define FMOE_SEL(f) Q.f = it.shared ? a.p1.f : a.p0.f
  FMOE_SEL(A); FMOE_SEL(As); FMOE_SEL(lda); FMOE_SEL(ldas); FMOE_SEL(map1); FMOE_SEL(map2); FMOE_SEL(map1_limit);
  FMOE_SEL(Bp); FMOE_SEL(Sp); FMOE_SEL(group_stride); FMOE_SEL(scale_stride); FMOE_SEL(units); FMOE_SEL(N); FMOE_SEL(K);
  FMOE_SEL(H); FMOE_SEL(Hs); FMOE_SEL(ldh); FMOE_SEL(ldhs); FMOE_SEL(expert_groups); FMOE_SEL(C); FMOE_SEL(ldc);
  FMOE_SEL(a_group_off); FMOE_SEL(as_group_off); FMOE_SEL(c_group_off);
#undef FMOE_SEL
  if (it.shared) {   // a shared expert's part of the hidden rows, its output (down)
    Q.A += (size_t)it.group * Q.a_group_off;
    Q.As += (size_t)it.group * Q.as_group_off;
    Q.C += (size_t)it.group * Q.c_group_off;
  }
  return Q;
}

constexpr int FEW_ROWS = 32, MANY_ROWS = 128;
constexpr int FEW_STAGES = 3, MANY_STAGES = 4;   // ring of k tiles, of rows and of weights (few: with four registers go to memory)
constexpr int lds_bytes(int rows, int stages) { return stages * (rows * RBK + (rows > 64 ? rows : 64) * 4); }

// Bound: the weights (400 tokens, d 2048, 128 experts of 768, 12 rows an expert: 43 + 26 us with the launches, 5.0 TB/s).
template <bool SWIGLU>
__global__ __launch_bounds__(256, 3) void ffn_rows8_few_kernel(RowsArgs a) {
  __shared__ __align__(16) char smem[lds_bytes(FEW_ROWS, FEW_STAGES)];
  const QuantItem it = find_tile<true>(a, (int)blockIdx.x);
  if (it.group < 0) return;
  const RowsProblem P = rows_problem(a, it);
  if (it.rows <= 16) rows_tile<SWIGLU, 1, FEW_ROWS, FEW_STAGES, false>(P, it.row0, it.rows, it.group, 4 * it.unit, smem);   // uniform
  else rows_tile<SWIGLU, 2, FEW_ROWS, FEW_STAGES, false>(P, it.row0, it.rows, it.group, 4 * it.unit, smem);
}
// Bound: matrix instructions, by the power they take: 16384 tokens, two experts of 8192, d 4096 883 + 468 us, 2.4 PFLOP/s (a bf16 library
// product of 8192^3 1.18), matrix units 70 % busy at a clock of 1.6 GHz.  With short reductions and few rows also an item's start and end:
// 8192 tokens, d 2048, 128 experts of 768 125 + 88 us, matrix units 50 and 32 % busy.
// (The build looks at the registers of a kernel of this name.)
template <bool SWIGLU>
__global__ __launch_bounds__(256, 2) void ffn_rows8_many_kernel(RowsArgs a) {
  __shared__ __align__(16) char smem[lds_bytes(MANY_ROWS, MANY_STAGES)];
  const QuantItem it = find_tile<true>(a, (int)blockIdx.x);
  if (it.group < 0) return;
  const RowsProblem P = rows_problem(a, it);
  switch ((it.rows + 31) >> 5) {   // live 32-row bands of the tile, uniform
    case 1: rows_tile<SWIGLU, 2, MANY_ROWS, MANY_STAGES, true>(P, it.row0, it.rows, it.group, 4 * it.unit, smem); break;
    case 2: rows_tile<SWIGLU, 4, MANY_ROWS, MANY_STAGES, true>(P, it.row0, it.rows, it.group, 4 * it.unit, smem); break;
    case 3: rows_tile<SWIGLU, 6, MANY_ROWS, MANY_STAGES, true>(P, it.row0, it.rows, it.group, 4 * it.unit, smem); break;
    default: rows_tile<SWIGLU, 8, MANY_ROWS, MANY_STAGES, true>(P, it.row0, it.rows, it.group, 4 * it.unit, smem); break;
  }
}

// Feature of row r of fragment i in column unit cu
template <bool PAIR>
__device__ __forceinline__ int unit_feature(int cu, int i, int r) {
  return PAIR ? 32 * cu + 8 * (r >> 2) + 4 * (i >> 1) + (r & 3) : 64 * cu + 16 * (r >> 2) + 4 * i + (r & 3);
}
// Source rows [group][n][k]: codes two to a byte, scales one byte per 32 k.  PAIR: gate (fragments 0 and 2) and up.  Past N and K
// the codes are 0 and the scales 1.
template <bool PAIR>
__global__ __launch_bounds__(256) void pack_rows8_kernel(const u32x4_t* __restrict__ codes0, const uint8_t* __restrict__ scales0,
                                                         const u32x4_t* __restrict__ codes1, const uint8_t* __restrict__ scales1,
                                                         u32x4_t* __restrict__ dst, uint32_t* __restrict__ dst_scales, int G,
                                                         int N, int K, int units) {
  const int NT = rows_tiles(K), KG = K / FMOE_QUANT_GROUP;
  const size_t total = (size_t)G * units * NT * (FRAGS * 64), total_scales = (size_t)G * units * NT * 64;
  for (size_t u = (size_t)blockIdx.x * blockDim.x + threadIdx.x; u < total + total_scales; u += (size_t)gridDim.x * blockDim.x) {
    const bool scales = u >= total;
    size_t q = scales ? u - total : u;
    const int lane = (int)(q & 63), row = lane & 15;
    q >>= 6;
    const int f = scales ? 0 : (int)(q % FRAGS);
    if (!scales) q /= FRAGS;
    const int k = (int)(q % NT) * 4 + (lane >> 4);   // 32 codes: a 16-byte unit of the source
    q /= NT;
    const int cu = (int)(q % units), g = (int)(q / units);
    if (!scales) {
      const int n = unit_feature<PAIR>(cu, f, row);
      u32x4_t v = {0u, 0u, 0u, 0u};
      if (n < N && k < KG) v = (PAIR && (f & 1) ? codes1 : codes0)[((size_t)g * N + n) * KG + k];
      dst[u] = v;
    } else {
      uint32_t v = 0;
#pragma unroll
      for (int i = 0; i < FRAGS; ++i) {
        const int n = unit_feature<PAIR>(cu, i, row);
        uint32_t s = 127u;
        if (n < N && k < KG) s = (PAIR && (i & 1) ? scales1 : scales0)[((size_t)g * N + n) * KG + k];
        v |= s << (8 * i);
      }
      dst_scales[u - total] = v;
    }
  }
}

inline int column_units(const PackedMatrix& m, int which) { return (which & 1) == 0 ? (m.N + 31) / 32 : (m.N + 63) / 64; }
inline size_t group_words(const PackedMatrix& m, int which) { return (size_t)column_units(m, which) * rows_tiles(m.K) * 64; }
inline size_t group_units(const PackedMatrix& m, int which) { return group_words(m, which) * FRAGS; }
inline int scale_bytes(int K) { return rows_tiles(K) * 4; }   // of a row of K values

}  // namespace

size_t fmoe_rows8_bytes(const fmoe_ctx* ctx, int which) {
  const PackedMatrix m = packed_matrix(ctx->cfg, which);
  return (size_t)m.groups * (group_units(m, which) * 16 + group_words(m, which) * 4);
}

int launch_pack_rows8(fmoe_ctx* ctx, const fmoe_quant_tensor* const* w, hipStream_t stream) {
  for (int which = 0; which < 4; ++which) {
    const PackedMatrix m = packed_matrix(ctx->cfg, which);
    if (m.groups == 0) continue;
    const bool pair = (which & 1) == 0;
    const fmoe_quant_tensor* a = w[which == 0 ? 0 : which == 1 ? 2 : which == 2 ? 3 : 5];
    const fmoe_quant_tensor* b = pair ? w[which == 0 ? 1 : 4] : nullptr;
    char* const base = static_cast<char*>(ctx->pr[which]);
    const size_t blocks = (size_t)m.groups * (group_units(m, which) + group_words(m, which)) / 256 + 1;
    const dim3 grid((unsigned)(blocks < 65536 ? blocks : 65536)), block(256);
#define FMOE_PACK(PAIR)                                                                                                 \
  hipLaunchKernelGGL(pack_rows8_kernel<PAIR>, grid, block, 0, stream, static_cast<const u32x4_t*>(a->codes), a->scales, \
                     PAIR ? static_cast<const u32x4_t*>(b->codes) : nullptr, PAIR ? b->scales : nullptr,                \
                     reinterpret_cast<u32x4_t*>(base),                                                                  \
                     reinterpret_cast<uint32_t*>(base + (size_t)m.groups * group_units(m, which) * 16), m.groups, m.N, m.K,  \
                     column_units(m, which))
    if (pair) FMOE_PACK(true);
    else FMOE_PACK(false);
#undef FMOE_PACK
  }
  FMOE_HIP_CHECK(hipGetLastError());
  return FMOE_OK;
}

int launch_expert_ffn_rows8(const fmoe_ctx* ctx, const uint8_t* codes, const uint8_t* scales, const int32_t* kept_idx, int n_cap,
                            const int32_t* n_dev, const int32_t* expert_offsets, const int32_t* perm_src, void* y, void* y_shared,
                            void* ws, const fmoe_ws_layout& L, hipStream_t stream) {
  const fmoe_config& c = ctx->cfg;
  const int d = c.d_model, E = c.n_experts, F = c.d_ffn, Fs = c.d_ffn_shared, Ft = c.n_shared * Fs;
  const int row_cap = n_cap * ctx->kmax;
  if (n_cap == 0 || (row_cap == 0 && Ft == 0)) return FMOE_OK;
  char* const base = static_cast<char*>(ws);
  auto problem = [&](int which) {
    const PackedMatrix m = packed_matrix(c, which);
    RowsProblem q{};
    if (m.groups == 0) return q;
    const char* packed = static_cast<const char*>(ctx->pr[which]);
    q.Bp = reinterpret_cast<const u32x4_t*>(packed);
    q.Sp = reinterpret_cast<const uint32_t*>(packed + (size_t)m.groups * group_units(m, which) * 16);
    q.group_stride = (long long)group_units(m, which);
    q.scale_stride = (long long)group_words(m, which);
    q.units = column_units(m, which); q.N = m.N; q.K = m.K;
    return q;
  };
  // hidden rows: codes, then scale bytes, in the workspace's room for bf16 ones
  uint8_t* const h = reinterpret_cast<uint8_t*>(base + L.h);
  uint8_t* const h_shared = reinterpret_cast<uint8_t*>(base + L.h_shared);
  uint8_t* const hs = h + (size_t)row_cap * F;
  uint8_t* const hs_shared = h_shared + (size_t)n_cap * Ft;
  const int sF = scale_bytes(F), sFs = Ft > 0 ? scale_bytes(Fs) : 0;
  RowsArgs g1{}, g2{};
  g1.p0 = problem(0); g1.p1 = problem(2); g2.p0 = problem(1); g2.p1 = problem(3);
  {
    RowsProblem &p = g1.p0, &q = g1.p1;
    p.A = q.A = codes; p.lda = q.lda = (uint32_t)d;
    p.As = q.As = scales; p.ldas = q.ldas = (uint32_t)scale_bytes(d);
    p.map1 = perm_src; p.map1_limit = n_cap;
    p.map2 = q.map2 = kept_idx;
    p.H = h; p.Hs = hs; p.ldh = (uint32_t)F; p.ldhs = (uint32_t)sF; p.expert_groups = F / 32;
    q.H = h_shared; q.Hs = hs_shared; q.ldh = (uint32_t)Ft; q.ldhs = (uint32_t)(c.n_shared * sFs); q.expert_groups = Fs / 32;
  }
  {
    RowsProblem &p = g2.p0, &q = g2.p1;
    p.A = h; p.As = hs; p.lda = (uint32_t)F; p.ldas = (uint32_t)sF;
    p.C = static_cast<bf16_t*>(y); p.ldc = d;
    q.A = h_shared; q.As = hs_shared; q.lda = (uint32_t)(Ft > 0 ? Ft : 1); q.ldas = (uint32_t)(c.n_shared * sFs);
    q.a_group_off = Fs; q.as_group_off = sFs;
    q.C = static_cast<bf16_t*>(y_shared); q.ldc = d; q.c_group_off = (long long)n_cap * d;
  }
  // Tiles of 128 rows from so many rows an expert on, if those are items enough (tiles that the call can have times items of the narrower
  // product).  us, tiles of 32 / 128, gate/up and down with the launches: 1280, 64 of 896 20 rows an expert 32 / 31, 75 rows 50 / 43;
  // 2048, 64 of 1408 94 rows 121 / 91, 192 rows 195 / 134; 512, 256 of 512 125 rows 75 / 71; few items: 4096, 8 of 1536 150 rows
  // (204) 50 / 47, 375 rows (376) 103 / 74; 1280, 16 of 896 100 rows (140) 25 / 29, 400 rows (330) 51 / 43; 512, 64 of 512
  // 150 rows (278) 31 / 31.  (Tiles of 64 between: at best 3 % from 9 to 75 rows.)
  const long long units1 = (g1.p0.units + 3) / 4, units2 = (g2.p0.units + 3) / 4;
  const bool many = ctx->ffn_shape ? ctx->ffn_shape == 2
                                   : row_cap >= 64 * E && (E + row_cap / MANY_ROWS) * (units1 < units2 ? units1 : units2) >= 300;
  auto launch = [&](auto swiglu, RowsArgs a) {
    constexpr bool S = decltype(swiglu)::value;
    a.expert_offsets = expert_offsets; a.n_dev = n_dev;
    a.E = E; a.n_cap = n_cap; a.row_cap = row_cap;
    static_assert(FEW_ROWS == 1 << 5 && MANY_ROWS == 1 << 7, "rows of a tile");
    a.log2_bm = many ? 7 : 5;
    a.cols = (a.p0.units + 3) / 4;   // items of four column units
    if (Ft > 0) {
      a.shared_groups = S ? 1 : c.n_shared;
      a.shared_cols = (a.p1.units + 3) / 4;
    }
    const long long tiles = (row_cap < E ? row_cap : E) + (row_cap >> a.log2_bm);   // that the routed experts can have
    const long long shared_tiles = ((long long)n_cap + (1 << a.log2_bm) - 1) >> a.log2_bm;
    const long long eighths = (tiles * a.cols + 7) / 8 + (shared_tiles * a.shared_cols * a.shared_groups + 7) / 8;
    const dim3 grid((unsigned)(eighths * 8)), block(256);
    if (many) hipLaunchKernelGGL(ffn_rows8_many_kernel<S>, grid, block, 0, stream, a);
    else hipLaunchKernelGGL(ffn_rows8_few_kernel<S>, grid, block, 0, stream, a);
  };
  {
    fmoe_prof_scope prof(ctx, many ? SLOT_GEMM1_DENSE : SLOT_GEMM1, stream);
    launch(std::true_type{}, g1);
  }
  {
    fmoe_prof_scope prof(ctx, many ? SLOT_GEMM2_DENSE : SLOT_GEMM2, stream);
    launch(std::false_type{}, g2);
  }
  FMOE_HIP_CHECK(hipGetLastError());
  return FMOE_OK;
}
