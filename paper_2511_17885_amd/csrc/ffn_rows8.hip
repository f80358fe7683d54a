// The expert FFNs of Eq.4 on rows in 8 bits (e4m3, a power of two per 32 neighbours: rows8_dev.h) and weights in 4 bits
// (quant.hip), also the hidden rows h = silu(gate) * up between the two products, which are rounded to 8 bits on their way.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 takes both formats as they are, and the two scales of every 32 products: nothing is converted.
// It does in a step of 128 k what the bf16 instruction does in four of 32, in half the time.  Lane l has of a row (l % 16)
// the 16-byte pieces l / 16 and l / 16 + 4 of a k tile of 128, of a column the 32 codes from 32 (l / 16) on; its scale operands
// have in one of their four bytes, which the instruction names, the power of two of the l / 16-th 32 of the row and the column.
// The instruction cuts the products of eight neighbouring k at 2^-13 of the largest power of two among them and adds the eights up in
// fp32 (found on the card): nothing is lost but of products 2^8 and more below a neighbour's, and less than the rounding of the
// rows to 8 bits has taken from them.
//
// Packing (fmoe_set_weights_quant_rows): of a column block (16 features, gate and up; or 32 output features), a k tile and a fragment
// (gate / up, or features 0..15 / 16..31) lane l has one 16-byte unit, all units in one linear stream; of two k tiles the four
// scale bytes of its column are one word.
//
// A workgroup has a tile of rows and, per wavefront, one or two column blocks.  As in ffn.hip: rows global -> LDS directly, in a
// ring of four k tiles (128 bytes a row, pieces exchanged so that operand reads meet no bank twice); weights into registers,
// as many tiles ahead; a barrier per k tile.  Work items are found from the experts' offsets (quant_items.h).

#include "ffn_dev.h"
#include "quant_items.h"
#include "rows8_dev.h"

namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));

#include "rows8_regs.inc"   // rows_acc<IDX>

constexpr int RBK = 128;       // k per tile
constexpr int RSTAGES = 4;     // ring of k tiles, of rows and of weights
constexpr int RAHEAD = RSTAGES - 1;

struct RowsProblem {
  const uint8_t *A, *As;       // rows [*, lda] bytes and their scale bytes [*, ldas]
  uint32_t lda, ldas;
  const int32_t *map1, *map2;  // row -> index (perm_src) -> token (kept_idx), or null
  int map1_limit;
  const u32x4_t* Bp;
  const uint32_t* Sp;
  long long group_stride, scale_stride;   // units and words between groups
  int nbw, N, K;
  uint8_t *H, *Hs;             // gate/up: the hidden rows
  uint32_t ldh, ldhs;
  int expert_cols;             // columns of one expert in H (shared experts stand side by side)
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
__host__ __device__ inline int rows_pairs(int K) { return (rows_tiles(K) + 1) / 2; }

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
template <int OPB>
__device__ __forceinline__ f32x4_t mfma_rows(i32x8_t a, uint32_t sa, u32x4_t b, uint32_t sb, f32x4_t c) {
  typedef int i32x4_t __attribute__((ext_vector_type(4)));
  const i32x4_t b4 = __builtin_bit_cast(i32x4_t, b);
  const i32x8_t b8 = __builtin_shufflevector(b4, b4, 0, 1, 2, 3, -1, -1, -1, -1);   // 4-bit operands have four registers
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b8, c, 0, 4, 0, (int)sa, OPB, (int)sb);
}

// Hidden rows of a tile: silu(gate) * up, 32 columns a group, through LDS (the ring, free by now), a band of 32 rows at a time.
template <int NAB, int NCB, typename ACC>
__device__ __forceinline__ void store_hidden(const RowsProblem& P, const fmoe_tile& tile, int col0, int cols, ACC acc, char* smem) {
  constexpr int BC = 64 * NCB, CS = BC + 4;
  float* const buf = reinterpret_cast<float*>(smem);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  static_for<0, NAB>([&](auto bandc) {
    constexpr int band = decltype(bandc)::value;
    __syncthreads();   // every wavefront is done with what was there
    static_for<0, 2>([&](auto hc) {
      static_for<0, NCB>([&](auto jc) {
        constexpr int rb = 2 * band + decltype(hc)::value, j = decltype(jc)::value;
        const f32x4_t g = acc(jc, std::integral_constant<int, rb>{}, std::integral_constant<int, 0>{});
        const f32x4_t u = acc(jc, std::integral_constant<int, rb>{}, std::integral_constant<int, 1>{});
#pragma unroll
        for (int v = 0; v < 4; ++v)
          buf[(decltype(hc)::value * 16 + 4 * (lane >> 4) + v) * CS + j * 64 + wave * 16 + (lane & 15)] = silu_mul_bf16(g[v], u[v]);
      });
    });
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NCB; ++i) {
      const int unit = tid + 256 * i, r = unit / (BC / 8), cu = unit % (BC / 8);
      const int row = band * 32 + r, col = col0 + cu * 8;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = buf[r * CS + cu * 8 + e];
      uint32_t scale;
      const uint2 c = rows8::quantize(v, scale);
      if (row < tile.rows && cu * 8 < cols && col < P.N) {   // groups are whole: the same for four lanes
        const size_t at = (size_t)(tile.row0 + row);
        *reinterpret_cast<uint2*>(P.H + at * P.ldh + col) = c;
        if ((cu & 3) == 0) {
          const int expert = col / P.expert_cols, g = (col - expert * P.expert_cols) >> 5, last = (P.expert_cols >> 5) - 1;
          uint8_t* const s = P.Hs + at * P.ldhs + expert * ((P.expert_cols + 127) / 128 * 4) + g;
          s[0] = (uint8_t)scale;
          if (g == last)
            for (int k = g + 1; k & 3; ++k) s[k - g] = 127;   // the word's unused bytes
        }
      }
    }
  });
}

// One work item: NAB live bands of 32 rows, LDS stages of ROWS, NCB column tiles of 64 (gate/up) or 128 columns from ct0 on.
// HALF: of the only band the first 16 rows.
template <bool SWIGLU, int NAB, int NCB, int ROWS, bool HALF = false>
__device__ __forceinline__ void rows_tile(const RowsProblem& P, const fmoe_tile& tile, int group, int ct0, int ct_limit, char* smem) {
  static_assert(32 * NAB <= ROWS, "the rows fit in a stage");
  constexpr int NRB = HALF ? 1 : 2 * NAB;
  constexpr int SROWS = ROWS > 64 ? ROWS : 64;                  // scale words a stage
  constexpr int PER_TILE = NAB + 1 + 2 * NCB;                   // loads of a k tile (without those of weight scales)
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int K = P.K, NT = rows_tiles(K), NP = rows_pairs(K);
  const int col_tiles = (P.nbw + 3) / 4;
  char* const rows_lds = smem;
  char* const scales_lds = smem + RSTAGES * ROWS * RBK;

  const __amdgpu_buffer_rsrc_t b_rsrc = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<u32x4_t*>(P.Bp) + (size_t)group * P.group_stride, 0, 0xffffffff, 0x00020000);
  const __amdgpu_buffer_rsrc_t s_rsrc = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint32_t*>(P.Sp) + (size_t)group * P.scale_stride, 0, 0xffffffff, 0x00020000);
  const __amdgpu_buffer_rsrc_t a_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(P.A), 0, 0xffffffff, 0x00020000);
  const __amdgpu_buffer_rsrc_t as_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(P.As), 0, 0xffffffff, 0x00020000);
  uint32_t bbase[NCB], sbase[NCB];   // scalar
#pragma unroll
  for (int j = 0; j < NCB; ++j) {    // column tiles past the packing: the last one again, never stored
    const uint32_t cb = (uint32_t)(ct0 + j < col_tiles ? ct0 + j : col_tiles - 1) * 4u + (uint32_t)wave;
    bbase[j] = cb * (uint32_t)NT * 2048u;
    sbase[j] = cb * (uint32_t)NP * 256u;
  }
  const uint32_t lane16 = (uint32_t)lane * 16u, lane4 = (uint32_t)lane * 4u;

  u32x4_t breg[RSTAGES][NCB][2];
  uint32_t sreg[2][NCB];             // of the k tiles' pair 2i and 2i + 1
  auto load_b = [&](int slot, int t, int j, int f) {
    breg[slot][j][f] = __builtin_amdgcn_raw_buffer_load_b128(
        b_rsrc, lane16, bbase[j] + (uint32_t)(t < NT ? t : NT - 1) * 2048u + (uint32_t)f * 1024u, 0);
  };
  auto load_s = [&](int slot, int pair, int j) {
    sreg[slot][j] = __builtin_amdgcn_raw_buffer_load_b32(s_rsrc, lane4, sbase[j] + (uint32_t)(pair < NP ? pair : NP - 1) * 256u, 0);
  };
  // Rows this lane fetches: 32 it + 8 wave + lane / 8 of the tile; scale words of row 64 (wave % 2) + lane (or lane % 64 where the
  // stage has 64: the wavefronts then fetch the same).  Past the tile its last row.
  const uint32_t most = 0xffffffffu / P.lda - 1u;
  const int sr = (ROWS > 64 ? 64 * (wave & 1) : 0) + lane;
  int src[NAB + 1];
#pragma unroll
  for (int it = 0; it <= NAB; ++it) {
    const int r = it < NAB ? 32 * it + 8 * wave + (lane >> 3) : sr;
    src[it] = tile.row0 + (r < tile.rows ? r : tile.rows - 1);
    if (P.map1) src[it] = P.map1[src[it]];
  }
  order_loads();
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < NCB; ++j) load_s(i, i, j);
#pragma unroll
  for (int t = 0; t < RAHEAD; ++t)
#pragma unroll
    for (int j = 0; j < NCB; ++j) {
      load_b(t, t, j, 0);
      load_b(t, t, j, 1);
    }
  order_loads();
  uint32_t a_src[NAB], a_last[NAB], as_src;   // of the lane's piece in k tile 0, and in the last one less its start
  const int piece = ((lane & 7) ^ ((4 * wave + (lane >> 4)) & 7)) * 16;
  const int k_last = (NT - 1) * RBK, piece_last = k_last + piece < K ? piece : K - 16 - k_last;   // past K the row's end again
#pragma unroll
  for (int it = 0; it <= NAB; ++it) {
    int s = src[it];
    if (P.map1 && P.map1_limit > 0) s = s < 0 ? 0 : (s >= P.map1_limit ? P.map1_limit - 1 : s);
    if (P.map2) s = P.map2[s];
    const uint32_t at = (uint32_t)s < most ? (uint32_t)s : most;
    if (it < NAB) {
      a_last[it] = at * P.lda + (uint32_t)piece_last;
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
  for (int t = 0; t < RAHEAD; ++t) {
#pragma unroll
    for (int it = 0; it < NAB; ++it) load_a(t, t, it);
    load_as(t, t);
    order_loads();
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)FMOE_LPTR(rows_lds), lds1 = (uint32_t)(uintptr_t)FMOE_LPTR(scales_lds);
  const uint32_t frag_row = lds0 + (uint32_t)(lane & 15) * RBK;
  const uint32_t frag_a0 = frag_row + (uint32_t)(((lane >> 4)) ^ ((lane & 15) >> 1)) * 16;
  const uint32_t frag_a1 = frag_row + (uint32_t)(((lane >> 4) + 4) ^ ((lane & 15) >> 1)) * 16;
  const uint32_t frag_s = lds1 + (uint32_t)(lane & 15) * 4 + (uint32_t)(lane >> 4);

  // Accumulators: the compiler's with one column tile, hand-placed ones with two (number (j*NRB + rb)*2 + f), which it would
  // put in part into scratch memory
  constexpr bool NAMED = NCB == 2;
  f32x4_t acc[NCB][NAMED ? 1 : NRB][2];
  if constexpr (NAMED) {
    dense_claim_acc();
  } else {
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) acc[0][rb][0] = acc[0][rb][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  // k tile t, U = t % RSTAGES: products, and the loads of tile t + RAHEAD; of the LAST tiles, fewer than RSTAGES, products only
  u32x4_t fa[2][2];
  uint32_t fs[2];
  auto ktile = [&](auto uc, auto last, int t) {
    constexpr int U = decltype(uc)::value;
    constexpr bool LAST = decltype(last)::value;
    // loads newer than this tile's rows, see ffn_quant.hip
    constexpr int LATER = U < RAHEAD ? RAHEAD - 1 - U : 0;
    if constexpr (LAST) {
      if (t < RAHEAD) FMOE_WAIT_VM(LATER * (NAB + 1));   // uniform
      else FMOE_WAIT_VM(LATER * PER_TILE);
    } else {
      if (t < RAHEAD) FMOE_WAIT_VM(LATER * (NAB + 1) + U * PER_TILE);
      else FMOE_WAIT_VM((RAHEAD - 1) * PER_TILE);
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
          if (i < NAB) load_a((U + RAHEAD) % RSTAGES, t + RAHEAD, i);
          else if (i == NAB) load_as((U + RAHEAD) % RSTAGES, t + RAHEAD);
          else load_b((U + RAHEAD) % RSTAGES, t + RAHEAD, (i - NAB - 1) >> 1, (i - NAB - 1) & 1);
        }
      }
      __builtin_amdgcn_sched_barrier(0);   // the next operand is on its way behind the products
      static_for<0, NCB>([&](auto jc) {
        constexpr int j = decltype(jc)::value;
        const i32x8_t a = joined(fa[cur][0], fa[cur][1]);
        if constexpr (NAMED) {
          rows_acc<(j * NRB + rb) * 2>::template add<2 * (U & 1)>(a, fs[cur], breg[U][j][0], sreg[U / 2][j]);
          rows_acc<(j * NRB + rb) * 2 + 1>::template add<2 * (U & 1) + 1>(a, fs[cur], breg[U][j][1], sreg[U / 2][j]);
        } else {
          acc[j][rb][0] = mfma_rows<2 * (U & 1)>(a, fs[cur], breg[U][j][0], sreg[U / 2][j], acc[j][rb][0]);
          acc[j][rb][1] = mfma_rows<2 * (U & 1) + 1>(a, fs[cur], breg[U][j][1], sreg[U / 2][j], acc[j][rb][1]);
        }
      });
    });
    if constexpr (!LAST && (U & 1) == 1) {   // the pair is done: the next but one takes its place
#pragma unroll
      for (int j = 0; j < NCB; ++j) load_s(U / 2, t / 2 + 2, j);
    }
  };
  int t0 = 0;
  for (; t0 + RSTAGES <= NT; t0 += RSTAGES)
    static_for<0, RSTAGES>([&](auto uc) { ktile(uc, std::false_type{}, t0 + decltype(uc)::value); });
  static_for<0, RSTAGES - 1>([&](auto uc) {
    if (t0 + decltype(uc)::value < NT) ktile(uc, std::true_type{}, t0 + decltype(uc)::value);   // uniform
  });
  FMOE_WAIT_VM(0);   // the loads issued past the end have landed before the ring is reused
  // the last matrix instructions have retired before hand-placed accumulators are read, see ffn.hip
  if constexpr (NAMED) asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 7" ::: "memory");
  auto result = [&](auto jc, auto rbc, auto fc) {
    constexpr int rb = decltype(rbc)::value;
    if constexpr (rb >= NRB) return f32x4_t{0.f, 0.f, 0.f, 0.f};   // rows that are not stored
    else if constexpr (NAMED) return read_acc<(decltype(jc)::value * NRB + rb) * 2 + decltype(fc)::value>();
    else return acc[decltype(jc)::value][rb][decltype(fc)::value];
  };
  if constexpr (SWIGLU) {
    store_hidden<NAB, NCB>(P, tile, ct0 * 64, (ct_limit - ct0) * 64, result, smem);
  } else {
    StreamProblem S{};
    S.C = P.C;
    S.ldc = P.ldc;
    S.N = P.N;
    static_for<0, NCB>([&](auto jc) {
      if (ct0 + decltype(jc)::value < ct_limit)   // uniform
        store_tile<false, NAB, RSTAGES>(S, tile, ct0 + decltype(jc)::value, [&](auto rbc, auto fc) { return result(jc, rbc, fc); },
                                        reinterpret_cast<bf16_t*>(smem));
    });
  }
}

// field by field, so that the descriptors stay in scalar registers
__device__ __forceinline__ RowsProblem rows_problem(const RowsArgs& a, const QuantItem& it) {
  RowsProblem Q;
#define FMOE_SEL(f) Q.f = it.shared ? a.p1.f : a.p0.f
  FMOE_SEL(A); FMOE_SEL(As); FMOE_SEL(lda); FMOE_SEL(ldas); FMOE_SEL(map1); FMOE_SEL(map2); FMOE_SEL(map1_limit);
  FMOE_SEL(Bp); FMOE_SEL(Sp); FMOE_SEL(group_stride); FMOE_SEL(scale_stride); FMOE_SEL(nbw); FMOE_SEL(N); FMOE_SEL(K);
  FMOE_SEL(H); FMOE_SEL(Hs); FMOE_SEL(ldh); FMOE_SEL(ldhs); FMOE_SEL(expert_cols); FMOE_SEL(C); FMOE_SEL(ldc);
  FMOE_SEL(a_group_off); FMOE_SEL(as_group_off); FMOE_SEL(c_group_off);
#undef FMOE_SEL
  if (it.shared) {   // a shared expert's part of the hidden rows, its output (down)
    Q.A += (size_t)it.group * Q.a_group_off;
    Q.As += (size_t)it.group * Q.as_group_off;
    Q.C += (size_t)it.group * Q.c_group_off;
  }
  return Q;
}

constexpr int FEW_ROWS = 32, SOME_ROWS = 64, MANY_ROWS = 128;
constexpr int lds_bytes(int rows) { return RSTAGES * (rows * RBK + (rows > 64 ? rows : 64) * 4); }

template <bool SWIGLU>
__global__ __launch_bounds__(256, 4) void ffn_rows8_few_kernel(RowsArgs a) {
  __shared__ __align__(16) char smem[lds_bytes(FEW_ROWS)];
  const QuantItem it = find_tile(a, (int)blockIdx.x);
  if (it.group < 0) return;
  const RowsProblem P = rows_problem(a, it);
  fmoe_tile tile{};
  tile.row0 = it.row0;
  tile.rows = it.rows;
  if (it.rows <= 16) rows_tile<SWIGLU, 1, 1, FEW_ROWS, true>(P, tile, it.group, it.unit, it.unit + 1, smem);   // uniform
  else rows_tile<SWIGLU, 1, 1, FEW_ROWS>(P, tile, it.group, it.unit, it.unit + 1, smem);
}
template <bool SWIGLU>
__global__ __launch_bounds__(256, 4) void ffn_rows8_some_kernel(RowsArgs a) {
  __shared__ __align__(16) char smem[lds_bytes(SOME_ROWS)];
  const QuantItem it = find_tile(a, (int)blockIdx.x);
  if (it.group < 0) return;
  const RowsProblem P = rows_problem(a, it);
  fmoe_tile tile{};
  tile.row0 = it.row0;
  tile.rows = it.rows;
  if (it.rows <= 32) rows_tile<SWIGLU, 1, 1, SOME_ROWS>(P, tile, it.group, it.unit, it.unit + 1, smem);
  else rows_tile<SWIGLU, 2, 1, SOME_ROWS>(P, tile, it.group, it.unit, it.unit + 1, smem);
}
// (The build looks at the registers of a kernel of this name.)
template <bool SWIGLU>
__global__ __launch_bounds__(256, 2) void ffn_rows8_many_kernel(RowsArgs a) {
  __shared__ __align__(16) char smem[lds_bytes(MANY_ROWS)];
  const QuantItem it = find_tile(a, (int)blockIdx.x);
  if (it.group < 0) return;
  const RowsProblem P = rows_problem(a, it);
  fmoe_tile tile{};
  tile.row0 = it.row0;
  tile.rows = it.rows;
  const int tiles = (P.nbw + 3) / 4, ct0 = 2 * it.unit, limit = ct0 + 2 < tiles ? ct0 + 2 : tiles;
  switch ((tile.rows + 31) >> 5) {   // live 32-row bands of the tile, uniform
    case 1: rows_tile<SWIGLU, 1, 2, MANY_ROWS>(P, tile, it.group, ct0, limit, smem); break;
    case 2: rows_tile<SWIGLU, 2, 2, MANY_ROWS>(P, tile, it.group, ct0, limit, smem); break;
    case 3: rows_tile<SWIGLU, 3, 2, MANY_ROWS>(P, tile, it.group, ct0, limit, smem); break;
    default: rows_tile<SWIGLU, 4, 2, MANY_ROWS>(P, tile, it.group, ct0, limit, smem); break;
  }
}

// Source rows [group][n][k]: codes two to a byte, scales one byte per 32 k.  PAIR: gate and up (fragments 0 and 1), else
// fragment f = features 16f..16f+15 of the column block.  Past N and K the codes are 0 and the scales 1.
template <bool PAIR>
__global__ __launch_bounds__(256) void pack_rows8_kernel(const u32x4_t* __restrict__ codes0, const uint8_t* __restrict__ scales0,
                                                         const u32x4_t* __restrict__ codes1, const uint8_t* __restrict__ scales1,
                                                         u32x4_t* __restrict__ dst, uint32_t* __restrict__ dst_scales, int G,
                                                         int N, int K, int nb) {
  const int NT = rows_tiles(K), NP = rows_pairs(K), KG = K / FMOE_QUANT_GROUP;
  const size_t total = (size_t)G * nb * NT * 128, total_scales = (size_t)G * nb * NP * 64;
  for (size_t u = (size_t)blockIdx.x * blockDim.x + threadIdx.x; u < total + total_scales; u += (size_t)gridDim.x * blockDim.x) {
    const bool scales = u >= total;
    size_t q = scales ? u - total : u;
    const int lane = (int)(q & 63), col = lane & 15, kg = lane >> 4;
    q >>= 6;
    if (!scales) {
      const int f = (int)(q & 1);
      q >>= 1;
      const int kt = (int)(q % NT);
      q /= NT;
      const int b = (int)(q % nb), g = (int)(q / nb);
      const int n = PAIR ? b * 16 + col : b * 32 + f * 16 + col, k = kt * 4 + kg;   // 32 codes: a 16-byte unit of the source
      u32x4_t v = {0u, 0u, 0u, 0u};
      if (n < N && k < KG) v = (PAIR && f ? codes1 : codes0)[((size_t)g * N + n) * KG + k];
      dst[u] = v;
    } else {
      const int pair = (int)(q % NP);
      q /= NP;
      const int b = (int)(q % nb), g = (int)(q / nb);
      uint32_t v = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int f = i & 1, n = PAIR ? b * 16 + col : b * 32 + f * 16 + col, k = (2 * pair + (i >> 1)) * 4 + kg;
        uint32_t s = 127u;
        if (n < N && k < KG) s = (PAIR && f ? scales1 : scales0)[((size_t)g * N + n) * KG + k];
        v |= s << (8 * i);
      }
      dst_scales[u - total] = v;
    }
  }
}

inline int padded_blocks(const PackedMatrix& m) { return (m.nbw + 3) / 4 * 4; }
inline size_t group_units(const PackedMatrix& m) { return (size_t)padded_blocks(m) * rows_tiles(m.K) * 128; }
inline size_t group_words(const PackedMatrix& m) { return (size_t)padded_blocks(m) * rows_pairs(m.K) * 64; }
inline int scale_bytes(int K) { return rows_tiles(K) * 4; }   // of a row of K values

}  // namespace

size_t fmoe_rows8_bytes(const fmoe_ctx* ctx, int which) {
  const PackedMatrix m = packed_matrix(ctx->cfg, which);
  return (size_t)m.groups * (group_units(m) * 16 + group_words(m) * 4);
}

int launch_pack_rows8(fmoe_ctx* ctx, const fmoe_quant_tensor* const* w, hipStream_t stream) {
  for (int which = 0; which < 4; ++which) {
    const PackedMatrix m = packed_matrix(ctx->cfg, which);
    if (m.groups == 0) continue;
    const bool pair = (which & 1) == 0;
    const fmoe_quant_tensor* a = w[which == 0 ? 0 : which == 1 ? 2 : which == 2 ? 3 : 5];
    const fmoe_quant_tensor* b = pair ? w[which == 0 ? 1 : 4] : nullptr;
    char* const base = static_cast<char*>(ctx->pr[which]);
    const size_t blocks = (size_t)m.groups * (group_units(m) + group_words(m)) / 256 + 1;
    const dim3 grid((unsigned)(blocks < 65536 ? blocks : 65536)), block(256);
#define FMOE_PACK(PAIR)                                                                                                 \
  hipLaunchKernelGGL(pack_rows8_kernel<PAIR>, grid, block, 0, stream, static_cast<const u32x4_t*>(a->codes), a->scales, \
                     PAIR ? static_cast<const u32x4_t*>(b->codes) : nullptr, PAIR ? b->scales : nullptr,                \
                     reinterpret_cast<u32x4_t*>(base), reinterpret_cast<uint32_t*>(base + (size_t)m.groups * group_units(m) * 16), \
                     m.groups, m.N, m.K, padded_blocks(m))
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
    q.Sp = reinterpret_cast<const uint32_t*>(packed + (size_t)m.groups * group_units(m) * 16);
    q.group_stride = (long long)group_units(m);
    q.scale_stride = (long long)group_words(m);
    q.nbw = m.nbw; q.N = m.N; q.K = m.K;
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
    p.H = h; p.Hs = hs; p.ldh = (uint32_t)F; p.ldhs = (uint32_t)sF; p.expert_cols = F;
    q.H = h_shared; q.Hs = hs_shared; q.ldh = (uint32_t)Ft; q.ldhs = (uint32_t)(c.n_shared * sFs); q.expert_cols = Fs;
  }
  {
    RowsProblem &p = g2.p0, &q = g2.p1;
    p.A = h; p.As = hs; p.lda = (uint32_t)F; p.ldas = (uint32_t)sF;
    p.C = static_cast<bf16_t*>(y); p.ldc = d;
    q.A = h_shared; q.As = hs_shared; q.lda = (uint32_t)(Ft > 0 ? Ft : 1); q.ldas = (uint32_t)(c.n_shared * sFs);
    q.a_group_off = Fs; q.as_group_off = sFs;
    q.C = static_cast<bf16_t*>(y_shared); q.ldc = d; q.c_group_off = (long long)n_cap * d;
  }
  const long long per_expert = row_cap / E;
  const int form = ctx->ffn_shape ? 2 * (ctx->ffn_shape - 1) : per_expert < 16 ? 0 : per_expert < 150 ? 1 : 2;
  auto launch = [&](auto swiglu, RowsArgs a) {
    constexpr bool S = decltype(swiglu)::value;
    a.expert_offsets = expert_offsets; a.n_dev = n_dev;
    a.E = E; a.n_cap = n_cap; a.row_cap = row_cap;
    a.log2_bm = 5 + form;
    const int per_unit = form == 2 ? 8 : 4;   // column blocks of a unit
    a.cols = (a.p0.nbw + per_unit - 1) / per_unit;
    if (Ft > 0) {
      a.shared_groups = S ? 1 : c.n_shared;
      a.shared_cols = (a.p1.nbw + per_unit - 1) / per_unit;
    }
    const long long tiles = (row_cap < E ? row_cap : E) + (row_cap >> a.log2_bm);   // that the routed experts can have
    const long long shared_tiles = ((long long)n_cap + (1 << a.log2_bm) - 1) >> a.log2_bm;
    const long long items = tiles * a.cols + shared_tiles * a.shared_cols * a.shared_groups;
    const dim3 grid((unsigned)((items + 7) / 8 * 8)), block(256);
    if (form == 0) hipLaunchKernelGGL(ffn_rows8_few_kernel<S>, grid, block, 0, stream, a);
    else if (form == 1) hipLaunchKernelGGL(ffn_rows8_some_kernel<S>, grid, block, 0, stream, a);
    else hipLaunchKernelGGL(ffn_rows8_many_kernel<S>, grid, block, 0, stream, a);
  };
  {
    fmoe_prof_scope prof(ctx, form == 2 ? SLOT_GEMM1_DENSE : SLOT_GEMM1, stream);
    launch(std::true_type{}, g1);
  }
  {
    fmoe_prof_scope prof(ctx, form == 2 ? SLOT_GEMM2_DENSE : SLOT_GEMM2, stream);
    launch(std::false_type{}, g2);
  }
  FMOE_HIP_CHECK(hipGetLastError());
  return FMOE_OK;
}
