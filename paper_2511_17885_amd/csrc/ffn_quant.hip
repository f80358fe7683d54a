// The expert FFNs of Eq.4 with weights in 4 bits (quant.hip: +-{0, .5, 1, 1.5, 2, 3, 4, 6} times a power of two per 32
// values along the reduction), activations in bf16.
//
// A weight is a bf16 number exactly, so the products are those of the bf16 kernels: a wavefront turns eight codes into an
// operand of v_mfma_f32_16x16x32_bf16 by four conversion instructions that apply the scale as well, and the matrix
// instruction does the rest, in the same order of k.  A context with 4-bit weights gives the same bits as a bf16 context
// that is given the dequantized ones.  So h = silu(gate) * up is rounded to bf16 on its way to the down product, as there: the
// outputs are 0.0024 of their size from the 64-bit ones where their own rounding makes 0.0017.  Two bf16 parts of h would keep
// it, for twice the matrix instructions of the down product and other bits than a bf16 context.
//
// Packing (fmoe_set_weights_quant, matrix-core operand order as in ffn.hip): of a column block (16 features, gate and up;
// or 32 output features) and a k tile of 64, lane l has one 16-byte unit: word 2s + f = the eight codes of k step s and
// fragment f that the bf16 packing holds as 16 bytes.  The scales of a k tile, the same four of each column, are a word,
// and four k tiles' words are one 16-byte unit per column: 17 bits per four weights in two linear streams.

#include "ffn_dev.h"
#include "quant_items.h"

namespace {

struct QuantProblem {
  StreamProblem s;            // Bp: codes, group_stride in 16-byte units
  const u32x4_t* Sp;          // scales
  long long scale_stride;     // 16-byte units between groups
};

struct QuantArgs {
  QuantProblem p0, p1;        // routed experts; shared group (tile.group >= E)
  int E;
  const fmoe_tile* tiles;
  const int32_t* n_tiles;     // device
  int cols;                   // work items per tile entry in this launch
  int cols_entry;             // column tiles per tile entry
};

__host__ __device__ inline int quant_tiles(int K) { return (K + SBK - 1) / SBK; }
__host__ __device__ inline int quant_scale_tiles(int K) { return (quant_tiles(K) + 3) / 4; }

// One wavefront, one column block, sixteen rows: codes, scales and rows straight into registers in matrix order, no LDS and
// no barrier, for calls of at most THIN_ROWS tokens, where the weights are all there is to move.  Rows past the tile reuse
// its last one, row indices are clamped as in gather_offsets.  Bound: in each of the two launches a chain of latencies (offsets,
// row indices, rows and the first weights), then the weights.  d 2048, 64 experts of 1408 and two shared, one token: 8.0 + 5.6
// us for 36 MB.
constexpr int THIN_ROWS = 16;
constexpr int THIN_SLOTS = 8;    // k tiles (64 wide) of codes, and of rows, in flight

template <bool SWIGLU>
__device__ __forceinline__ void thin_quant_tile(const QuantProblem& Q, int row0, int rows, int group, int cb) {
  constexpr int S = THIN_SLOTS;
  static_assert(S % 4 == 0, "a unit of scales serves four k tiles");
  const StreamProblem& P = Q.s;
  const int lane = threadIdx.x;
  const int K = P.K, N = P.N;
  const int NT = quant_tiles(K), NT4 = quant_scale_tiles(K);
  // The streams' descriptors end with the column block: loads past the last k tile return zeros and fetch nothing (the
  // whole offset is the lanes': a scalar one would be taken off the size first)
  const __amdgpu_buffer_rsrc_t b_rsrc = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<u32x4_t*>(P.Bp) + (size_t)group * P.group_stride + (size_t)cb * NT * 64, 0, NT * 1024, 0x00020000);
  const __amdgpu_buffer_rsrc_t s_rsrc = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<u32x4_t*>(Q.Sp) + (size_t)group * Q.scale_stride + (size_t)cb * NT4 * 16, 0, NT4 * 256, 0x00020000);
  const __amdgpu_buffer_rsrc_t a_rsrc =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(P.A), 0, 0xffffffff, 0x00020000);
  const uint32_t lane16 = (uint32_t)lane * 16u, column16 = (uint32_t)(lane & 15) * 16u;
  const int kq = (lane >> 4) * 8;
  u32x4_t breg[S], sreg[S / 4], areg[S][2];
  auto load_b = [&](int slot, int t) { breg[slot] = __builtin_amdgcn_raw_buffer_load_b128(b_rsrc, lane16 + (uint32_t)t * 1024u, 0, 0); };
  auto load_s = [&](int slot, int t4) {
    sreg[slot] = __builtin_amdgcn_raw_buffer_load_b128(s_rsrc, column16 + (uint32_t)t4 * 256u, 0, 0);
  };
  // byte offsets of the lane's pieces in k tile 0, and in the last one less its start; past the end the last tile again
  uint32_t a_src[2], a_last[2];
  auto load_a = [&](int slot, int t) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
      areg[slot][s] = __builtin_amdgcn_raw_buffer_load_b128(a_rsrc, t < NT - 1 ? a_src[s] : a_last[s],
                                                            (t < NT ? t : NT - 1) * (SBK * 2), 0);
  };
  // the weights do not need the row indices (two dependent loads)
  const uint32_t a_max_row = 0xffffffffu / ((uint32_t)P.lda * 2u) - 1u;
  int src = row0 + ((lane & 15) < rows ? (lane & 15) : rows - 1);
  if (P.map1) src = P.map1[src];
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int t = 0; t < S; ++t) {
    if (t % 4 == 0) load_s(t / 4, t / 4);
    load_b(t, t);
  }
  __builtin_amdgcn_sched_barrier(0);
  if (P.map1 && P.map1_limit > 0) src = src < 0 ? 0 : (src >= P.map1_limit ? P.map1_limit - 1 : src);
  if (P.map2) src = P.map2[src];
  const uint32_t a_row = ((uint32_t)src < a_max_row ? (uint32_t)src : a_max_row) * (uint32_t)P.lda * 2u;
#pragma unroll
  for (int s = 0; s < 2; ++s) {   // k past K re-reads the row's end, where the packed weights are zero
    const int k_last = (NT - 1) * SBK, piece = s * 32 + kq;
    a_src[s] = a_row + (uint32_t)piece * 2u;
    a_last[s] = a_row + (uint32_t)(k_last + piece < K ? piece : K - 8 - k_last) * 2u;
  }
#pragma unroll
  for (int t = 0; t < S; ++t) load_a(t, t);
  __builtin_amdgcn_sched_barrier(0);

  f32x4_t acc[2] = {f32x4_t{0.f, 0.f, 0.f, 0.f}, f32x4_t{0.f, 0.f, 0.f, 0.f}};
  auto multiply = [&](int slot) {
    const uint32_t sc = sreg[slot / 4][slot % 4];
    const bf16x8_t a0 = __builtin_bit_cast(bf16x8_t, areg[slot][0]), a1 = __builtin_bit_cast(bf16x8_t, areg[slot][1]);
    acc[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, __builtin_bit_cast(bf16x8_t, dequantize<0>(breg[slot][0], sc)), acc[0], 0, 0, 0);
    acc[1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a0, __builtin_bit_cast(bf16x8_t, dequantize<1>(breg[slot][1], sc)), acc[1], 0, 0, 0);
    acc[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, __builtin_bit_cast(bf16x8_t, dequantize<2>(breg[slot][2], sc)), acc[0], 0, 0, 0);
    acc[1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a1, __builtin_bit_cast(bf16x8_t, dequantize<3>(breg[slot][3], sc)), acc[1], 0, 0, 0);
  };
  int t0 = 0;
  for (; t0 + S <= NT; t0 += S) {   // no exit inside, so that the waits can count on the rings' order
#pragma unroll
    for (int u = 0; u < S; ++u) {
      multiply(u);
      __builtin_amdgcn_sched_barrier(0);
      load_b(u, t0 + u + S);
      load_a(u, t0 + u + S);
      if (u % 4 == 3) load_s(u / 4, (t0 + S) / 4 + u / 4);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // fewer than S tiles are left, all of their codes and rows on the way
#pragma unroll
  for (int u = 0; u < S - 1; ++u) {
    if (t0 + u >= NT) break;   // uniform
    multiply(u);
  }
  // accumulator register v of lane l: row 4*(l/16) + v, column l%16
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    const int row = 4 * (lane >> 4) + v;
    if (row >= rows) continue;
    bf16_t* crow = P.C + (size_t)(row0 + row) * P.ldc;
    if (SWIGLU) {
      const int col = cb * 16 + (lane & 15);
      if (col < N) crow[col] = f32_to_bf16(silu_mul_bf16(acc[0][v], acc[1][v]));
    } else {
      const int col = cb * 32 + (lane & 15);
      if (col < N) crow[col] = f32_to_bf16(acc[0][v]);
      if (col + 16 < N) crow[col + 16] = f32_to_bf16(acc[1][v]);
    }
  }
}

template <int I, int N, typename C, typename F>
__device__ __forceinline__ void while_for(C&& c, F&& f) {   // static_for that ends at the first i for which c(i) is not true
  if constexpr (I < N) {
    if (c(std::integral_constant<int, I>{})) {
      f(std::integral_constant<int, I>{});
      while_for<I + 1, N>(c, f);
    }
  }
}

// One work item of a workgroup: a tile of rows (NAB live bands of 32, LDS stages of ROWS) times NCB column tiles, column block
// w of each for wavefront w.  Rows go through a ring of LDS stages as in ffn.hip; codes and scales into registers, all as
// many k tiles ahead; a k tile is one barrier.  Every load of the loop is unconditional (past the end the last tile
// again), so the number of loads in flight at a wait is a compile-time constant.  Row blocks are taken two at a time, the next
// pair's operands requested from LDS before the present pair's products.  HALF: of the only band the first 16 rows.
template <bool SWIGLU, int NAB, int NCB, int STAGES, int ROWS, bool HALF = false>
__device__ __forceinline__ void quant_tile(const QuantProblem& Q, const fmoe_tile& tile, int group, int ct0, int ct_limit,
                                           bf16_t* As) {
  static_assert(STAGES == 4 || STAGES == 8, "a unit of scales serves four k tiles");
  static_assert(32 * NAB <= ROWS, "the rows fit in a stage");
  static_assert(!HALF || NAB == 1, "half a band is half of the only one");
  constexpr int NRB = HALF ? 1 : 2 * NAB;
  constexpr int PB = HALF ? 1 : 2;   // row blocks taken together
  constexpr int AHEAD = STAGES - 1, UNITS = STAGES / 4;
  constexpr int PER_TILE = NAB + NCB;
  const StreamProblem& P = Q.s;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int K = P.K;
  const int NT = quant_tiles(K), NT4 = quant_scale_tiles(K);
  const int col_tiles = (P.nbw + 3) / 4;

  const __amdgpu_buffer_rsrc_t b_rsrc = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<u32x4_t*>(P.Bp) + (size_t)group * P.group_stride, 0, 0xffffffff, 0x00020000);
  const __amdgpu_buffer_rsrc_t s_rsrc = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<u32x4_t*>(Q.Sp) + (size_t)group * Q.scale_stride, 0, 0xffffffff, 0x00020000);
  const __amdgpu_buffer_rsrc_t a_rsrc =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(P.A), 0, 0xffffffff, 0x00020000);
  uint32_t bbase[NCB], sbase[NCB];   // scalar
#pragma unroll
  for (int j = 0; j < NCB; ++j) {    // column tiles past the packing: the last one again, never stored
    const uint32_t cb = (uint32_t)(ct0 + j < col_tiles ? ct0 + j : col_tiles - 1) * 4u + (uint32_t)wave;
    bbase[j] = cb * (uint32_t)NT * 1024u;
    sbase[j] = cb * (uint32_t)NT4 * 256u;
  }
  const uint32_t lane16 = (uint32_t)lane * 16u, column16 = (uint32_t)(lane & 15) * 16u;
  const int a_kc = ((lane & 7) ^ ((4 * wave + (lane >> 4)) & 7)) * 8;

  u32x4_t breg[STAGES][NCB], scales[UNITS][NCB], next_scales[NCB];
  uint32_t a_src[NAB], a_last[NAB];   // byte offsets of the lane's pieces in k tile 0, and in the last one less its start
  auto loadB1 = [&](int slot, int t, int j) {
    breg[slot][j] = __builtin_amdgcn_raw_buffer_load_b128(b_rsrc, lane16, bbase[j] + (uint32_t)(t < NT ? t : NT - 1) * 1024u, 0);
  };
  auto loadS1 = [&](int t4, int j) {
    return __builtin_amdgcn_raw_buffer_load_b128(s_rsrc, column16, sbase[j] + (uint32_t)(t4 < NT4 ? t4 : NT4 - 1) * 256u, 0);
  };
  auto loadA1 = [&](int stage, int t, int it) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        a_rsrc, FMOE_LPTR(As + stage * (ROWS * SBK) + (32 * it + 8 * wave) * SBK), 16,
        t < NT - 1 ? a_src[it] : a_last[it], (uint32_t)(t < NT ? t : NT - 1) * (SBK * 2u), 0, 0);
  };
  const uint32_t lds0 = (uint32_t)(uintptr_t)FMOE_LPTR(As);
  const uint32_t frag_row = lds0 + (uint32_t)(lane & 15) * (SBK * 2);
  const uint32_t frag_a0 = frag_row + (uint32_t)(((lane >> 4)) ^ ((lane & 15) >> 1)) * 16;
  const uint32_t frag_a1 = frag_row + (uint32_t)(((lane >> 4) + 4) ^ ((lane & 15) >> 1)) * 16;

  // prologue: weights between the two loads of the row indices, then the first activations
  int src[NAB];
  gather_first<NAB>(P, tile, src);
  order_loads();
#pragma unroll
  for (int q = 0; q < UNITS; ++q)
#pragma unroll
    for (int j = 0; j < NCB; ++j) scales[q][j] = loadS1(q, j);
#pragma unroll
  for (int t = 0; t < AHEAD; ++t)
#pragma unroll
    for (int j = 0; j < NCB; ++j) loadB1(t, t, j);
  order_loads();
  gather_offsets<NAB>(P, src, a_src);
  // k past K re-reads the row's end, where the packed weights are zero
  const int k_last = (NT - 1) * SBK, piece_last = k_last + a_kc < K ? a_kc : K - 8 - k_last;
#pragma unroll
  for (int it = 0; it < NAB; ++it) {
    a_last[it] = a_src[it] + (uint32_t)piece_last * 2u;
    a_src[it] += (uint32_t)a_kc * 2u;
  }
#pragma unroll
  for (int t = 0; t < AHEAD; ++t) {
#pragma unroll
    for (int it = 0; it < NAB; ++it) loadA1(t, t, it);
    order_loads();
  }

  // Accumulators: the compiler's with one column tile, hand-placed ones with two (number (j*NRB + rb)*2 + f), which it would
  // put in part into scratch memory
  constexpr bool NAMED = NCB == 2;
  f32x4_t acc[NAMED ? 1 : NRB][2];
  if constexpr (NAMED) {
    dense_claim_acc();
  } else {
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) acc[rb][0] = acc[rb][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  u32x4_t fa[2][PB];
  u32x4_t fb[NCB][2];
  // k tile t, U = t % STAGES: products, and the loads of tile t + AHEAD; of the LAST tiles, fewer than STAGES, products only,
  // since all of theirs are on the way.  (Loads of theirs would be past the end, and the compiler drops those into registers that
  // nothing reads: the counts below would be too large.)  Scales: with one unit in registers the next one is
  // requested with the unit's first tile; with two a unit's successor but one takes its place behind its last tile.
  auto ktile = [&](auto uc, auto last, int t) {
    constexpr int U = decltype(uc)::value;
    constexpr bool LAST = decltype(last)::value;
    constexpr bool SCALES = UNITS == 1 ? U == 0 : U % 4 == 3;
    constexpr int NL = LAST ? 0 : PER_TILE + (SCALES ? NCB : 0);   // loads this tile issues
    constexpr int unit = (U / 4) % UNITS;
    // Loads newer than this tile's rows: behind the prologue, whose rows come after all its weights, the later rows of it
    // and what the tiles so far have issued; then what the AHEAD - 1 tiles before have issued.  (Loads of scales are counted
    // only where they are sure to be among them.)
    constexpr int LATER = U < AHEAD ? AHEAD - 1 - U : 0;   // tiles requested behind this one, ahead of tile t - U
    if constexpr (LAST) {
      if (t < AHEAD) FMOE_WAIT_VM(LATER * NAB);   // uniform
      else FMOE_WAIT_VM(LATER * PER_TILE);
    } else {
      if (t < AHEAD) FMOE_WAIT_VM(LATER * NAB + U * PER_TILE);
      else FMOE_WAIT_VM((AHEAD - 1) * PER_TILE);
    }
    block_barrier();   // every wavefront's share of the tile is in LDS; all are done with the tile before
    constexpr int off = U * (ROWS * SBK * 2);
    lds_issue_frags_at<PB, off>(frag_a0, fa[0]);
    static_for<0, 2 * NAB>([&](auto pc) {
      constexpr int p = decltype(pc)::value, s = p / NAB, h = p % NAB, cur = p & 1, nxt = cur ^ 1;
      if constexpr (h == 0) {
#pragma unroll
        for (int j = 0; j < NCB; ++j) {
          uint32_t c0 = breg[U][j][2 * s], c1 = breg[U][j][2 * s + 1];
          if constexpr (NAMED) asm volatile("" : "+v"(c0), "+v"(c1));   // not converted earlier: there are no registers for it
          fb[j][0] = dequantize<2 * s>(c0, scales[unit][j][U % 4]);
          fb[j][1] = dequantize<2 * s + 1>(c1, scales[unit][j][U % 4]);
          // a conversion's result must not be read by the very next instruction, and the compiler does not see that the
          // hand-placed matrix instructions do
          if constexpr (NAMED) asm volatile("s_nop 0" : "+v"(fb[j][0]), "+v"(fb[j][1]));
        }
      }
      lds_settle_frags<PB>(fa[cur]);
      if constexpr (h + 1 < NAB) lds_issue_frags_at<PB, off + (h + 1) * 4096>(s ? frag_a1 : frag_a0, fa[nxt]);
      else if constexpr (s == 0) lds_issue_frags_at<PB, off>(frag_a1, fa[nxt]);
#pragma unroll
      for (int i = 0; i < NL; ++i) {   // load i of the tile goes out with pair i * (2 NAB) / NL
        if ((i * 2 * NAB) / NL != p) continue;
        if (i < NAB) loadA1((U + AHEAD) % STAGES, t + AHEAD, i);
        else if (i < PER_TILE) loadB1((U + AHEAD) % STAGES, t + AHEAD, i - NAB);
        else if constexpr (UNITS == 1) next_scales[i - PER_TILE] = loadS1(t / 4 + 1, i - PER_TILE);
        else scales[unit][i - PER_TILE] = loadS1(t / 4 + UNITS, i - PER_TILE);   // (behind the tile's conversions)
      }
      static_for<0, NCB>([&](auto jc) {
        constexpr int j = decltype(jc)::value;
        const bf16x8_t b0 = __builtin_bit_cast(bf16x8_t, fb[j][0]), b1 = __builtin_bit_cast(bf16x8_t, fb[j][1]);
        static_for<0, PB>([&](auto rc) {
          constexpr int rb = PB * h + decltype(rc)::value;
          const bf16x8_t a8 = __builtin_bit_cast(bf16x8_t, fa[cur][decltype(rc)::value]);
          if constexpr (NAMED) {
            mfma_at<(j * NRB + rb) * 2>(a8, b0);
            mfma_at<(j * NRB + rb) * 2 + 1>(a8, b1);
          } else {
            acc[rb][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a8, b0, acc[rb][0], 0, 0, 0);
            acc[rb][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a8, b1, acc[rb][1], 0, 0, 0);
          }
        });
      });
    });
    if constexpr (UNITS == 1 && U == 3 && !LAST) {
#pragma unroll
      for (int j = 0; j < NCB; ++j) scales[0][j] = next_scales[j];
    }
  };
  int t0 = 0;
  for (; t0 + STAGES <= NT; t0 += STAGES)
    static_for<0, STAGES>([&](auto uc) { ktile(uc, std::false_type{}, t0 + decltype(uc)::value); });
  while_for<0, STAGES - 1>([&](auto uc) { return t0 + decltype(uc)::value < NT; },   // uniform
                           [&](auto uc) { ktile(uc, std::true_type{}, t0 + decltype(uc)::value); });
  FMOE_WAIT_VM(0);   // the loads issued past the end have landed before the ring is reused
  // the last matrix instructions have retired before hand-placed accumulators are read, see ffn.hip
  if constexpr (NAMED) asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 7" ::: "memory");
  static_for<0, NCB>([&](auto jc) {
    constexpr int j = decltype(jc)::value;
    if (ct0 + j < ct_limit)   // uniform
      store_tile<SWIGLU, NAB, STAGES>(P, tile, ct0 + j, [&](auto rbc, auto fc) {
        constexpr int rb = decltype(rbc)::value, f = decltype(fc)::value;
        if constexpr (rb >= NRB) return f32x4_t{0.f, 0.f, 0.f, 0.f};   // rows that are not stored
        else if constexpr (NAMED) return read_acc<(j * NRB + rb) * 2 + f>();
        else return acc[rb][f];
      }, As);
  });
}

// field by field, so that the descriptors stay in scalar registers
template <typename ARGS>
__device__ __forceinline__ QuantProblem select_problem(const ARGS& a, bool shared) {
  QuantProblem Q;
#define FMOE_SEL(f) Q.f = shared ? a.p1.f : a.p0.f
  FMOE_SEL(s.A); FMOE_SEL(s.lda); FMOE_SEL(s.map1); FMOE_SEL(s.map2); FMOE_SEL(s.map1_limit); FMOE_SEL(s.Bp);
  FMOE_SEL(s.group_stride); FMOE_SEL(s.nbw); FMOE_SEL(s.ks); FMOE_SEL(s.C); FMOE_SEL(s.ldc); FMOE_SEL(s.N);
  FMOE_SEL(s.K); FMOE_SEL(s.n_col_tiles); FMOE_SEL(s.a_group_off); FMOE_SEL(s.c_group_off); FMOE_SEL(Sp);
  FMOE_SEL(scale_stride);
#undef FMOE_SEL
  return Q;
}

// The forms for few rows find their work item from the experts' offsets: no launch to build lists, which would take as long as
// a GEMM of a token or two.  Items: the shared groups', then those of the routed experts in ascending order, an expert's row
// tiles next to each other for every column unit, since they share its weights.  With row tiles the sequence is cut into eight
// contiguous shares, one per XCD (consecutive workgroups go round the XCDs).
struct QuantListArgs {
  QuantProblem p0, p1;             // routed experts; shared group
  const int32_t* expert_offsets;   // null without room for rows
  const int32_t* n_dev;            // or null
  int E, n_cap, row_cap;
  int cols;                        // column units of an expert
  int shared_groups, shared_cols;  // shared groups in this launch, column units of one
  int log2_bm;                     // rows of a row tile (narrow kernel)
};
// One row tile an expert, whatever its rows; workgroup = place in the sequence.  Without the sums over all experts and the
// shares: a token or two are all latency (one token, d 2048, 64 experts of 1408 and two shared 15.1 -> 13.6 us).
__device__ __forceinline__ QuantItem find_expert(const QuantListArgs& a, int item) {
  constexpr int Q = FMOE_MAX_EXPERTS / 64;
  const int lane = threadIdx.x & 63;
  QuantItem it{-1, 0, 0, 0, false};
  const int shared_items = a.shared_groups * a.shared_cols;
  if (item < shared_items) {
    it.shared = true;
    it.group = item / a.shared_cols;
    it.unit = item - it.group * a.shared_cols;
    it.rows = resolve_count(a.n_cap, a.n_dev);
    return it;
  }
  if (a.row_cap == 0) return it;                // a launch is whole eights of workgroups, the offsets may be null
  int ahead = (item - shared_items) / a.cols;   // experts with rows ahead of this item's
  it.unit = item - shared_items - ahead * a.cols;
  int r0[Q], r1[Q];
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    r0[q] = r1[q] = 0;
    if (64 * q + lane < a.E) {
      r0[q] = a.expert_offsets[64 * q + lane];
      r1[q] = a.expert_offsets[64 * q + lane + 1];
    }
  }
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const bool some = r0[q] >= 0 && r1[q] > r0[q] && r1[q] <= a.row_cap;
    const unsigned long long mask = __ballot(some);
    const int here = __popcll(mask);
    if (it.group < 0 && ahead < here) {   // uniform
      const int rank = __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0));
      const int at = __ffsll((long long)__ballot(some && rank == ahead)) - 1;
      it.group = 64 * q + at;
      it.row0 = __builtin_amdgcn_readlane(r0[q], at);
      it.rows = __builtin_amdgcn_readlane(r1[q], at) - it.row0;
    }
    ahead -= here;
  }
  return it;
}
// The item's problem, with the slices of a shared expert of the hidden buffer and the output (down GEMM).
template <typename ARGS>
__device__ __forceinline__ QuantProblem item_problem(const ARGS& a, bool shared, int group) {
  QuantProblem Q = select_problem(a, shared);
  if (shared) {
    Q.s.A += (size_t)group * Q.s.a_group_off;
    Q.s.C += (size_t)group * Q.s.c_group_off;
  }
  return Q;
}

template <bool SWIGLU>
__global__ __launch_bounds__(64, 2) void ffn_quant_thin_kernel(QuantListArgs a) {
  const QuantItem it = find_expert(a, (int)blockIdx.x);
  if (it.group < 0) return;
  const QuantProblem Q = item_problem(a, it.shared, it.group);
  // one turn unless a caller's own row lists name a token several times for one expert
  for (int done = 0; done < it.rows; done += THIN_ROWS)
    thin_quant_tile<SWIGLU>(Q, it.row0 + done, it.rows - done < THIN_ROWS ? it.rows - done : THIN_ROWS, it.group, it.unit);
}

// One column tile and four workgroups a CU, for a few rows an expert, where the weights have to be on their way in great
// numbers.  Row tiles of 32, seven k tiles ahead; or of 64: those of more than 32 rows in the same ring as stages twice as
// large, three ahead, so that an expert's weights are read and converted once and not twice.  Bound: the weights for a row or
// two an expert (d 2048, 64 experts of 1408 and two shared, 8 tokens: 15.7 + 10.8 us for 111 MB, 4.2 TB/s), from some ten on no
// one unit (d 1280, 64 of 896, two shared, 416 tokens: 27.2 + 16.9 us; the weights: 25).  By counters of that call's gate/up, a
// SIMD issues something in 62 % of its cycles, vector instructions (conversions and addresses, matrix instructions among them) in 32 %;
// matrix units 24 % busy, LDS 13 %, memory 2.9 TB/s; wavefronts wait 44 % of their time for a turn or for the instruction
// before, 35 % for loads and at barriers, and three quarters of the places for wavefronts are taken.
constexpr int NARROW_ROWS = 32, MIDDLE_ROWS = 64, NARROW_STAGES = 8;
template <bool SWIGLU>
__global__ __launch_bounds__(256, 4) void ffn_quant_narrow_kernel(QuantListArgs a) {
  __shared__ __align__(16) bf16_t As[NARROW_STAGES * NARROW_ROWS * SBK];
  const QuantItem it = find_tile(a, (int)blockIdx.x);
  if (it.group < 0) return;
  const QuantProblem Q = item_problem(a, it.shared, it.group);
  fmoe_tile tile{};
  tile.row0 = it.row0;
  tile.rows = it.rows;
  if (it.rows <= 16)   // uniform
    quant_tile<SWIGLU, 1, 1, NARROW_STAGES, NARROW_ROWS, true>(Q, tile, it.group, it.unit, it.unit + 1, As);
  else if (it.rows <= NARROW_ROWS)
    quant_tile<SWIGLU, 1, 1, NARROW_STAGES, NARROW_ROWS>(Q, tile, it.group, it.unit, it.unit + 1, As);
  else
    quant_tile<SWIGLU, 2, 1, NARROW_STAGES / 2, MIDDLE_ROWS>(Q, tile, it.group, it.unit, it.unit + 1, As);
}

// Tiles of 128 rows and two column tiles, dealt out as deal.h says; column tiles are taken two at a time (a.cols = such pairs
// per tile entry).  Bound: the matrix instructions, at the rate of a large library product (4096 tokens, d 2048, 64 experts of
// 1408 and two shared: 208 + 119 us, 1146 TFLOP/s over both and the lists; a product of 8192^3 1158).  (The build looks at the
// registers of a kernel of this name.)
template <bool SWIGLU>
__global__ __launch_bounds__(256, 2) void ffn_quant_dense_kernel(QuantArgs a) {
  __shared__ __align__(16) bf16_t As[4 * SBM * SBK];
  int pair, strip_cols;
  bool single;
  const int ti = dense_entry((int)blockIdx.x, a.n_tiles[0], a.n_tiles[2], a.cols, pair, single, strip_cols);
  if (ti < 0) return;
  fmoe_tile tile = load_entry(a.tiles, ti);
  const bool shared = tile.group >= a.E;
  const int group = shared ? tile.group - a.E : tile.group;
  const QuantProblem Q = item_problem(a, shared, group);
  // column tiles this entry really has, and pairs of them
  const int ct_here = (Q.s.n_col_tiles - tile.col0 < a.cols_entry) ? (Q.s.n_col_tiles - tile.col0) : a.cols_entry;
  const int pairs = (ct_here + 1) / 2;
  if (pair >= pairs) return;
  int row_tile = tile.rt;
  if (tile.nrt > 1) dense_run_order(tile.rt, tile.nrt, pairs, strip_cols, row_tile, pair);
  take_row_tile(tile, row_tile, SBM);
  const int ct0 = tile.col0 + pair * 2, ct_limit = tile.col0 + ct_here;
  switch ((tile.rows + 31) >> 5) {   // live 32-row bands of the tile, uniform per block
    case 1: quant_tile<SWIGLU, 1, 2, 4, SBM>(Q, tile, group, ct0, ct_limit, As); break;
    case 2: quant_tile<SWIGLU, 2, 2, 4, SBM>(Q, tile, group, ct0, ct_limit, As); break;
    case 3: quant_tile<SWIGLU, 3, 2, 4, SBM>(Q, tile, group, ct0, ct_limit, As); break;
    default: quant_tile<SWIGLU, 4, 2, 4, SBM>(Q, tile, group, ct0, ct_limit, As); break;
  }
}

// Source rows [group][n][k]: codes two to a byte, scales one byte per 32 k.  PAIR: gate and up (fragments 0 and 1), else
// fragment f = features 16f..16f+15 of the column block.  Past N and K the codes are 0 and the scales 1.
template <bool PAIR>
__global__ __launch_bounds__(256) void pack_quant_kernel(const uint32_t* __restrict__ codes0, const uint8_t* __restrict__ scales0,
                                                         const uint32_t* __restrict__ codes1, const uint8_t* __restrict__ scales1,
                                                         u32x4_t* __restrict__ dst, u32x4_t* __restrict__ dst_scales, int G,
                                                         int N, int K, int nbt) {
  const int NT = quant_tiles(K), NT4 = quant_scale_tiles(K), KG = (K + FMOE_QUANT_GROUP - 1) / FMOE_QUANT_GROUP;
  const size_t total = (size_t)G * nbt * NT * 256, total_scales = (size_t)G * nbt * NT4 * 64;
  for (size_t u = (size_t)blockIdx.x * blockDim.x + threadIdx.x; u < total + total_scales;
       u += (size_t)gridDim.x * blockDim.x) {
    const bool scales = u >= total;
    size_t q = scales ? u - total : u;
    const int lane = scales ? (int)(q & 15) : (int)(q & 63);
    q >>= scales ? 4 : 6;
    const int kt = (int)(q % (scales ? NT4 : NT));
    q /= scales ? NT4 : NT;
    const int b = (int)(q % (nbt * 4)), g = (int)(q / (nbt * 4));
    u32x4_t v = {0u, 0u, 0u, 0u};
    if (!scales) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {   // k step i/2, fragment i%2
        const int f = i & 1, n = PAIR ? b * 16 + (lane & 15) : b * 32 + f * 16 + (lane & 15);
        const int k = kt * SBK + (i >> 1) * 32 + 8 * (lane >> 4);
        if (n < N && k < K) v[i] = (PAIR && f ? codes1 : codes0)[(((size_t)g * N + n) * K + k) >> 3];
      }
      dst[u] = v;
    } else {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int f = i & 1, n = PAIR ? b * 16 + lane : b * 32 + f * 16 + lane;
          const int kg = (kt * 4 + t) * 2 + (i >> 1);
          uint32_t s = 127u;
          if (n < N && kg < KG) s = (PAIR && f ? scales1 : scales0)[((size_t)g * N + n) * KG + kg];
          v[t] |= s << (8 * i);
        }
      dst_scales[u - total] = v;
    }
  }
}

// 16-byte units of one packed group: column tiles (of four column blocks) times k tiles
inline size_t code_units(int nbw, int K) { return (size_t)((nbw + 3) / 4) * quant_tiles(K) * 256; }
inline size_t scale_units(int nbw, int K) { return (size_t)((nbw + 3) / 4) * quant_scale_tiles(K) * 64; }

}  // namespace

size_t fmoe_quant_bytes(const fmoe_ctx* ctx, int which, size_t* codes) {
  const PackedMatrix m = packed_matrix(ctx->cfg, which);
  const size_t c = (size_t)m.groups * code_units(m.nbw, m.K) * 16;
  if (codes) *codes = c;
  return c + (size_t)m.groups * scale_units(m.nbw, m.K) * 16;
}

int launch_pack_quant(fmoe_ctx* ctx, const fmoe_quant_tensor* const* w, hipStream_t stream) {
  for (int which = 0; which < 4; ++which) {
    const PackedMatrix m = packed_matrix(ctx->cfg, which);
    if (m.groups == 0) continue;
    const bool pair = (which & 1) == 0;
    const fmoe_quant_tensor* a = w[which == 0 ? 0 : which == 1 ? 2 : which == 2 ? 3 : 5];
    const fmoe_quant_tensor* b = pair ? w[which == 0 ? 1 : 4] : nullptr;
    size_t codes;
    const size_t threads = fmoe_quant_bytes(ctx, which, &codes) / 16;
    char* const base = static_cast<char*>(ctx->pq[which]);
    const size_t blocks = threads / 256 + 1;
    const dim3 grid((unsigned)(blocks < 65536 ? blocks : 65536)), block(256);
#define FMOE_PACK(PAIR)                                                                                                 \
  hipLaunchKernelGGL(pack_quant_kernel<PAIR>, grid, block, 0, stream, static_cast<const uint32_t*>(a->codes), a->scales, \
                     PAIR ? static_cast<const uint32_t*>(b->codes) : nullptr, PAIR ? b->scales : nullptr,               \
                     reinterpret_cast<u32x4_t*>(base), reinterpret_cast<u32x4_t*>(base + codes), m.groups, m.N, m.K,    \
                     (m.nbw + 3) / 4)
    if (pair) FMOE_PACK(true);
    else FMOE_PACK(false);
#undef FMOE_PACK
  }
  FMOE_HIP_CHECK(hipGetLastError());
  return FMOE_OK;
}

// Which form a call takes, by what it can route (capacities).  All times: us, gate/up and down, weights from memory;
// "2048, 64 of 1408": d_model, experts, their hidden size.
//  * Thin for at most THIN_ROWS tokens (no expert has more rows) that touch up to so many bytes of weights: a wavefront an
//    item and no LDS, the shortest way from launch to result; with more to stream, the narrow form has more on its way.
//    Thin / narrow (MB: what the rule counts): 2048, 64 of 1408 and two shared one token 13.4 / 16.9 (37), 2 tokens 19.4 / 21.0
//    (64), 3 tokens 24.6 / 24.9 (92), 4 tokens 28 / 28 (119); 128 of 768 one token 12.5 / 15.2 (20), 4
//    tokens 21.1 / 21.4 (80), 5 tokens 25.3 / 24.3 (100); 1280, 64 of 896, two shared 4 tokens 13.9 / 15.8 (48), 8 tokens 16.8 / 18.3
//    (92); 4096, 8 of 1536, one shared one token 15.5 / 20.6 (30), 8 tokens 24.2 / 25.1 and 16 tokens 27.6 / 25.8 (90).
//  * Dense from so many rows an expert, so much work (rows times weights of a matrix: what it gains has to make up for its
//    launch that builds lists and for two workgroups a CU instead of four) and so many items on, row tiles the call can have
//    (one of every expert with rows, and the further ones) times pairs of column tiles of the narrower GEMM.  Tiles of 64 /
//    dense (10^9 rows times weights): 2048, 64 of 1408 and two shared 100 rows an expert 165 / 180 (18), 150 rows 226 / 228 (28),
//    200 rows 285 / 272 (37); 128 of 768 150 rows 205 / 215 (30), 200 rows 256 / 251 (40); 2560, 72 of 1536 125 rows 297 / 296
//    (35), 158 rows 363 / 340 (45); with less work 1280, 64 of 896, two shared 169 rows 117 / 124 (12), 200 rows 130 / 132 (15),
//    244 rows 154 / 147 (18); 512, 256 of 512 200 rows 119 / 130 (13), 300 rows 166 / 165 (20); 768, 64 of 768 250 rows 76 / 78 (9),
//    500 rows 130 / 127 (19); 4096, 8 of 1536 225 rows 109 / 122 (11), 375 rows 162 / 155 (19); 1288, 16 of 904 400 rows 71 / 82
//    (7), 800 rows 139 / 135 (15), 1200 rows 209 / 182 (22).
//  * Of the forms with one column tile, tiles of 64 rows from so many rows an expert on, if those also are items enough (rows
//    that the call can have, in tiles of 64, times column tiles of the narrower GEMM).  32 / 64: 2048, 64 of 1408, two shared 9
//    rows 66 / 66, 28 rows 94 / 91, 47 rows 121 / 113; 1280, 64 of 896, two shared 19 rows 42 / 42, 39 rows 55 / 54, 56 rows
//    66 / 64; 512, 256 of 512 16 rows 40 / 38, 47 rows 60 / 54; 128 of 768 50 rows 119 / 113; with few items 4096, 8 of 1536 37
//    rows (288) 42 / 47, 50 rows (336) 51 / 50, 62 rows (360) 54 / 51, 100 rows (480) 71 / 67; 1288, 16 of 904, one shared 50
//    rows (308) 24 / 26, 62 rows (341) 26 / 27.
constexpr size_t QUANT_THIN_BYTES = 92u << 20;
constexpr long long QUANT_DENSE_ROWS = 150;
constexpr long long QUANT_DENSE_WORK = 16000000000;
constexpr long long QUANT_DENSE_ITEMS = 300;
constexpr long long QUANT_MIDDLE_ROWS = 16;
constexpr long long QUANT_MIDDLE_ITEMS = 350;
quant_form quant_ffn_form(const fmoe_ctx* ctx, int n_cap) {
  const fmoe_config& c = ctx->cfg;
  if (ctx->ffn_shape == 2) return QUANT_DENSE;
  const bool few = ctx->ffn_shape == 1;
  const long long rows = (long long)n_cap * ctx->kmax, experts = rows < c.n_experts ? rows : c.n_experts;
  if (!few && n_cap <= THIN_ROWS) {
    const size_t expert = (fmoe_quant_bytes(ctx, 0, nullptr) + fmoe_quant_bytes(ctx, 1, nullptr)) / c.n_experts;
    const size_t shared = fmoe_quant_bytes(ctx, 2, nullptr) + fmoe_quant_bytes(ctx, 3, nullptr);
    return (size_t)experts * expert + shared <= QUANT_THIN_BYTES ? QUANT_THIN : QUANT_NARROW;
  }
  const int tiles1 = (c.d_ffn + 63) / 64, tiles2 = (c.d_model + 127) / 128, pairs1 = (tiles1 + 1) / 2, pairs2 = (tiles2 + 1) / 2;
  if (!few && rows >= QUANT_DENSE_ROWS * c.n_experts && (double)rows * c.d_model * c.d_ffn >= QUANT_DENSE_WORK &&
      (experts + rows / SBM) * (pairs1 < pairs2 ? pairs1 : pairs2) >= QUANT_DENSE_ITEMS)
    return QUANT_DENSE;
  return rows >= QUANT_MIDDLE_ROWS * c.n_experts &&
                 (experts + rows / MIDDLE_ROWS) * (tiles1 < tiles2 ? tiles1 : tiles2) >= QUANT_MIDDLE_ITEMS
             ? QUANT_MIDDLE : QUANT_NARROW;
}

int run_ffn_quant(const fmoe_ctx* ctx, const void* x, const int32_t* kept_idx, int n_cap, const int32_t* n_dev,
                  const int32_t* expert_offsets, const int32_t* perm_src, void* y, void* y_shared, char* base,
                  const fmoe_ws_layout& L, const fmoe_ffn_geom& geo, hipStream_t stream) {
  const fmoe_config& c = ctx->cfg;
  const int d = c.d_model, E = c.n_experts, F = c.d_ffn;
  const int Ft = c.n_shared * c.d_ffn_shared;
  if ((size_t)n_cap * ctx->kmax * F * 2 > 0xffffffffull || (size_t)n_cap * Ft * 2 > 0xffffffffull)
    return fmoe_fail(FMOE_ERR_UNSUPPORTED, "expert FFN: a hidden buffer of %d rows exceeds 4 GiB", n_cap);
  int32_t* tile_count = reinterpret_cast<int32_t*>(base + L.tile_count);
  auto problem = [&](int which) {
    const PackedMatrix m = packed_matrix(c, which);
    QuantProblem q{};
    if (m.groups == 0) return q;
    size_t codes;
    (void)fmoe_quant_bytes(ctx, which, &codes);
    const char* packed = static_cast<const char*>(ctx->pq[which]);
    q.s.Bp = reinterpret_cast<const u32x4_t*>(packed);
    q.Sp = reinterpret_cast<const u32x4_t*>(packed + codes);
    q.s.nbw = m.nbw; q.s.N = m.N; q.s.K = m.K;
    q.s.group_stride = (long long)code_units(m.nbw, m.K);
    q.scale_stride = (long long)scale_units(m.nbw, m.K);
    return q;
  };
  QuantArgs g1{}, g2{};
  g1.E = g2.E = E;
  g1.tiles = reinterpret_cast<fmoe_tile*>(base + L.tiles);
  g2.tiles = reinterpret_cast<fmoe_tile*>(base + L.tiles2);
  g1.n_tiles = tile_count;
  g2.n_tiles = tile_count + 1;
  g1.p0 = problem(0); g1.p1 = problem(2); g2.p0 = problem(1); g2.p1 = problem(3);
  {
    StreamProblem &p = g1.p0.s, &q = g1.p1.s;
    p.A = q.A = static_cast<const bf16_t*>(x); p.lda = q.lda = d;
    p.map1 = perm_src; p.map1_limit = n_cap;
    p.map2 = q.map2 = kept_idx;
    p.C = reinterpret_cast<bf16_t*>(base + L.h); p.ldc = F; p.n_col_tiles = geo.cols1;
    q.C = reinterpret_cast<bf16_t*>(base + L.h_shared); q.ldc = Ft; q.n_col_tiles = geo.scols1;
  }
  {
    StreamProblem &p = g2.p0.s, &q = g2.p1.s;
    p.A = reinterpret_cast<const bf16_t*>(base + L.h); p.lda = F;
    p.C = static_cast<bf16_t*>(y); p.ldc = d; p.n_col_tiles = geo.cols2;
    q.A = reinterpret_cast<const bf16_t*>(base + L.h_shared); q.lda = Ft; q.a_group_off = c.d_ffn_shared;
    q.C = static_cast<bf16_t*>(y_shared); q.ldc = d; q.c_group_off = (long long)n_cap * d; q.n_col_tiles = geo.scols2;
  }
  const quant_form form = quant_ffn_form(ctx, n_cap);
  const bool dense = form == QUANT_DENSE;
  const int row_cap = n_cap * ctx->kmax;
  auto launch = [&](auto swiglu, QuantArgs g, int cols) {
    constexpr bool S = decltype(swiglu)::value;
    if (dense) {
      g.cols_entry = cols;
      g.cols = (cols + 1) / 2;
      hipLaunchKernelGGL(ffn_quant_dense_kernel<S>, dim3(dense_blocks(geo.tile_cap, g.cols)), dim3(256), 0, stream, g);
      return;
    }
    // column units: column blocks in the thin form, tiles of four in the narrow one
    const bool thin = form == QUANT_THIN;
    const int log2_bm = form == QUANT_MIDDLE ? 6 : 5;
    static_assert(MIDDLE_ROWS == 1 << 6 && NARROW_ROWS == 1 << 5, "rows of a tile");
    QuantListArgs h{g.p0, g.p1, expert_offsets, n_dev, E, n_cap, row_cap, 0, 0, 0, log2_bm};
    h.cols = thin ? g.p0.s.nbw : (g.p0.s.nbw + 3) / 4;
    if (Ft > 0) {
      h.shared_groups = S ? 1 : c.n_shared;
      h.shared_cols = thin ? g.p1.s.nbw : (g.p1.s.nbw + 3) / 4;
    }
    const long long tiles = (row_cap < E ? row_cap : E) + (thin ? 0 : row_cap >> log2_bm);   // that the routed experts can have
    const long long shared_tiles = thin ? n_cap > 0 : ((long long)n_cap + (1 << log2_bm) - 1) >> log2_bm;
    const long long items = tiles * h.cols + shared_tiles * h.shared_cols * h.shared_groups;
    if (items == 0) return;
    const unsigned blocks = (unsigned)((items + 7) / 8 * 8);
    if (thin) hipLaunchKernelGGL(ffn_quant_thin_kernel<S>, dim3(blocks), dim3(64), 0, stream, h);
    else hipLaunchKernelGGL(ffn_quant_narrow_kernel<S>, dim3(blocks), dim3(256), 0, stream, h);
  };
  {
    fmoe_prof_scope prof(ctx, dense ? SLOT_GEMM1_DENSE : SLOT_GEMM1, stream);
    launch(std::true_type{}, g1, geo.cols1);
  }
  {
    fmoe_prof_scope prof(ctx, dense ? SLOT_GEMM2_DENSE : SLOT_GEMM2, stream);
    launch(std::false_type{}, g2, geo.cols2);
  }
  return FMOE_OK;
}
