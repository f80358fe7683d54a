// A whole layer for a few tokens (at most FMOE_DECODE_TOKENS, a decoding step): the addition and norm in front of it, router, choice of
// experts, their products, gates and residual.
//
//   decode_logits    h = x + delta, n = norm(h) (norm_dev.h), logits of n in 64 bits, rounded once: every workgroup takes 4 experts and
//                    one to four tokens, so that the router matrix is read by many CUs at once and no chain of additions holds it up
//   select_units     the choice (select.hip), and the list of the experts that any token has listed
//   decode_gate_up   one to four wavefronts per expert of the list and column block of 16: all tokens are the rows of the matrix
//                    instruction, whose hidden rows are kept for those that list the expert
//   decode_down      per 32 output columns four workgroups, whose wavefronts share the experts (and where there are fewer, their
//                    reductions); the rows stay tokens (of whose hidden rows a second plane has the other 8 bits), so that gate * product
//                    is added up in registers, then over the wavefronts
//                    in LDS
//   decode_join      the four sums and the residual, in a fixed order.  (Left to the last of the four workgroups to arrive, which takes
//                    fences between L2s that are not coherent with each other: 50 us for the down launch instead of 8.)
// Bound: the weights of the experts that the tokens touch; for a token or two a chain of launches and latencies.

#include "ffn_dev.h"
#include "norm_dev.h"
#include "quant_items.h"

namespace {

constexpr int TOKENS = FMOE_DECODE_TOKENS;

// ---------------------------------------------------------------------------------------------------------- norm and logits

struct LogitArgs {
  const bf16_t *x, *delta;
  const void* w;            // norm weight or null
  int w_bf16;
  float eps;
  double inv_d;
  int T, d, E, groups;      // groups of 16 k in the packed router
  const float *wp, *bias;
  bf16_t *h, *n;            // [T, d] or null
  float* logits;            // [T, E]
};

constexpr int LOGIT_WAVES = 8, LOGIT_EXPERTS = 4;

// Router weights as route.hip packs them: expert block of 16, group of 16 k, lane l: expert l % 16, k = l / 16 + 4 j, j = 0..3.
// A wavefront's load is four experts of four groups.
template <int TB>
__global__ __launch_bounds__(64 * LOGIT_WAVES) void decode_logits_kernel(LogitArgs a) {
  extern __shared__ __align__(16) bf16_t rows[];                // n of TB tokens, in the order of the packed weights
  __shared__ double s_sum[LOGIT_WAVES], s_part[LOGIT_WAVES][TB][LOGIT_EXPERTS];
  constexpr int WPT = LOGIT_WAVES / TB, AHEAD = 4;              // wavefronts a token; loads of weights in flight
  constexpr int STEP = LOGIT_WAVES * 4;                         // groups that the workgroup's loads cover at a time
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int t0 = (int)blockIdx.y * TB, e0 = (int)blockIdx.x * LOGIT_EXPERTS, padded = a.groups * 16;
  const int quarter = (lane >> 2) & 3, g_first = wave * 4 + (lane >> 4);
  const f32x4_t* const wp = reinterpret_cast<const f32x4_t*>(a.wp) + (size_t)(e0 >> 4) * a.groups * 64 + quarter * 16 + (e0 & 15) + (lane & 3);
  // a token's row: its WPT wavefronts, units of eight
  const int tb = wave / WPT, first = (wave % WPT) * 64 + lane, t = t0 + tb < a.T ? t0 + tb : a.T - 1;
  const size_t base = (size_t)t * a.d;
  const int units = a.d >> 3;
  bf16_t* const row = rows + (size_t)tb * padded;
  constexpr int HELD = 2;                                       // units a lane holds; longer rows are read again
  auto load_row = [&](int u, rms::Unit<bf16_t>& h, rms::Unit<bf16_t>& dl) {
    h.load(a.x + base + u * 8);
    if (a.delta != nullptr) dl.load(a.delta + base + u * 8);
  };
  auto add_delta = [&](rms::Unit<bf16_t>& h, const rms::Unit<bf16_t>& dl) {
    if (a.delta == nullptr) return;
#pragma unroll
    for (int e = 0; e < 8; e += 2)
      h.set2(e, rms::add_rounded<bf16_t>(h.get(e), dl.get(e)), rms::add_rounded<bf16_t>(h.get(e + 1), dl.get(e + 1)));
  };
  auto sum_of = [&](int u, rms::Unit<bf16_t>& h) {
    rms::Unit<bf16_t> dl;
    load_row(u, h, dl);
    add_delta(h, dl);
  };
  auto load_weight = [&](int u, float (&f)[8]) {
    if (a.w_bf16) rms::load_weights<bf16_t>(a.w, u * 8, f);     // uniform
    else rms::load_weights<float>(a.w, u * 8, f);
  };
  rms::Unit<bf16_t> held[HELD], held_delta[HELD];
  float weight[HELD][8];                                        // of the norm
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    held[i].zero();
    held_delta[i].zero();
    if (first + 64 * WPT * i < units) {
      load_row(first + 64 * WPT * i, held[i], held_delta[i]);
      if (a.w != nullptr) load_weight(first + 64 * WPT * i, weight[i]);
    }
  }
  __builtin_amdgcn_sched_barrier(0);
  f32x4_t w[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) {                             // on their way behind the norm (its rows were asked for first); past the end the last group
    const int g = g_first + STEP * i;
    w[i] = wp[(size_t)(g < a.groups ? g : a.groups - 1) * 64];
  }
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int i = 0; i < HELD; ++i) add_delta(held[i], held_delta[i]);
  rms::Scale r{1.0f, 0.0f, 0};
  if (a.w != nullptr) {
    auto add = [&](const rms::Unit<bf16_t>& h) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double v = (double)h.get(e);
        sum = fma(v, v, sum);
      }
    };
#pragma unroll
    for (int i = 0; i < HELD; ++i) add(held[i]);
    for (int u = first + 64 * WPT * HELD; u < units; u += 64 * WPT) {
      rms::Unit<bf16_t> h;
      sum_of(u, h);
      add(h);
    }
    sum = rms::wave_sum(sum);
    if (lane == 0) s_sum[wave] = sum;
    __syncthreads();
    sum = 0.0;
#pragma unroll
    for (int i = 0; i < WPT; ++i) sum += s_sum[tb * WPT + i];
    r = rms::row_scale(sum, a.inv_d, a.eps);
  }
  const bool mine = e0 == 0 && t0 + tb < a.T;                   // the first workgroups write the rows
  // element e of unit u: group u / 2, k = 8 (u % 2) + e of it, which lane group e % 4 wants as its number 2 (u % 2) + e / 4
  auto lay_out = [&](int u, const rms::Unit<bf16_t>& n) {
    bf16_t* const to = row + (u >> 1) * 16 + 2 * (u & 1);
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<uint32_t*>(to + 4 * q) = (__float_as_uint(n.get(q)) >> 16) | (__float_as_uint(n.get(q + 4)) & 0xffff0000u);
  };
  auto place = [&](int u, const rms::Unit<bf16_t>& h, const float (&f)[8]) {
    rms::Unit<bf16_t> n = h;
    if (a.w != nullptr) {
#pragma unroll
      for (int e = 0; e < 8; e += 2)
        n.set2(e, rms::value_rounded<bf16_t>(h.get(e), f[e], r), rms::value_rounded<bf16_t>(h.get(e + 1), f[e + 1], r));
    }
    if (mine && a.h != nullptr) h.store(a.h + base + u * 8);
    if (mine && a.n != nullptr) n.store(a.n + base + u * 8);
    lay_out(u, n);
  };
#pragma unroll
  for (int i = 0; i < HELD; ++i)
    if (first + 64 * WPT * i < units) place(first + 64 * WPT * i, held[i], weight[i]);
  for (int u = first + 64 * WPT * HELD; u < units; u += 64 * WPT) {
    rms::Unit<bf16_t> h;
    float f[8];
    sum_of(u, h);
    if (a.w != nullptr) load_weight(u, f);
    place(u, h, f);
  }
  for (int u = units + first; u < padded >> 3; u += 64 * WPT) {
    rms::Unit<bf16_t> zero;
    zero.zero();
    lay_out(u, zero);
  }
  __syncthreads();

  double acc[TB];
#pragma unroll
  for (int i = 0; i < TB; ++i) acc[i] = 0.0;
  for (int g0 = g_first; g0 < a.groups; g0 += STEP * AHEAD) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int g = g0 + STEP * i;
      if (g < a.groups) {
#pragma unroll
        for (int b = 0; b < TB; ++b) {
          const uint2 v = *reinterpret_cast<const uint2*>(rows + (size_t)b * padded + g * 16 + quarter * 4);
#pragma unroll
          for (int j = 0; j < 4; ++j) {   // a product of two bf16 numbers is exact in fp32
            const uint32_t p = j < 2 ? v.x : v.y;
            acc[b] += (double)(__uint_as_float(j & 1 ? p & 0xffff0000u : p << 16) * w[i][j]);
          }
        }
      }
      const int next = g + STEP * AHEAD;
      if (next < a.groups) w[i] = wp[(size_t)next * 64];
    }
  }
#pragma unroll
  for (int b = 0; b < TB; ++b) {
    double v = acc[b];   // of the sixteen lanes with the same expert
    v += row_rotate<4>(v);
    v += row_rotate<8>(v);
    v = rms::add_32_apart(rms::add_16_apart(v));
    if (lane < LOGIT_EXPERTS) s_part[wave][b][lane] = v;
  }
  __syncthreads();
  if (tid < LOGIT_EXPERTS * TB) {
    const int b = tid / LOGIT_EXPERTS, e = e0 + tid % LOGIT_EXPERTS;
    double v = 0.0;
#pragma unroll
    for (int i = 0; i < LOGIT_WAVES; ++i) v += s_part[i][b][tid % LOGIT_EXPERTS];
    if (t0 + b < a.T && e < a.E) a.logits[(size_t)(t0 + b) * a.E + e] = (float)(a.bias != nullptr ? v + (double)a.bias[e] : v);
  }
}

// ------------------------------------------------------------------------------------------------------------- products

// Weights of one packed matrix, bf16 (ffn.hip) or 4 bits (ffn_quant.hip): what a wavefront needs of a column block
struct DecodeMatrix {
  const u32x4_t *Bp, *Sp;
  long long group_stride, scale_stride;   // 16-byte units between groups
  int nbw, N, K;                          // column blocks, output features, reduction
};

// acc[j][f] += rows x weights over the k tiles (64 wide) first .. last-1 of column block cb + j, j < NCB (the last one again past the
// end): fragment f is gate / up or a half of 32 columns, lane l has row l % 16 from `a` (the lane's own address; K elements).  A ring
// of k tiles in registers, with as many bytes of weights on their way with one column block as with two; loads past the last tile
// return zeros and fetch nothing.
template <bool QUANT, int NCB>
__device__ __forceinline__ void accumulate(const DecodeMatrix& M, int group, int cb, int first, int last, const bf16_t* a,
                                           f32x4_t (&acc)[NCB][2]) {
  constexpr int S = (QUANT ? 8 : 4) / NCB, PIECES = QUANT ? 1 : 4, SU = S / 4 > 0 ? S / 4 : 1;
  static_assert(!QUANT || S % 4 == 0, "a unit of scales serves four k tiles");
  const int lane = threadIdx.x & 63, NT = (M.K + SBK - 1) / SBK, NT4 = (NT + 3) / 4, tiles = last - first;
  constexpr int TILE = QUANT ? 1024 : 16384;   // bytes between k tiles
  __amdgpu_buffer_rsrc_t b_rsrc[NCB], s_rsrc[NCB];
#pragma unroll
  for (int j = 0; j < NCB; ++j) {
    const int c = cb + j < M.nbw ? cb + j : M.nbw - 1;
    const char* const b0 = reinterpret_cast<const char*>(M.Bp + (size_t)group * M.group_stride) +
                           (QUANT ? (size_t)c * NT * 1024 : (size_t)(c >> 2) * NT * 16384 + (c & 3) * 4096) + (size_t)first * TILE;
    b_rsrc[j] = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(b0), 0, QUANT ? tiles * 1024 : (tiles - 1) * 16384 + 4096, 0x00020000);
    s_rsrc[j] = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<u32x4_t*>(QUANT ? M.Sp + (size_t)group * M.scale_stride + ((size_t)c * NT4 + first / 4) * 16 : nullptr), 0,
        QUANT ? (tiles + 3) / 4 * 256 : 0, 0x00020000);
  }
  const uint32_t lane16 = (uint32_t)lane * 16u, column16 = (uint32_t)(lane & 15) * 16u;
  const int kq = (lane >> 4) * 8;
  u32x4_t breg[S][NCB][PIECES], sreg[SU][NCB], areg[S][2];
  auto load_b = [&](int slot, int t) {
#pragma unroll
    for (int j = 0; j < NCB; ++j)
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
        breg[slot][j][i] = __builtin_amdgcn_raw_buffer_load_b128(b_rsrc[j], lane16 + (uint32_t)(t * TILE + i * 1024), 0, 0);
  };
  auto load_s = [&](int slot, int t4) {
#pragma unroll
    for (int j = 0; j < NCB; ++j)
      sreg[slot][j] = __builtin_amdgcn_raw_buffer_load_b128(s_rsrc[j], column16 + (uint32_t)t4 * 256u, 0, 0);
  };
  auto load_a = [&](int slot, int t) {   // k past K re-reads the row's end, where the packed weights are zero
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int k = (first + t) * SBK + s * 32 + kq;
      areg[slot][s] = *reinterpret_cast<const u32x4_t*>(a + (k < M.K ? k : M.K - 8));
    }
  };
  auto multiply = [&](int slot) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const bf16x8_t av = __builtin_bit_cast(bf16x8_t, areg[slot][s]);
#pragma unroll
      for (int j = 0; j < NCB; ++j) {
        u32x4_t b[2];
        if constexpr (QUANT) {
          const uint32_t sc = sreg[slot / 4][j][slot % 4];
          b[0] = s == 0 ? dequantize<0>(breg[slot][j][0][0], sc) : dequantize<2>(breg[slot][j][0][2], sc);
          b[1] = s == 0 ? dequantize<1>(breg[slot][j][0][1], sc) : dequantize<3>(breg[slot][j][0][3], sc);
        } else {
          b[0] = breg[slot][j][2 * s];
          b[1] = breg[slot][j][2 * s + 1];
        }
#pragma unroll
        for (int f = 0; f < 2; ++f)
          acc[j][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, __builtin_bit_cast(bf16x8_t, b[f]), acc[j][f], 0, 0, 0);
      }
    }
  };
#pragma unroll
  for (int t = 0; t < S; ++t) {
    if constexpr (QUANT) {
      if (t % 4 == 0) load_s(t / 4, t / 4);
    }
    load_b(t, t);
  }
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int t = 0; t < S; ++t) load_a(t, t);
  __builtin_amdgcn_sched_barrier(0);
  int t0 = 0;
  for (; t0 + S <= tiles; t0 += S) {   // no exit inside, so that the waits can count on the rings' order
#pragma unroll
    for (int u = 0; u < S; ++u) {
      multiply(u);
      __builtin_amdgcn_sched_barrier(0);
      load_b(u, t0 + u + S);
      load_a(u, t0 + u + S);
      if constexpr (QUANT) {
        if (u % 4 == 3) load_s(u / 4, (t0 + S) / 4 + u / 4);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
#pragma unroll
  for (int u = 0; u < S - 1; ++u) {
    if (t0 + u >= tiles) break;   // uniform
    multiply(u);
  }
}

// The list's length and unit u (which may be behind the last), held within bounds (units.h), in scalar registers
__device__ __forceinline__ int list_length(const fmoe_unit_list* list, const ListBounds& b) { return units_within(list->n, b); }
__device__ __forceinline__ fmoe_unit load_unit(const fmoe_unit_list* list, int u, const ListBounds& b) {
  typedef const __attribute__((address_space(4))) int32_t* const_ptr;
  const const_ptr p = (const_ptr)(uintptr_t)(list->unit + u);
  return unit_within(fmoe_unit{p[0], p[1], (uint32_t)p[2]}, b);
}
// Of the n units those that two tokens eight apart list: number i, how many there are
__device__ __forceinline__ int full_unit(const fmoe_unit_list* list, int i, int n) {
  typedef const __attribute__((address_space(4))) int32_t* const_ptr;
  return full_unit_within(((const_ptr)(uintptr_t)list->full)[i], n);
}
__device__ __forceinline__ int full_length(const fmoe_unit_list* list, int n) { return full_units_within(list->n_full, n); }

// Hidden rows h = silu(gate) * up are kept in two bf16 planes, h rounded to bf16 and what that leaves rounded again: 16 bits, 2^-16 of a
// value at most lost, far less than the rounding of the output.  (One plane's rounding is as much as the output's; the down launch with
// one / two, us: one token, d 2048, 64 experts of 1408, two shared, in 4 bits 6.4 / 6.9, 16 tokens 12.6 / 14.8; 8 tokens, 128 of 768 in bf16
// 20.9 / 21.2.)  What a value too large for bf16 leaves is taken for 0.
__device__ __forceinline__ void store_hidden(bf16_t* row, int plane, int col, float h) {
  const bf16_t hi = f32_to_bf16(h);
  const float top = bf16_to_f32(hi);
  row[col] = hi;
  row[plane + col] = rms::finite(top) ? f32_to_bf16(h - top) : 0;
}

struct GateUpArgs {
  DecodeMatrix routed, shared;
  const bf16_t* n;              // [T, K]
  const fmoe_unit_list* list;   // or null: no experts are listed
  ListBounds bounds;
  bf16_t *h, *h_shared;         // hidden rows [., 2, routed.N] of the pairs by expert and token; [T, 2, shared.N]
};

// NCB column blocks a wavefront: with two the rows, sixteen of them, are read half as often.
template <bool QUANT, int NCB>
__global__ __launch_bounds__(64) void decode_gate_up_kernel(GateUpArgs a) {
  const int lane = threadIdx.x, T = a.bounds.T;
  const int shared_items = (a.shared.nbw + NCB - 1) / NCB, items = (a.routed.nbw + NCB - 1) / NCB;
  int cb = (int)blockIdx.x;
  const bool shared = cb < shared_items;
  fmoe_unit unit{0, 0, (1u << T) - 1u};
  if (!shared) {
    cb -= shared_items;
    const int u = cb / items;
    cb -= u * items;
    if (u >= list_length(a.list, a.bounds)) return;
    unit = load_unit(a.list, u, a.bounds);
  }
  cb *= NCB;
  DecodeMatrix M;
#define FMOE_SEL(f) M.f = shared ? a.shared.f : a.routed.f
  FMOE_SEL(Bp); FMOE_SEL(Sp); FMOE_SEL(group_stride); FMOE_SEL(scale_stride); FMOE_SEL(nbw); FMOE_SEL(N); FMOE_SEL(K);
#undef FMOE_SEL
  bf16_t* const h = shared ? a.h_shared : a.h;
  const int token = (lane & 15) < T ? lane & 15 : T - 1;
  f32x4_t acc[NCB][2];
#pragma unroll
  for (int j = 0; j < NCB; ++j) acc[j][0] = acc[j][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  accumulate<QUANT, NCB>(M, unit.expert, cb, 0, (M.K + SBK - 1) / SBK, a.n + (size_t)token * M.K, acc);
#pragma unroll
  for (int v = 0; v < 4; ++v) {   // accumulator register v of lane l: row 4*(l/16) + v, column l%16
    const int t = 4 * (lane >> 4) + v;
    if (!((unit.mask >> t) & 1u)) continue;
    bf16_t* const row = h + (size_t)(unit.row0 + __popc(unit.mask & ((1u << t) - 1u))) * 2 * M.N;
#pragma unroll
    for (int j = 0; j < NCB; ++j) {
      const int col = (cb + j) * 16 + (lane & 15);
      if (col < M.N) store_hidden(row, M.N, col, silu_mul_bf16(acc[j][0][v], acc[j][1][v]));
    }
  }
}

// v plus that of the lane 32 away
__device__ __forceinline__ float plus_32_apart(float v) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

struct DownArgs {
  DecodeMatrix routed, shared;   // (a group per shared expert)
  int n_shared;
  const bf16_t *h, *h_shared;
  int plane, plane_shared;       // columns of a hidden row
  const fmoe_unit_list* list;    // or null
  ListBounds bounds;
  float* part;                   // [SPLITS, T, d]
};

// Workgroups that share 32 output columns.  us a call, 1 / 2 / 4 / 8 of them (in a graph, weights from memory): one token, d 1280, 64 experts
// of 896, two shared, 4 bits 22.2 / 21.7 / 20.4 / 20.5; d 2048, 64 of 1408, two shared, 4 bits 2 tokens 31.3 / 28.0 / 26.8 / 29.3, 8 tokens
// 59 / 48 / 43 / 46; 16 tokens 84 / 66 / 58 / 60; 128 of 768, bf16 one token 36.8 / 35.1 / 33.6 / 33.7, 8 tokens 100 / 84 / 78 / 81.
constexpr int SPLITS = 4, DOWN_WAVES = 8;

template <bool QUANT>
__global__ __launch_bounds__(64 * DOWN_WAVES) void decode_down_kernel(DownArgs a) {
  __shared__ float s_out[DOWN_WAVES][TOKENS][36];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), T = a.bounds.T;
  const int cb = (int)blockIdx.x, split = (int)blockIdx.y, d = a.routed.N;
  const int listed = a.list != nullptr ? list_length(a.list, a.bounds) : 0, units = listed + a.n_shared, waves = DOWN_WAVES * SPLITS;
  // parts of a reduction: as many as there are wavefronts for
  const int parts = units > 0 && units < waves ? waves / units : 1, items = units * parts;
  f32x4_t total[2] = {f32x4_t{0.f, 0.f, 0.f, 0.f}, f32x4_t{0.f, 0.f, 0.f, 0.f}};
  // Rows are tokens, whose other plane is in the row eight away.  Where two tokens eight apart list an expert (all with a shared
  // one), its tokens from 8 on are an item of their own, behind the others.
  const int again = T > 8 ? a.n_shared + (listed > 0 ? full_length(a.list, listed) : 0) : 0;
  for (int item = wave * SPLITS + split; item < items + again * parts; item += waves) {   // uniform
    const bool second = item >= items;
    const int place = second ? item - items : item, part = place % parts;
    int u = place / parts;
    const bool shared = u < a.n_shared;
    if (second && !shared) u = a.n_shared + full_unit(a.list, u - a.n_shared, listed);
    DecodeMatrix M;
#define FMOE_SEL(f) M.f = shared ? a.shared.f : a.routed.f
    FMOE_SEL(Bp); FMOE_SEL(Sp); FMOE_SEL(group_stride); FMOE_SEL(scale_stride); FMOE_SEL(nbw); FMOE_SEL(N); FMOE_SEL(K);
#undef FMOE_SEL
    fmoe_unit unit{u, 0, (1u << T) - 1u};
    f32x4_t gate = {1.f, 1.f, 1.f, 1.f};
    if (!shared) {
      unit = load_unit(a.list, u - a.n_shared, a.bounds);
      gate = *reinterpret_cast<const f32x4_t*>(&a.list->gate[u - a.n_shared][4 * (lane >> 4)]);
    }
    const bool both = (unit.mask & (unit.mask >> 8)) != 0u;
    const uint32_t mask = both ? unit.mask & (second ? 0xff00u : 0xffu) : unit.mask;
    const int NT = (M.K + SBK - 1) / SBK, per = ((NT + parts - 1) / parts + 3) / 4 * 4;   // whole units of scales
    const int first = part * per, last = first + per < NT ? first + per : NT;
    if (first >= last) continue;
    // a row with neither plane of a token takes the first row of the expert, and leaves its products out
    const int t = lane & 15, plane = shared ? a.plane_shared : a.plane;
    const bool own = (mask >> t) & 1u, rest = !own && ((mask >> (t ^ 8)) & 1u);
    const int row = own || rest ? __popc(unit.mask & ((1u << (rest ? t ^ 8 : t)) - 1u)) : 0;
    const bf16_t* const h = shared ? a.h_shared + (size_t)row * 2 * plane + (size_t)u * M.K : a.h + (size_t)(unit.row0 + row) * 2 * plane;
    f32x4_t acc[1][2] = {{f32x4_t{0.f, 0.f, 0.f, 0.f}, f32x4_t{0.f, 0.f, 0.f, 0.f}}};
    accumulate<QUANT, 1>(M, unit.expert, cb, first, last, h + (rest ? plane : 0), acc);
#pragma unroll
    for (int f = 0; f < 2; ++f)
#pragma unroll
      for (int v = 0; v < 4; ++v) acc[0][f][v] = plus_32_apart(acc[0][f][v]);   // rows eight apart
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      if (!((mask >> (4 * (lane >> 4) + v)) & 1u)) continue;
      total[0][v] = fmaf(gate[v], acc[0][0][v], total[0][v]);
      total[1][v] = fmaf(gate[v], acc[0][1][v], total[1][v]);
    }
  }
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    s_out[wave][4 * (lane >> 4) + v][lane & 15] = total[0][v];
    s_out[wave][4 * (lane >> 4) + v][16 + (lane & 15)] = total[1][v];
  }
  __syncthreads();
  static_assert(TOKENS * 32 == 64 * DOWN_WAVES, "an output a thread");
  const int t = (int)threadIdx.x >> 5, c = threadIdx.x & 31, col = cb * 32 + c;
  if (t >= T || col >= d) return;
  float sum = 0.0f;
#pragma unroll
  for (int w = 0; w < DOWN_WAVES; ++w) sum += s_out[w][t][c];
  a.part[((size_t)split * T + t) * d + col] = sum;
}

// out = residual + the sums of the workgroups that share columns, in order: two outputs a thread, all their loads at once.
__global__ __launch_bounds__(64) void decode_join_kernel(const float* __restrict__ part, int n, const bf16_t* residual, bf16_t* out) {
  const int i = ((int)blockIdx.x * 64 + (int)threadIdx.x) * 2;   // n is a multiple of eight
  if (i >= n) return;
  float2 v[SPLITS];
#pragma unroll
  for (int s = 0; s < SPLITS; ++s) v[s] = *reinterpret_cast<const float2*>(part + (size_t)s * n + i);
  const uint32_t r = residual != nullptr ? *reinterpret_cast<const uint32_t*>(residual + i) : 0u;
  float2 sum = v[0];
#pragma unroll
  for (int s = 1; s < SPLITS; ++s) sum = float2{sum.x + v[s].x, sum.y + v[s].y};
  if (residual != nullptr) sum = float2{__uint_as_float(r << 16) + sum.x, __uint_as_float(r & 0xffff0000u) + sum.y};
  *reinterpret_cast<uint32_t*>(out + i) = (uint32_t)f32_to_bf16(sum.x) | ((uint32_t)f32_to_bf16(sum.y) << 16);
}

DecodeMatrix decode_matrix(const fmoe_ctx* ctx, int which) {
  const PackedMatrix m = packed_matrix(ctx->cfg, which);
  DecodeMatrix q{};
  if (m.groups == 0) return q;
  q.nbw = m.nbw; q.N = m.N; q.K = m.K;
  if (ctx->quant) {
    size_t codes;
    const size_t bytes = fmoe_quant_bytes(ctx, which, &codes);
    const char* const base = static_cast<const char*>(ctx->pq[which]);
    q.Bp = reinterpret_cast<const u32x4_t*>(base);
    q.Sp = reinterpret_cast<const u32x4_t*>(base + codes);
    q.group_stride = (long long)(codes / 16 / m.groups);
    q.scale_stride = (long long)((bytes - codes) / 16 / m.groups);
  } else {
    const void* const packed[4] = {ctx->pk_gate_up, ctx->pk_down, ctx->pk_sgate_up, ctx->pk_sdown};
    q.Bp = static_cast<const u32x4_t*>(packed[which]);
    q.group_stride = (long long)(fmoe_packed_bytes(ctx, which) / 16 / m.groups);
  }
  return q;
}

// Workspace behind the layer's
struct ExtraLayout {
  size_t list, part, h, h_shared, total;
};
ExtraLayout extra_layout(const fmoe_ctx* ctx, int T) {
  const fmoe_config& c = ctx->cfg;
  ExtraLayout L{};
  auto take = [&](size_t bytes) { const size_t at = L.total; L.total += (bytes + 255) / 256 * 256; return at; };
  L.list = take(sizeof(fmoe_unit_list));
  L.part = take((size_t)SPLITS * T * c.d_model * 4);
  L.h = take((size_t)T * ctx->kmax * c.d_ffn * 4);
  L.h_shared = take((size_t)T * c.n_shared * c.d_ffn_shared * 4);
  return L;
}

}  // namespace

size_t decode_extra_bytes(const fmoe_ctx* ctx, int T) { return extra_layout(ctx, T).total; }

int launch_layer_decode(const fmoe_ctx* ctx, const fmoe_select_params* params, const fmoe_norm_params* norm, const void* x,
                        const void* delta, const uint8_t* is_visual, const float* select_bias, int T, int add_residual, void* out,
                        int32_t* topk_idx, float* topk_gate, void* ws, const fmoe_ws_layout& L, hipStream_t stream) {
  const fmoe_config& c = ctx->cfg;
  const int d = c.d_model, E = c.n_experts, F = c.d_ffn, Ft = c.n_shared * c.d_ffn_shared;
  char* const base = static_cast<char*>(ws);
  char* const behind = base + L.total;
  const ExtraLayout X = extra_layout(ctx, T);
  bf16_t* const n_ws = reinterpret_cast<bf16_t*>(base + L.x_merged);
  bf16_t* const h_ws = reinterpret_cast<bf16_t*>(base + L.y);          // (T rows; y has no other use here)
  float* const logits = reinterpret_cast<float*>(base + L.probs);
  if (topk_idx == nullptr) topk_idx = reinterpret_cast<int32_t*>(base + L.topk_idx);
  if (topk_gate == nullptr) topk_gate = reinterpret_cast<float*>(base + L.topk_gate);
  const ListBounds bounds{E, T, T * ctx->kmax};
  fmoe_unit_list* const list = reinterpret_cast<fmoe_unit_list*>(behind + X.list);
  const bf16_t* const xb = static_cast<const bf16_t*>(x);
  const bool sum = delta != nullptr, normed = norm != nullptr;
  const bf16_t* const h = sum ? h_ws : xb;
  const bf16_t* const n = normed ? n_ws : h;
  {
    LogitArgs a{xb, static_cast<const bf16_t*>(delta), normed ? norm->weight : nullptr, normed && norm->weight_dtype == FMOE_BF16,
                normed ? norm->eps : 0.0f, 1.0 / (double)d, T, d, E, (d + 127) / 128 * 8, ctx->router_wp, ctx->router_bias, sum ? h_ws : nullptr,
                normed ? n_ws : nullptr, logits};
    const size_t row = (size_t)a.groups * 32, room = 48 << 10;   // bytes of a token's row in LDS
    const int ebs = (E + LOGIT_EXPERTS - 1) / LOGIT_EXPERTS;
    int tb = ebs * T <= 256 ? 1 : ebs * T <= 512 ? 2 : 4;         // a workgroup a CU, then fewer passes over the weights
    while (row * tb > room) tb >>= 1;
    const dim3 grid(ebs, (T + tb - 1) / tb), block(64 * LOGIT_WAVES);
    fmoe_prof_scope prof(ctx, SLOT_ROUTE, stream);
    if (tb == 4) hipLaunchKernelGGL(decode_logits_kernel<4>, grid, block, row * 4, stream, a);
    else if (tb == 2) hipLaunchKernelGGL(decode_logits_kernel<2>, grid, block, row * 2, stream, a);
    else hipLaunchKernelGGL(decode_logits_kernel<1>, grid, block, row, stream, a);
  }
  if (ctx->kmax > 0) {
    const fmoe_select_params softmax{0, 1, 1, 0, 1.0f};
    const int rc = launch_select(ctx, params != nullptr ? params : &softmax, logits, FMOE_F32, is_visual, select_bias, T, nullptr,
                                 topk_idx, topk_gate, stream, list);
    if (rc != FMOE_OK) return rc;
  }
  GateUpArgs g{};
  g.routed = decode_matrix(ctx, 0); g.shared = decode_matrix(ctx, 2);
  g.n = n; g.list = ctx->kmax > 0 ? list : nullptr; g.bounds = bounds;
  g.h = reinterpret_cast<bf16_t*>(behind + X.h); g.h_shared = reinterpret_cast<bf16_t*>(behind + X.h_shared);
  const int pairs = T * ctx->kmax, units = pairs < E ? pairs : E;
  {
    // Column blocks a wavefront.  4 bits, where sixteen rows are more to read than the weights beside them; one / two, us a call: d 2048,
    // 64 experts of 1408, two shared 2 tokens 26.6 / 30.1, 4 tokens 32.3 / 33.5, 8 tokens 47.0 / 43.3, 16 tokens 72 / 58; d 1280, 64
    // of 896 12 tokens 34.6 / 32.7; bf16 weights (four times the bytes): 128 of 768 2 tokens 42.9 / 46.2, 8 tokens 78.2 / 78.4
    const int blocks = g.shared.nbw + units * g.routed.nbw, ncb = ctx->quant && T > 4 ? 2 : 1;
    const dim3 grid((g.shared.nbw + ncb - 1) / ncb + units * ((g.routed.nbw + ncb - 1) / ncb));
    fmoe_prof_scope prof(ctx, SLOT_GEMM1, stream);
    if (blocks > 0) {
      if (!ctx->quant) hipLaunchKernelGGL((decode_gate_up_kernel<false, 1>), grid, dim3(64), 0, stream, g);
      else if (ncb == 1) hipLaunchKernelGGL((decode_gate_up_kernel<true, 1>), grid, dim3(64), 0, stream, g);
      else hipLaunchKernelGGL((decode_gate_up_kernel<true, 2>), grid, dim3(64), 0, stream, g);
    }
  }
  DownArgs a{};
  a.routed = decode_matrix(ctx, 1); a.shared = decode_matrix(ctx, 3);
  a.n_shared = c.n_shared;
  a.h = g.h; a.h_shared = g.h_shared; a.plane = F; a.plane_shared = Ft;
  a.list = g.list;
  a.bounds = bounds;
  a.part = reinterpret_cast<float*>(behind + X.part);
  {
    fmoe_prof_scope prof(ctx, SLOT_GEMM2, stream);
    const dim3 grid(a.routed.nbw, SPLITS), block(64 * DOWN_WAVES);
    if (ctx->quant) hipLaunchKernelGGL(decode_down_kernel<true>, grid, block, 0, stream, a);
    else hipLaunchKernelGGL(decode_down_kernel<false>, grid, block, 0, stream, a);
  }
  {
    fmoe_prof_scope prof(ctx, SLOT_COMBINE, stream);
    hipLaunchKernelGGL(decode_join_kernel, dim3((T * d / 2 + 63) / 64), dim3(64), 0, stream, a.part, T * d,
                       add_residual ? h : nullptr, static_cast<bf16_t*>(out));
  }
  FMOE_HIP_CHECK(hipGetLastError());
  return FMOE_OK;
}
