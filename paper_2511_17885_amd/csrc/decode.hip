// A whole layer for a few tokens (at most FMOE_DECODE_TOKENS, a decoding step): the addition and norm in front of it, router, choice of
// experts, their products, gates and residual.
//
//   decode_logits    h = x + delta, n = norm(h) (norm_dev.h), logits of n in 64 bits, rounded once: every workgroup takes 16 experts and
//                    one to four tokens, so that the router matrix is read by many CUs at once and no chain of additions holds it up
//   select_kernel    the choice (select.hip)
//   decode_gate_up   a wavefront per expert that any token lists and column block of 16: all tokens are the rows of the matrix
//                    instruction, whose hidden rows are kept for those that list the expert
//   decode_down      a workgroup per 32 output columns: its wavefronts share the experts (where there are fewer, also their
//                    reductions), the rows stay tokens, so that gate * product is added up in registers, then over the wavefronts
//                    in LDS in a fixed order; with more experts than a workgroup has wavefronts several of them share the columns
//                    and decode_join adds their sums
// Bound: the weights of the experts that the tokens touch; for a token or two a chain of launches and latencies.

#include "ffn_dev.h"
#include "norm_dev.h"
#include "quant_items.h"

namespace {

using rms::finite;

constexpr int TOKENS = FMOE_DECODE_TOKENS;

// ---------------------------------------------------------------------------------------------------------- norm and logits

struct LogitArgs {
  const bf16_t *x, *delta;
  const void* w;            // norm weight or null
  int w_bf16;
  float eps;
  int T, d, E, groups;      // groups of 16 k in the packed router
  const float *wp, *bias;
  bf16_t *h, *n;            // [T, d] or null
  float* logits;            // [T, E]
};

constexpr int LOGIT_WAVES = 16;

// Router weights as route.hip packs them: expert block of 16, group of 16 k, lane l: expert l % 16, k = l / 16 + 4 j, j = 0..3.
template <int TB>
__global__ __launch_bounds__(64 * LOGIT_WAVES) void decode_logits_kernel(LogitArgs a) {
  extern __shared__ __align__(16) bf16_t rows[];                // n of TB tokens, in the order of the packed weights
  __shared__ double s_sum[LOGIT_WAVES], s_part[LOGIT_WAVES][TB][16];
  constexpr int WPT = LOGIT_WAVES / TB, AHEAD = 8;              // wavefronts a token; groups of weights in flight
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int t0 = (int)blockIdx.y * TB, eb = (int)blockIdx.x, padded = a.groups * 16;
  const f32x4_t* const wp = reinterpret_cast<const f32x4_t*>(a.wp) + (size_t)eb * a.groups * 64 + lane;
  f32x4_t w[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) {                             // on their way behind the norm; past the end the last group
    const int g = wave + LOGIT_WAVES * i;
    w[i] = wp[(size_t)(g < a.groups ? g : a.groups - 1) * 64];
  }
  // a token's row: its WPT wavefronts, units of eight
  const int tb = wave / WPT, first = (wave % WPT) * 64 + lane, t = t0 + tb < a.T ? t0 + tb : a.T - 1;
  const size_t base = (size_t)t * a.d;
  const int units = a.d >> 3;
  bf16_t* const row = rows + (size_t)tb * padded;
  constexpr int HELD = 2;                                       // units a lane holds; longer rows are read again
  auto sum_of = [&](int u, rms::Unit<bf16_t>& h) {
    h.load(a.x + base + u * 8);
    if (a.delta != nullptr) {
      rms::Unit<bf16_t> dl;
      dl.load(a.delta + base + u * 8);
#pragma unroll
      for (int e = 0; e < 8; e += 2)
        h.set2(e, rms::add_rounded<bf16_t>(h.get(e), dl.get(e)), rms::add_rounded<bf16_t>(h.get(e + 1), dl.get(e + 1)));
    }
  };
  rms::Unit<bf16_t> held[HELD];
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    held[i].zero();
    if (first + 64 * WPT * i < units) sum_of(first + 64 * WPT * i, held[i]);
  }
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
    r = rms::row_scale(sum, a.d, a.eps);
  }
  const bool mine = eb == 0 && t0 + tb < a.T;                   // the first workgroups write the rows
  // element e of unit u: group u / 2, k = 8 (u % 2) + e of it, which lane group e % 4 wants as its number 2 (u % 2) + e / 4
  auto lay_out = [&](int u, const rms::Unit<bf16_t>& n) {
    bf16_t* const to = row + (u >> 1) * 16 + 2 * (u & 1);
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<uint32_t*>(to + 4 * q) = (__float_as_uint(n.get(q)) >> 16) | (__float_as_uint(n.get(q + 4)) & 0xffff0000u);
  };
  auto place = [&](int u, const rms::Unit<bf16_t>& h) {
    rms::Unit<bf16_t> n = h;
    if (a.w != nullptr) {
      float f[8];
      if (a.w_bf16) rms::load_weights<bf16_t>(a.w, u * 8, f);   // uniform
      else rms::load_weights<float>(a.w, u * 8, f);
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
    if (first + 64 * WPT * i < units) place(first + 64 * WPT * i, held[i]);
  for (int u = first + 64 * WPT * HELD; u < units; u += 64 * WPT) {
    rms::Unit<bf16_t> h;
    sum_of(u, h);
    place(u, h);
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
  const int q4 = (lane >> 4) * 4;
  for (int g0 = wave; g0 < a.groups; g0 += LOGIT_WAVES * AHEAD) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int g = g0 + LOGIT_WAVES * i;
      if (g < a.groups) {   // uniform
#pragma unroll
        for (int b = 0; b < TB; ++b) {
          const uint2 v = *reinterpret_cast<const uint2*>(rows + (size_t)b * padded + g * 16 + q4);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t p = j < 2 ? v.x : v.y;
            acc[b] = fma((double)__uint_as_float(j & 1 ? p & 0xffff0000u : p << 16), (double)w[i][j], acc[b]);
          }
        }
      }
      const int next = g + LOGIT_WAVES * AHEAD;
      if (next < a.groups) w[i] = wp[(size_t)next * 64];
    }
  }
#pragma unroll
  for (int b = 0; b < TB; ++b) {
    double v = acc[b];
    v += __shfl_xor(v, 16, 64);
    v += __shfl_xor(v, 32, 64);
    if (lane < 16) s_part[wave][b][lane] = v;
  }
  __syncthreads();
  if (tid < 16 * TB) {
    const int b = tid >> 4, e = eb * 16 + (tid & 15);
    double v = 0.0;
#pragma unroll
    for (int i = 0; i < LOGIT_WAVES; ++i) v += s_part[i][b][tid & 15];
    if (t0 + b < a.T && e < a.E) a.logits[(size_t)(t0 + b) * a.E + e] = (float)(a.bias != nullptr ? v + (double)a.bias[e] : v);
  }
}

// -------------------------------------------------------------------------------------------------------- experts of the step

struct Unit {               // an expert that a token lists
  int expert, row0;         // its first hidden row
  uint32_t mask;            // tokens
};

// The experts that are listed, ascending, from the lists of all tokens; by all threads of a workgroup.  Returns how many.
__device__ __forceinline__ int find_units(const int32_t* idx, int T, int Kmax, int E, uint32_t* s_mask, Unit* s_unit, int* s_n) {
  static_assert(FMOE_MAX_EXPERTS == 256, "four experts a lane");
  for (int i = threadIdx.x; i < FMOE_MAX_EXPERTS; i += blockDim.x) s_mask[i] = 0u;
  __syncthreads();
  for (int i = threadIdx.x; i < T * Kmax; i += blockDim.x) {
    const int e = idx[i];
    if (e >= 0 && e < E) atomicOr(&s_mask[e], 1u << (i / Kmax));
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x;
    uint32_t m[4];
    int rows = 0, some = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      m[q] = s_mask[4 * lane + q];
      rows += __popc(m[q]);
      some += m[q] != 0u;
    }
    int row = wave_scan(rows) - rows, rank = wave_scan(some) - some;
    if (lane == 63) *s_n = rank + some;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (m[q] == 0u) continue;
      s_unit[rank++] = Unit{4 * lane + q, row, m[q]};
      row += __popc(m[q]);
    }
  }
  __syncthreads();
  return *s_n;
}

// Weights of one packed matrix, bf16 (ffn.hip) or 4 bits (ffn_quant.hip): what a wavefront needs of a column block
struct DecodeMatrix {
  const u32x4_t *Bp, *Sp;
  long long group_stride, scale_stride;   // 16-byte units between groups
  int nbw, N, K;                          // column blocks, output features, reduction
};

// acc[f] += rows x weights over the k tiles (64 wide) first .. last-1 of column block cb: fragment f is gate / up or a half of 32
// columns, lane l has row l % 16 from `a` (the lane's own address; K elements).  A ring of k tiles in registers; loads past the last
// tile return zeros and fetch nothing.
template <bool QUANT>
__device__ __forceinline__ void accumulate(const DecodeMatrix& M, int group, int cb, int first, int last, const bf16_t* a,
                                           f32x4_t (&acc)[2]) {
  constexpr int S = QUANT ? 8 : 4, PIECES = QUANT ? 1 : 4;
  const int lane = threadIdx.x & 63, NT = (M.K + SBK - 1) / SBK, NT4 = (NT + 3) / 4;
  const size_t tile_bytes = QUANT ? 1024 : 16384;
  const char* const b0 = reinterpret_cast<const char*>(M.Bp + (size_t)group * M.group_stride) +
                         (QUANT ? (size_t)cb * NT * 1024 : (size_t)(cb >> 2) * NT * 16384 + (cb & 3) * 4096) + first * tile_bytes;
  const int tiles = last - first;
  const __amdgpu_buffer_rsrc_t b_rsrc =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(b0), 0, (int)(QUANT ? tiles * 1024 : (tiles - 1) * 16384 + 4096), 0x00020000);
  const __amdgpu_buffer_rsrc_t s_rsrc = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<u32x4_t*>(QUANT ? M.Sp + (size_t)group * M.scale_stride + ((size_t)cb * NT4 + first / 4) * 16 : nullptr), 0,
      QUANT ? (tiles + 3) / 4 * 256 : 0, 0x00020000);
  const uint32_t lane16 = (uint32_t)lane * 16u, column16 = (uint32_t)(lane & 15) * 16u;
  const int kq = (lane >> 4) * 8;
  u32x4_t breg[S][PIECES], sreg[S / 4], areg[S][2];
  auto load_b = [&](int slot, int t) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
      breg[slot][i] = __builtin_amdgcn_raw_buffer_load_b128(b_rsrc, lane16 + (uint32_t)(t * (int)tile_bytes + i * 1024), 0, 0);
  };
  auto load_s = [&](int slot, int t4) { sreg[slot] = __builtin_amdgcn_raw_buffer_load_b128(s_rsrc, column16 + (uint32_t)t4 * 256u, 0, 0); };
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
      u32x4_t b[2];
      if constexpr (QUANT) {
        const uint32_t sc = sreg[slot / 4][slot % 4];
        b[0] = s == 0 ? dequantize<0>(breg[slot][0][0], sc) : dequantize<2>(breg[slot][0][2], sc);
        b[1] = s == 0 ? dequantize<1>(breg[slot][0][1], sc) : dequantize<3>(breg[slot][0][3], sc);
      } else {
        b[0] = breg[slot][2 * s];
        b[1] = breg[slot][2 * s + 1];
      }
#pragma unroll
      for (int f = 0; f < 2; ++f)
        acc[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, __builtin_bit_cast(bf16x8_t, b[f]), acc[f], 0, 0, 0);
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

struct GateUpArgs {
  DecodeMatrix routed, shared;
  const bf16_t* n;          // [T, K]
  const int32_t* idx;       // [T, Kmax]
  int T, Kmax, E;
  bf16_t *h, *h_shared;     // hidden rows [., routed.N] of the pairs by expert and token; [T, shared.N]
};

template <bool QUANT>
__global__ __launch_bounds__(64, 2) void decode_gate_up_kernel(GateUpArgs a) {
  __shared__ uint32_t s_mask[FMOE_MAX_EXPERTS];
  __shared__ Unit s_unit[FMOE_MAX_EXPERTS];
  __shared__ int s_n;
  const int lane = threadIdx.x;
  int cb = (int)blockIdx.x;
  const bool shared = cb < a.shared.nbw;
  Unit unit{0, 0, (1u << a.T) - 1u};
  if (!shared) {
    cb -= a.shared.nbw;
    const int u = cb / a.routed.nbw;
    cb -= u * a.routed.nbw;
    if (u >= find_units(a.idx, a.T, a.Kmax, a.E, s_mask, s_unit, &s_n)) return;
    unit.expert = __builtin_amdgcn_readfirstlane(s_unit[u].expert);
    unit.row0 = __builtin_amdgcn_readfirstlane(s_unit[u].row0);
    unit.mask = (uint32_t)__builtin_amdgcn_readfirstlane((int)s_unit[u].mask);
  }
  DecodeMatrix M;
#define FMOE_SEL(f) M.f = shared ? a.shared.f : a.routed.f
  FMOE_SEL(Bp); FMOE_SEL(Sp); FMOE_SEL(group_stride); FMOE_SEL(scale_stride); FMOE_SEL(nbw); FMOE_SEL(N); FMOE_SEL(K);
#undef FMOE_SEL
  bf16_t* const h = shared ? a.h_shared : a.h;
  const int token = (lane & 15) < a.T ? lane & 15 : a.T - 1;
  f32x4_t acc[2] = {f32x4_t{0.f, 0.f, 0.f, 0.f}, f32x4_t{0.f, 0.f, 0.f, 0.f}};
  accumulate<QUANT>(M, unit.expert, cb, 0, (M.K + SBK - 1) / SBK, a.n + (size_t)token * M.K, acc);
  const int col = cb * 16 + (lane & 15);
#pragma unroll
  for (int v = 0; v < 4; ++v) {   // accumulator register v of lane l: row 4*(l/16) + v, column l%16
    const int t = 4 * (lane >> 4) + v;
    if (((unit.mask >> t) & 1u) && col < M.N)
      h[(size_t)(unit.row0 + __popc(unit.mask & ((1u << t) - 1u))) * M.N + col] = f32_to_bf16(silu_mul_bf16(acc[0][v], acc[1][v]));
  }
}

struct DownArgs {
  DecodeMatrix routed, shared;   // (a group per shared expert)
  int n_shared;
  const bf16_t *h, *h_shared;
  int ld_shared;
  const int32_t* idx;
  const float* gate;
  int T, Kmax, E, splits;
  const bf16_t* residual;        // [T, d] or null
  bf16_t* out;                   // [T, d]
  float* part;                   // [splits, T, d] with more than one split
};

template <bool QUANT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void decode_down_kernel(DownArgs a) {
  __shared__ uint32_t s_mask[FMOE_MAX_EXPERTS];
  __shared__ Unit s_unit[FMOE_MAX_EXPERTS];
  __shared__ int s_n;
  __shared__ float s_gate[TOKENS * FMOE_MAX_TOPK];
  __shared__ int32_t s_idx[TOKENS * FMOE_MAX_TOPK];
  __shared__ float s_out[WAVES][TOKENS][36];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int cb = (int)blockIdx.x, split = (int)blockIdx.y, d = a.routed.N;
  const int pairs = a.T * a.Kmax;
  for (int i = threadIdx.x; i < pairs; i += 64 * WAVES) {
    s_gate[i] = a.gate[i];
    s_idx[i] = a.idx[i];
  }
  const int n_units = a.Kmax > 0 ? find_units(a.idx, a.T, a.Kmax, a.E, s_mask, s_unit, &s_n) : 0;
  const int units = n_units + a.n_shared, waves = WAVES * a.splits;
  // parts of a reduction: as many as there are wavefronts for, whole groups of four k tiles each
  const int parts = units > 0 && units < waves ? waves / units : 1;
  f32x4_t total[2] = {f32x4_t{0.f, 0.f, 0.f, 0.f}, f32x4_t{0.f, 0.f, 0.f, 0.f}};
  for (int item = split * WAVES + wave; item < units * parts; item += waves) {   // uniform
    const int u = item / parts, part = item - u * parts;
    const bool shared = u < a.n_shared;
    DecodeMatrix M;
#define FMOE_SEL(f) M.f = shared ? a.shared.f : a.routed.f
    FMOE_SEL(Bp); FMOE_SEL(Sp); FMOE_SEL(group_stride); FMOE_SEL(scale_stride); FMOE_SEL(nbw); FMOE_SEL(N); FMOE_SEL(K);
#undef FMOE_SEL
    Unit unit{u, 0, (1u << a.T) - 1u};
    if (!shared) {
      const Unit& s = s_unit[u - a.n_shared];
      unit.expert = __builtin_amdgcn_readfirstlane(s.expert);
      unit.row0 = __builtin_amdgcn_readfirstlane(s.row0);
      unit.mask = (uint32_t)__builtin_amdgcn_readfirstlane((int)s.mask);
    }
    const int NT = (M.K + SBK - 1) / SBK, per = ((NT + parts - 1) / parts + 3) / 4 * 4;
    const int first = part * per, last = first + per < NT ? first + per : NT;
    if (first >= last) continue;
    // rows are tokens; one that does not list the expert takes the row of the first that does, which its gate leaves out
    const int t = lane & 15;
    const int row = (unit.mask >> t) & 1u ? __popc(unit.mask & ((1u << t) - 1u)) : 0;
    const bf16_t* const src = shared ? a.h_shared + (size_t)row * a.ld_shared + (size_t)u * M.K : a.h + (size_t)(unit.row0 + row) * M.K;
    f32x4_t acc[2] = {f32x4_t{0.f, 0.f, 0.f, 0.f}, f32x4_t{0.f, 0.f, 0.f, 0.f}};
    accumulate<QUANT>(M, unit.expert, cb, first, last, src, acc);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int to = 4 * (lane >> 4) + v;
      float g = 1.0f;
      if (!shared) {
        for (int s = 0; s < a.Kmax; ++s)
          if (to < a.T && s_idx[to * a.Kmax + s] == unit.expert) g = s_gate[to * a.Kmax + s];
      }
      if ((unit.mask >> to) & 1u) {
        total[0][v] = fmaf(g, acc[0][v], total[0][v]);
        total[1][v] = fmaf(g, acc[1][v], total[1][v]);
      }
    }
  }
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    s_out[wave][4 * (lane >> 4) + v][lane & 15] = total[0][v];
    s_out[wave][4 * (lane >> 4) + v][16 + (lane & 15)] = total[1][v];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.T * 32; i += 64 * WAVES) {
    const int t = i >> 5, c = i & 31, col = cb * 32 + c;
    if (col >= d) continue;
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sum += s_out[w][t][c];
    const size_t at = (size_t)t * d + col;
    if (a.splits > 1) a.part[((size_t)split * a.T) * d + at] = sum;
    else a.out[at] = f32_to_bf16(a.residual != nullptr ? bf16_to_f32(a.residual[at]) + sum : sum);
  }
}

__global__ __launch_bounds__(256) void decode_join_kernel(const float* __restrict__ part, int splits, int n, const bf16_t* residual,
                                                          bf16_t* out) {
  const int i = ((int)blockIdx.x * 256 + (int)threadIdx.x) * 4;   // n is a multiple of eight
  if (i >= n) return;
  f32x4_t sum = *reinterpret_cast<const f32x4_t*>(part + i);
  for (int s = 1; s < splits; ++s) {
    const f32x4_t v = *reinterpret_cast<const f32x4_t*>(part + (size_t)s * n + i);
    sum = f32x4_t{sum[0] + v[0], sum[1] + v[1], sum[2] + v[2], sum[3] + v[3]};
  }
  uint2 r = {0u, 0u};
  if (residual != nullptr) r = *reinterpret_cast<const uint2*>(residual + i);
  const float o[4] = {__uint_as_float(r.x << 16) + sum[0], __uint_as_float(r.x & 0xffff0000u) + sum[1],
                      __uint_as_float(r.y << 16) + sum[2], __uint_as_float(r.y & 0xffff0000u) + sum[3]};
  *reinterpret_cast<uint2*>(out + i) = uint2{(uint32_t)f32_to_bf16(o[0]) | ((uint32_t)f32_to_bf16(o[1]) << 16),
                                             (uint32_t)f32_to_bf16(o[2]) | ((uint32_t)f32_to_bf16(o[3]) << 16)};
}

constexpr int DOWN_WAVES = 8;
int down_splits(const fmoe_ctx* ctx, int T) {
  const int pairs = T * ctx->kmax, E = ctx->cfg.n_experts;
  const int units = (pairs < E ? pairs : E) + ctx->cfg.n_shared;   // that the call can have
  const int splits = (units + DOWN_WAVES - 1) / DOWN_WAVES;
  return splits < 1 ? 1 : splits > 8 ? 8 : splits;
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

}  // namespace

// Bytes of partial sums behind the layer's workspace
size_t decode_part_bytes(const fmoe_ctx* ctx, int T) {
  const int splits = down_splits(ctx, T);
  return splits > 1 ? (size_t)splits * T * ctx->cfg.d_model * 4 : 0;
}

int launch_layer_decode(const fmoe_ctx* ctx, const fmoe_select_params* params, const fmoe_norm_params* norm, const void* x,
                        const void* delta, const uint8_t* is_visual, const float* select_bias, int T, int add_residual, void* out,
                        int32_t* topk_idx, float* topk_gate, void* ws, const fmoe_ws_layout& L, hipStream_t stream) {
  const fmoe_config& c = ctx->cfg;
  const int d = c.d_model, E = c.n_experts, F = c.d_ffn, Ft = c.n_shared * c.d_ffn_shared;
  char* const base = static_cast<char*>(ws);
  bf16_t* const n_ws = reinterpret_cast<bf16_t*>(base + L.x_merged);
  bf16_t* const h_ws = reinterpret_cast<bf16_t*>(base + L.y);          // (T rows; y has no other use here)
  float* const logits = reinterpret_cast<float*>(base + L.probs);
  if (topk_idx == nullptr) topk_idx = reinterpret_cast<int32_t*>(base + L.topk_idx);
  if (topk_gate == nullptr) topk_gate = reinterpret_cast<float*>(base + L.topk_gate);
  const bf16_t* const xb = static_cast<const bf16_t*>(x);
  const bool sum = delta != nullptr, normed = norm != nullptr;
  const bf16_t* const h = sum ? h_ws : xb;
  const bf16_t* const n = normed ? n_ws : h;
  {
    LogitArgs a{xb, static_cast<const bf16_t*>(delta), normed ? norm->weight : nullptr, normed && norm->weight_dtype == FMOE_BF16,
                normed ? norm->eps : 0.0f, T, d, E, (d + 127) / 128 * 8, ctx->router_wp, ctx->router_bias, sum ? h_ws : nullptr,
                normed ? n_ws : nullptr, logits};
    const size_t row = (size_t)a.groups * 32, room = 48 << 10;   // bytes of a token's row in LDS
    const int tb = T >= 4 && row * 4 <= room ? 4 : T >= 2 && row * 2 <= room ? 2 : 1;
    const dim3 grid((E + 15) / 16, (T + tb - 1) / tb), block(64 * LOGIT_WAVES);
    fmoe_prof_scope prof(ctx, SLOT_ROUTE, stream);
    if (tb == 4) hipLaunchKernelGGL(decode_logits_kernel<4>, grid, block, row * 4, stream, a);
    else if (tb == 2) hipLaunchKernelGGL(decode_logits_kernel<2>, grid, block, row * 2, stream, a);
    else hipLaunchKernelGGL(decode_logits_kernel<1>, grid, block, row, stream, a);
  }
  if (ctx->kmax > 0) {
    const fmoe_select_params softmax{0, 1, 1, 0, 1.0f};
    const int rc = launch_select(ctx, params != nullptr ? params : &softmax, logits, FMOE_F32, is_visual, select_bias, T, nullptr,
                                 topk_idx, topk_gate, stream);
    if (rc != FMOE_OK) return rc;
  }
  GateUpArgs g{};
  g.routed = decode_matrix(ctx, 0); g.shared = decode_matrix(ctx, 2);
  g.n = n; g.idx = topk_idx; g.T = T; g.Kmax = ctx->kmax; g.E = E;
  g.h = reinterpret_cast<bf16_t*>(base + L.h); g.h_shared = reinterpret_cast<bf16_t*>(base + L.h_shared);
  const int pairs = T * ctx->kmax, units = pairs < E ? pairs : E;
  {
    fmoe_prof_scope prof(ctx, SLOT_GEMM1, stream);
    const unsigned blocks = (unsigned)g.shared.nbw + (unsigned)units * (unsigned)g.routed.nbw;
    if (blocks > 0 && ctx->quant) hipLaunchKernelGGL(decode_gate_up_kernel<true>, dim3(blocks), dim3(64), 0, stream, g);
    else if (blocks > 0) hipLaunchKernelGGL(decode_gate_up_kernel<false>, dim3(blocks), dim3(64), 0, stream, g);
  }
  const int splits = down_splits(ctx, T);
  DownArgs a{};
  a.routed = decode_matrix(ctx, 1); a.shared = decode_matrix(ctx, 3);
  a.n_shared = c.n_shared;
  a.h = g.h; a.h_shared = g.h_shared; a.ld_shared = Ft;
  a.idx = topk_idx; a.gate = topk_gate;
  a.T = T; a.Kmax = ctx->kmax; a.E = E; a.splits = splits;
  a.residual = add_residual ? h : nullptr;
  a.out = static_cast<bf16_t*>(out);
  a.part = reinterpret_cast<float*>(base + L.total);
  const dim3 grid(a.routed.nbw, splits), block(64 * DOWN_WAVES);
  {
    fmoe_prof_scope prof(ctx, SLOT_GEMM2, stream);
    if (ctx->quant) hipLaunchKernelGGL((decode_down_kernel<true, DOWN_WAVES>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((decode_down_kernel<false, DOWN_WAVES>), grid, block, 0, stream, a);
  }
  if (splits > 1) {
    fmoe_prof_scope prof(ctx, SLOT_COMBINE, stream);
    hipLaunchKernelGGL(decode_join_kernel, dim3((T * d / 4 + 255) / 256), dim3(256), 0, stream, a.part, splits, T * d, a.residual, a.out);
  }
  FMOE_HIP_CHECK(hipGetLastError());
  return FMOE_OK;
}
