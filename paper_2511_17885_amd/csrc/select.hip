// Experts of a token from its router logits: scores (softmax or sigmoid), a balance bias that decides but does not weigh,
// groups of experts, the list of the k largest, gates; and the gradient of gates and scores with respect to the logits.
//
//   score  s_e = softmax_e(z) or 1 / (1 + exp(-z_e));  key u_e = s_e + b_e, without a bias the order of z_e itself
//   gates  c * softmax over the list of log(s) (renormalised) or c * s
// log(s) is z (softmax: the row's normaliser cancels) or -log(1 + exp(-z)); as a softmax over the list the renormalised
// gates need no division by a sum of scores that may have underflowed.
//
// Keys that come from a score are defined in 64 bits: two scores in 32 bits can be equal or change places where the
// logits differ, and with thousands of tokens some pair of neighbours does.  They are compared in 32 bits first, with the
// exponential and reciprocal of the hardware.  A key is then off by at most 2^-21 of the largest score a token can have and
// half a rounding of its own; where two keys that are next to each other in the list, or on either side of its end, or
// two groups on either side of theirs, are not further apart than twice that (taken twice), the wavefront does it again in
// 64 bits.  One wavefront in a hundred does for 256 experts with a bias of deviation 0.1.
//
// Sixteen lanes have a token (four tokens a wavefront), lane j of them the experts 64 q + 4 j + i: a row is read in
// pieces of 16 bytes, and a reduction over the row is one over a lane's registers and four steps inside the vector unit.

#include <float.h>

#include <type_traits>

#include "common.h"
#include "rows.h"

namespace {

constexpr int ROWS = 16;   // tokens per block

struct SelectArgs {
  const void* z;
  const uint8_t* is_visual;   // or null: text
  const float* bias;          // or null
  int T, E, k_text, k_visual, Kmax;
  int sigmoid, renorm, groups, topk_groups, sum_two;
  int group_size, group_mul;  // e / group_size == e * group_mul >> 16 for e < 256
  float scale;
  float* scores;              // or null
  int32_t* idx;
  float* gate;
};

// A logit as the definitions take it: NaN is masked like -inf, +inf is the largest finite number.
__device__ __forceinline__ float clean(float z) { return z > -INFINITY ? fminf(z, FLT_MAX) : -INFINITY; }

__device__ __forceinline__ float log_sigmoid(float z) { return fminf(z, 0.0f) - log1pf(expf(-fabsf(z))); }

// A lane's elements of a row of E, four at a time where rows are whole fours (their starts then are aligned); past the end
// the first ones again.
template <typename T, int NQ>
__device__ __forceinline__ void read_row(const T* __restrict__ row, int E, int j, T (&v)[4 * NQ]) {
  typedef T four_t __attribute__((ext_vector_type(4)));
  if ((E & 3) == 0) {   // uniform
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int e = 64 * q + 4 * j;
      const four_t w = *reinterpret_cast<const four_t*>(row + (e < E ? e : 0));
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * q + i] = w[i];
    }
  } else {
#pragma unroll
    for (int r = 0; r < 4 * NQ; ++r) {
      const int e = 64 * (r >> 2) + 4 * j + (r & 3);
      v[r] = row[e < E ? e : 0];
    }
  }
}
template <typename T, int NQ>
__device__ __forceinline__ void write_row(T* __restrict__ row, int E, int j, const T (&v)[4 * NQ]) {
  typedef T four_t __attribute__((ext_vector_type(4)));
  if ((E & 3) == 0) {
#pragma unroll
    for (int q = 0; q < NQ; ++q)
      if (64 * q + 4 * j < E)
        *reinterpret_cast<four_t*>(row + 64 * q + 4 * j) = four_t{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
  } else {
#pragma unroll
    for (int r = 0; r < 4 * NQ; ++r)
      if (64 * (r >> 2) + 4 * j + (r & 3) < E) row[64 * (r >> 2) + 4 * j + (r & 3)] = v[r];
  }
}
// A lane's logits of row t; experts past E are masked.
template <typename ZT, int NQ>
__device__ __forceinline__ void load_row(const ZT* __restrict__ z, int t, int E, int j, float (&v)[4 * NQ]) {
  ZT raw[4 * NQ];
  read_row<ZT, NQ>(z + (size_t)t * E, E, j, raw);
#pragma unroll
  for (int r = 0; r < 4 * NQ; ++r) v[r] = 64 * (r >> 2) + 4 * j + (r & 3) < E ? clean(to_f32(raw[r])) : -INFINITY;
}

// Of a row's logits: the largest (0 if all are masked) and the sum of exp(z - largest).
template <int N>
__device__ __forceinline__ float row_largest(const float (&z)[N]) {
  float m = z[0];
#pragma unroll
  for (int r = 1; r < N; ++r) m = larger(m, z[r]);
  m = row_max(m);
  return m > -INFINITY ? m : 0.0f;
}
template <int N>
__device__ __forceinline__ float row_exp_sum(const float (&z)[N], float m) {
  float s = 0.0f;
#pragma unroll
  for (int r = 0; r < N; ++r) s += expf(z[r] - m);
  return row_sum_butterfly(s);
}

// Expert of register r of a lane.
__device__ __forceinline__ int expert_of(int r, int j) { return 64 * (r >> 2) + 4 * j + (r & 3); }

// LDS written by lanes of this wavefront is read by others of it.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Masks the experts of a token's groups that do not stay.  key: what a group's score is made of; order: what ranks the
// experts; ks: the token's row in LDS.  Returns whether the scores on either side of the line are further apart than `slack`
// plus `relative` times their size (32 bits; not asked for in 64).
template <typename T, int N>
__device__ __forceinline__ bool keep_groups(const SelectArgs& a, int j, const T (&key)[N], T (&order)[N], T* ks, T slack,
                                            T relative) {
#pragma unroll
  for (int r = 0; r < N; ++r) ks[expert_of(r, j)] = key[r];
  wave_sync();
  // lane g has group g: its largest key, or the sum of its two largest
  T one = -INFINITY, two = -INFINITY;
  if (j < a.groups) {
    const T* const own = ks + j * a.group_size;
    for (int i = 0; i < a.group_size; ++i) {
      const T v = own[i];
      two = v > one ? one : larger(two, v);
      one = larger(one, v);
    }
  }
  const T score = (a.sum_two && two > -INFINITY) ? one + two : one;
  // rank among the groups: larger scores, or equal ones of lower groups, are ahead
  int ahead = 0;
  for (int g = 0; g < a.groups; ++g) {
    const T o = __shfl(score, (threadIdx.x & 48) + g, 64);
    ahead += (o > score || (o == score && g < j)) ? 1 : 0;
  }
  const bool in = j < a.groups && ahead < a.topk_groups;
  const unsigned mask = (unsigned)(__ballot(in) >> (threadIdx.x & 48)) & 0xffffu;
#pragma unroll
  for (int r = 0; r < N; ++r)
    if (!((mask >> ((expert_of(r, j) * a.group_mul >> 16) & 15)) & 1u)) order[r] = -INFINITY;   // (past E masked already)
  if (a.topk_groups == a.groups) return true;
  const T last = -row_max(in ? -score : (T)-INFINITY), next = row_max(j < a.groups && !in ? score : (T)-INFINITY);
  return next == -INFINITY || last - next > slack + relative * (fabs(last) + fabs(next));
}

// k rounds of the largest that is left (ties: lowest expert); lane j keeps entry j: its expert (-1: none) and key.
template <typename T, int N>
__device__ __forceinline__ int list_largest(int k, int rounds, int j, T (&order)[N], T& my_key) {
  int mine = -1;
  my_key = -INFINITY;
  for (int round = 0; round < rounds; ++round) {
    T v = order[0];
#pragma unroll
    for (int r = 1; r < N; ++r) v = larger(v, order[r]);
    const T top = row_max(v);
    int e = 0x7fff;
#pragma unroll
    for (int r = N - 1; r >= 0; --r) e = order[r] == top ? expert_of(r, j) : e;
    e = row_min(e);
    if (j == round && round < k && top > -INFINITY) {
      mine = e;
      my_key = top;
    }
    if (round < k) {
#pragma unroll
      for (int r = 0; r < N; ++r) order[r] = expert_of(r, j) == e ? (T)-INFINITY : order[r];
    }
  }
  return mine;
}

// KEYED: the keys are scores with a bias, or sums of scores rank the groups; else the logits are the keys.
template <typename ZT, int NQ, bool KEYED>
__global__ __launch_bounds__(256) void select_kernel(SelectArgs a) {
  constexpr int N = 4 * NQ, STRIDE = 64 * NQ + 4;
  typedef std::conditional_t<KEYED, double, float> wide_t;
  __shared__ wide_t ks[ROWS][STRIDE];   // keys, for groups
  const int j = threadIdx.x & 15, tok = threadIdx.x >> 4;
  const bool tv = (int)blockIdx.x * ROWS + tok < a.T;
  const int t = tv ? (int)blockIdx.x * ROWS + tok : a.T - 1;
  const ZT* const logits = static_cast<const ZT*>(a.z);
  float z[N];
  load_row<ZT, NQ>(logits, t, a.E, j, z);
  const bool visual = a.is_visual != nullptr && a.is_visual[t] != 0;
  const int k = visual ? a.k_visual : a.k_text;

  float m = 0.0f, inv = 1.0f;   // softmax scores are exp(z - m) * inv
  if (!a.sigmoid && (KEYED || a.scores != nullptr || !a.renorm)) {
    m = row_largest(z);
    const float sum = row_exp_sum(z, m);
    inv = sum > 0.0f ? 1.0f / sum : 0.0f;
  }
  if (a.scores != nullptr && tv) {
    float s[N];
#pragma unroll
    for (int r = 0; r < N; ++r) s[r] = a.sigmoid ? 1.0f / (1.0f + expf(-z[r])) : expf(z[r] - m) * inv;
    write_row<float, NQ>(a.scores + (size_t)t * a.E, a.E, j, s);
  }

  int mine;
  if constexpr (KEYED) {
    float bias[N];
    if (a.bias != nullptr) {   // uniform
      read_row<float, NQ>(a.bias, a.E, j, bias);
    } else {
#pragma unroll
      for (int r = 0; r < N; ++r) bias[r] = 0.0f;
    }
    bool sure = true;
    {
      const float largest = a.sigmoid ? 1.0f : inv;
      const float slack = largest * 0x1p-19f;
      constexpr float RELATIVE = 0x1p-22f;
      float key[N], order[N];
#pragma unroll
      for (int r = 0; r < N; ++r) {
        const float s = a.sigmoid ? __builtin_amdgcn_rcpf(1.0f + __expf(-z[r])) : __expf(z[r] - m) * inv;
        key[r] = z[r] > -INFINITY && bias[r] > -INFINITY ? s + bias[r] : -INFINITY;
        order[r] = a.bias != nullptr ? key[r] : z[r];
      }
      if (a.groups > 1)
        sure = keep_groups<float, N>(a, j, key, order, reinterpret_cast<float*>(ks[tok]), 2.0f * slack, 2.0f * RELATIVE);
      float my_key;
      mine = list_largest<float, N>(k, a.Kmax, j, order, my_key);
      if (a.bias != nullptr) {
        // the largest that is not listed; then every entry against the one behind it
        float rest = order[0];
#pragma unroll
        for (int r = 1; r < N; ++r) rest = larger(rest, order[r]);
        rest = row_max(rest);
        const int listed = __popc((unsigned)(__ballot(mine >= 0) >> (threadIdx.x & 48)) & 0xffffu);
        const float behind = __shfl(my_key, (threadIdx.x & 48) + ((j + 1) & 15), 64);
        const float next = j + 1 < listed ? behind : rest;
        sure = sure && (mine < 0 || next == -INFINITY || my_key - next > slack + RELATIVE * (fabsf(my_key) + fabsf(next)));
      }
    }
    if (__any(!sure)) {
      double key[N], order[N], sum = 0.0, my_key;
      if (!a.sigmoid) {
#pragma unroll
        for (int r = 0; r < N; ++r) sum += exp((double)z[r] - (double)m);
        sum = row_sum_butterfly(sum);
      }
#pragma unroll
      for (int r = 0; r < N; ++r) {
        const double s = a.sigmoid ? 1.0 / (1.0 + exp(-(double)z[r])) : exp((double)z[r] - (double)m) / sum;
        key[r] = z[r] > -INFINITY && bias[r] > -INFINITY ? s + (double)bias[r] : -INFINITY;
        order[r] = a.bias != nullptr ? key[r] : (double)z[r];
      }
      wave_sync();
      if (a.groups > 1) (void)keep_groups<double, N>(a, j, key, order, ks[tok], 0.0, 0.0);
      mine = list_largest<double, N>(k, a.Kmax, j, order, my_key);
    }
  } else {
    float key[N], my_key;
#pragma unroll
    for (int r = 0; r < N; ++r) key[r] = z[r];
    if (a.groups > 1) (void)keep_groups<float, N>(a, j, key, z, ks[tok], 0.0f, 0.0f);
    mine = list_largest<float, N>(k, a.Kmax, j, z, my_key);
  }

  const float zl = mine >= 0 ? clean(to_f32(logits[(size_t)t * a.E + mine])) : -INFINITY;
  float g;
  if (a.renorm) {
    const float l = mine >= 0 ? (a.sigmoid ? log_sigmoid(zl) : zl) : -INFINITY;
    const float lm = row_max(l);
    const float p = mine >= 0 ? expf(l - lm) : 0.0f;
    const float sum = row_sum_butterfly(p);   // (every lane takes part)
    g = mine >= 0 ? p / sum : 0.0f;
  } else {
    g = mine < 0 ? 0.0f : a.sigmoid ? 1.0f / (1.0f + expf(-zl)) : expf(zl - m) * inv;
  }
  if (tv && j < a.Kmax) {
    a.idx[(size_t)t * a.Kmax + j] = mine;
    a.gate[(size_t)t * a.Kmax + j] = mine >= 0 ? g * a.scale : 0.0f;
  }
}

// To the type of the logits; NaN, which an incoming gradient may hold, stays NaN.
template <typename ZT> __device__ __forceinline__ ZT gradient(float v);
template <> __device__ __forceinline__ float gradient<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16_t gradient<bf16_t>(float v) { return v == v ? f32_to_bf16(v) : (bf16_t)0x7fc0; }

struct SelectBackwardArgs {
  const void* z;
  const int32_t* idx;
  const float* d_gate;
  const float* d_scores;   // or null
  int T, E, Kmax;
  int sigmoid, renorm;
  float scale;
  void* d_z;
};

// Gradient of  sum d_gate * gate + sum d_scores * score  with respect to the logits, for the list that was chosen.  With
// p the softmax over the list of l = log(s) and a = c * d_gate, renormalised gates give dl = p (a - sum p a), and
// dz = dl (softmax) or dl * (1 - s) (sigmoid).  What reaches the scores, ds (d_scores, and a at the listed experts where
// gates are not renormalised), gives dz = s (ds - sum s ds) (softmax) or s (1 - s) ds (sigmoid).
// DENSE: every logit is needed (d_scores, or softmax gates that are not renormalised); else those of the list.
template <typename ZT, int NQ, bool DENSE>
__global__ __launch_bounds__(256) void select_backward_kernel(SelectBackwardArgs a) {
  constexpr int N = 4 * NQ, STRIDE = 64 * NQ + 4;
  __shared__ float row[ROWS][STRIDE];   // what the list adds to its experts
  const int j = threadIdx.x & 15, tok = threadIdx.x >> 4;
  const bool tv = (int)blockIdx.x * ROWS + tok < a.T;
  const int t = tv ? (int)blockIdx.x * ROWS + tok : a.T - 1;
  const ZT* const zrow = static_cast<const ZT*>(a.z) + (size_t)t * a.E;
#pragma unroll
  for (int r = 0; r < N; ++r) row[tok][64 * (r >> 2) + 4 * j + (r & 3)] = 0.0f;
  int e = -1;
  float ga = 0.0f;
  if (j < a.Kmax) {
    e = a.idx[(size_t)t * a.Kmax + j];
    ga = a.d_gate[(size_t)t * a.Kmax + j] * a.scale;
  }
  const bool in = e >= 0 && e < a.E;
  const float zl = in ? clean(to_f32(zrow[in ? e : 0])) : -INFINITY;
  float v = in ? ga : 0.0f;   // to the scores
  if (a.renorm || (a.sigmoid && !DENSE)) {
    if (a.renorm) {
      const float l = a.sigmoid ? log_sigmoid(zl) : zl;
      const float lm = row_max(in ? l : -INFINITY);
      float p = in && l > -INFINITY ? expf(l - lm) : 0.0f;
      const float sum = row_sum_butterfly(p);
      p = sum > 0.0f ? p / sum : 0.0f;
      v = p * (v - row_sum_butterfly(p * v));
      if (a.sigmoid) v = v / (1.0f + expf(zl));
    } else {
      v = zl > -INFINITY ? v / (1.0f + expf(-zl)) / (1.0f + expf(zl)) : 0.0f;
    }
  }
  __syncthreads();
  if (in) atomicAdd(&row[tok][e], v);   // the entries of a list are distinct
  __syncthreads();
  float d[N];
#pragma unroll
  for (int r = 0; r < N; ++r) d[r] = row[tok][64 * (r >> 2) + 4 * j + (r & 3)];
  if constexpr (DENSE) {
    float z[N];
    load_row<ZT, NQ>(static_cast<const ZT*>(a.z), t, a.E, j, z);
    float ds[N];
    if (a.d_scores != nullptr) {   // uniform
      read_row<float, NQ>(a.d_scores + (size_t)t * a.E, a.E, j, ds);
    } else {
#pragma unroll
      for (int r = 0; r < N; ++r) ds[r] = 0.0f;
    }
    if (!a.renorm) {
#pragma unroll
      for (int r = 0; r < N; ++r) {
        ds[r] += d[r];
        d[r] = 0.0f;
      }
    }
    if (a.sigmoid) {
#pragma unroll
      for (int r = 0; r < N; ++r)
        d[r] = z[r] > -INFINITY ? d[r] + ds[r] / (1.0f + expf(-z[r])) / (1.0f + expf(z[r])) : 0.0f;
    } else {
      const float m = row_largest(z);
      const float sum = row_exp_sum(z, m);
      const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
      float dot = 0.0f;
#pragma unroll
      for (int r = 0; r < N; ++r) {
        z[r] = z[r] > -INFINITY ? expf(z[r] - m) * inv : -1.0f;   // the score; -1: masked
        dot += z[r] > 0.0f ? z[r] * ds[r] : 0.0f;
      }
      dot = row_sum_butterfly(dot);
#pragma unroll
      for (int r = 0; r < N; ++r) d[r] = z[r] >= 0.0f ? d[r] + z[r] * (ds[r] - dot) : 0.0f;
    }
  }
  if (tv) {
    ZT out[N];
#pragma unroll
    for (int r = 0; r < N; ++r) out[r] = gradient<ZT>(d[r]);
    write_row<ZT, NQ>(static_cast<ZT*>(a.d_z) + (size_t)t * a.E, a.E, j, out);
  }
}

template <typename ZT, int NQ>
void run_select(const SelectArgs& a, bool keyed, hipStream_t stream) {
  const dim3 grid((a.T + ROWS - 1) / ROWS), block(256);
  if (keyed) hipLaunchKernelGGL((select_kernel<ZT, NQ, true>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((select_kernel<ZT, NQ, false>), grid, block, 0, stream, a);
}
template <typename ZT>
void run_select_by_size(const SelectArgs& a, bool keyed, hipStream_t stream) {
  if (a.E <= 64) run_select<ZT, 1>(a, keyed, stream);
  else if (a.E <= 128) run_select<ZT, 2>(a, keyed, stream);
  else run_select<ZT, 4>(a, keyed, stream);
}

template <typename ZT, int NQ>
void run_backward(const SelectBackwardArgs& a, bool dense, hipStream_t stream) {
  const dim3 grid((a.T + ROWS - 1) / ROWS), block(256);
  if (dense) hipLaunchKernelGGL((select_backward_kernel<ZT, NQ, true>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((select_backward_kernel<ZT, NQ, false>), grid, block, 0, stream, a);
}
template <typename ZT>
void run_backward_by_size(const SelectBackwardArgs& a, bool dense, hipStream_t stream) {
  if (a.E <= 64) run_backward<ZT, 1>(a, dense, stream);
  else if (a.E <= 128) run_backward<ZT, 2>(a, dense, stream);
  else run_backward<ZT, 4>(a, dense, stream);
}

}  // namespace

int launch_select(const fmoe_ctx* ctx, const fmoe_select_params* p, const void* logits, int dtype,
                  const uint8_t* is_visual, const float* bias, int T, float* scores, int32_t* topk_idx,
                  float* topk_gate, hipStream_t stream) {
  const fmoe_config& c = ctx->cfg;
  SelectArgs a{};
  a.z = logits; a.is_visual = is_visual; a.bias = bias;
  a.T = T; a.E = c.n_experts; a.k_text = c.k_text; a.k_visual = c.k_visual; a.Kmax = ctx->kmax;
  a.sigmoid = p->score; a.renorm = c.renormalize; a.groups = p->n_groups; a.topk_groups = p->topk_groups;
  a.sum_two = p->group_score;
  a.group_size = c.n_experts / p->n_groups;
  a.group_mul = (65536 + a.group_size - 1) / a.group_size;
  a.scale = p->gate_scale;
  a.scores = scores; a.idx = topk_idx; a.gate = topk_gate;
  const bool keyed = bias != nullptr || (p->n_groups > 1 && p->group_score == 1);
  if (dtype == FMOE_BF16) run_select_by_size<bf16_t>(a, keyed, stream);
  else run_select_by_size<float>(a, keyed, stream);
  FMOE_HIP_CHECK(hipGetLastError());
  return FMOE_OK;
}

int launch_select_backward(const fmoe_ctx* ctx, const fmoe_select_params* p, const void* logits, int dtype,
                           const int32_t* topk_idx, const float* d_gate, const float* d_scores, int T, void* d_logits,
                           hipStream_t stream) {
  const fmoe_config& c = ctx->cfg;
  SelectBackwardArgs a{};
  a.z = logits; a.idx = topk_idx; a.d_gate = d_gate; a.d_scores = d_scores;
  a.T = T; a.E = c.n_experts; a.Kmax = ctx->kmax;
  a.sigmoid = p->score; a.renorm = c.renormalize; a.scale = p->gate_scale;
  a.d_z = d_logits;
  const bool dense = d_scores != nullptr || !(c.renormalize || p->score);
  if (dtype == FMOE_BF16) run_backward_by_size<bf16_t>(a, dense, stream);
  else run_backward_by_size<float>(a, dense, stream);
  FMOE_HIP_CHECK(hipGetLastError());
  return FMOE_OK;
}
