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
// exponential and reciprocal of the hardware.  Two sigmoid scores are then off by less than 2^-21 together; two softmax scores
// that go with close keys by less than 27 * 2^-24 of the largest score the row can have (22 for the normaliser, whose error
// they share); 2^-19 of it is allowed for, and half a rounding of each key.  Where keys in a token's list or behind its end are
// closer than that, its entries and the next one are put in order in 64 bits, a lane an entry; where that is not enough (more
// than one key close behind the list) its whole wavefront lists the token again.  Where the scores of groups on either side of
// the line are that close, the wavefront chooses the token's groups.  Of 22016 tokens with 256 experts in eight groups and a
// bias of deviation 0.1 some twenty are of the first kind and a few of the last.
//
// Sixteen lanes have a token (four tokens a wavefront), lane j of them the experts 64 q + 4 j + i: a row is read in
// pieces of 16 bytes, and a reduction over the row is one over a lane's registers and four steps inside the vector unit.
//
// Bound: vector instructions (some thousand a wavefront, 256 experts) behind one wait for the logits, and for few tokens the
// launch.  22016 tokens, 256 experts, sigmoid, bias, eight groups: 16.5 us, 1.4 TB/s.  Step by step: everything in 64 bits
// 41.4; keys in 32 bits and only what is close in 64, rows four at a time 34.6; lists by integers sorted in a lane, so that
// a round is one reduction 24.1; fewer instructions for keys, integers and gates 21.5; reductions of the whole wavefront without
// LDS 19.0; close entries put in order instead of listed again 18.6; only the groups chosen again 16.6; row maxima as
// integers 16.5.  The few tokens in 64 bits still are 1.8 of it, at the end of the launch.  A wavefront that takes several rows
// in turn, the next ones' logits on their way, took 25 where this took 21.5.  The gradient reads and writes rows once and is bound by
// that: 22016 x 256 in fp32 6.7 us, 3.7 TB/s.

#include <float.h>
#include <limits.h>

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
__device__ __forceinline__ float clean(float z) { return fminf(fmaxf(z, -INFINITY), FLT_MAX); }

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
// (Past the caches: the gradient of 22016 x 256 logits 7.8 -> 6.8 us.)
template <typename T, int NQ>
__device__ __forceinline__ void write_row(T* __restrict__ row, int E, int j, const T (&v)[4 * NQ]) {
  typedef T four_t __attribute__((ext_vector_type(4)));
  if ((E & 3) == 0) {
#pragma unroll
    for (int q = 0; q < NQ; ++q)
      if (64 * q + 4 * j < E)
        __builtin_nontemporal_store(four_t{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]},
                                    reinterpret_cast<four_t*>(row + 64 * q + 4 * j));
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

// Largest over the row of a number that is not NaN, as integers of the same order: an instruction a step.
__device__ __forceinline__ float row_top(float v) {
  int o = __float_as_int(v);
  o = row_max(o ^ ((o >> 31) & 0x7fffffff));
  return __int_as_float(o ^ ((o >> 31) & 0x7fffffff));
}

// Of a row: the largest, of its logits also 0 if all are masked, and the sum of exp(z - largest).
template <int N>
__device__ __forceinline__ float row_peak(const float (&z)[N]) {
  float m = z[0];
#pragma unroll
  for (int r = 1; r < N; ++r) m = fmaxf(m, z[r]);
  return row_top(m);
}
template <int N>
__device__ __forceinline__ float row_largest(const float (&z)[N]) {
  const float m = row_peak(z);
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

// v of the lane whose number differs in bit LOG2 (0 or 1), or, among lanes that agree within their fours, of the other four
// of the same eight (2).
template <int LOG2>
__device__ __forceinline__ float lane_partner(float v) {
  constexpr int CTRL = LOG2 == 0 ? 0xb1 : LOG2 == 1 ? 0x4e : 0x141;   // quad permutations, half-row mirror
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true));
}
// The two largest so far, and two more.
__device__ __forceinline__ void two_largest(float& one, float& two, float o1, float o2) {
  two = fmaxf(fminf(one, o1), fmaxf(two, o2));
  one = fmaxf(one, o1);
}

// ---- one token by a whole wavefront, in 64 bits: what the definition says, for the few that are close.  A wavefront that
// comes here is one the launch waits for, so what counts is latency: reductions go through the rows of 16 and four lane
// reads, not through LDS.
__device__ __forceinline__ double read_lane(double v, int lane) {
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane), __builtin_amdgcn_readlane(__double2loint(v), lane));
}
__device__ __forceinline__ double wave_max(double v) {
  v = row_max(v);
  return larger(larger(read_lane(v, 0), read_lane(v, 16)), larger(read_lane(v, 32), read_lane(v, 48)));
}
__device__ __forceinline__ double wave_sum(double v) {
  v = row_sum_butterfly(v);
  return (read_lane(v, 0) + read_lane(v, 16)) + (read_lane(v, 32) + read_lane(v, 48));
}
__device__ __forceinline__ int wave_min(int v) {
  v = row_min(v);
  return min(min(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16)),
             min(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48)));
}
// Keys of experts 4 l .. 4 l + 3 of token t in lane l.
template <typename ZT, bool KEYED, bool SIGMOID>
__device__ __forceinline__ void keys_wide(const SelectArgs& a, int t, double (&z)[4], double (&key)[4]) {
  const int lane = threadIdx.x & 63;
  const ZT* const row = static_cast<const ZT*>(a.z) + (size_t)t * a.E;
#pragma unroll
  for (int i = 0; i < 4; ++i) z[i] = 4 * lane + i < a.E ? clean(to_f32(row[4 * lane + i])) : -INFINITY;
  double m = 0.0, sum = 1.0;
  if (KEYED && !SIGMOID) {
    m = wave_max(larger(larger(z[0], z[1]), larger(z[2], z[3])));
    if (!(m > -INFINITY)) m = 0.0;
    sum = wave_sum((exp(z[0] - m) + exp(z[1] - m)) + (exp(z[2] - m) + exp(z[3] - m)));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = 4 * lane + i;
    key[i] = z[i];
    if (KEYED) {
      const float b = a.bias != nullptr && e < a.E ? a.bias[e] : 0.0f;
      const double s = SIGMOID ? 1.0 / (1.0 + exp(-z[i])) : exp(z[i] - m) / sum;
      key[i] = z[i] > -INFINITY && b > -INFINITY ? s + (double)b : -INFINITY;
    }
  }
}
// Bits 4 g: the groups g of token t that stay.  ks: room for E doubles.
template <typename ZT, bool SIGMOID>
__device__ unsigned long long groups_wide(const SelectArgs& a, int t, double* ks) {
  const int lane = threadIdx.x & 63;
  double z[4], key[4];
  keys_wide<ZT, true, SIGMOID>(a, t, z, key);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (4 * lane + i < a.E) ks[4 * lane + i] = key[i];
  wave_sync();
  double one = -INFINITY, two = -INFINITY;   // lane 4 g + q: of group g the elements q, q + 4, ..
  const int g0 = lane >> 2;
  for (int i = lane & 3; i < a.group_size && g0 < a.groups; i += 4) {
    const double v = ks[g0 * a.group_size + i];
    two = v > one ? one : larger(two, v);
    one = larger(one, v);
  }
#pragma unroll
  for (int s = 1; s <= 2; s <<= 1) {   // (of equal ones both count)
    const double o1 = __shfl_xor(one, s, 64), o2 = __shfl_xor(two, s, 64);
    two = larger(o1 > one ? one : o1, larger(two, o2));
    one = larger(one, o1);
  }
  wave_sync();
  const double score = (a.sum_two && two > -INFINITY) ? one + two : one;
  int ahead = 0;
  for (int g = 0; g < a.groups; ++g) {
    const double o = read_lane(score, 4 * g);
    ahead += (o > score || (o == score && g < g0)) ? 1 : 0;
  }
  return __ballot(g0 < a.groups && ahead < a.topk_groups);
}
// Lane i of the result: entry i of the token's list.  stays(e): whether the group of expert e stays.
template <typename ZT, bool KEYED, bool SIGMOID, typename F>
__device__ int list_wide(const SelectArgs& a, int t, int k, F&& stays) {
  const int lane = threadIdx.x & 63;
  double z[4], order[4];
  keys_wide<ZT, KEYED, SIGMOID>(a, t, z, order);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (a.bias == nullptr) order[i] = z[i];
    if (!stays(4 * lane + i)) order[i] = -INFINITY;
  }
  int mine = -1;
  for (int round = 0; round < k; ++round) {
    const double top = wave_max(larger(larger(order[0], order[1]), larger(order[2], order[3])));
    if (!(top > -INFINITY)) break;
    int e = 0x7fff;
#pragma unroll
    for (int i = 3; i >= 0; --i) e = order[i] == top ? 4 * lane + i : e;
    e = wave_min(e);   // ties: lowest expert
    if (lane == round) mine = e;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (4 * lane + i == e) order[i] = -INFINITY;
  }
  return mine;
}

// Masks the experts of a token's groups that do not stay.  key: what a group's score is made of; order: what ranks the
// experts; rows: the tokens' rows in LDS.  Where keys are SCORED and the scores on either side of the line are not further
// apart than `slack` plus `relative` times the largest keys that went into any, the token's groups are chosen in 64 bits.
// 2^log2p lanes have a group; bits g << log2p of the result: the groups that stay.
__device__ __forceinline__ int lanes_of_group(const SelectArgs& a) {
  return a.groups <= 2 ? 3 : a.groups <= 4 ? 2 : a.groups <= 8 ? 1 : 0;   // uniform; logarithm
}
__device__ __forceinline__ bool stays(const SelectArgs& a, unsigned mask, int log2p, int e) {   // (past E masked already)
  return (mask >> (((e * a.group_mul >> 16) << log2p) & 15)) & 1u;
}
template <typename ZT, bool SCORED, bool SIGMOID, int N, int STRIDE>
__device__ __forceinline__ unsigned keep_groups(const SelectArgs& a, int t, int tok, int j, const float (&key)[N],
                                                float (&order)[N], float (&rows)[ROWS][STRIDE], float slack, float relative) {
  float* const ks = rows[tok];
  typedef float four_t __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int q = 0; q < N / 4; ++q)
    *reinterpret_cast<four_t*>(ks + 64 * q + 4 * j) = four_t{key[4 * q], key[4 * q + 1], key[4 * q + 2], key[4 * q + 3]};
  wave_sync();
  const int log2p = lanes_of_group(a);
  const int g = j >> log2p, part = j & ((1 << log2p) - 1);
  const bool fours = (a.group_size & 3) == 0;
  float one = -INFINITY, two = -INFINITY;
  if (g < a.groups) {
    const float* const own = ks + g * a.group_size;
    if (fours) {
      for (int i = 4 * part; i < a.group_size; i += 4 << log2p) {
        const four_t v = *reinterpret_cast<const four_t*>(own + i);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          two = fmaxf(two, fminf(one, v[x]));
          one = fmaxf(one, v[x]);
        }
      }
    } else {
      for (int i = part; i < a.group_size; i += 1 << log2p) {
        const float v = own[i];
        two = fmaxf(two, fminf(one, v));
        one = fmaxf(one, v);
      }
    }
  }
  if (log2p > 0) two_largest(one, two, lane_partner<0>(one), lane_partner<0>(two));
  if (log2p > 1) two_largest(one, two, lane_partner<1>(one), lane_partner<1>(two));
  if (log2p > 2) two_largest(one, two, lane_partner<2>(one), lane_partner<2>(two));
  // (keys of the type's lowest value: a sum past it is not the score of a group that has none)
  const float score = (a.sum_two && two > -INFINITY) ? fmaxf(one + two, -FLT_MAX) : one;
  // rank among the groups: larger scores, or equal ones of lower groups, are ahead
  wave_sync();   // the keys have been read
  if (part == 0) ks[g] = score;
  wave_sync();
  int ahead = 0;
  for (int h = 0; h < a.groups; ++h) {
    const float o = ks[h];
    ahead += (o > score || (o == score && h < g)) ? 1 : 0;
  }
  wave_sync();   // the scores have been read
  bool in = g < a.groups && ahead < a.topk_groups;
  if constexpr (SCORED) {
    const float last = -row_top(in ? -score : -INFINITY), next = row_top(g < a.groups && !in ? score : -INFINITY);
    const float size = row_top(fabsf(one > -INFINITY ? one : 0.0f) + fabsf(two > -INFINITY ? two : 0.0f));
    const bool sure = a.topk_groups == a.groups || next == -INFINITY || last - next > slack + relative * size;
    unsigned long long again = __ballot(!sure);
    while (again != 0) {   // uniform
      const int first = (__ffsll((long long)again) - 1) & 48;   // the token's first lane
      again &= ~(0xffffull << first);
      const unsigned long long stay =
          groups_wide<ZT, SIGMOID>(a, __shfl(t, first, 64), reinterpret_cast<double*>(rows[tok & 12]));
      if ((threadIdx.x & 48) == (unsigned)first) in = (stay >> (4 * g)) & 1u;
    }
  }
  const unsigned mask = (unsigned)(__ballot(in) >> (threadIdx.x & 48)) & 0xffffu;
  if (fours) {
#pragma unroll
    for (int q = 0; q < N / 4; ++q) {
      const bool on = stays(a, mask, log2p, 64 * q + 4 * j);
#pragma unroll
      for (int i = 0; i < 4; ++i) order[4 * q + i] = on ? order[4 * q + i] : -INFINITY;
    }
  } else {
#pragma unroll
    for (int r = 0; r < N; ++r) order[r] = stays(a, mask, log2p, expert_of(r, j)) ? order[r] : -INFINITY;
  }
  return mask;
}

// The list by integers that hold key and expert, all different: a lane's are sorted once, then every round takes the largest
// head and its lane moves up.  Lane j keeps entry j; `rest`: the largest that is not listed.  Below 0: masked.
constexpr int NONE = INT_MIN;
template <int N, int DEPTH>
__device__ __forceinline__ void pop_rounds(int rounds, int j, int (&s)[N], int& mine) {
  for (int round = 0; round < rounds; ++round) {
    const int top = row_max(s[0]);
    mine = j == round ? top : mine;
    const bool won = s[0] == top;
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) {
      const int here = s[i], next = i + 1 < N ? s[i + 1 < N ? i + 1 : 0] : NONE;   // (values: not a choice of places)
      s[i] = won ? next : here;
    }
  }
}
template <int N>
__device__ __forceinline__ int list_packed(int rounds, int j, int (&s)[N], int& rest) {
  // Batcher's merge exchange, largest first
#pragma unroll
  for (int p = 1; p < N; p *= 2) {
#pragma unroll
    for (int k = p; k >= 1; k /= 2) {
#pragma unroll
      for (int x = k % p; x + k < N; x += 2 * k) {
#pragma unroll
        for (int i = 0; i < k; ++i) {
          const int lo = x + i, hi = x + i + k;
          if (hi < N && lo / (2 * p) == hi / (2 * p)) {
            const int big = max(s[lo], s[hi]), small = min(s[lo], s[hi]);
            s[lo] = big;
            s[hi] = small;
          }
        }
      }
    }
  }
  int mine = NONE;
  // a lane is asked for at most `rounds` heads, and one more for `rest`
  if (N > 10 && rounds <= 9) pop_rounds<N, N < 10 ? N : 10>(rounds, j, s, mine);
  else pop_rounds<N, N>(rounds, j, s, mine);
  rest = row_max(s[0]);
  return mine;
}
__device__ __forceinline__ int unpack_expert(int packed) { return packed < 0 ? -1 : 255 - (packed & 255); }
__device__ __forceinline__ int masked_below_zero(int packed, float order) { return packed | (order > -INFINITY ? 0 : NONE); }

// Key and expert in one integer: the distance to the row's largest key `top` in steps, KEY_STEPS over RANGE, then the expert,
// lower ones larger.  Keys further below than RANGE, and masked ones, have no steps.
// The largest key has to stay below 2^23 steps, or its integer is negative.  For |top| below 8 ranges, range - top is below 9
// ranges and off by at most 2^-24 of itself, 4.5 steps; the product with the scale (which is exact in either range) by as much;
// the fused sum by half a step: at most KEY_STEPS + 9.5 (8 at every such number), and the key has 32 to spare.
constexpr float KEY_RANGE = 4.0f;      // of scores (0 .. 1) with a bias
constexpr float LOGIT_RANGE = 64.0f;
constexpr float KEY_STEPS = 0x1p23f - 32.0f;
template <int N>
__device__ __forceinline__ void pack_below(const float (&order)[N], float top, float range, int j, int (&s)[N]) {
  const float scale = KEY_STEPS / range, offset = (range - top) * scale;
  const int lane_part = (15 - j) * 4;
#pragma unroll
  for (int r = 0; r < N; ++r) {
    unsigned q;   // the instruction saturates at 0, also for -inf and NaN; a cast would leave that undefined
    asm("v_cvt_u32_f32 %0, %1" : "=v"(q) : "v"(fmaf(order[r], scale, offset)));
    s[r] = (int)((q << 8) | lane_part) | (192 - 64 * (r >> 2) + 3 - (r & 3));   // .. 255 - expert
  }
}
// Whether entries j < k of the list differ from the ones behind them by more than `steps` and all are in range.
__device__ __forceinline__ bool apart(int mine, int rest, int k, int rounds, int j, int steps) {
  const int behind = row_rotate<15>(mine);   // of lane j + 1
  const int next = j + 1 < rounds ? behind : rest;
  return (j >= k) | (((mine >> 8) > 0) & ((mine >> 8) - (next >> 8) > steps));
}

// f(v, i) of the fifteen other lanes of the row
template <int ROT = 1, typename F>
__device__ __forceinline__ void static_for_rotations(double v, int i, F&& f) {
  if constexpr (ROT < 16) {
    f(row_rotate<ROT>(v), row_rotate<ROT>(i));
    static_for_rotations<ROT + 1>(v, i, f);
  }
}

// The entries of four tokens' lists (experts, -1: none; a token in sixteen lanes) put in order by their keys in 64 bits.
// SCORED: keys are scores with a bias, else logits.
template <typename ZT, int NQ, bool SCORED, bool SIGMOID>
__device__ __forceinline__ int sort_entries(const SelectArgs& a, int t, int j, int entry) {
  const ZT* const row = static_cast<const ZT*>(a.z) + (size_t)t * a.E;
  const int e = entry >= 0 ? entry : 0;
  const double z = clean(to_f32(row[e]));
  double key = z;
  if constexpr (SCORED) {
    const double b = a.bias[e];
    if constexpr (SIGMOID) {
      key = 1.0 / (1.0 + exp(-z)) + b;
    } else {
      float all[4 * NQ];
      load_row<ZT, NQ>(static_cast<const ZT*>(a.z), t, a.E, j, all);
      const double m = row_largest(all);
      double sum = 0.0;
#pragma unroll 4
      for (int r = 0; r < 4 * NQ; ++r) sum += exp((double)all[r] - m);
      sum = row_sum_butterfly(sum);
      key = exp(z - m) / sum + b;
    }
  }
  if (entry < 0) key = -INFINITY;
  const int id = entry < 0 ? FMOE_MAX_EXPERTS + j : entry;
  int rank = 0;   // entries of the token ahead of this lane's
  const auto against = [&](double k, int i) { rank += ((k > key) | ((k == key) & (i < id))) ? 1 : 0; };
  static_for_rotations(key, id, against);
  // every rank occurs once in a token: each lane takes what the one of its rank has
  return __builtin_amdgcn_ds_permute(((threadIdx.x & 48) + rank) << 2, entry);
}

// KEYED: the keys are scores with a bias, or sums of scores rank the groups; else the logits are the keys.
// ks: keys, for groups.  Returns the expert of the lane's place in the token's list, or -1 (also past T), and its gate.
template <typename ZT, int NQ, bool KEYED, bool SIGMOID>
__device__ __forceinline__ int select_rows(const SelectArgs& a, float (&ks)[ROWS][64 * NQ + 4], float& gate) {
  constexpr int N = 4 * NQ;
  const int j = threadIdx.x & 15, tok = threadIdx.x >> 4;
  const bool tv = (int)blockIdx.x * ROWS + tok < a.T;
  const int t = tv ? (int)blockIdx.x * ROWS + tok : a.T - 1;
  const ZT* const logits = static_cast<const ZT*>(a.z);
  float z[N];
  load_row<ZT, NQ>(logits, t, a.E, j, z);
  const bool visual = a.is_visual != nullptr && a.is_visual[t] != 0;
  const int k = visual ? a.k_visual : a.k_text;

  float m = 0.0f, inv = 1.0f;   // softmax scores are exp(z - m) * inv
  if (!SIGMOID && (KEYED || a.scores != nullptr || !a.renorm)) {
    m = row_largest(z);
    const float sum = row_exp_sum(z, m);
    inv = sum > 0.0f ? 1.0f / sum : 0.0f;
  }
  if (a.scores != nullptr && tv) {
    float s[N];
#pragma unroll
    for (int r = 0; r < N; ++r) s[r] = SIGMOID ? 1.0f / (1.0f + expf(-z[r])) : expf(z[r] - m) * inv;
    write_row<float, NQ>(a.scores + (size_t)t * a.E, a.E, j, s);
  }

  // the list in 32 bits
  float order[N];
  unsigned groups = 0xffffu;   // that stay
  if constexpr (KEYED) {
    float bias[N], key[N];
    if (a.bias != nullptr) {   // uniform
      read_row<float, NQ>(a.bias, a.E, j, bias);
    } else {
#pragma unroll
      for (int r = 0; r < N; ++r) bias[r] = 0.0f;
    }
    const float slack = (SIGMOID ? 1.0f : inv) * 0x1p-19f;
#pragma unroll
    for (int r = 0; r < N; ++r) {
      const float s = SIGMOID ? __builtin_amdgcn_rcpf(1.0f + __expf(-z[r])) : __expf(z[r] - m) * inv;
      const float u = fmaxf(s + bias[r], -INFINITY);   // bias NaN or -inf: masked
      key[r] = z[r] > -INFINITY ? u : -INFINITY;
    }
    if (a.bias != nullptr) {
#pragma unroll
      for (int r = 0; r < N; ++r) order[r] = key[r];
    } else {
#pragma unroll
      for (int r = 0; r < N; ++r) order[r] = z[r];
    }
    if (a.groups > 1) groups = keep_groups<ZT, true, SIGMOID>(a, t, tok, j, key, order, ks, 2.0f * slack, 0x1p-21f);
  } else {
#pragma unroll
    for (int r = 0; r < N; ++r) order[r] = z[r];
    if (a.groups > 1) groups = keep_groups<ZT, false, SIGMOID>(a, t, tok, j, z, order, ks, 0.0f, 0.0f);
  }
  int packed[N], rest, mine;
  if constexpr (!KEYED && sizeof(ZT) == 2) {
    // a bf16 logit's sixteen bits and the expert are one integer: exact, equal ones in order of the expert
#pragma unroll
    for (int r = 0; r < N; ++r) {
      int o = __float_as_int(order[r] == FLT_MAX ? INFINITY : order[r] + 0.0f);   // as it came; -0 is +0
      o ^= (o >> 31) & 0x7fffffff;                                                  // in order as a signed integer
      packed[r] = masked_below_zero((((o >> 16) + 0x8000) << 8) | (255 - expert_of(r, j)), order[r]);
    }
    const int entry = list_packed(a.Kmax, j, packed, rest);
    mine = j < k ? unpack_expert(entry) : -1;
  } else {
    const float peak = row_peak(order);
    const bool scored = KEYED && a.bias != nullptr;   // uniform
    const float range = scored ? KEY_RANGE : LOGIT_RANGE;
    pack_below(order, peak, range, j, packed);
    const int rounds = a.Kmax < 16 ? a.Kmax + 1 : 16;   // one more than is listed, if there is a lane for it
    const int entry = list_packed(rounds, j, packed, rest);
    mine = (entry >> 8) > 0 ? unpack_expert(entry) : -1;   // (without steps: masked, or further below than all in range)
    // The way from key to integer is monotonic, so logits whose integers differ are in order.  Two scored keys can be off by
    // `slack` and half a rounding each, and their integers lose less than two steps more.  (The offset's rounding is the same
    // for all, and while the peak is below 8 ranges the largest integer stays below 2^23: KEY_STEPS.)
    int steps = 0;
    if constexpr (KEYED)
      if (scored) {
        const float off = (SIGMOID ? 1.0f : inv) * 0x1p-19f + 0x1p-23f * (fabsf(peak) + KEY_RANGE);
        steps = (int)fminf(off * (0x1p23f / KEY_RANGE), 1e6f) + 3;
      }
    const bool none = peak == -INFINITY;   // nothing to choose from
    bool sorted = apart(entry, rest, k, rounds, j, steps) | none;
    // do the entries hold the list for certain?  Their integers then are in range, and the k-th is apart from the rest
    bool held = (j != k - 1) | (((entry >> 8) > 0) & ((entry >> 8) - (rest >> 8) > steps));
    if (__any(!held & ((entry >> 8) == 0) & !none)) {   // uniform
      // no k-th entry in range: the list is complete if what is not in range is masked
      bool lost = false;
#pragma unroll
      for (int r = 0; r < N; ++r) lost |= (order[r] > -INFINITY) & (peak - order[r] > 0.99f * range);
      const bool complete = ((__ballot(lost) >> (threadIdx.x & 48)) & 0xffffu) == 0;
      held |= complete & ((entry >> 8) == 0);
      sorted |= complete & ((entry >> 8) == 0);
    }
    const bool sure = (held & (fabsf(peak) < 8.0f * range)) | none;
    if (none) mine = -1;
    if (__any(!sorted & sure)) {   // uniform
      bool by_score = false;
      if constexpr (KEYED) by_score = scored;
      if (by_score) mine = sort_entries<ZT, NQ, KEYED, SIGMOID>(a, t, j, mine);
      else mine = sort_entries<ZT, NQ, false, SIGMOID>(a, t, j, mine);
    }
    mine = j < k ? mine : -1;
    unsigned long long again = __ballot(!sure);
    while (again != 0) {   // uniform
      const int first = (__ffsll((long long)again) - 1) & 48;   // the token's first lane
      again &= ~(0xffffull << first);
      const unsigned on = (unsigned)__shfl((int)groups, first, 64);
      const int log2p = lanes_of_group(a);
      const int list = list_wide<ZT, KEYED, SIGMOID>(a, __shfl(t, first, 64), __shfl(k, first, 64),
                                                     [&](int e) { return a.groups <= 1 || stays(a, on, log2p, e); });
      const int mine_again = __shfl(list, j, 64);
      mine = (threadIdx.x & 48) == (unsigned)first ? mine_again : mine;
    }
  }

  const float zl = mine >= 0 ? clean(to_f32(logits[(size_t)t * a.E + mine])) : -INFINITY;
  float g;
  if (a.renorm) {
    // Sigmoid: shares of the scores themselves where none of the token's own underflows.  (By its own logits, so that its
    // gates are the same whatever tokens are beside it.)
    const unsigned long long low = SIGMOID ? __ballot(mine >= 0 && zl < -60.0f) : ~0ull;
    float p = 0.0f;
    if (SIGMOID) p = mine >= 0 ? 1.0f / (1.0f + expf(-zl)) : 0.0f;
    if (low != 0) {   // uniform
      const float l = mine >= 0 ? (SIGMOID ? log_sigmoid(zl) : zl) : -INFINITY;
      const float lm = row_top(l);
      const float shifted = mine >= 0 ? expf(l - lm) : 0.0f;
      p = ((low >> (threadIdx.x & 48)) & 0xffffu) != 0 ? shifted : p;
    }
    const float sum = row_sum_butterfly(p);   // (every lane takes part)
    g = mine >= 0 ? p / sum : 0.0f;
  } else {
    g = mine < 0 ? 0.0f : SIGMOID ? 1.0f / (1.0f + expf(-zl)) : expf(zl - m) * inv;
  }
  gate = mine >= 0 ? g * a.scale : 0.0f;
  if (tv && j < a.Kmax) {
    a.idx[(size_t)t * a.Kmax + j] = mine;
    a.gate[(size_t)t * a.Kmax + j] = gate;
  }
  return tv && j < a.Kmax ? mine : -1;
}

template <typename ZT, int NQ, bool KEYED, bool SIGMOID>
__global__ __launch_bounds__(256) void select_kernel(SelectArgs a) {
  __shared__ __align__(16) float ks[ROWS][64 * NQ + 4];
  float gate;
  (void)select_rows<ZT, NQ, KEYED, SIGMOID>(a, ks, gate);
}

// The same for tokens of one workgroup, and the experts that any of them lists, ascending, as work for the launches behind it.
template <int NQ, bool KEYED, bool SIGMOID>
__global__ __launch_bounds__(256) void select_units_kernel(SelectArgs a, fmoe_unit_list* list) {
  __shared__ __align__(16) float ks[ROWS][64 * NQ + 4];
  __shared__ uint32_t s_mask[FMOE_MAX_EXPERTS];
  __shared__ int s_rank[FMOE_MAX_EXPERTS];
  static_assert(ROWS >= FMOE_DECODE_TOKENS && FMOE_MAX_EXPERTS == 256, "tokens of a workgroup; four experts a lane");
  s_mask[threadIdx.x] = 0u;
  float gate;
  const int mine = select_rows<float, NQ, KEYED, SIGMOID>(a, ks, gate), tok = threadIdx.x >> 4;
  __syncthreads();
  if (mine >= 0) atomicOr(&s_mask[mine], 1u << tok);
  __syncthreads();
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x;
    uint32_t m[4];
    int rows = 0, some = 0, full = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      m[q] = s_mask[4 * lane + q];
      rows += __popc(m[q]);
      some += m[q] != 0u;
      full += (m[q] & (m[q] >> 8)) != 0u;
    }
    int row = wave_scan(rows) - rows, rank = wave_scan(some) - some, at = wave_scan(full) - full;
    if (lane == 63) {
      list->n = rank + some;
      list->n_full = at + full;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (m[q] == 0u) continue;
      s_rank[4 * lane + q] = rank;
      if ((m[q] & (m[q] >> 8)) != 0u) list->full[at++] = rank;
      list->unit[rank++] = fmoe_unit{4 * lane + q, row, m[q]};
      row += __popc(m[q]);
    }
  }
  __syncthreads();
  if (mine >= 0) list->gate[s_rank[mine]][tok] = gate;
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
      const float lm = row_top(in ? l : -INFINITY);
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

template <int NQ>
void run_select_units(const SelectArgs& a, bool keyed, fmoe_unit_list* list, hipStream_t stream) {
#define FMOE_SELECT(KEYED, SIGMOID) \
  hipLaunchKernelGGL((select_units_kernel<NQ, KEYED, SIGMOID>), dim3(1), dim3(256), 0, stream, a, list)
  if (keyed && a.sigmoid) FMOE_SELECT(true, true);
  else if (keyed) FMOE_SELECT(true, false);
  else if (a.sigmoid) FMOE_SELECT(false, true);
  else FMOE_SELECT(false, false);
#undef FMOE_SELECT
}

template <typename ZT, int NQ>
void run_select(const SelectArgs& a, bool keyed, hipStream_t stream) {
  const dim3 grid((a.T + ROWS - 1) / ROWS), block(256);
#define FMOE_SELECT(KEYED, SIGMOID) \
  hipLaunchKernelGGL((select_kernel<ZT, NQ, KEYED, SIGMOID>), grid, block, 0, stream, a)
  if (keyed && a.sigmoid) FMOE_SELECT(true, true);
  else if (keyed) FMOE_SELECT(true, false);
  else if (a.sigmoid) FMOE_SELECT(false, true);
  else FMOE_SELECT(false, false);
#undef FMOE_SELECT
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
                  float* topk_gate, hipStream_t stream, fmoe_unit_list* units) {
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
  if (units != nullptr) {   // fp32 logits of at most FMOE_DECODE_TOKENS tokens
    if (a.E <= 64) run_select_units<1>(a, keyed, units, stream);
    else if (a.E <= 128) run_select_units<2>(a, keyed, units, stream);
    else run_select_units<4>(a, keyed, units, stream);
  } else if (dtype == FMOE_BF16) run_select_by_size<bf16_t>(a, keyed, stream);
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
