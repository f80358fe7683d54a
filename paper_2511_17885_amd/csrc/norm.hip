// Root-mean-square norm of rows with the addition in front of it, its output in the storage type or in 8 bits, and its gradient.
// Compiled with floating-point contraction off: the roundings that norm_dev.h relies on are written out.
//
// Bound: memory.  A wavefront has a row in registers (up to 4096 elements; a workgroup of four wavefronts has one of up to 16384,
// or where there are few rows), reads it once and writes its outputs once.  22016 rows of 2048 in bf16: 58 us, 6.2 TB/s (a copy of
// 1 GiB 5.2); gradient 68 us with the sums of the weight's; 8192 rows to 8 bits 26.8 us, 4.4 TB/s: some 25 vector instructions an
// element for the exact rounding beside the loads.  (Called again and again, so that outputs are where the last call's were, which the
// memory-side cache still has in part; four sets of inputs and outputs in turn, as below: 68 us for the first of these.)

#include "norm_dev.h"
#include "rows8_dev.h"

namespace {

using namespace rms;

constexpr int MAX_D = FMOE_NORM_MAX_D;

struct NormArgs {
  const void *x, *delta, *w;
  int T, d;
  float eps;
  double inv_d;
  void *h, *n;          // h may be null (nobody wants the sum), n with rows in 8 bits
  uint32_t* codes;      // [T, d] bytes
  uint8_t* scales;      // [T, scale_stride]
  int scale_stride;     // groups of 32, rounded up to words
};

// A sum over the wavefronts of a workgroup that share a row (WPR of them); s_part: 4 doubles
template <int WPR>
__device__ __forceinline__ double row_total(double v, double* s_part) {
  v = wave_sum(v);
  if constexpr (WPR > 1) {
    const int wave = threadIdx.x >> 6;
    __syncthreads();   // the last sum has been read
    if ((threadIdx.x & 63) == 0) s_part[wave] = v;
    __syncthreads();
    v = (s_part[0] + s_part[1]) + (s_part[2] + s_part[3]);
  }
  return v;
}

// NU units of eight a lane; WPR wavefronts a row (1 or all 4).
template <typename XT, typename WT, int NU, int WPR, bool ROWS8, bool PASS>
__global__ __launch_bounds__(256) void rms_norm_kernel(NormArgs a) {
  __shared__ double s_part[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = WPR == 1 ? (int)blockIdx.x * 4 + wave : (int)blockIdx.x;
  if (row >= a.T) return;   // uniform over those who share a row
  const int first = WPR == 1 ? lane : (int)threadIdx.x;
  constexpr int STEP = 64 * WPR;
  const int units = a.d >> 3;
  const size_t base = (size_t)row * a.d;
  Unit<XT> h[NU], dl[NU];
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    const int u = first + STEP * i;
    h[i].zero();
    if (u < units) h[i].template load<PASS>(static_cast<const XT*>(a.x) + base + u * 8);
  }
  if (a.delta != nullptr) {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int u = first + STEP * i;
      dl[i].zero();
      if (u < units) dl[i].template load<PASS>(static_cast<const XT*>(a.delta) + base + u * 8);
    }
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
      for (int e = 0; e < 8; e += 2)
        h[i].set2(e, add_rounded<XT>(h[i].get(e), dl[i].get(e)), add_rounded<XT>(h[i].get(e + 1), dl[i].get(e + 1)));
  }
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < NU; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const double v = (double)h[i].get(e);
      sum = fma(v, v, sum);
    }
  const Scale r = row_scale(row_total<WPR>(sum, s_part), a.inv_d, a.eps);
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    const int u = first + STEP * i;
    const bool in = u < units;
    float w[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (in) {
      load_weights<WT>(a.w, u * 8, w);
      if (a.h != nullptr) h[i].template store<PASS>(static_cast<XT*>(a.h) + base + u * 8);
    }
    if constexpr (!ROWS8) {
      Unit<XT> n;
#pragma unroll
      for (int e = 0; e < 8; e += 2)
        n.set2(e, value_rounded<XT>(h[i].get(e), w[e], r), value_rounded<XT>(h[i].get(e + 1), w[e + 1], r));
      if (in) n.store(static_cast<XT*>(a.n) + base + u * 8);
    } else {
      // values rounded to odd keep what the choice of the scale and the rounding to 4 significant bits need
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float hi, lo;
        value(h[i].get(e), w[e], r, hi, lo);
        v[e] = in ? odd(hi, lo) : 0.0f;
      }
      uint32_t scale;
      const uint2 c = rows8::quantize(v, scale, [](uint32_t m) { return rows8::quad_max(m); });
      if (in) *reinterpret_cast<uint2*>(reinterpret_cast<char*>(a.codes) + base + u * 8) = c;
      if ((u & 3) == 0 && (u >> 2) < a.scale_stride) a.scales[(size_t)row * a.scale_stride + (u >> 2)] = (uint8_t)scale;
    }
  }
}

struct NormBackwardArgs {
  const void *h, *w, *dn, *dh;
  int T, d;
  float eps;
  double inv_d;
  void* dx;
  float* part;          // [blocks, d] or null: no gradient of the weight
};

// With c = h r and g = dn w: dx = dh + r (g - c mean(g c)); a workgroup's rows add dn c up for the weight, one partial sum each.
template <typename XT, typename WT, int NU, int WPR, bool PASS>
__global__ __launch_bounds__(256) void rms_norm_backward_kernel(NormBackwardArgs a) {
  __shared__ double s_part[4];
  __shared__ float s_dw[WPR == 1 ? 64 * NU * 8 : 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int first = WPR == 1 ? lane : (int)threadIdx.x;
  constexpr int STEP = 64 * WPR;
  const int units = a.d >> 3;
  float dw[NU][8];
#pragma unroll
  for (int i = 0; i < NU; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[i][e] = 0.0f;
  Unit<WT> w[NU];
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    w[i].zero();
    if (first + STEP * i < units) w[i].load(static_cast<const WT*>(a.w) + (first + STEP * i) * 8);
  }
  const int rows_a_step = WPR == 1 ? (int)gridDim.x * 4 : (int)gridDim.x;
  for (int row = WPR == 1 ? (int)blockIdx.x * 4 + wave : (int)blockIdx.x; row < a.T; row += rows_a_step) {
    const size_t base = (size_t)row * a.d;
    Unit<XT> h[NU], g[NU], dh[NU];
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int u = first + STEP * i;
      h[i].zero();
      g[i].zero();
      dh[i].zero();
      if (u < units) {
        h[i].template load<PASS>(static_cast<const XT*>(a.h) + base + u * 8);
        g[i].template load<PASS>(static_cast<const XT*>(a.dn) + base + u * 8);
        if (a.dh != nullptr) dh[i].template load<PASS>(static_cast<const XT*>(a.dh) + base + u * 8);
      }
    }
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double v = (double)h[i].get(e);
        sum = fma(v, v, sum);
      }
    const Scale r = row_scale(row_total<WPR>(sum, s_part), a.inv_d, a.eps);
    float dot = 0.0f;
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float c = __builtin_amdgcn_ldexpf(h[i].get(e), r.q) * r.hi;
        const float dn = g[i].get(e);
        dot = fmaf(dn * w[i].get(e), c, dot);
        dw[i][e] = fmaf(dn, c, dw[i][e]);
      }
    const float m = (float)(row_total<WPR>((double)dot, s_part) * a.inv_d);
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int u = first + STEP * i;
      Unit<XT> out;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float c = __builtin_amdgcn_ldexpf(h[i].get(e), r.q) * r.hi;
        const float t = __builtin_amdgcn_ldexpf(fmaf(-c, m, g[i].get(e) * w[i].get(e)) * r.hi, r.q);
        v[e] = a.dh != nullptr ? t + dh[i].get(e) : t;
      }
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        if constexpr (sizeof(XT) == 2) out.set2(e, nearest_bf16(v[e]), nearest_bf16(v[e + 1]));
        else out.set2(e, v[e], v[e + 1]);
      }
      if (u < units) out.template store<PASS>(static_cast<XT*>(a.dx) + base + u * 8);
    }
  }
  if (a.part == nullptr) return;
  float* const part = a.part + (size_t)blockIdx.x * a.d;
  if constexpr (WPR == 1) {   // the wavefronts' sums one after the other
    for (int turn = 0; turn < 4; ++turn) {
      if (wave == turn) {
#pragma unroll
        for (int i = 0; i < NU; ++i)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int at = (i * 8 + e) * 64 + lane;   // no two lanes on a bank
            dw[i][e] = turn == 0 ? dw[i][e] : s_dw[at] + dw[i][e];
            if (turn < 3) s_dw[at] = dw[i][e];
          }
      }
      __syncthreads();
    }
    if (wave != 3) return;
  }
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    const int u = first + STEP * i;
    if (u >= units) continue;
    reinterpret_cast<f32x4_t*>(part + u * 8)[0] = f32x4_t{dw[i][0], dw[i][1], dw[i][2], dw[i][3]};
    reinterpret_cast<f32x4_t*>(part + u * 8)[1] = f32x4_t{dw[i][4], dw[i][5], dw[i][6], dw[i][7]};
  }
}

// The partial sums of every column, in a fixed order: a workgroup has 16 columns, four a lane, and takes 64 partial sums at a time.
__global__ __launch_bounds__(256) void rms_norm_weight_kernel(const float* __restrict__ part, int parts, int d,
                                                              float* __restrict__ dw) {
  __shared__ double s[64][17];
  const int c = (threadIdx.x & 3) * 4, first = threadIdx.x >> 2, k = (int)blockIdx.x * 16 + c;   // (d is a multiple of eight)
  double sum[4] = {0.0, 0.0, 0.0, 0.0};
  if (k < d) {
#pragma unroll 8
    for (int p = first; p < parts; p += 64) {
      const f32x4_t v = *reinterpret_cast<const f32x4_t*>(part + (size_t)p * d + k);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += (double)v[e];
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) s[first][c + e] = sum[e];
  __syncthreads();
  const int col = (int)blockIdx.x * 16 + (int)threadIdx.x;
  if (threadIdx.x >= 16 || col >= d) return;
  double total = 0.0;
#pragma unroll
  for (int p = 0; p < 64; ++p) total += s[p][threadIdx.x];
  dw[col] = (float)total;
}

// Do the inputs and h, which nobody asks for again soon, pass the caches by?  (n is read by the next launch and stays.)  us with / without
// (in a graph, four sets of tensors in turn): bf16, d 2048, 22016 rows 68.4 / 71.9, 8192 rows 29.0 / 30.8, in 8 bits 30.0 / 34.1; gradient
// 22016 rows 69.8 / 76.6, 8192 rows 32.8 / 34.9, 4096 rows (67 MB) 22.8 / 20.5.
bool passes(size_t bytes) { return bytes >= ((size_t)100 << 20); }

// Wavefronts a row: all four of a workgroup for rows that one cannot hold, and where rows of more than 128 units are few.  us with one / four:
// bf16, d 2048, 4096 rows 15.5 / 14.2, in 8 bits 18.9 / 15.9, 2048 rows 11.5 / 10.2, 600 rows 6.9 / 5.4; d 1280 100 rows 5.5 / 4.4; d 1288 in
// fp32 1601 rows 9.7 / 9.6; d 1024 4096 rows 10.3 / 11.0, in 8 bits 11.7 / 13.1; d 512 3000 rows 5.6 / 7.7.  (The figures end at d 2048.)
int waves_per_row(int T, int d) { return d > 4096 || (d > 1024 && T <= 4096) ? 4 : 1; }
// The gradient, with two sums a row between which four wavefronts would wait for each other: d 2048 bf16 22016 rows 69.8 / 86.7, 4096 rows
// 20.5 / 21.9, 200 rows 8.3 / 8.2; d 1280 in fp32 600 rows 10.2 / 11.5, 1600 rows 14.6 / 13.9.  (The figures end at d 2048.)
int waves_per_gradient(int d) { return d > 4096 ? 4 : 1; }

template <typename XT, typename WT, bool ROWS8>
void run_norm(const NormArgs& a, hipStream_t stream) {
  const int wpr = waves_per_row(a.T, a.d);
  const int units = ROWS8 ? (a.d + 127) / 128 * 16 : a.d / 8, per_lane = (units + 64 * wpr - 1) / (64 * wpr);
  const dim3 grid(wpr == 1 ? (a.T + 3) / 4 : a.T), block(256);
  const bool pass = wpr == 1 && passes((size_t)a.T * a.d * sizeof(XT) * (a.delta != nullptr ? 4 : 2));
#define FMOE_NORM(NU)                                                                                                 \
  do {                                                                                                                \
    if (pass) hipLaunchKernelGGL((rms_norm_kernel<XT, WT, NU, 1, ROWS8, true>), grid, block, 0, stream, a);           \
    else if (wpr == 1) hipLaunchKernelGGL((rms_norm_kernel<XT, WT, NU, 1, ROWS8, false>), grid, block, 0, stream, a); \
    else hipLaunchKernelGGL((rms_norm_kernel<XT, WT, NU, 4, ROWS8, false>), grid, block, 0, stream, a);               \
  } while (0)
  if (per_lane <= 1) FMOE_NORM(1);
  else if (per_lane <= 2) FMOE_NORM(2);
  else if (per_lane <= 3) FMOE_NORM(3);
  else if (per_lane <= 4) FMOE_NORM(4);
  else FMOE_NORM(8);
#undef FMOE_NORM
}
template <typename XT, typename WT>
void run_backward(const NormBackwardArgs& a, int blocks, hipStream_t stream) {
  const int wpr = waves_per_gradient(a.d);
  const int per_lane = (a.d / 8 + 64 * wpr - 1) / (64 * wpr);
  const dim3 grid(blocks), block(256);
  const bool pass = wpr == 1 && passes((size_t)a.T * a.d * sizeof(XT) * (a.dh != nullptr ? 4 : 3));
#define FMOE_NORM(NU)                                                                                                   \
  do {                                                                                                                  \
    if (pass) hipLaunchKernelGGL((rms_norm_backward_kernel<XT, WT, NU, 1, true>), grid, block, 0, stream, a);           \
    else if (wpr == 1) hipLaunchKernelGGL((rms_norm_backward_kernel<XT, WT, NU, 1, false>), grid, block, 0, stream, a); \
    else if constexpr (NU > 2) /* four wavefronts: rows of more than 512 units */                                       \
      hipLaunchKernelGGL((rms_norm_backward_kernel<XT, WT, NU, 4, false>), grid, block, 0, stream, a);                  \
  } while (0)
  if (per_lane <= 1) FMOE_NORM(1);
  else if (per_lane <= 2) FMOE_NORM(2);
  else if (per_lane <= 3) FMOE_NORM(3);
  else if (per_lane <= 4) FMOE_NORM(4);
  else FMOE_NORM(8);
#undef FMOE_NORM
}

}  // namespace

// Workgroups of the backward kernel, and so partial sums of the weight's gradient
int norm_backward_blocks(int T, int d) {
  const int rows = waves_per_gradient(d) == 1 ? (T + 3) / 4 : T;
  return rows < 512 ? rows : 512;
}

int launch_rms_norm(const void* x, const void* delta, const void* weight, int dtype, int weight_dtype, int T, int d, float eps,
                    void* h, void* n, void* codes, uint8_t* scales, hipStream_t stream) {
  static_assert(MAX_D == 256 * 8 * 8, "a workgroup holds a row");
  const NormArgs a{x, delta, weight, T, d, eps, 1.0 / (double)d, h, n, static_cast<uint32_t*>(codes), scales, (d + 127) / 128 * 4};
  const bool b = dtype == FMOE_BF16, wb = weight_dtype == FMOE_BF16;
  if (codes != nullptr) {
    if (b && wb) run_norm<bf16_t, bf16_t, true>(a, stream);
    else if (b) run_norm<bf16_t, float, true>(a, stream);
    else if (wb) run_norm<float, bf16_t, true>(a, stream);
    else run_norm<float, float, true>(a, stream);
  } else {
    if (b && wb) run_norm<bf16_t, bf16_t, false>(a, stream);
    else if (b) run_norm<bf16_t, float, false>(a, stream);
    else if (wb) run_norm<float, bf16_t, false>(a, stream);
    else run_norm<float, float, false>(a, stream);
  }
  FMOE_HIP_CHECK(hipGetLastError());
  return FMOE_OK;
}

int launch_rms_norm_backward(const void* h, const void* weight, const void* d_n, const void* d_h, int dtype, int weight_dtype,
                             int T, int d, float eps, void* d_x, float* d_weight, float* part, hipStream_t stream) {
  const int blocks = norm_backward_blocks(T, d);
  const NormBackwardArgs a{h, weight, d_n, d_h, T, d, eps, 1.0 / (double)d, d_x, d_weight != nullptr ? part : nullptr};
  if (T > 0) {
    const bool b = dtype == FMOE_BF16, wb = weight_dtype == FMOE_BF16;
    if (b && wb) run_backward<bf16_t, bf16_t>(a, blocks, stream);
    else if (b) run_backward<bf16_t, float>(a, blocks, stream);
    else if (wb) run_backward<float, bf16_t>(a, blocks, stream);
    else run_backward<float, float>(a, blocks, stream);
  }
  if (d_weight != nullptr)
    hipLaunchKernelGGL(rms_norm_weight_kernel, dim3((d + 15) / 16), dim3(256), 0, stream, part, blocks, d, d_weight);
  FMOE_HIP_CHECK(hipGetLastError());
  return FMOE_OK;
}
