// Device code that the bf16 expert-GEMM kernels share: tile geometry, descriptors, row gather, LDS operand reads, output
// tiles, hand-placed accumulators.
#pragma once

#include <type_traits>

#include "common.h"
#include "deal.h"
#include "tiles.h"

namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8_t;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4_t;
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));   // one 16-byte chunk

// silu(g) * u for values that are rounded next, to bf16, 16 or 8 bits: the hardware reciprocal (1 ulp of fp32) instead of
// the correctly rounded one, a third of the instructions (1.7 % of the gate/up kernel at 2064 rows per expert).  With the
// hardware's exponential off by 2^-20 (1 + |g|) of its size at most.
__device__ __forceinline__ float silu_mul_bf16(float g, float u) {
  return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)) * u;
}

// ======================================================================== bf16: weight-stream kernel
constexpr int SBM = 128;        // rows per tile: 8 MFMA row blocks of 16
constexpr int SBK = 64;         // k per tile: two 32-wide MFMA steps; one LDS row = 128 bytes
constexpr int A_STAGES = 4;     // LDS ring of activation k-tiles (weight-stream shape)
constexpr int B_SLOTS = 4;      // register ring of weight k-tiles (weight-stream shape)
// The dense shape of the kernel, for row lists of a few hundred rows per expert and more (where LDS and
// the CU's load path rather than the weight stream hold the weight-stream shape back: it reads every
// activation fragment from LDS once per column block and fetches every activation tile once per four
// column blocks): a workgroup owns 128 rows x 8 column blocks, each wavefront DNCB = 2 column blocks.  A
// wavefront's activation fragments then feed twice as many matrix instructions, which halves the LDS
// reads and the activation fetches per flop.  Two workgroups still share a CU (one hides the other's
// start-up and epilogue), so a wavefront has 256 registers: 128 accumulation registers that the kernel
// names itself and 128 vector registers for a k-step ring of weights, one group of fragments and
// addresses, which is why the wavefront-uniform part of every address is kept in scalar registers.
constexpr int DNCB = 2;         // column blocks per wavefront
constexpr int DA_STAGES = 4;    // LDS ring of activation k tiles (64 wide)
constexpr int DB_SLOTS = 4;     // register ring of weight k steps (32 wide)
constexpr int NON_TEMPORAL = 2; // cache hint of a buffer load
constexpr size_t WEIGHTS_PASS_BYTES = 384u << 20;   // one and a half times the memory-side cache, see deal.h

struct StreamProblem {
  const bf16_t* A;            // [*, lda]
  int lda;
  const int32_t* map1;        // row -> index (perm_src) or null
  const int32_t* map2;        // index -> token (kept_idx) or null
  int map1_limit;             // clamp for map1 values (exclusive), <= 0: none
  const u32x4_t* Bp;          // packed weights
  long long group_stride;     // 16-byte units between groups
  int nbw;                    // column blocks per group in the packing
  int ks;                     // 32-wide k steps per column block in the packing (K padded to 64)
  bf16_t* C;                  // [*, ldc]
  int ldc;
  int N, K;
  int n_col_tiles;
  int a_group_off;            // shared group g reads A columns from g*a_group_off (elements)
  long long c_group_off;      // and writes C at g*c_group_off (elements)
};

struct StreamArgs {
  StreamProblem p0;           // routed experts
  StreamProblem p1;           // shared group (tile.group == E)
  int E;
  const fmoe_tile* tiles;
  const int32_t* n_tiles;     // device
  int cols;                   // work items per tile entry in this launch (column tiles, or groups of them)
  int cols_entry;             // column tiles per tile entry
  int weights_pass;           // dense shape: the layer's weights do not stay in the memory-side cache anyway
};

// A list entry, by scalar loads of all its words at once (the lists are read-only in these kernels, which the
// compiler cannot see past their stores).
__device__ __forceinline__ fmoe_tile load_entry(const fmoe_tile* tiles, int ti) {
  typedef const __attribute__((address_space(4))) int32_t* const_ptr;
  const const_ptr p = (const_ptr)(uintptr_t)(tiles + ti);
  fmoe_tile t;
  t.group = p[0]; t.row0 = p[1]; t.rows = p[2]; t.col0 = p[3]; t.rt = p[4]; t.nrt = p[5];
  return t;
}
// Narrows an entry to row tile r of its run (bm rows per tile).
__device__ __forceinline__ void take_row_tile(fmoe_tile& t, int r, int bm) {
  t.row0 += r * bm;
  t.rows = t.rows - r * bm < bm ? t.rows - r * bm : bm;
}

// s_waitcnt vmcnt(n) with the other counters left alone (gfx9 encoding: vmcnt = bits 15:14 | 3:0)
#define FMOE_WAIT_VM(n) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(n) : "memory")
__device__ __forceinline__ void wait_vm_upto(int n) {   // n not known at compile time (loop tails)
  switch (n < 0 ? 0 : n) {
    case 0: FMOE_WAIT_VM(0); break;
    case 1: case 2: case 3: FMOE_WAIT_VM(1); break;
    case 4: case 5: case 6: case 7: FMOE_WAIT_VM(4); break;
    case 8: case 9: case 10: case 11: FMOE_WAIT_VM(8); break;
    case 12: case 13: case 14: case 15: FMOE_WAIT_VM(12); break;
    case 16: case 17: case 18: case 19: FMOE_WAIT_VM(16); break;
    default: FMOE_WAIT_VM(20); break;
  }
}
// NRB operand fragments (16 bytes per lane each, 2048 bytes apart) from LDS byte address `addr`,
// valid on return.  Written as one block of machine instructions so that the compiler, which knows
// nothing about the asynchronous global->LDS loads that filled the tile, neither adds waits for them
// here nor touches the destination registers before the LDS counter has drained.
template <int NRB>
__device__ __forceinline__ void lds_read_frags(uint32_t addr, u32x4_t (&f)[NRB]) {
  static_assert(NRB == 2 || NRB == 3 || NRB == 4 || NRB == 6 || NRB == 8, "supported fragment counts");
  if constexpr (NRB == 2) {
    asm volatile("ds_read_b128 %0, %2\n\tds_read_b128 %1, %2 offset:2048\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(f[0]), "=&v"(f[1]) : "v"(addr) : "memory");
  } else if constexpr (NRB == 3) {
    asm volatile("ds_read_b128 %0, %3\n\tds_read_b128 %1, %3 offset:2048\n\t"
                 "ds_read_b128 %2, %3 offset:4096\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]) : "v"(addr) : "memory");
  } else if constexpr (NRB == 4) {
    asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:2048\n\t"
                 "ds_read_b128 %2, %4 offset:4096\n\tds_read_b128 %3, %4 offset:6144\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3]) : "v"(addr) : "memory");
  } else if constexpr (NRB == 6) {
    asm volatile("ds_read_b128 %0, %6\n\tds_read_b128 %1, %6 offset:2048\n\t"
                 "ds_read_b128 %2, %6 offset:4096\n\tds_read_b128 %3, %6 offset:6144\n\t"
                 "ds_read_b128 %4, %6 offset:8192\n\tds_read_b128 %5, %6 offset:10240\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3]), "=&v"(f[4]), "=&v"(f[5])
                 : "v"(addr) : "memory");
  } else {
    asm volatile("ds_read_b128 %0, %8\n\tds_read_b128 %1, %8 offset:2048\n\t"
                 "ds_read_b128 %2, %8 offset:4096\n\tds_read_b128 %3, %8 offset:6144\n\t"
                 "ds_read_b128 %4, %8 offset:8192\n\tds_read_b128 %5, %8 offset:10240\n\t"
                 "ds_read_b128 %6, %8 offset:12288\n\tds_read_b128 %7, %8 offset:14336\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3]), "=&v"(f[4]), "=&v"(f[5]),
                   "=&v"(f[6]), "=&v"(f[7])
                 : "v"(addr) : "memory");
  }
}
// The same reads without the wait and with a compile-time byte offset OFF on top of the address register
// (one register then serves every stage of the ring): lds_issue_frags_at starts them, lds_settle_frags
// waits for them and is the point from which the compiler may use the registers (they are in/out
// operands of the wait).
template <int NRB, int OFF>
__device__ __forceinline__ void lds_issue_frags_at(uint32_t addr, u32x4_t (&f)[NRB]) {
  static_assert(NRB >= 1 && NRB <= 4, "supported fragment counts");
  static_assert(OFF >= 0 && OFF + (NRB - 1) * 2048 < 65536, "offset field of an LDS instruction");
  if constexpr (NRB == 1) {
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=&v"(f[0]) : "v"(addr), "n"(OFF) : "memory");
  } else if constexpr (NRB == 2) {
    asm volatile("ds_read_b128 %0, %2 offset:%3\n\tds_read_b128 %1, %2 offset:%4"
                 : "=&v"(f[0]), "=&v"(f[1]) : "v"(addr), "n"(OFF), "n"(OFF + 2048) : "memory");
  } else if constexpr (NRB == 3) {
    asm volatile("ds_read_b128 %0, %3 offset:%4\n\tds_read_b128 %1, %3 offset:%5\n\tds_read_b128 %2, %3 offset:%6"
                 : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2])
                 : "v"(addr), "n"(OFF), "n"(OFF + 2048), "n"(OFF + 4096) : "memory");
  } else {
    asm volatile("ds_read_b128 %0, %4 offset:%5\n\tds_read_b128 %1, %4 offset:%6\n\t"
                 "ds_read_b128 %2, %4 offset:%7\n\tds_read_b128 %3, %4 offset:%8"
                 : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3])
                 : "v"(addr), "n"(OFF), "n"(OFF + 2048), "n"(OFF + 4096), "n"(OFF + 6144) : "memory");
  }
}
template <int NRB>
__device__ __forceinline__ void lds_settle_frags(u32x4_t (&f)[NRB]) {
  static_assert(NRB >= 1 && NRB <= 4, "supported fragment counts");
  if constexpr (NRB == 1) {
    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(f[0]) : : "memory");
  } else if constexpr (NRB == 2) {
    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(f[0]), "+v"(f[1]) : : "memory");
  } else if constexpr (NRB == 3) {
    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(f[0]), "+v"(f[1]), "+v"(f[2]) : : "memory");
  } else {
    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(f[0]), "+v"(f[1]), "+v"(f[2]), "+v"(f[3]) : : "memory");
  }
}
#define FMOE_LPTR(p) ((__attribute__((address_space(3))) void*)(p))

// One (row tile, column tile) work item.  NAB = number of live 32-row bands of the tile (1..4):
// a compile-time constant, so the k loop below is straight-line code with a fixed number of loads,
// LDS reads and matrix instructions per step, and rows past the last live band cost nothing.
//   weights:     register ring of B_SLOTS k-tiles per wavefront (B_SLOTS-1 in flight)
//   activations: LDS ring of A_STAGES k-tiles filled by direct global->LDS loads (no register hop,
//                no LDS store instructions; A_STAGES-1 in flight).  Such a load drops the 64 lanes'
//                16-byte pieces at consecutive LDS addresses, so which (row, k chunk) a lane fetches
//                decides the LDS layout: rows are 128 bytes, and row r keeps its 16-byte chunk c at
//                position c ^ ((r >> 1) & 7), which makes the 16 rows x 16 bytes read for one matrix
//                operand fall on 16 different bank groups without any padding.
// Workgroup barrier without the memory fence of __syncthreads(): a fence would wait for EVERY
// outstanding global->LDS load (they count as stores to LDS), i.e. drain the prefetch ring each
// step.  What the barrier has to order here is covered explicitly: a wavefront waits for its own
// loads of the tile about to be read (FMOE_WAIT_VM) before the barrier, and its LDS reads of the
// previous tile have returned (lds_read_frags) before it.
__device__ __forceinline__ void block_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <int I, int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {   // f(integral_constant<int, i>) for i in [I, N)
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    static_for<I + 1, N>(f);
  }
}

// Byte offsets (into the buffer descriptor over P.A) of the activation rows this lane fetches: rows
// 32*it + 8*wave + lane/8 of the tile, through the two-level gather; rows past the tile reuse its last row.
// In two halves, a load each, between which the dense shape requests its first weights.
template <int NAB>
__device__ __forceinline__ void gather_first(const StreamProblem& P, const fmoe_tile& tile, int (&src)[NAB]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int it = 0; it < NAB; ++it) {
    const int r = 32 * it + 8 * wave + (lane >> 3);
    src[it] = tile.row0 + (r < tile.rows ? r : tile.rows - 1);
    if (P.map1) src[it] = P.map1[src[it]];
  }
}
template <int NAB>
__device__ __forceinline__ void gather_offsets(const StreamProblem& P, const int (&src)[NAB], uint32_t (&a_src)[NAB]) {
  const uint32_t a_max_row = 0xffffffffu / ((uint32_t)P.lda * 2u) - 1u;
#pragma unroll
  for (int it = 0; it < NAB; ++it) {
    int s = src[it];
    if (P.map1 && P.map1_limit > 0) s = s < 0 ? 0 : (s >= P.map1_limit ? P.map1_limit - 1 : s);
    if (P.map2) s = P.map2[s];
    s = (uint32_t)s < a_max_row ? s : (int)a_max_row;   // offsets stay below 4 GiB whatever the input
    a_src[it] = (uint32_t)s * (uint32_t)P.lda * 2u;
  }
}
// Nothing is moved across: what is requested before is requested first.
__device__ __forceinline__ void order_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Epilogue of one 128-row x 4-column-block output tile (column tile nt of the packing): accumulator
// register v of lane l holds row 4*(l/16) + v, column l%16 of a 16x16 block.  The tile is transposed
// through LDS (the activation ring, free once every wavefront has passed the opening barrier) so that
// global memory sees whole 128/256-byte row segments instead of 32-byte pieces.
template <bool SWIGLU, int NAB, int STAGES, typename ACC>
__device__ __forceinline__ void store_tile(const StreamProblem& P, const fmoe_tile& tile, int nt, ACC acc,
                                           bf16_t* As) {   // acc(rb, f): accumulator of row block rb, fragment f
  constexpr int NRB = 2 * NAB;
  constexpr int BC = SWIGLU ? 64 : 128;    // output columns of the block
  constexpr int CS = BC + 8;               // LDS row stride (elements): rows 4 apart land 16 banks apart
  static_assert(SBM * CS <= STAGES * SBM * SBK, "output tile fits in the activation ring");
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int N = P.N;
  __syncthreads();   // every wavefront is done with what the ring held
  static_for<0, NRB>([&](auto rbc) {
    constexpr int rb = decltype(rbc)::value;
    const f32x4_t c0 = acc(rbc, std::integral_constant<int, 0>{});
    const f32x4_t c1 = acc(rbc, std::integral_constant<int, 1>{});
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int row = rb * 16 + 4 * (lane >> 4) + v;
      if (SWIGLU) {
        As[row * CS + wave * 16 + (lane & 15)] = f32_to_bf16(silu_mul_bf16(c0[v], c1[v]));
      } else {
        As[row * CS + wave * 32 + (lane & 15)] = f32_to_bf16(c0[v]);
        As[row * CS + wave * 32 + 16 + (lane & 15)] = f32_to_bf16(c1[v]);
      }
    }
  });
  __syncthreads();
  constexpr int CPR = BC / 8;              // 16-byte chunks per row
  constexpr int RPP = 256 / CPR;           // rows per pass of the block
  const int col = nt * BC + (tid % CPR) * 8;
  const bool vec_ok = ((P.ldc & 7) == 0) && (col + 8 <= N) &&
                      ((reinterpret_cast<uintptr_t>(P.C) & 15) == 0);
#pragma unroll
  for (int r0 = 0; r0 < 32 * NAB; r0 += RPP) {
    const int row = r0 + tid / CPR;
    if (row >= tile.rows || col >= N) continue;
    const bf16_t* src = &As[row * CS + (tid % CPR) * 8];
    bf16_t* dst = P.C + (size_t)(tile.row0 + row) * P.ldc + col;
    if (vec_ok) {
      // streaming store: the next kernel reads the tile, this one never does, and in L2 it would only
      // displace the weights and activation tiles the other workgroups are sharing
      __builtin_nontemporal_store(*reinterpret_cast<const u32x4_t*>(src), reinterpret_cast<u32x4_t*>(dst));
    } else {
      for (int i = 0; i < 8 && col + i < N; ++i) dst[i] = src[i];
    }
  }
}

// The dense shape keeps its 32 accumulators in accumulation registers that it names itself: accumulator
// IDX is a[4*IDX : 4*IDX+3].  Left to the compiler, the accumulators share the vector register budget
// with everything else and part of them travels through scratch memory; named, they cost the
// allocator nothing, and, being volatile, the instructions keep their place in the step.  The compiler
// does not see what these instructions do, so it is told: dense_claim_acc() lists a0..a127 as written
// (a wavefront is then given them, and the compiler half of its 256 registers), and every matrix
// instruction lists its four registers as destroyed (mfma_at<IDX>), so that the compiler cannot keep a
// value of its own in one of them across the k loop -- it did once: a row index of the epilogue, which
// came back as accumulator bits and sent the output store to a wild address.  On top of that the build
// reads the generated code of the dense kernels from the first to the last line and fails if the
// compiler itself placed anything in an accumulation register, and the parity tests run this shape on
// every size.
template <int IDX>
__device__ __forceinline__ f32x4_t read_acc() {
  float r0, r1, r2, r3;
  asm volatile("v_accvgpr_read_b32 %0, a[%4]\n\tv_accvgpr_read_b32 %1, a[%5]\n\t"
               "v_accvgpr_read_b32 %2, a[%6]\n\tv_accvgpr_read_b32 %3, a[%7]"
               : "=v"(r0), "=v"(r1), "=v"(r2), "=v"(r3)
               : "n"(4 * IDX), "n"(4 * IDX + 1), "n"(4 * IDX + 2), "n"(4 * IDX + 3));
  return f32x4_t{r0, r1, r2, r3};
}
#include "dense_regs.inc"   // dense_claim_acc(): zeroes a0..a127 and lists them as written; mfma_at<IDX>()

}  // namespace
