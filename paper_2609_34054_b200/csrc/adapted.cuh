// The projection of a batch whose rows belong to different agents, Y[m] = X[m] W + s (X[m] A_a(m)) B_a(m):  what its kernels share,
// and the rank-r product T = s X A_a of every row with its own agent's A (bf16, [M][rank, at least 16]).
//
// T is small work (2 M K r flops) that the main kernel needs only at its end.  For few rows it runs beside it: the shrink kernel lets its
// dependent start as soon as all its own blocks run - behind its own wait for the kernel ahead, so whatever
// the dependent reads before ITS wait was complete before either started - and uses little shared memory and at most half of an SM's registers (90 .. 128 a
// thread; the forms of 16 or 32 rows, and most in 8 bits, spill 4 .. 116 bytes at that limit), so that a block of the main kernel fits on the same SM (not
// one of the few-row kernel for 17 .. 32 rows, with 178 registers, in 8 bits 255 and 108 bytes of spills).  For many rows it is a kernel on the tensor cores of its own (adapted_shrink.cuh).
// For a decode step it is latency and no more (8 rows of 4096, eight agents of rank 32: 4.3 us beside a main kernel of 7), and so it is for 777 rows of 1024 (5.7).
// T is rounded to bf16, the operand type of the MMA that takes it: 2^-8 of the adapter's term, which is added to a sum that is
// rounded to bf16 as a whole.
#pragma once
#include "adapted_plan.h"
#include "norm.cuh"
#include "tc_common.cuh"

namespace precc {

struct AdaptedParams {
  int M, N, K, rank, rank_pad;                // rank_pad: rank, at least 16 (the K of one MMA)
  int rank_shift;                             // log2 of rank
  int n_agents;
  const int32_t* agent_id;                    // [M], or null: no adapters in this call
  const void* x;                              // [M][K] bf16 or e4m3
  const float* x_scale;                       // 8 bits: [M]
  const float* w_scale;                       // 8 bits: [N]
  const void* A;                              // packed bf16 [K/64][n_agents * rank][64], or e4m3 [K/128][2: value, rest][n_agents * rank][128]
  const float* a_scale;                       // 8 bits: [n_agents * rank]
  const __nv_bfloat16* B;                     // [n_agents][rank][N] (8 bits: divided by w_scale)
  __nv_bfloat16* T;                           // [M][rank_pad]
  __nv_bfloat16* y;                           // [M][N]
  float s;
  int tile_rows;                              // shrink kernel: rows of a block
  int BN, stages, tmem_cols;
  int kps;                                    // shrink kernel of many rows: k-blocks in a slot of its ring
  uint32_t* status;
};

// A walk over the slots of a ring: the slot, and the parity of its present round.  (Counted along: a division by the number of slots, which is
// not known when the kernel is compiled, would cost the issuing warps more than the instructions they issue.)
// The loops that issue copies and MMAs run in one elected thread from end to end.  With an election in every step, and the whole warp waiting on
// the barriers, a step of four MMAs took 364 .. 388 cycles; so it takes 263 up to 128 columns, and what the MMAs take beyond.
struct RingWalk {
  int s = 0;
  uint32_t parity = 0;
  bool filled = false;                        // the first round is over: slots have to be waited for
  __device__ __forceinline__ void next(int slots) {
    if (++s == slots) { s = 0; parity ^= 1u; filled = true; }
  }
  __device__ __forceinline__ void skip(int n, int slots) {
    const int to = s + n, rounds = to / slots;
    s = to - rounds * slots;
    parity ^= rounds & 1;
    filled |= rounds > 0;
  }
};

// 8 bits: a sum in units of its column's and its row's scale.  One scale after the other, and subnormal numbers kept: the product of the two may leave
// fp32's range where the result does not (the norm leaves row scales down to 2^-126).
__device__ __forceinline__ float unscale(float v, float w_scale, float x_scale) { return mul_full(mul_full(v, w_scale), x_scale); }

// An agent id as the kernels use it: out of range counts as "no adapter" (reported by the shrink kernel).
__device__ __forceinline__ int agent_of(const AdaptedParams& p, long long row) {
  if (row >= p.M) return -1;
  const int a = p.agent_id[row];
  return a >= 0 && a < p.n_agents ? a : -1;
}

// The agents of the 256 rows from m0 on, as far as `rows` of them (id[i]: row 32 i + lane).  Asked for at once and looked at later: eight loads
// behind conditions of their own wait for one another, 4 us a tile.
__device__ __forceinline__ void load_agents(const AdaptedParams& p, long long m0, int lane, int (&id)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) id[i] = __ldg(p.agent_id + min(m0 + 32 * i + lane, (long long)p.M - 1));
}
// One bit for each agent among them; ids out of range, and rows past M or `rows`, become -1.
__device__ __forceinline__ unsigned long long agents_present(const AdaptedParams& p, long long m0, int rows, int lane, int (&id)[8]) {
  unsigned lo = 0, hi = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const bool on = 32 * i + lane < rows && m0 + 32 * i + lane < p.M && id[i] >= 0 && id[i] < p.n_agents;
    if (!on) id[i] = -1;
    lo |= on && id[i] < 32 ? 1u << (id[i] & 31) : 0u;
    hi |= on && id[i] >= 32 ? 1u << (id[i] & 31) : 0u;
  }
  return (static_cast<unsigned long long>(__reduce_or_sync(0xffffffffu, hi)) << 32) | __reduce_or_sync(0xffffffffu, lo);
}

// D(16x8, fp32) += A(16x32, e4m3, row) * B(32x8, e4m3, col)
__device__ __forceinline__ void mma_e4m3_16832(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Four of the instructions above cover 128 bytes of K: 64 bf16 or 128 e4m3.
template <bool Q8>
__device__ __forceinline__ void mma_step(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (Q8) mma_e4m3_16832(d, a, b0, b1);
  else mma_bf16_16816(d, a, b0, b1);
}

constexpr int SHRINK_WARPS = 8;
constexpr int SHRINK_THREADS = SHRINK_WARPS * 32;

// T of up to 8 NT rows (fewer where that fills more SMs: a block takes the agents among its rows one after the other).  MT: 16-wide pieces of the rank.  The K extent is split over the warps of a block and the blocks of a cluster;
// partial sums meet in shared memory in a fixed order.  The rows are the N axis of mma.sync and the coordinates of the rank its M axis, so a row
// is computed in its own column of the product and nothing of another agent's adapter reaches it: for every agent among the rows
// the product is taken with the rows of that agent (the others' columns are zero and dropped).
// Fragments come straight from global memory, 16 bytes a lane: of the 128 bytes of a step a lane of a quad takes pieces t and t + 4, and as A and X
// agree on which, the order of K inside a step does not matter.
// 8 bits: A is the sum of two e4m3 matrices with a common scale per coordinate, the value and what its rounding left (see
// pack_adapter_e4m3_kernel), so that it keeps the bits of bf16; the second is simply more steps of K.
template <int MT, int NT, bool Q8>
__global__ void __launch_bounds__(SHRINK_THREADS, 2)
adapted_shrink_kernel(const AdaptedParams p) {
  constexpr int RT = 8 * NT, R = 16 * MT;
  constexpr int MW = MT > 2 ? 2 : MT, KW = SHRINK_WARPS * MW / MT;      // pieces of the rank of a warp; warps that share the K extent
  __shared__ float red[KW][RT][R];
  __shared__ float part[RT][R];
  uint32_t rank_c, KS;
  asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(rank_c));
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;\n" : "=r"(KS));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int kw = warp % KW, m0 = warp / KW * MW;
  const long long row0 = (long long)(blockIdx.x / KS) * p.tile_rows;
  pdl_wait();
  pdl_launch_dependents();

  int id = -1;
  if (lane < p.tile_rows && row0 + lane < p.M) {
    const int raw = p.agent_id[row0 + lane];
    if (raw < -1 || raw >= p.n_agents) { if (warp == 0 && rank_c == 0) atomicOr(p.status, StatusBits::BAD_INDEX); }
    else id = raw;
  }
  unsigned todo = __ballot_sync(0xffffffffu, id >= 0);
  const unsigned with_adapter = todo;
  constexpr int PARTS = Q8 ? 2 : 1;
  const int steps = p.K / (Q8 ? 128 : 64) * PARTS;
  const int v0 = (int)((long long)rank_c * steps / KS), v1 = (int)((long long)(rank_c + 1) * steps / KS);
  const int a_rows = p.n_agents * p.rank;
  const long long row_bytes = (long long)p.K * (Q8 ? 1 : 2);

  // step v of agent a: fragments of this warp's part of A, and of the rows of that agent
  auto fetch = [&](int a, unsigned mine, int v, uint4 (&av)[MW][2][2], uint4 (&xv)[NT][2]) {
#pragma unroll
    for (int m = 0; m < MW; ++m)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = (m0 + m) * 16 + h * 8 + g;
        const uint4* src = static_cast<const uint4*>(p.A) + ((long long)v * a_rows + a * p.rank + r) * 8;      // (step v = value or rest of k-block v / 2)
#pragma unroll
        for (int c = 0; c < 2; ++c) av[m][h][c] = r < p.rank ? __ldg(src + t + 4 * c) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const bool on = (mine >> (n * 8 + g)) & 1u;
      const uint4* src = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(p.x) + (row0 + n * 8 + g) * row_bytes + (long long)(v / PARTS) * AP_ROW_BYTES);
#pragma unroll
      for (int c = 0; c < 2; ++c) xv[n][c] = on ? __ldg(src + t + 4 * c) : make_uint4(0, 0, 0, 0);
    }
  };
  float acc[MW][NT][4];
  auto clear = [&]() {
#pragma unroll
    for (int m = 0; m < MW; ++m)
#pragma unroll
      for (int n = 0; n < NT; ++n) { acc[m][n][0] = acc[m][n][1] = acc[m][n][2] = acc[m][n][3] = 0.f; }
  };
  auto multiply = [&](const uint4 (&av)[MW][2][2], const uint4 (&xv)[NT][2]) {
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int m = 0; m < MW; ++m) {
          const uint32_t a0[4] = {av[m][0][c].x, av[m][1][c].x, av[m][0][c].y, av[m][1][c].y};
          const uint32_t a1[4] = {av[m][0][c].z, av[m][1][c].z, av[m][0][c].w, av[m][1][c].w};
          mma_step<Q8>(acc[m][n], a0, xv[n][c].x, xv[n][c].y);
          mma_step<Q8>(acc[m][n], a1, xv[n][c].z, xv[n][c].w);
        }
  };
  auto leave = [&](unsigned mine) {                // a row belongs to one agent: its column goes to its place once
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = n * 8 + 2 * t + e;
        if ((mine >> r) & 1u) {
#pragma unroll
          for (int m = 0; m < MW; ++m) { red[kw][r][(m0 + m) * 16 + g] = acc[m][n][e]; red[kw][r][(m0 + m) * 16 + 8 + g] = acc[m][n][2 + e]; }
        }
      }
  };
  auto next_agent = [&](unsigned& mine) {          // -1: none left
    mine = 0;
    if (!todo) return -1;
    const int a = __shfl_sync(0xffffffffu, id, __ffs(todo) - 1);
    mine = __ballot_sync(0xffffffffu, id == a);
    todo &= ~mine;
    return a;
  };
  unsigned mine;
  int a = next_agent(mine);
  clear();
  if constexpr (NT == 1) {
    // few rows, so often an agent of its own for each: the next step's fragments, be it of the next agent, are on their way while one is multiplied
    uint4 a0[MW][2][2], x0[NT][2], a1[MW][2][2], x1[NT][2];
    int v = v0 + kw;
    if (v >= v1) { while (a >= 0) { leave(mine); a = next_agent(mine); } }
    if (a >= 0) fetch(a, mine, v, a0, x0);
    auto step = [&](const uint4 (&av)[MW][2][2], const uint4 (&xv)[NT][2], uint4 (&an)[MW][2][2], uint4 (&xn)[NT][2]) {
      const unsigned now = mine;
      const bool last = v + KW >= v1;
      if (last) { a = next_agent(mine); v = v0 + kw; } else { v += KW; }
      if (a >= 0) fetch(a, mine, v, an, xn);
      multiply(av, xv);
      if (last) { leave(now); clear(); }
    };
    while (a >= 0) {
      step(a0, x0, a1, x1);
      if (a >= 0) step(a1, x1, a0, x0);
    }
  } else {
    for (; a >= 0; a = next_agent(mine)) {
#pragma unroll 2
      for (int v = v0 + kw; v < v1; v += KW) {
        uint4 av[MW][2][2], xv[NT][2];
        fetch(a, mine, v, av, xv);
        multiply(av, xv);
      }
      leave(mine);
      clear();
    }
  }
  // the scales of what this thread finishes below, on their way while the sums meet
  constexpr int MINE = RT * R / SHRINK_THREADS > 0 ? RT * R / SHRINK_THREADS : 1;
  float scale[MINE];
#pragma unroll
  for (int k = 0; k < MINE; ++k) {
    const int i = threadIdx.x + ((int)rank_c + k * (int)KS) * SHRINK_THREADS, r = i / R, c = i % R;      // (R is 16 or more: at most two rows a warp)
    scale[k] = p.s;
    if constexpr (Q8) {
      const int a = __shfl_sync(0xffffffffu, id, r & 31);
      if (i < RT * R && a >= 0 && c < p.rank) scale[k] *= __ldg(p.a_scale + a * p.rank + c);
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < RT * R; i += SHRINK_THREADS) {
    const int r = i / R, c = i % R;
    float v = 0.f;
    if ((with_adapter >> r) & 1u) {
#pragma unroll
      for (int w = 0; w < KW; ++w) v += red[w][r][c];
    }
    part[r][c] = v;
  }
  if (KS > 1) {
    asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
  } else {
    __syncthreads();
  }
  // every block of the cluster finishes a share of the elements, adding the blocks' sums in rank order
#pragma unroll
  for (int j = 0; j < MINE; ++j) {
    const int i = threadIdx.x + ((int)rank_c + j * (int)KS) * SHRINK_THREADS, r = i / R, c = i % R;
    if (i >= RT * R || !((with_adapter >> r) & 1u)) continue;
    const uint32_t local = smem_u32(&part[r][c]);
    float u[8], v = 0.f;
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) {             // (asked for at once: one read after the other costs its latency every time)
      u[k] = 0.f;
      if (k < KS) asm volatile("ld.shared::cluster.f32 %0, [%1];\n" : "=f"(u[k]) : "r"(dsmem_addr(local, k)));
    }
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) v += u[k];
    // (rank 8: the other eight of an MMA's sixteen coordinates are zeros, in a row with an infinity too, where the product gave 0 * inf)
    p.T[(row0 + r) * p.rank_pad + c] = __float2bfloat16(c < p.rank ? scale[j] * v : 0.f);
  }
  if (KS > 1) {
    asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
  }
}

}  // namespace precc
