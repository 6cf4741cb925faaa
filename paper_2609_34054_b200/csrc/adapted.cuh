// The projection of a batch whose rows belong to different agents, Y[m] = X[m] W + s (X[m] A_a(m)) B_a(m):  what its kernels share,
// and the rank-r product T = s X A_a of every row with its own agent's A (bf16, [M][rank, at least 16]).
//
// T is small work (2 M K r flops) that the main kernel needs only at its end, so it runs beside it: this kernel lets its
// dependent start as soon as all its own blocks run - behind its own wait for the kernel ahead, so whatever
// the dependent reads before ITS wait was complete before either started - and uses little shared memory and few registers, so
// that a block of the main kernel fits on the same SM.
// T is rounded to bf16, the operand type of the MMA that takes it: 2^-8 of the adapter's term, which is added to a sum that is
// rounded to bf16 as a whole.
#pragma once
#include <cuda_fp16.h>

#include "norm.cuh"
#include "tc_common.cuh"

namespace precc {

constexpr int AP_MAX_AGENTS = 64;
constexpr int AP_ROW_BYTES = 128;             // bytes of K in a step: 64 bf16 or 128 e4m3

struct AdaptedParams {
  int M, N, K, rank, rank_pad;                // rank_pad: rank, at least 16 (the K of one MMA)
  int n_agents;
  const int32_t* agent_id;                    // [M], or null: no adapters in this call
  const void* x;                              // [M][K] bf16 or e4m3
  const float* x_scale;                       // 8 bits: [M]
  const float* w_scale;                       // 8 bits: [N]
  const __nv_bfloat16* A;                     // packed [K/64][n_agents * rank][64]
  const __nv_bfloat16* B;                     // [n_agents][rank][N] (8 bits: divided by w_scale)
  __nv_bfloat16* T;                           // [M][rank_pad]
  __nv_bfloat16* y;                           // [M][N]
  float s;
  int tile_rows;                              // shrink kernel: rows of a block
  int BN, stages, tmem_cols;
  uint32_t* status;
};

// An agent id as the kernels use it: out of range counts as "no adapter" (reported by the shrink kernel).
__device__ __forceinline__ int agent_of(const AdaptedParams& p, long long row) {
  if (row >= p.M) return -1;
  const int a = p.agent_id[row];
  return a < p.n_agents ? a : -1;
}

// Eight e4m3 values as bf16 (exact).
__device__ __forceinline__ void e4m3x8_to_bf16(uint32_t lo, uint32_t hi, uint32_t (&o)[4]) {
  const uint32_t w[2] = {lo, hi};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint16_t two = static_cast<uint16_t>(w[i >> 1] >> (16 * (i & 1)));
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(h) : "h"(two));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    o[i] = pack_bf16(f.x, f.y);
  }
}

constexpr int SHRINK_WARPS = 8;
constexpr int SHRINK_THREADS = SHRINK_WARPS * 32;

// T of up to 8 NT rows (fewer where that fills more SMs: a block takes the agents among its rows one after the other).  MT: 16-wide pieces of the rank.  The K extent is split over the warps of a block and the blocks of a cluster;
// partial sums meet in shared memory in a fixed order.  The rows are the N axis of mma.sync and the coordinates of the rank its M axis, so a row
// is computed in its own column of the product and nothing of another agent's adapter reaches it: for every agent among the rows
// the product is taken with the rows of that agent (the others' columns are zero and dropped).
// Fragments come straight from global memory, 16 bytes a lane: within 64 values of K a lane of a quad takes two runs of eight, and as A and X agree
// on which, the order of K inside a step does not matter.
template <int MT, int NT, bool Q8>
__global__ void __launch_bounds__(SHRINK_THREADS, 2)
adapted_shrink_kernel(const AdaptedParams p) {
  constexpr int RT = 8 * NT, R = 16 * MT;
  __shared__ float red[SHRINK_WARPS][RT][R];
  __shared__ float part[RT][R];
  uint32_t rank_c, KS;
  asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(rank_c));
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;\n" : "=r"(KS));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
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
  const int nkb = p.K / 64;
  const int kb0 = (int)((long long)rank_c * nkb / KS), kb1 = (int)((long long)(rank_c + 1) * nkb / KS);
  const int a_rows = p.n_agents * p.rank;

  while (todo) {
    const int a = __shfl_sync(0xffffffffu, id, __ffs(todo) - 1);
    const unsigned mine = __ballot_sync(0xffffffffu, id == a);
    todo &= ~mine;
    float acc[MT][NT][4];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int n = 0; n < NT; ++n) { acc[m][n][0] = acc[m][n][1] = acc[m][n][2] = acc[m][n][3] = 0.f; }
#pragma unroll 2
    for (int kb = kb0 + warp; kb < kb1; kb += SHRINK_WARPS) {
      // bf16: 16-byte pieces t and t + 4 of the 128; e4m3: 16 values 16 t .. 16 t + 15, i.e. pieces 2 t and 2 t + 1 of A
      uint4 av[MT][2][2];
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = m * 16 + h * 8 + g;
          const uint4* src = reinterpret_cast<const uint4*>(p.A + ((long long)kb * a_rows + a * p.rank + r) * 64);
#pragma unroll
          for (int c = 0; c < 2; ++c)
            av[m][h][c] = r < p.rank ? __ldg(src + (Q8 ? 2 * t + c : t + 4 * c)) : make_uint4(0, 0, 0, 0);
        }
      uint4 xv[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const bool on = (mine >> (n * 8 + g)) & 1u;
        const long long row = row0 + n * 8 + g;
        xv[n][0] = xv[n][1] = make_uint4(0, 0, 0, 0);
        if constexpr (Q8) {
          if (on) {
            const uint4 q = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(p.x) + row * p.K + (long long)kb * 64) + t);
            uint32_t lo[4], hi[4];
            e4m3x8_to_bf16(q.x, q.y, lo);
            e4m3x8_to_bf16(q.z, q.w, hi);
            xv[n][0] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            xv[n][1] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
          }
        } else if (on) {
          const uint4* src = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.x) + row * p.K + (long long)kb * 64);
          xv[n][0] = __ldg(src + t);
          xv[n][1] = __ldg(src + t + 4);
        }
      }
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            const uint32_t a0[4] = {av[m][0][c].x, av[m][1][c].x, av[m][0][c].y, av[m][1][c].y};
            const uint32_t a1[4] = {av[m][0][c].z, av[m][1][c].z, av[m][0][c].w, av[m][1][c].w};
            mma_bf16_16816(acc[m][n], a0, xv[n][c].x, xv[n][c].y);
            mma_bf16_16816(acc[m][n], a1, xv[n][c].z, xv[n][c].w);
          }
    }
    // a row belongs to one agent: its column goes to its place once
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = n * 8 + 2 * t + e;
        if ((mine >> r) & 1u) {
#pragma unroll
          for (int m = 0; m < MT; ++m) { red[warp][r][m * 16 + g] = acc[m][n][e]; red[warp][r][m * 16 + 8 + g] = acc[m][n][2 + e]; }
        }
      }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < RT * R; i += SHRINK_THREADS) {
    const int r = i / R, c = i % R;
    float v = 0.f;
    if ((with_adapter >> r) & 1u) {
#pragma unroll
      for (int w = 0; w < SHRINK_WARPS; ++w) v += red[w][r][c];
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
  for (int i = threadIdx.x + (int)rank_c * SHRINK_THREADS; i < RT * R; i += SHRINK_THREADS * (int)KS) {
    const int r = i / R, c = i % R;
    if (!((with_adapter >> r) & 1u)) continue;
    float v = 0.f;
    const uint32_t local = smem_u32(&part[r][c]);
    for (uint32_t k = 0; k < KS; ++k) {
      float u;
      asm volatile("ld.shared::cluster.f32 %0, [%1];\n" : "=f"(u) : "r"(dsmem_addr(local, k)));
      v += u;
    }
    p.T[(row0 + r) * p.rank_pad + c] = __float2bfloat16(p.s * v);
  }
  if (KS > 1) {
    asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
  }
}

}  // namespace precc
