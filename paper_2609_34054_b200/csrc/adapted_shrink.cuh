// T = s X A_a of every row with its own agent's A, for many rows: one pass over X on tcgen05.
//
// HBM-bound at M x K values of X.  A block takes TN rows (as many as spread them over all SMs) over the whole K extent.  The coordinates of the rank are
// the M axis of the MMA, 128 lanes that hold the coordinates of up to 128 / r agents, and the rows of X its N axis: a row is computed with every
// agent among the rows of its block, and the lanes of its own agent are the ones that are written.  Rows of one request follow one
// another, so a block mostly sees one or two agents.  Where it sees more than 128 lanes hold, a step loads A for
// several accumulators at once (CHUNKS), and beyond that the block goes over X again.
// 8 bits: A is the sum of two e4m3 matrices (value and rest); both are added into the same accumulator.
#pragma once
#include "adapted.cuh"

namespace precc {

constexpr int AS_THREADS = 192;                          // producer, MMA issuer, four epilogue warps
constexpr int AS_LANES = 128;
constexpr int AS_MAX_STAGES = 8;
template <bool Q8>
constexpr int AS_CHUNKS = Q8 ? 2 : 4;                    // accumulators of a pass at most
template <bool Q8>
constexpr int AS_CHUNK_BYTES = AS_LANES * AP_ROW_BYTES * (Q8 ? 2 : 1);

__device__ __forceinline__ void umma_e4m3(uint32_t tmem_d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}\n"
      ::"r"(tmem_d), "l"(da), "l"(db), "r"(idesc), "r"(accumulate) : "memory");
}

// p.BN: rows of a block (a multiple of 16, at most 256 / 128 where more than one accumulator is used); ring_bytes: shared memory for the ring
template <bool Q8>
__global__ void __launch_bounds__(AS_THREADS, 1)
adapted_shrink_tc_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_a, const AdaptedParams p,
                         const int ring_bytes) {
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  __shared__ __align__(8) uint64_t bars[2 * AS_MAX_STAGES + 2];
  __shared__ uint32_t tmem_holder;
  __shared__ int8_t row_agent[256];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int TN = p.BN;
  const long long m0 = (long long)blockIdx.x * TN;
  const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8 * AS_MAX_STAGES, acc_full = empty0 + 8 * AS_MAX_STAGES, acc_empty = acc_full + 8;
  const int nkb = p.K / (Q8 ? 128 : 64);
  if (threadIdx.x == 0) {
    for (int s = 0; s < AS_MAX_STAGES; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, 1); }
    mbar_init(acc_full, 1);
    mbar_init(acc_empty, 4);
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
  }
  pdl_wait();
  pdl_launch_dependents();
  int id[8];
  const unsigned long long present = agents_of_rows(p, m0, TN, lane, id);
  if (warp == 2) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      row_agent[32 * i + lane] = (int8_t)max(id[i], -1);
      const long long m = m0 + 32 * i + lane;
      if (32 * i + lane < TN && m < p.M && (p.agent_id[m] < -1 || p.agent_id[m] >= p.n_agents)) atomicOr(p.status, StatusBits::BAD_INDEX);
    }
  }
  if (present == 0) return;                              // (the same in every thread)
  const int slots = AS_LANES / p.rank;                   // agents in an accumulator
  const int all_chunks = (__popcll(present) + slots - 1) / slots;
  const int chunks = min(all_chunks, min(AS_CHUNKS<Q8>, 512 / TN));       // accumulators of a pass
  const int x_bytes = TN * AP_ROW_BYTES, stage_bytes = (x_bytes + 1023) / 1024 * 1024 + chunks * AS_CHUNK_BYTES<Q8>;
  const int stages = min(AS_MAX_STAGES, ring_bytes / stage_bytes);
  const int passes = (all_chunks + chunks - 1) / chunks;
  uint32_t tmem_cols = 32;
  while ((int)tmem_cols < chunks * TN) tmem_cols <<= 1;
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&tmem_holder)), "r"(tmem_cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
  const uint32_t tmem_base = tmem_holder;
  const uint32_t smem0 = smem_u32(smem);
  const int a_off = (x_bytes + 1023) / 1024 * 1024;
  // takes the agents of the next pass off `rest`
  auto next_pass = [&](unsigned long long& rest) {
    unsigned long long now = 0;
    for (int i = 0; i < chunks * slots && rest; ++i) { now |= rest & (0 - rest); rest &= rest - 1; }
    return now;
  };

  if (warp == 0) {
    RingWalk at;
    unsigned long long rest = present;
    for (int pass = 0; pass < passes; ++pass) {
      const unsigned long long now = next_pass(rest);
      const uint32_t tx = x_bytes + __popcll(now) * p.rank * AP_ROW_BYTES * (Q8 ? 2 : 1);
      for (int kb = 0; kb < nkb; ++kb, at.next(stages)) {
        if (at.filled) mbar_wait(empty0 + 8 * at.s, at.parity ^ 1u, p.status);
        const uint32_t st = smem0 + at.s * stage_bytes, bar = full0 + 8 * at.s;
        if (elect_one()) {
          mbar_expect_tx(bar, tx);
          tma_load_2d(st, &map_x, kb * (Q8 ? 128 : 64), (int)m0, bar);
          int i = 0;
          for (unsigned long long left = now; left; left &= left - 1, ++i) {
            const int row = (__ffsll(left) - 1) * p.rank;
            const uint32_t dst = st + a_off + i / slots * AS_CHUNK_BYTES<Q8> + i % slots * p.rank * AP_ROW_BYTES;
            tma_load_3d(dst, &map_a, 0, row, kb, bar);
            if constexpr (Q8) tma_load_3d(dst + AS_LANES * AP_ROW_BYTES, &map_a, 0, p.n_agents * p.rank + row, kb, bar);
          }
        }
        __syncwarp();
      }
    }
  } else if (warp == 1) {
    const uint32_t idesc = Q8 ? umma_idesc_bf16(TN) & ~((1u << 7) | (1u << 10)) : umma_idesc_bf16(TN);      // (e4m3 is format 0)
    const uint64_t dx0 = umma_desc_sw128(smem0), da0 = umma_desc_sw128(smem0 + a_off);
    RingWalk at;
    for (int pass = 0; pass < passes; ++pass) {
      if (pass > 0) mbar_wait(acc_empty, (pass - 1) & 1, p.status);
      const int live = min(chunks, all_chunks - pass * chunks);
      for (int kb = 0; kb < nkb; ++kb, at.next(stages)) {
        mbar_wait(full0 + 8 * at.s, at.parity, p.status);
        asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
        if (elect_one()) {
          const uint64_t so = (uint64_t)((at.s * stage_bytes) >> 4);
          for (int c = 0; c < live; ++c) {
            const uint64_t da = da0 + so + (uint64_t)((c * AS_CHUNK_BYTES<Q8>) >> 4);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              if constexpr (Q8) {
                umma_e4m3(tmem_base + c * TN, da + 2 * k, dx0 + so + 2 * k, idesc, (kb | k) ? 1u : 0u);
                umma_e4m3(tmem_base + c * TN, da + ((AS_LANES * AP_ROW_BYTES) >> 4) + 2 * k, dx0 + so + 2 * k, idesc, 1u);
              } else {
                umma_bf16(tmem_base + c * TN, da + 2 * k, dx0 + so + 2 * k, idesc, (kb | k) ? 1u : 0u);
              }
            }
          }
          umma_commit(empty0 + 8 * at.s);
          if (kb == nkb - 1) umma_commit(acc_full);
        }
        __syncwarp();
      }
    }
  } else {
    const int quad = warp & 3, slot = (quad * 32 + lane) / p.rank, coord = (quad * 32 + lane) % p.rank;
    unsigned long long rest = present;
    for (int pass = 0; pass < passes; ++pass) {
      unsigned long long now = next_pass(rest);
      const int live = min(chunks, all_chunks - pass * chunks);
      mbar_wait_relaxed(acc_full, pass & 1, p.status);
      asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
      for (int c = 0; c < live; ++c) {
        int agent = -2;                                  // of this lane (no row has agent -2)
        for (int i = 0; i < slots && now; ++i, now &= now - 1)
          if (i == slot) agent = __ffsll(now) - 1;
        float scale = p.s;
        if constexpr (Q8) { if (agent >= 0) scale *= p.a_scale[agent * p.rank + coord]; }
        for (int r0 = 0; r0 < TN; r0 += 16) {
          uint32_t v[16];
          tmem_ld16(tmem_base + c * TN + r0 + (static_cast<uint32_t>(quad * 32) << 16), v);
          asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory");
#pragma unroll
          for (int q = 0; q < 16; ++q) {
            if (row_agent[r0 + q] != agent) continue;
            __nv_bfloat16* dst = p.T + (m0 + r0 + q) * p.rank_pad + coord;
            *dst = __float2bfloat16(scale * __uint_as_float(v[q]));
            if (p.rank < p.rank_pad) dst[p.rank] = __float2bfloat16(0.f);       // (rank 8 of 16)
          }
        }
      }
      asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
      __syncwarp();
      if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];\n" ::"r"(acc_empty) : "memory");
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem_base), "r"(tmem_cols) : "memory");
  }
}

}  // namespace precc
