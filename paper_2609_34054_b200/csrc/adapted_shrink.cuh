// T = s X A_a of every row with its own agent's A, for many rows: one pass over X on tcgen05.
//
// HBM-bound at M x K values of X.  A block takes TN rows (as many as spread them over all SMs) over the whole K extent, or, where that would leave SMs
// idle, the blocks of a cluster share the K extent and add their sums in rank order.  The coordinates of the rank are
// the M axis of the MMA, 128 lanes that hold the coordinates of up to 128 / r agents, and the rows of X its N axis: a row is computed with every
// agent among the rows of its block, and the lanes of its own agent are the ones that are written.  Rows of one request follow one
// another, so a block mostly sees one or two agents.  Where it sees more than 128 lanes hold, a step loads A for
// several accumulators at once (CHUNKS), and beyond that the block goes over X again.
// 8 bits: A is the sum of two e4m3 matrices (value and rest); both are added into the same accumulator.
// Measured: 32768 x 4096 in bf16, runs of eight agents of rank 32, 49 us (5.5 TB/s of X); 8192 x 4096 19.2, where start and epilogue are a third.
// K-blocks begun at another place in every block change nothing.
#pragma once
#include "adapted.cuh"

namespace precc {

constexpr int AS_THREADS = 192;                          // producer, MMA issuer, four epilogue warps

__device__ __forceinline__ void umma_e4m3(uint32_t tmem_d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}\n"
      ::"r"(tmem_d), "l"(da), "l"(db), "r"(idesc), "r"(accumulate) : "memory");
}

// A slot of the ring holds `kps` neighbouring k-blocks, which one copy fetches as up to 512 bytes of every row (128 bytes a row and copy leave DRAM at
// two thirds of its rate), and of A the lanes that are used and no more (the MMA reads 128 lanes whatever lies behind them; the tail behind the ring is larger
// than what it reads past the last slot).
// A lane of the accumulator is a coordinate and a column a row, so 64 rows at a time go through shared memory, where each row finds the
// coordinates of its agent side by side (writing them out of the accumulator, two bytes a row under a condition each, took 3.6 us for 64 rows).
// p.BN: rows of a block (a multiple of 16, at most 256 / 128 where more than one accumulator is used); ring_bytes: shared memory for the ring
template <bool Q8>
__global__ void __launch_bounds__(AS_THREADS, 1)
adapted_shrink_tc_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_a, const AdaptedParams p,
                         const int ring_bytes) {
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  __shared__ __align__(8) uint64_t bars[2 * AS_MAX_STAGES + 2];
  __shared__ uint32_t tmem_holder;
  __shared__ __align__(16) int8_t row_agent[256];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t KS_u;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;\n" : "=r"(KS_u));
  const int TN = p.BN, KS = (int)KS_u, rank_c = (int)cluster_ctarank();
  const long long m0 = (long long)(blockIdx.x / KS) * TN;
  float* dump = reinterpret_cast<float*>(smem + ring_bytes);         // [64 rows][lanes]
  float* part = reinterpret_cast<float*>(smem + ring_bytes + AS_TAIL_BYTES);         // KS > 1: [TN][rank]
  const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8 * AS_MAX_STAGES, acc_full = empty0 + 8 * AS_MAX_STAGES, acc_empty = acc_full + 8;
  const int steps_all = (p.K / (Q8 ? 128 : 64) + p.kps - 1) / p.kps;               // (k-blocks past K arrive as zeros)
  const int step0 = (int)((long long)rank_c * steps_all / KS), steps = (int)((long long)(rank_c + 1) * steps_all / KS) - step0;
  if (threadIdx.x == 0) {
    prefetch_map(&map_x);
    prefetch_map(&map_a);
    mbar_init(acc_full, 1);
    mbar_init(acc_empty, 4);
  }
  if (warp == 0) {
    if (lane < AS_MAX_STAGES) { mbar_init(full0 + 8 * lane, 1); mbar_init(empty0 + 8 * lane, 1); }
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&tmem_holder)), "r"(p.tmem_cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  pdl_wait();
  pdl_launch_dependents();
  int id[8];
  load_agents(p, m0, lane, id);
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) bad |= 32 * i + lane < TN && m0 + 32 * i + lane < p.M && (id[i] < -1 || id[i] >= p.n_agents);
  const unsigned long long present = agents_present(p, m0, TN, lane, id);
  if (warp == 2) {
    if (bad && rank_c == 0) atomicOr(p.status, StatusBits::BAD_INDEX);
#pragma unroll
    for (int i = 0; i < 8; ++i) row_agent[32 * i + lane] = (int8_t)id[i];
  }
  // (no agents: nothing is loaded, multiplied or written, and the same in every thread of the cluster)
  const int slots = AS_LANES >> p.rank_shift, n_present = __popcll(present);        // slots: agents in an accumulator
  const int all_chunks = (n_present + slots - 1) >> (7 - p.rank_shift);
  // accumulators of a pass: what tensor memory holds, and what leaves room for two slots of the ring (one always fits once, see plan_shrink_tc)
  const int room = (ring_bytes / (2 * p.kps) - TN * AP_ROW_BYTES) / as_chunk_bytes(Q8);
  const int chunks = max(1, min(min(all_chunks, room), min(as_chunks(Q8), p.tmem_cols / TN)));
  const int passes = (all_chunks + chunks - 1) / chunks;
  const int lane_bytes = (all_chunks > 1 ? AS_LANES : n_present * p.rank) * AP_ROW_BYTES, chunk_bytes = lane_bytes * (Q8 ? 2 : 1);
  const int a_off = p.kps * TN * AP_ROW_BYTES, a_bytes = chunks * chunk_bytes;      // (TN: a multiple of 16)
  const int stage_bytes = a_off + p.kps * a_bytes;
  const int stages = min(AS_MAX_STAGES, ring_bytes / stage_bytes);
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
  const uint32_t tmem_base = tmem_holder;
  const uint32_t smem0 = smem_u32(smem);
  // takes the agents of the next pass off `rest`
  auto next_pass = [&](unsigned long long& rest) {
    unsigned long long now = 0;
    for (int i = 0; i < chunks * slots && rest; ++i) { now |= rest & (0 - rest); rest &= rest - 1; }
    return now;
  };

  if (warp == 0) {
    if (elect_one()) {
      RingWalk at;
      unsigned long long rest = present;
      for (int pass = 0; pass < passes; ++pass) {
        const unsigned long long now = next_pass(rest);
        const uint32_t tx = p.kps * (TN + __popcll(now) * p.rank * (Q8 ? 2 : 1)) * AP_ROW_BYTES;
        for (int it = 0; it < steps; ++it, at.next(stages)) {
          if (at.filled) mbar_wait(empty0 + 8 * at.s, at.parity ^ 1u, p.status);
          const uint32_t st = smem0 + at.s * stage_bytes, bar = full0 + 8 * at.s;
          const int kb = (step0 + it) * p.kps;
          mbar_expect_tx(bar, tx);
          tma_load_3d(st, &map_x, 0, (int)m0, kb, bar);
          for (int j = 0; j < p.kps; ++j) {
            uint32_t dst = st + a_off + j * a_bytes;
            int slot = 0;
            for (unsigned long long left = now; left; left &= left - 1) {
              const int row = (__ffsll(left) - 1) << p.rank_shift;
              tma_load_3d(dst, &map_a, 0, row, kb + j, bar);
              if constexpr (Q8) tma_load_3d(dst + lane_bytes, &map_a, 0, p.n_agents * p.rank + row, kb + j, bar);
              dst += p.rank * AP_ROW_BYTES;
              if (++slot == slots) { slot = 0; dst += chunk_bytes - lane_bytes; }
            }
          }
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    const uint32_t idesc = Q8 ? umma_idesc_bf16(TN) & ~((1u << 7) | (1u << 10)) : umma_idesc_bf16(TN);      // (e4m3 is format 0)
    const uint64_t dx0 = umma_desc_sw128(smem0), da0 = umma_desc_sw128(smem0 + a_off);
    if (elect_one()) {
      RingWalk at;
      for (int pass = 0; pass < passes; ++pass) {
        if (pass > 0) mbar_wait(acc_empty, (pass - 1) & 1, p.status);
        const int live = min(chunks, all_chunks - pass * chunks);
        for (int it = 0; it < steps; ++it, at.next(stages)) {
          mbar_wait(full0 + 8 * at.s, at.parity, p.status);
          asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
          uint64_t dx = dx0 + (uint64_t)((at.s * stage_bytes) >> 4), da_step = da0 + (uint64_t)((at.s * stage_bytes) >> 4);
          for (int j = 0; j < p.kps; ++j, dx += TN * AP_ROW_BYTES >> 4, da_step += a_bytes >> 4) {
            uint64_t da = da_step;
            for (int c = 0; c < live; ++c, da += chunk_bytes >> 4) {
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                if constexpr (Q8) {
                  umma_e4m3(tmem_base + c * TN, da + 2 * k, dx + 2 * k, idesc, (it | j | k) ? 1u : 0u);
                  umma_e4m3(tmem_base + c * TN, da + (lane_bytes >> 4) + 2 * k, dx + 2 * k, idesc, 1u);
                } else {
                  umma_bf16(tmem_base + c * TN, da + 2 * k, dx + 2 * k, idesc, (it | j | k) ? 1u : 0u);
                }
              }
            }
          }
          umma_commit(empty0 + 8 * at.s);
        }
        umma_commit(acc_full);
      }
    }
    __syncwarp();
  } else {
    const int quad = warp & 3, et = threadIdx.x - 64;
    const int pieces = p.rank >> 2;                      // of four coordinates in a row
    unsigned long long rest = present;
    for (int pass = 0; pass < passes; ++pass) {
      unsigned long long now = next_pass(rest);
      const int live = min(chunks, all_chunks - pass * chunks);
      mbar_wait_relaxed(acc_full, pass & 1, p.status);
      asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
      for (int c = 0; c < live; ++c) {
        unsigned long long mine = 0;                     // the agents of this accumulator
        for (int i = 0; i < slots && now; ++i) { mine |= now & (0 - now); now &= now - 1; }
        const bool lanes_used = quad * 32 < __popcll(mine) << p.rank_shift;
        for (int b0 = 0; b0 < TN; b0 += AS_DUMP_ROWS) {
          const int nb = min(AS_DUMP_ROWS, TN - b0);
          float* col = dump + quad * 32 + lane;
          for (int r0 = 0; lanes_used && r0 < nb; r0 += 16, col += 16 * AS_DUMP_PITCH) {
            uint32_t v[16];
            tmem_ld16(tmem_base + c * TN + b0 + r0 + (static_cast<uint32_t>(quad * 32) << 16), v);
            asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory");
#pragma unroll
            for (int q = 0; q < 16; ++q) col[q * AS_DUMP_PITCH] = __uint_as_float(v[q]);
          }
          asm volatile("bar.sync 1, 128;\n" ::: "memory");
          for (int i = et; i < nb * pieces; i += 128) {
            const int r = i >> (p.rank_shift - 2), k = (i & (pieces - 1)) * 4, a = row_agent[b0 + r];
            if (a < 0 || !((mine >> a) & 1ull)) continue;
            const int at = __popcll(mine & ((1ull << a) - 1)) << p.rank_shift;
            float4 v = *reinterpret_cast<const float4*>(dump + r * AS_DUMP_PITCH + at + k);
            float4 w = make_float4(p.s, p.s, p.s, p.s);
            if constexpr (Q8) {
              const float* sc = p.a_scale + (a << p.rank_shift) + k;        // (a caller's pointer, on a 4-byte boundary and no more)
              w = make_float4(p.s * __ldg(sc), p.s * __ldg(sc + 1), p.s * __ldg(sc + 2), p.s * __ldg(sc + 3));
            }
            v = make_float4(v.x * w.x, v.y * w.y, v.z * w.z, v.w * w.w);
            if (KS > 1) {
              *reinterpret_cast<float4*>(part + ((b0 + r) << p.rank_shift) + k) = v;
            } else {
              __nv_bfloat16* dst = p.T + (m0 + b0 + r) * p.rank_pad + k;
              *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
              if (p.rank < p.rank_pad) *reinterpret_cast<uint2*>(dst + p.rank) = make_uint2(0u, 0u);       // (rank 8 of 16)
            }
          }
          asm volatile("bar.sync 1, 128;\n" ::: "memory");
        }
      }
      asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
      __syncwarp();
      if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];\n" ::"r"(acc_empty) : "memory");
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();
  if (KS > 1) {                                          // every block finishes a share of the elements
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
    const int pieces = p.rank >> 2;
    for (int i = rank_c * AS_THREADS + threadIdx.x; i < TN * pieces; i += KS * AS_THREADS) {
      const int r = i >> (p.rank_shift - 2), k = (i & (pieces - 1)) * 4;
      if (row_agent[r] < 0) continue;
      const uint32_t local = smem_u32(part + (r << p.rank_shift) + k);
      float4 u[8], v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        u[j] = v;
        if (j < KS) asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];\n" : "=f"(u[j].x), "=f"(u[j].y), "=f"(u[j].z), "=f"(u[j].w) : "r"(dsmem_addr(local, j)));
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) { v.x += u[j].x; v.y += u[j].y; v.z += u[j].z; v.w += u[j].w; }
      __nv_bfloat16* dst = p.T + (m0 + r) * p.rank_pad + k;
      *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
      if (p.rank < p.rank_pad) *reinterpret_cast<uint2*>(dst + p.rank) = make_uint2(0u, 0u);
    }
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");      // nobody leaves while its sums are read
  }
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem_base), "r"(p.tmem_cols) : "memory");
  }
}

}  // namespace precc
