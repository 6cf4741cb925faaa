// The main kernel of the adapted projection for many rows: persistent pairs of SMs, 256 rows x BN columns a tile (tcgen05 cta_group::2,
// two accumulators in tensor memory).  The ring, its hand-offs and the tile walk are those of the pair form of the plain projection GEMM.
//
// The adapters are more K: behind the last step of W a tile takes one step of depth rank_pad for every agent among its rows, with
// T rows as the A operand and that agent's B (columns contiguous in memory, so an MN-major operand) as the other.  The rows of a tile
// are the lanes of the accumulator, and the MMA leaves the lanes of other agents' rows alone (its lane mask): no other adapter, were it
// infinite or NaN, touches a row, and T needs no zeros for the rows of others.
// Bound by the tensor pipe: 8192 rows of 4096 x 4096 in bf16 in 165 .. 172 us without adapters (1.6 .. 1.67 PFLOP/s, a large library product's rate; the pipe is active 81 .. 83 %
// of the time), 99 us in 8 bits; with eight agents' runs of rank 32, the shrink kernel included, 197 .. 203.  In a long loop the power limit takes
// clocks: 235.  512 rows are 17.5 us, as 64 tiles leave ten pairs of SMs idle and each loads at L2's rate.
#pragma once
#include "adapted.cuh"

namespace precc {

constexpr int AP_EPI_WARPS = 8;                       // two on each quarter of the lanes, half of the columns each
constexpr int AP_THREADS = (2 + AP_EPI_WARPS) * 32;   // producer, MMA issuer, epilogue warps
__device__ __forceinline__ void umma_pair_e4m3(uint32_t tmem_d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}\n"
      ::"r"(tmem_d), "l"(da), "l"(db), "r"(idesc), "r"(accumulate) : "memory");
}
// D += A B on the lanes whose bit in `off` is clear.
__device__ __forceinline__ void umma_pair_bf16_lanes(uint32_t tmem_d, uint64_t da, uint64_t db, uint32_t idesc, const uint32_t (&off)[8]) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, 1, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, {%4, %5, %6, %7, %8, %9, %10, %11}, p;\n\t}\n"
      ::"r"(tmem_d), "l"(da), "l"(db), "r"(idesc), "r"(off[0]), "r"(off[1]), "r"(off[2]), "r"(off[3]), "r"(off[4]), "r"(off[5]),
        "r"(off[6]), "r"(off[7]) : "memory");
}

template <bool Q8>
__global__ void __launch_bounds__(AP_THREADS, 2)
adapted_pair_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                    const __grid_constant__ CUtensorMap map_t, const __grid_constant__ CUtensorMap map_b, const AdaptedParams p) {
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const uint32_t smem0 = smem_u32(smem);
  const int half_n = p.BN / 2;
  const int stage_bytes = ap_stage_bytes(p.BN);
  const uint32_t step_tx = 2u * (AP_A_BYTES + half_n * AP_ROW_BYTES);
  const int b_boxes = (half_n + 63) / 64;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + (size_t)p.stages * stage_bytes);
  const uint32_t full0 = smem_u32(bars);
  const uint32_t empty0 = full0 + 8 * p.stages;
  const uint32_t acc_full = empty0 + 8 * p.stages;
  const uint32_t acc_empty = acc_full + 16;
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(bars + 2 * p.stages + 4);
  __shared__ int slot_agents[AP_MAX_STAGES];              // of the tile that begins in this slot
  __shared__ __align__(16) uint32_t slot_lanes[AP_MAX_STAGES][8];   // of an adapter's step: the lanes that are not its agent's
  __shared__ __align__(16) float w_scale_s[2][256];       // 8 bits: the scales of a tile's columns

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
  const int nkb = p.K / (Q8 ? 128 : 64);
  const int n_tiles_n = (p.N + p.BN - 1) / p.BN;
  const long long n_tiles = (long long)((p.M + AP_BM - 1) / AP_BM) * n_tiles_n;
  const bool adapters = p.agent_id != nullptr;

  if (threadIdx.x == 0) {
    prefetch_map(&map_x);
    prefetch_map(&map_w);
    if (adapters) { prefetch_map(&map_t); prefetch_map(&map_b); }
    for (int s = 0; s < p.stages; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, 1); }
    mbar_init(acc_full, 1); mbar_init(acc_full + 8, 1);
    mbar_init(acc_empty, 2 * AP_EPI_WARPS); mbar_init(acc_empty + 8, 2 * AP_EPI_WARPS);
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(tmem_holder)), "r"(p.tmem_cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n" ::: "memory");
  }
  if (!adapters) pdl_wait();       // with adapters the kernel ahead is the shrink kernel, which starts this one behind its own wait
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();
  pair_sync();
  asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
  const uint32_t tmem_base = *tmem_holder;
  if (!adapters) pdl_launch_dependents();

  if (warp == 0) {
    // ---- producer.  It also tells the issuer, slot by slot, how many agents a tile has and which lanes are theirs, so that the issuing thread never waits for
    // anything but its barriers (worked out there, between two tiles, it cost 5 % of a tile in 8 bits).
    const uint32_t full0_lead = map_to_rank(full0, 0);
    RingWalk at;
    bool waited = false;
    int id[8];
    if (adapters && pair < n_tiles) load_agents(p, (long long)(pair / n_tiles_n) * AP_BM, lane, id);
    for (long long t = pair; t < n_tiles; t += n_pairs) {
      const int mt = (int)(t / n_tiles_n) * AP_BM;
      const int m0 = mt + (int)rank * GEMM_BM, n0 = (int)(t % n_tiles_n) * p.BN + (int)rank * half_n;
      const unsigned long long present = adapters ? agents_present(p, mt, AP_BM, lane, id) : 0ull;
      if (elect_one()) {
        RingWalk w = at;
        for (int kb = 0; kb < nkb; ++kb, w.next(p.stages)) {
          if (w.filled) mbar_wait(empty0 + 8 * w.s, w.parity ^ 1u, p.status);
          const uint32_t sa = smem0 + w.s * stage_bytes, bar = full0_lead + 8 * w.s;
          if (kb == 0) slot_agents[w.s] = __popcll(present);
          if (rank == 0) mbar_expect_tx(full0 + 8 * w.s, step_tx);
          tma_pair_load_3d(sa, &map_x, 0, m0, kb, bar);
          tma_pair_load_3d(sa + AP_A_BYTES, &map_w, 0, n0, kb, bar);
        }
      }
      __syncwarp();
      at.skip(nkb, p.stages);
      if (!adapters) continue;
      if (!waited) {                   // T is complete; also with no adapter in this tile, so that this grid ends after the shrink kernel
        pdl_wait();
        pdl_launch_dependents();
        waited = true;
      }
      for (unsigned long long left = present; left; left &= left - 1, at.next(p.stages)) {
        const int a = __ffsll(left) - 1;
        if (at.filled) mbar_wait(empty0 + 8 * at.s, at.parity ^ 1u, p.status);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint32_t off = ~__ballot_sync(0xffffffffu, id[j] == a);
          if (lane == j) slot_lanes[at.s][j] = off;
        }
        __syncwarp();
        if (elect_one()) {
          const uint32_t sa = smem0 + at.s * stage_bytes, bar = full0_lead + 8 * at.s;
          if (rank == 0) mbar_expect_tx(full0 + 8 * at.s, 2u * (GEMM_BM + b_boxes * 64) * p.rank_pad * 2);
          tma_pair_load_2d(sa, &map_t, 0, m0, bar);
          for (int j = 0; j < b_boxes; ++j) tma_pair_load_3d(sa + AP_A_BYTES + j * p.rank_pad * 128, &map_b, n0 + 64 * j, 0, a, bar);
        }
        __syncwarp();
      }
      if (t + n_pairs < n_tiles) load_agents(p, (t + n_pairs) / n_tiles_n * AP_BM, lane, id);
    }
  } else if (warp == 1) {
    if (rank == 0 && elect_one()) {
      const uint32_t idesc = Q8 ? umma_pair_idesc_bf16(p.BN) & ~((1u << 7) | (1u << 10)) : umma_pair_idesc_bf16(p.BN);   // (e4m3 is format 0)
      const uint32_t idesc_b = umma_pair_idesc_bf16(p.BN) | (1u << 16);                                                 // B operand MN-major
      const uint64_t da0 = umma_desc_sw128(smem0);
      const uint64_t db0 = umma_desc_sw128(smem0 + AP_A_BYTES);
      const uint64_t dt0 = umma_desc_kmajor(smem0, p.rank_pad * 2);
      const uint64_t de0 = umma_desc_mnmajor(smem0 + AP_A_BYTES, 128, p.rank_pad * 128);
      RingWalk w;
      int i = 0;
      for (long long t = pair; t < n_tiles; t += n_pairs, ++i) {
        const int buf = i & 1;
        const uint32_t d = tmem_base + buf * p.BN;
        if (i >= 2) mbar_wait(acc_empty + 8 * buf, ((i >> 1) - 1) & 1, p.status);
        int agents = 0;
        for (int kb = 0; kb < nkb; ++kb, w.next(p.stages)) {
          mbar_wait(full0 + 8 * w.s, w.parity, p.status);
          asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
          const uint64_t so = (uint64_t)((w.s * stage_bytes) >> 4);
          if (kb == 0) agents = slot_agents[w.s];
#pragma unroll
          for (int k = 0; k < 4; ++k) {             // 32 bytes of K a step: 16 bf16 or 32 e4m3
            if constexpr (Q8) umma_pair_e4m3(d, da0 + so + 2 * k, db0 + so + 2 * k, idesc, (kb | k) ? 1u : 0u);
            else umma_pair_bf16(d, da0 + so + 2 * k, db0 + so + 2 * k, idesc, (kb | k) ? 1u : 0u);
          }
          umma_pair_commit_both(empty0 + 8 * w.s);
        }
        for (; agents > 0; --agents, w.next(p.stages)) {
          mbar_wait(full0 + 8 * w.s, w.parity, p.status);
          asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
          const uint64_t so = (uint64_t)((w.s * stage_bytes) >> 4);
          uint32_t off[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) off[j] = slot_lanes[w.s][j];
          for (int k = 0; k < p.rank_pad / 16; ++k) umma_pair_bf16_lanes(d, dt0 + so + 2 * k, de0 + so + 128 * k, idesc_b, off);
          umma_pair_commit_both(empty0 + 8 * w.s);
        }
        umma_pair_commit_both(acc_full + 8 * buf);
      }
    }
    __syncwarp();
  } else {
    // ---- epilogue: a thread holds a row of the accumulator and stores 64 bytes of Y at a time; the next 32 columns are on their way meanwhile
    const int lane_base = (warp & 3) * 32, et = threadIdx.x - 64;
    const int c_begin = (warp - 2) / 4 * half_n, c_end = c_begin + half_n;      // (half_n: a multiple of 32)
    const uint32_t acc_empty_lead = map_to_rank(acc_empty, 0);
    int i = 0;
    for (long long t = pair; t < n_tiles; t += n_pairs, ++i) {
      const int buf = i & 1;
      const int m = (int)(t / n_tiles_n) * AP_BM + (int)rank * GEMM_BM + lane_base + lane, n0 = (int)(t % n_tiles_n) * p.BN;
      const bool row_ok = m < p.M;
      float xs = 1.f;
      if constexpr (Q8) {
        if (et < p.BN) w_scale_s[buf][et] = n0 + et < p.N ? p.w_scale[n0 + et] : 0.f;
        xs = row_ok ? p.x_scale[m] : 0.f;
        asm volatile("bar.sync 1, 256;\n" ::: "memory");       // (a buffer is written again two tiles later, behind another of these)
      }
      __nv_bfloat16* yr = p.y + (long long)m * p.N + n0;
      mbar_wait_relaxed(acc_full + 8 * buf, (i >> 1) & 1, p.status);
      asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
      const uint32_t acc = tmem_base + buf * p.BN + (static_cast<uint32_t>(lane_base) << 16);
      auto store = [&](const uint32_t (&r)[32], int c) {
        if (!row_ok) return;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float v[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(r[8 * q + k]);
          if constexpr (Q8) {
            const float4 u = *reinterpret_cast<const float4*>(&w_scale_s[buf][c + 8 * q]), w = *reinterpret_cast<const float4*>(&w_scale_s[buf][c + 8 * q + 4]);
            v[0] = unscale(v[0], u.x, xs); v[1] = unscale(v[1], u.y, xs); v[2] = unscale(v[2], u.z, xs); v[3] = unscale(v[3], u.w, xs);
            v[4] = unscale(v[4], w.x, xs); v[5] = unscale(v[5], w.y, xs); v[6] = unscale(v[6], w.z, xs); v[7] = unscale(v[7], w.w, xs);
          }
          if (n0 + c + 8 * q < p.N) *reinterpret_cast<uint4*>(yr + c + 8 * q) = pack_bf16x8(v);       // (N is a multiple of 8)
        }
      };
      uint32_t r0[32], r1[32];
      tmem_ld32(acc + c_begin, r0);
      for (int c = c_begin; c < c_end; c += 64) {
        asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory");
        if (c + 32 < c_end) tmem_ld32(acc + c + 32, r1);
        store(r0, c);
        if (c + 32 < c_end) {
          asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory");
          if (c + 64 < c_end) tmem_ld32(acc + c + 64, r0);
          store(r1, c + 32);
        }
      }
      asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
      __syncwarp();
      if (lane == 0) asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];\n" ::"r"(acc_empty_lead + 8 * buf) : "memory");
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();
  pair_sync();
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;\n" ::"r"(tmem_base), "r"(p.tmem_cols) : "memory");
  }
}

}  // namespace precc
