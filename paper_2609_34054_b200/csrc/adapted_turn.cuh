// The main kernel of the adapted projection for the rows of a large batch or a short turn (17 .. some hundred): tiles of 128 output columns x
// TN rows with the weights on the M axis of tcgen05.mma, the K extent of a tile split over a cluster, slices merged by bulk copies
// between the blocks' shared memories in rank order.  Tile, split and merge are those of the turn projection into the caches.
//
// The adapters meet the sums in the block that finishes a row.  Its rows are sorted into groups of up to sixteen of one agent (while the
// main loop runs), and a warp multiplies a group's rows of T with 64 columns of that agent's B by mma.sync: rows of different agents never share a
// product.  B comes straight from global memory: a lane reads eight neighbouring columns of the four coordinates that the fragment wants
// of it, and column 8 g + j belongs to column g of the j-th MMA, so that it holds sixteen neighbouring columns of the result.
// Measured without / with adapters of rank 16, weights from HBM: 64 rows of 3584 x 3584 in bf16 8.8 / 14.0 us with the rows spread over eight agents, 12.7 with one (the
// bytes alone take 4.4); 61 rows of 4096 x 4096 with 64 agents of rank 64, whose A and B are twice the weights, 10.2 / 32.  What bounds
// it is latency: start, first copies, merge in the cluster, and ahead of it the start of the shrink kernel.
// Where a block has few rows the products are taken while the main loop runs, into a place of their own; else a warp's first one is, in registers, and
// all are added to the sums in shared memory.
#pragma once
#include "adapted_shrink.cuh"

namespace precc {

constexpr int AT_THREADS = (2 + AT_EPI_WARPS) * 32;      // producer, MMA issuer, eight merging warps

template <bool Q8>
__global__ void __launch_bounds__(AT_THREADS, 2)
adapted_turn_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const AdaptedParams p) {
  extern __shared__ __align__(1024) unsigned char smem[];
  if ((smem_u32(smem) & 1023u) != 0) {                   // the swizzle atoms and the peers' addresses rely on it
    if (threadIdx.x == 0) atomicOr(p.status, StatusBits::TIMEOUT);
    return;
  }
  const uint32_t smem0 = smem_u32(smem);
  const int KS = gridDim.x, rank = blockIdx.x;           // the cluster spans grid.x
  const int TN = p.BN;
  const int stage_bytes = pt_stage_bytes(TN, 1);
  constexpr int STEP = Q8 ? 128 : 64;
  const int low_bytes = at_low_bytes(TN, KS);
  float* low = reinterpret_cast<float*>(smem + pt_data_bytes(TN, KS, p.stages, 1));           // [own rows][128], where they are few
  AtTables& tab = *reinterpret_cast<AtTables*>(reinterpret_cast<unsigned char*>(low) + low_bytes);
  uint64_t* bars = reinterpret_cast<uint64_t*>(reinterpret_cast<unsigned char*>(&tab) + (sizeof(AtTables) + 15) / 16 * 16);
  const uint32_t full0 = smem_u32(bars);
  const uint32_t empty0 = full0 + 8 * PT_MAX_STAGES;
  const uint32_t acc_full = empty0 + 8 * PT_MAX_STAGES;
  const uint32_t ready_bar = acc_full + 8, recv_bar = acc_full + 16;
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(bars + 2 * PT_MAX_STAGES + 3);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int nkb = p.K / STEP;
  const int kb0 = (int)((long long)rank * nkb / KS);
  const int nkb_s = (int)((long long)(rank + 1) * nkb / KS) - kb0;
  const int m0 = blockIdx.z * TN, n0 = blockIdx.y * PT_COLS;
  const int n_rows = min(TN, p.M - m0);
  const int tw = pt_share(n_rows, KS);                   // rows finished by one block (the last ones may own fewer, or none)
  auto slice_rows = [&](int r) { return max(0, min(tw, n_rows - r * tw)); };
  const int own_rows = slice_rows(rank);
  float* dump = reinterpret_cast<float*>(smem);                               // [n_rows][128]
  float* recv = dump + (size_t)TN * PT_COLS;                                  // [KS-1][tw][128], slot = sender's rank with the own rank left out
  const bool adapters = p.agent_id != nullptr;

  if (threadIdx.x == 0) {
    prefetch_map(&map_w);
    prefetch_map(&map_x);
    for (int s = 0; s < p.stages; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, 1); }
    mbar_init(acc_full, 1);
    mbar_init(ready_bar, KS > 1 ? KS - 1 : 1);
    mbar_init(recv_bar, 1);
    mbar_expect_tx(recv_bar, (uint32_t)((KS - 1) * own_rows * PT_COLS * 4));   // the one arrival, and the bytes to come
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
    if (!adapters) pdl_wait();                           // with adapters the shrink kernel is ahead and has waited
    for (int it = 0; it < min(p.stages, nkb_s); ++it) {
      const uint32_t st = smem0 + it * stage_bytes;
      mbar_expect_tx(full0 + 8 * it, stage_bytes);
      tma_load_3d(st, &map_w, 0, n0, kb0 + it, full0 + 8 * it);
      tma_load_3d(st + PT_W_BYTES, &map_x, 0, m0, kb0 + it, full0 + 8 * it);
    }
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(tmem_holder)), "r"(p.tmem_cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  if (!adapters) pdl_wait();
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
  const uint32_t tmem_base = *tmem_holder;
  if (!adapters) pdl_launch_dependents();
  // every block's barriers exist before anybody arrives on them from outside (the wait comes with the first remote use)
  asm volatile("barrier.cluster.arrive.relaxed.aligned;\n" ::: "memory");

  if (warp == 0) {
    if (elect_one()) {
      RingWalk at;                                       // (the first round was requested above)
      for (int it = p.stages; it < nkb_s; ++it, at.next(p.stages)) {
        const uint32_t st = smem0 + at.s * stage_bytes, bar = full0 + 8 * at.s;
        mbar_wait(empty0 + 8 * at.s, at.parity, p.status);
        mbar_expect_tx(bar, stage_bytes);
        tma_load_3d(st, &map_w, 0, n0, kb0 + it, bar);
        tma_load_3d(st + PT_W_BYTES, &map_x, 0, m0, kb0 + it, bar);
      }
    }
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
  } else if (warp == 1) {
    const uint32_t idesc = Q8 ? umma_idesc_bf16(TN) & ~((1u << 7) | (1u << 10)) : umma_idesc_bf16(TN);     // (e4m3 is format 0)
    const uint64_t dw0 = umma_desc_sw128(smem0);
    const uint64_t dx0 = umma_desc_sw128(smem0 + PT_W_BYTES);
    if (elect_one()) {
      RingWalk at;
      for (int it = 0; it < nkb_s; ++it, at.next(p.stages)) {
        mbar_wait(full0 + 8 * at.s, at.parity, p.status);
        asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
        const uint64_t so = (uint64_t)((at.s * stage_bytes) >> 4);
#pragma unroll
        for (int k = 0; k < 4; ++k) {                    // 32 bytes of K a step
          if constexpr (Q8) umma_e4m3(tmem_base, dw0 + so + 2 * k, dx0 + so + 2 * k, idesc, (it | k) ? 1u : 0u);
          else umma_bf16(tmem_base, dw0 + so + 2 * k, dx0 + so + 2 * k, idesc, (it | k) ? 1u : 0u);
        }
        umma_commit(empty0 + 8 * at.s);
      }
      umma_commit(acc_full);                             // every MMA of the slice has completed: the ring is idle too
    }
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
  } else {
    const int quad = warp & 3, ew = warp - 2, half = ew >> 2;    // tensor-memory lanes of this warp; which of the two warps on them
    const int et = threadIdx.x - 64;                     // 0 .. 255 among the merging threads
    const int g = lane >> 2, t = lane & 3;
    auto sync_merging = [&]() { asm volatile("bar.sync 1, 256;\n" ::: "memory"); };
    int n_units = 0;                                     // a group x 64 columns
    float d[8][4];                                       // rows g, g + 8 x columns 16 t .. 16 t + 15 of a unit: [j][row, half] = column 16 t + 8 (e & 1) + j
    auto product = [&](int u) {
      const int gr = u >> 1, a = tab.agent[gr], n = n0 + (u & 1) * 64 + 8 * g;
      const int r0 = tab.rows[gr][g], r1 = tab.rows[gr][g + 8];
      const __nv_bfloat16* t0 = p.T + (long long)(m0 + rank * tw + r0) * p.rank_pad + 2 * t;
      const __nv_bfloat16* t1 = p.T + (long long)(m0 + rank * tw + r1) * p.rank_pad + 2 * t;
#pragma unroll
      for (int j = 0; j < 8; ++j) d[j][0] = d[j][1] = d[j][2] = d[j][3] = 0.f;
      const __nv_bfloat16* src = p.B + ((long long)a * p.rank + 2 * t) * p.N + n;
      auto fetch = [&](int k0, uint4 (&b)[4], uint32_t (&f)[4]) {        // coordinates k0 .. k0 + 15
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int r = k0 + (k & 1) + 8 * (k >> 1);
          b[k] = make_uint4(0, 0, 0, 0);
          if (2 * t + r < p.rank && n < p.N) b[k] = __ldg(reinterpret_cast<const uint4*>(src + (long long)r * p.N));
        }
        f[0] = r0 != AT_NO_ROW ? *reinterpret_cast<const uint32_t*>(t0 + k0) : 0u;
        f[1] = r1 != AT_NO_ROW ? *reinterpret_cast<const uint32_t*>(t1 + k0) : 0u;
        f[2] = r0 != AT_NO_ROW ? *reinterpret_cast<const uint32_t*>(t0 + k0 + 8) : 0u;
        f[3] = r1 != AT_NO_ROW ? *reinterpret_cast<const uint32_t*>(t1 + k0 + 8) : 0u;
      };
      auto multiply = [&](const uint4 (&b)[4], const uint32_t (&f)[4]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          auto word = [&](int k) { return j < 2 ? b[k].x : j < 4 ? b[k].y : j < 6 ? b[k].z : b[k].w; };
          const uint32_t pick = j & 1 ? 0x7632 : 0x5410;
          mma_bf16_16816(d[j], f, __byte_perm(word(0), word(1), pick), __byte_perm(word(2), word(3), pick));
        }
      };
      uint4 b0[4], b1[4];                                // the next sixteen coordinates are on their way while sixteen are multiplied
      uint32_t f0[4], f1[4];
      fetch(0, b0, f0);
      for (int k0 = 0; k0 < p.rank_pad; k0 += 32) {
        if (k0 + 16 < p.rank_pad) fetch(k0 + 16, b1, f1);
        multiply(b0, f0);
        if (k0 + 32 < p.rank_pad) fetch(k0 + 32, b0, f0);
        if (k0 + 16 < p.rank_pad) multiply(b1, f1);
      }
    };
    auto add_product = [&](int u, float* to) {           // to: the block's own rows
      const int gr = u >> 1;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = tab.rows[gr][g + 8 * e];
        if (r == AT_NO_ROW) continue;
        float* row = to + (size_t)r * PT_COLS + (u & 1) * 64 + 16 * t;
#pragma unroll
        for (int q = 0; q < 4; ++q) {                    // columns 4 q .. of the lane's sixteen
          float4 v = *reinterpret_cast<float4*>(row + 4 * q);
          const int j = 4 * (q & 1), h = 2 * e + (q >> 1);
          v.x += d[j][h]; v.y += d[j + 1][h]; v.z += d[j + 2][h]; v.w += d[j + 3][h];
          *reinterpret_cast<float4*>(row + 4 * q) = v;
        }
      }
    };
    if (adapters && own_rows > 0) {
      // ---- this block's rows in groups of one agent
      for (int i = et; i < AT_MAX_GROUPS * 8; i += 256) reinterpret_cast<uint32_t*>(tab.rows)[i] = 0xffffffffu;
      for (int i = et; i < AT_EPI_WARPS * AP_MAX_AGENTS / 4; i += 256) reinterpret_cast<uint32_t*>(tab.of_warp)[i] = 0u;
      const int a = et < own_rows ? agent_of(p, m0 + rank * tw + et) : -1;
      const unsigned same = __match_any_sync(0xffffffffu, a);
      const int before = __popc(same & ((1u << lane) - 1));
      sync_merging();
      if (a >= 0 && before == 0) tab.of_warp[ew][a] = (uint8_t)__popc(same);
      sync_merging();
      if (ew == 0) {                                     // groups of agents 2 lane and 2 lane + 1
        int c[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          int n = 0;
          for (int w = 0; w < AT_EPI_WARPS; ++w) n += tab.of_warp[w][2 * lane + i];
          c[i] = (n + 15) / 16;
        }
        int sum = c[0] + c[1];
        for (int m = 1; m < 32; m <<= 1) { const int o = __shfl_up_sync(0xffffffffu, sum, m); if (lane >= m) sum += o; }
        tab.first[2 * lane] = (uint8_t)(sum - c[0] - c[1]);
        tab.first[2 * lane + 1] = (uint8_t)(sum - c[1]);
        if (lane == 31) tab.n_groups = sum;
      }
      sync_merging();
      if (a >= 0) {
        int at = before;
        for (int w = 0; w < ew; ++w) at += tab.of_warp[w][a];
        const int gr = tab.first[a] + at / 16;
        tab.rows[gr][at % 16] = (uint16_t)et;
        tab.agent[gr] = (uint8_t)a;
      }
      sync_merging();
      n_units = 2 * tab.n_groups;
    }
    if (adapters) {
      pdl_wait();                                        // T is complete (in every block, so that this grid ends after the shrink kernel)
      if (et == 0) pdl_launch_dependents();
    }
    const bool early = low_bytes > 0 && n_units > 0;
    if (early) {
      for (int i = et; i < own_rows * PT_COLS / 4; i += 256) reinterpret_cast<float4*>(low)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      sync_merging();
      for (int u = ew; u < n_units; u += AT_EPI_WARPS) { product(u); add_product(u, low); }
    } else if (ew < n_units) {
      product(ew);
    }

    asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");       // the peers' barriers are initialised
    mbar_wait(acc_full, 0, p.status);
    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    // this block's ring is idle: the peers may send into the receive area that overlays it
    if (et < KS - 1) {
      const int peer = et < rank ? et : et + 1;
      asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];\n" ::"r"(dsmem_addr(ready_bar, peer)) : "memory");
    }
    // ---- dump slice by slice, the peers' first, the own one last; a peer's slice leaves while the next is dumped
    const uint32_t trow = tmem_base + (static_cast<uint32_t>(quad * 32) << 16);
    float* dcol = dump + quad * 32 + lane;
    for (int k = 1; k <= KS; ++k) {
      const int sl = rank + k < KS ? rank + k : rank + k - KS;
      const int c0 = sl * tw, nr = slice_rows(sl);
      for (int c = half * 8; c < nr; c += 32) {          // two groups of eight rows in flight per warp (the last one may run up to seven rows past n_rows: inside the tile, never read)
        uint32_t r0[8], r1[8];
        const bool two = c + 16 < nr;
        tmem_ld8(trow + c0 + c, r0);
        if (two) tmem_ld8(trow + c0 + c + 16, r1);
        asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory");
#pragma unroll
        for (int q = 0; q < 8; ++q) dcol[(size_t)(c0 + c + q) * PT_COLS] = __uint_as_float(r0[q]);
        if (two) {
#pragma unroll
          for (int q = 0; q < 8; ++q) dcol[(size_t)(c0 + c + 16 + q) * PT_COLS] = __uint_as_float(r1[q]);
        }
      }
      if (k < KS) asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");   // the copy engine reads what these threads wrote
      sync_merging();
      if (k < KS && et == 0) {
        if (k == 1) mbar_wait_cluster(ready_bar, 0, p.status);                     // every peer's ring is idle
        if (nr > 0) {
          const uint32_t src = smem_u32(dump) + (uint32_t)(c0 * PT_COLS * 4);
          const uint32_t dst = dsmem_addr(smem_u32(recv) + (uint32_t)((rank < sl ? rank : rank - 1) * tw * PT_COLS * 4), sl);
          asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n"
                       ::"r"(dst), "r"(src), "r"(nr * PT_COLS * 4), "r"(dsmem_addr(recv_bar, sl)) : "memory");
        }
      }
    }
    // ---- the adapters' share of the own rows
    if (!early && ew < n_units) {
      float* own = dump + (size_t)rank * tw * PT_COLS;
      add_product(ew, own);
      for (int u = ew + AT_EPI_WARPS; u < n_units; u += AT_EPI_WARPS) { product(u); add_product(u, own); }
    }
    if (n_units > 0) sync_merging();
    // ---- own rows + received rows, in rank order: sixteen threads per row, eight columns each
    const float* own = dump + (size_t)rank * tw * PT_COLS;
    const int piece = et & 15, gc = n0 + piece * 8;
    float ws[8], xs = 0.f;                               // 8 bits: the scales of this thread's columns and of its next row, ahead of the last wait
    if constexpr (Q8) {
      if (gc < p.N) {
        const float4 a = __ldg(reinterpret_cast<const float4*>(p.w_scale + gc)), b = __ldg(reinterpret_cast<const float4*>(p.w_scale + gc) + 1);
        ws[0] = a.x; ws[1] = a.y; ws[2] = a.z; ws[3] = a.w; ws[4] = b.x; ws[5] = b.y; ws[6] = b.z; ws[7] = b.w;
        if ((et >> 4) < own_rows) xs = __ldg(p.x_scale + m0 + rank * tw + (et >> 4));
      }
    }
    mbar_wait_cluster(recv_bar, 0, p.status);
    if (gc < p.N) {
      for (int r = et >> 4; r < own_rows; r += AT_EPI_WARPS * 2) {
        const long long m = m0 + rank * tw + r;
        float v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = 0.f;
        if (early) {
          const float4 a = *reinterpret_cast<const float4*>(low + r * PT_COLS + piece * 8), b = *reinterpret_cast<const float4*>(low + r * PT_COLS + piece * 8 + 4);
          v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        }
#pragma unroll
        for (int s = 0; s < GEMM_MAX_KS; ++s) {
          if (s < KS) {
            const float* src = (s == rank ? own : recv + (size_t)(s < rank ? s : s - 1) * tw * PT_COLS) + r * PT_COLS + piece * 8;
            const float4 a = *reinterpret_cast<const float4*>(src), b = *reinterpret_cast<const float4*>(src + 4);
            v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w; v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
          }
        }
        if constexpr (Q8) {
#pragma unroll
          for (int q = 0; q < 8; ++q) v[q] = unscale(v[q], ws[q], xs);
          if (r + AT_EPI_WARPS * 2 < own_rows) xs = __ldg(p.x_scale + m + AT_EPI_WARPS * 2);
        }
        *reinterpret_cast<uint4*>(p.y + m * p.N + gc) = pack_bf16x8(v);
      }
    }
    asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  }
  // the sends read the sender's shared memory: nobody leaves before every block has received everything
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem_base), "r"(p.tmem_cols) : "memory");
  }
}

}  // namespace precc
