// The main kernel of the adapted projection for a handful of rows (decode steps, up to 32): one pass over the weights.
//
// HBM-bound at K x N weights.  A block takes 16 output columns over the whole K extent, its eight warps every eighth k-block
// (so nothing is merged between blocks), and each warp asks for several k-blocks of weights before it uses the first: the
// fragments of mma.sync come straight from the packed weights into registers, 16 bytes a lane, which keeps more of the matrix in
// flight than a ring in shared memory would.  Output columns are the M axis of the MMA and the rows of X its N axis, so
// eight rows cost nothing over one.
// The adapters: warp u takes the u-th agent among the rows.  Its B slice (r x 16) is asked for with the first weights and meets that agent's rows
// of T once the shrink kernel is done; the rows of others are zero in the product and dropped from it.
// Measured, weights from HBM, us without / with adapters: 1 row of 2048 x 2048 in bf16 3.5 / 4.6 (rank 16; 8.4 MB: 2.4 TB/s without), 8 rows of 4096 x 9472 14.2 / 18.2
// (rank 16; 5.5 TB/s), 8 rows of 4096 x 4096 in 8 bits 5.9 / 9.1 (rank 32, eight agents).  What adapters add is the start of this
// kernel behind the shrink kernel's.  Started at once instead, with nothing but weights asked for before the wait for T, the calls came out
// slower (1 row 6.8, 8 rows in 8 bits 11.9): X, the ids and B then come behind T as well.
#pragma once
#include "adapted.cuh"

namespace precc {

constexpr int AF_WARPS = 8;
constexpr int AF_THREADS = AF_WARPS * 32;

// Weights are read once: past L1.
__device__ __forceinline__ uint4 ld_stream(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.L2::256B.v4.u32 {%0,%1,%2,%3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

constexpr int AF_COLS = 16;                       // output columns of a block: the M axis of one MMA

__host__ __device__ constexpr int af_smem_bytes(int nt, int rank_pad) {
  return (AF_WARPS + 1) * 8 * nt * (AF_COLS + 4) * 4 + AF_WARPS * rank_pad * (AF_COLS * 2 + 16);
}

// NT: eight-row pieces of X.  Steps of 128 bytes of K (64 bf16, 128 e4m3).
template <int NT, bool Q8>
__global__ void __launch_bounds__(AF_THREADS, NT < 4 ? 2 : 1)
adapted_few_kernel(const AdaptedParams p, const uint8_t* __restrict__ W) {
  constexpr int C = AF_COLS, S = C + 4;           // row of the partial sums, padded: the lanes of a store hit 32 banks
  constexpr int BP = C * 2 + 16;                  // bytes of a row of a B slice, padded for ldmatrix
  constexpr int U = NT == 1 ? 3 : 2;              // k-blocks of a warp in flight: what the registers of two blocks a SM hold
  extern __shared__ __align__(16) uint8_t smem[];
  float (*red)[8 * NT][S] = reinterpret_cast<float (*)[8 * NT][S]>(smem);                    // [warp]
  float (*low)[S] = red[AF_WARPS];                                                           // s (x A) B of every row
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t b_s = smem_u32(smem) + (AF_WARPS + 1) * 8 * NT * S * 4 + warp * p.rank_pad * BP;      // this warp's slice of B
  const int n0 = blockIdx.x * C;
  const bool adapters = p.agent_id != nullptr;
  if (!adapters) { pdl_wait(); pdl_launch_dependents(); }      // with adapters the shrink kernel is ahead and has waited

  const int nkb = p.K / (Q8 ? 128 : 64);
  const long long row_bytes = (long long)p.K * (Q8 ? 1 : 2);
  const uint8_t* x = static_cast<const uint8_t*>(p.x);
  float acc[NT][4];
#pragma unroll
  for (int n = 0; n < NT; ++n) { acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.f; }
  uint4 wv[U][2][2], xv[U][NT][2];                // [..][row g, row g + 8][piece t, piece t + 4]
  auto fetch = [&](int u, int kb) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int n = n0 + h * 8 + g;
      const uint4* src = reinterpret_cast<const uint4*>(W + ((long long)kb * p.N + n) * AP_ROW_BYTES);
#pragma unroll
      for (int c = 0; c < 2; ++c) wv[u][h][c] = kb < nkb && n < p.N ? ld_stream(src + t + 4 * c) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const uint4* src = reinterpret_cast<const uint4*>(x + (n * 8 + g) * row_bytes + (long long)kb * AP_ROW_BYTES);
#pragma unroll
      for (int c = 0; c < 2; ++c) xv[u][n][c] = kb < nkb && n * 8 + g < p.M ? __ldg(src + t + 4 * c) : make_uint4(0, 0, 0, 0);
    }
  };
#pragma unroll
  for (int u = 0; u < U; ++u) fetch(u, warp + u * AF_WARPS);

  // this warp's agents (every eighth among the rows, from the w-th on), and their slices of B
  int id = -1;
  if (adapters && lane < p.M) id = agent_of(p, lane);
  unsigned todo = __ballot_sync(0xffffffffu, id >= 0);
  const unsigned with_adapter = todo;
  unsigned mine[NT];
  int agent[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) { mine[i] = 0; agent[i] = -1; }
  for (int u = 0; todo; ++u) {
    const int a = __shfl_sync(0xffffffffu, id, __ffs(todo) - 1);
    const unsigned same = __ballot_sync(0xffffffffu, id == a);
    todo &= ~same;
#pragma unroll
    for (int i = 0; i < NT; ++i)
      if (u == warp + i * AF_WARPS) { mine[i] = same; agent[i] = a; }
  }
  auto fetch_b = [&](int a) {                     // (coordinates past the rank, columns past N: zeros)
    for (int i = lane; i < p.rank_pad * (C / 8); i += 32) {
      const int r = i / (C / 8), c = i % (C / 8) * 8;
      const bool on = r < p.rank && n0 + c < p.N;
      cp_async16(b_s + r * BP + c * 2, on ? p.B + ((long long)a * p.rank + r) * p.N + n0 + c : p.B, on ? 16 : 0);
    }
    cp_async_commit();
  };
  if (agent[0] >= 0) fetch_b(agent[0]);

  for (int kb = warp; kb < nkb; kb += U * AF_WARPS) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const uint32_t a0[4] = {wv[u][0][c].x, wv[u][1][c].x, wv[u][0][c].y, wv[u][1][c].y};
        const uint32_t a1[4] = {wv[u][0][c].z, wv[u][1][c].z, wv[u][0][c].w, wv[u][1][c].w};
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          mma_step<Q8>(acc[n], a0, xv[u][n][c].x, xv[u][n][c].y);
          mma_step<Q8>(acc[n], a1, xv[u][n][c].z, xv[u][n][c].w);
        }
      }
      fetch(u, kb + (u + U) * AF_WARPS);
    }
  }
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) red[warp][n * 8 + 2 * t + (e & 1)][g + 8 * (e >> 1)] = acc[n][e];

  constexpr int MINE = 8 * NT * C / AF_THREADS > 0 ? 8 * NT * C / AF_THREADS : 1;       // what this thread finishes (in one column), and its scales
  float xs[MINE], ws = 1.f;
  if constexpr (Q8) { if (n0 + (int)threadIdx.x % C < p.N) ws = __ldg(p.w_scale + n0 + threadIdx.x % C); }
#pragma unroll
  for (int j = 0; j < MINE; ++j) {
    const int r = (threadIdx.x + j * AF_THREADS) / C;
    xs[j] = 1.f;
    if constexpr (Q8) { if (r < p.M) xs[j] = __ldg(p.x_scale + r); }
  }
  if (adapters) {
    pdl_wait();                                   // T is complete
    if (threadIdx.x == 0) pdl_launch_dependents();
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      if (agent[i] < 0) continue;                 // (the same in every lane)
      if (i > 0) { __syncwarp(); fetch_b(agent[i]); }
      cp_async_wait<0>();
      __syncwarp();
#pragma unroll
      for (int half = 0; half < (NT + 1) / 2; ++half) {          // sixteen rows at a time
        if (!((mine[i] >> (16 * half)) & 0xffffu)) continue;
        float d[C / 8][4];
#pragma unroll
        for (int j = 0; j < C / 8; ++j) d[j][0] = d[j][1] = d[j][2] = d[j][3] = 0.f;
        for (int k0 = 0; k0 < p.rank_pad; k0 += 16) {
          uint32_t a[4];                          // rows g and g + 8 of T, coordinates 2t.. and 2t + 8..
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int r = 16 * half + g + 8 * (q & 1);
            const __nv_bfloat16* src = p.T + (long long)r * p.rank_pad + k0 + 2 * t + 8 * (q >> 1);
            a[q] = (mine[i] >> r) & 1u ? *reinterpret_cast<const uint32_t*>(src) : 0u;
          }
          uint32_t b[4];                          // 16 coordinates x 16 columns
          ldsm_x4_t(b, b_s + (k0 + (lane & 15)) * BP + (lane >> 4) * 16);
          mma_bf16_16816(d[0], a, b[0], b[1]);
          mma_bf16_16816(d[1], a, b[2], b[3]);
        }
#pragma unroll
        for (int j = 0; j < C / 8; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = 16 * half + g + 8 * (e >> 1);
            if ((mine[i] >> r) & 1u) low[r][8 * j + 2 * t + (e & 1)] = d[j][e];
          }
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < MINE; ++j) {
    const int i = threadIdx.x + j * AF_THREADS, r = i / C, c = i % C;
    if (r >= p.M || n0 + c >= p.N) continue;
    float v = (with_adapter >> r) & 1u ? low[r][c] : 0.f;
#pragma unroll
    for (int w = 0; w < AF_WARPS; ++w) v += red[w][r][c];
    p.y[(long long)r * p.N + n0 + c] = __float2bfloat16(Q8 ? unscale(v, ws, xs[j]) : v);
  }
}

}  // namespace precc
