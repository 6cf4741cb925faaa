// Which kernels take a call of the adapted projection and how its work is cut: arithmetic on sizes alone, free of CUDA, so that the rules can be
// compiled and checked without a GPU.
#pragma once
#include <algorithm>
#include <cstdint>

#include "proj_plan.h"

namespace precc {

constexpr int AP_MAX_AGENTS = 64;
constexpr int AP_ROW_BYTES = 128;             // bytes of K in a k-block: 64 bf16 or 128 e4m3

// ---- few rows (adapted_few.cuh): up to sixteen with at most two waves of blocks of sixteen columns (two blocks an SM), up to 32, where a block holds an SM, with one;
// past eight rows, where every step costs a warp more, none deeper than 4096 (eight steps of its eight warps in bf16, four in 8 bits).  us, few / turn kernel, rank 16, bf16:
// 8 rows, 4096 x 4096 10.7 / 13.9, 4096 x 9472 17.6 / 18.9, 8192 x 1024 9.1 / 11.0, but 4096 x 14336 24.5 / 22.3; 16 rows, 4096 x 4096 11.7 / 13.1,
// 4096 x 9472 19.0 / 19.9, 2048 x 2048 6.5 / 9.0, but 7168 x 2048 14.8 / 12.7; 32 rows, 2048 x 2048 8.7 / 10.3, 3584 x 1280 10.9 / 11.4, but 4096 x 4096
// 17.8 / 13.3 and 7168 x 2048 15.5 / 12.9.  In 8 bits the same, but for a second wave without adapters (8 rows, 4096 x 9472: 11.2 / 9.6), and but for the
// depth, where the sides cross later (rank 16 / without adapters: 16 rows, 4096 x 4096 9.4 / 13.1 and 6.2 / 7.4, 5120 x 2048 10.9 / 12.4 and 5.4 / 6.6, 8192 x 2048
// 12.9 / 13.3 and 6.9 / 7.5, 8192 x 1024 12.6 / 12.4 and 6.5 / 6.7; 32 rows, 4096 x 2048 11.2 / 12.4 and 6.2 / 6.5, 8192 x 2048 15.8 / 13.9 and 9.8 / 7.9): one
// depth for both types, as eight steps in 8 bits would be too deep for 32 rows.
constexpr int AF_MAX_ROWS = 32;
inline bool few_rows(int M, int K, int N, int sm_count) {
  return M <= 8 ? N <= 64 * sm_count : M <= AF_MAX_ROWS && K <= 4096 && N <= (M <= 16 ? 64 : 16) * sm_count;
}

// ---- turns (adapted_turn.cuh)
constexpr int AT_NO_ROW = 0xffff;
constexpr int AT_EPI_WARPS = 8;
constexpr int AT_MAX_GROUPS = PT_MAX_TN / 16 + AP_MAX_AGENTS;
struct AtTables {                             // a block's own rows in groups of up to sixteen of one agent
  uint16_t rows[AT_MAX_GROUPS][16];           // rows of a group (AT_NO_ROW: none), counted among the block's own rows
  uint8_t agent[AT_MAX_GROUPS];
  uint8_t of_warp[AT_EPI_WARPS][AP_MAX_AGENTS];          // rows of an agent among the 32 of a warp
  uint8_t first[AP_MAX_AGENTS];               // first group of an agent
  int n_groups;
};
constexpr int AT_LOW_ROWS = 32;               // own rows of a block whose adapters' share has a place beside the ring
PRECC_HD constexpr int at_low_bytes(int tn, int ks) { return pt_share(tn, ks) <= AT_LOW_ROWS ? AT_LOW_ROWS * PT_COLS * 4 : 0; }
PRECC_HD constexpr int at_smem_bytes(int tn, int ks, int stages) {
  return pt_data_bytes(tn, ks, stages, 1) + at_low_bytes(tn, ks) + ((int)sizeof(AtTables) + 15) / 16 * 16 + (2 * PT_MAX_STAGES + 4) * 8;
}

// ---- many rows (adapted_pair.cuh)
constexpr int AP_MAX_STAGES = 8;
constexpr int AP_BM = 2 * GEMM_BM;
constexpr int AP_A_BYTES = GEMM_BM * AP_ROW_BYTES;
PRECC_HD constexpr int ap_w_bytes(int bn) { return (bn / 2 + 63) / 64 * 64 * AP_ROW_BYTES; }   // (a step of B takes whole boxes of 64 columns)
PRECC_HD constexpr int ap_stage_bytes(int bn) { return AP_A_BYTES + ap_w_bytes(bn); }
PRECC_HD constexpr int ap_smem_bytes(int bn, int stages) { return stages * ap_stage_bytes(bn) + (2 * stages + 6) * 8 + 1024; }

// ---- the rank-r product of many rows (adapted_shrink.cuh)
constexpr int AS_LANES = 128;
constexpr int AS_MAX_STAGES = 24;
constexpr int AS_DUMP_ROWS = 64, AS_DUMP_PITCH = AS_LANES + 4;            // (in floats; the pitch spreads a row's pieces over the banks)
constexpr int AS_TAIL_BYTES = AS_DUMP_ROWS * AS_DUMP_PITCH * 4;
PRECC_HD constexpr int as_chunks(bool q8) { return q8 ? 2 : 4; }          // accumulators of a pass at most
PRECC_HD constexpr int as_chunk_bytes(bool q8) { return AS_LANES * AP_ROW_BYTES * (q8 ? 2 : 1); }

constexpr int SHRINK_SMEM = 38 * 1024;        // what a block of the small shrink kernel takes at most: left free beside the main kernel
constexpr int STATIC_SMEM = 4096;             // at least what the kernels declare of their own, and the system takes

enum AdaptedKernel { ADAPTED_FEW = 1, ADAPTED_TURN = 2, ADAPTED_PAIR = 3 };

// The rank-r product: by mma.sync beside the main kernel, or on tcgen05 ahead of it.  The first reads A again for every 16 or 32 rows, the second once for up
// to 256, but the main kernel starts only when it is done.  us of the whole call, mma.sync / tcgen05, 8 agents in runs: 4096 x 4096 bf16 rank 64, 2048 / 4096 / 8192
// rows: 61.9 / 61.4, 119 / 116, 216 / 201; rank 16: 56.2 / 59.4, 111 / 113, 197 / 195; 8 bits rank 64, 512 / 1024 / 4096 rows: 25.6 / 23.7, 32.4 / 29.2,
// 97 / 71; rank 16: 20.3 / 22.1, 26.3 / 27.3, 70 / 67 (8 bits read A twice, as value and rest).
inline bool shrink_on_tcgen05(int M, int rank, bool q8) { return (long long)M * rank >= (q8 ? 16384 : 262144); }

// Columns of a tile of the pair kernel, and the time it predicts in us: rounds of tiles over the pairs of SMs, per k-block what issue and copies take up to 96 columns
// and what L2 delivers beyond (256 x 256: 32 KB per SM and k-block).  Measured at 4096 x 4096 in bf16, 64 / 512 / 1024 / 8192 rows: 15.4 / 17.2 / 26.8 / 172 us,
// predicted 15.4 / 17.6 / 26.7 / 182.
struct PairPlan { int bn = 0; double cost = 1e30; };
inline PairPlan plan_pair(long long M, int N, int nkb, int sm_count) {
  PairPlan best;
  for (int bn : {256, 192, 128, 64}) {
    const long long tiles = ((M + AP_BM - 1) / AP_BM) * ((N + bn - 1) / bn), rounds = (tiles + sm_count / 2 - 1) / (sm_count / 2);
    const double cost = 4.5 + (double)rounds * nkb * (0.17 + 0.0011 * std::max(0, bn - 96));
    if (cost < best.cost - 1e-9) { best.bn = bn; best.cost = cost; }
  }
  return best;
}

// Tiles of the turn kernel: 128 columns x tn rows, the K extent over ks blocks of a cluster; predicted as the turn projection into the caches is (proj_plan.h), per wave
// of resident clusters, and 1.5 us a launch.  `limit`: shared memory of a block.  At 4096 x 4096 in bf16, 64 / 256 / 512 rows: measured 10.1 / 16.4 / 19.6,
// predicted 9.2 / 16.8 / 20.0.
struct AdaptedTurnPlan { int tn = 0, ks = 0, stages = 0; double cost = 1e30; };
inline AdaptedTurnPlan plan_adapted_turn(int M, int N, int nkb, int sm_count, int limit, const int* clusters) {
  AdaptedTurnPlan best;
  const long long groups = (N + PT_COLS - 1) / PT_COLS;
  for (int t = (M + PT_MAX_TN - 1) / PT_MAX_TN, last = 0; last != 16; ++t) {
    const int tn = ((M + t - 1) / t + 15) / 16 * 16;
    if (tn == last) continue;
    last = tn;
    const long long tiles = (M + tn - 1) / tn;
    if (tiles > 65535) break;                            // (a grid axis)
    for (int ks = 1; ks <= GEMM_MAX_KS && ks <= nkb; ++ks) {          // (every block of a cluster has a k-block)
      const int resident = ks == 1 ? sm_count : clusters[ks];
      if (resident < 1) continue;
      const long long waves = (groups * tiles + resident - 1) / resident;
      const int kb = (nkb + ks - 1) / ks;
      int st = std::min(kb, PT_MAX_STAGES);
      while (st > 0 && at_smem_bytes(tn, ks, st) > limit) --st;
      if (st < std::min(kb, 3)) continue;
      const double cost = (double)waves * (1.5 + kb * (0.37 + 0.00036 * tn) + 0.005 * pt_share(tn, ks) * (ks - 1) + 0.0113 * tn + 0.1 * ks);
      if (cost < best.cost) { best.tn = tn; best.ks = ks; best.stages = st; best.cost = cost; }
    }
  }
  return best;
}

// What the adapters cost the turn kernel beyond what they cost the pair kernel, in us (a difference: below zero where the pair kernel loses more by them).  Its products with B grow with the rank and the rows that a block
// finishes, while the pair kernel has nothing to do when the rank-r product of a deep K comes late (256 rows of 4096 x 4096 in bf16, rank 16 / 64: turn 19.4 / 24.1,
// pair 24.8 / 27.6; of 1024 x 1024: 10.9 / 14.4 against 10.8 / 12.1; 64 rows of 2048 x 2048 in 8 bits, rank 64: 14.9 / 12.3).
inline double turn_adapter_cost(int rank, int share, int K) {
  return rank > 0 ? 1.0 + 0.06 * (rank - 16) - 0.0023 * std::min(2048, std::max(0, K - 2048)) + rank * share / 2000.0 : 0.0;
}

// The main kernel of a call.  rank 0: no adapters.  Turns are compared up to 4096 rows; beyond, the pair kernel always wins.
struct AdaptedPlan { int kernel = 0, bn = 0, tn = 0, ks = 0, stages = 0; bool shrink_tc = false; };
inline AdaptedPlan plan_adapted(int M, int N, int K, int rank, bool q8, int sm_count, int max_smem, const int* clusters, int force_kernel = 0, int force_shrink = 0) {
  AdaptedPlan r;
  const int nkb = K / (q8 ? 128 : 64);
  r.shrink_tc = rank > 0 && (force_shrink ? force_shrink == 2 : shrink_on_tcgen05(M, rank, q8));
  const int limit = max_smem - (rank > 0 && !r.shrink_tc ? SHRINK_SMEM : 0);
  if (force_kernel == ADAPTED_FEW ? M <= AF_MAX_ROWS : force_kernel == 0 && few_rows(M, K, N, sm_count)) { r.kernel = ADAPTED_FEW; return r; }
  const PairPlan pair = plan_pair(M, N, nkb, sm_count);
  if (force_kernel != ADAPTED_PAIR && M <= 4096) {
    const AdaptedTurnPlan turn = plan_adapted_turn(M, N, nkb, sm_count, limit - 1024, clusters);
    if (turn.ks > 0 && (force_kernel == ADAPTED_TURN || turn.cost + turn_adapter_cost(rank, pt_share(turn.tn, turn.ks), K) <= pair.cost)) {
      r.kernel = ADAPTED_TURN; r.tn = turn.tn; r.ks = turn.ks; r.stages = turn.stages;
      return r;
    }
  }
  r.kernel = ADAPTED_PAIR; r.bn = pair.bn;
  r.stages = std::min(AP_MAX_STAGES, (limit - STATIC_SMEM) / ap_stage_bytes(pair.bn));
  return r;
}

// The small shrink kernel: rows of a block (at most `most`, 8 or more), and how many blocks share the K extent.  Fewer rows a block where that fills more SMs: a
// block takes the agents among its rows one after the other.
struct ShrinkPlan { int rows = 0, ks = 0; };
inline ShrinkPlan plan_shrink(int M, int K, int most, int sm_count) {
  ShrinkPlan r;
  r.ks = 8;
  while (r.ks > 1 && (K / 64 < r.ks * 8 || (M + most - 1LL) / most * r.ks > 2LL * sm_count)) r.ks >>= 1;
  r.rows = most;
  while (r.rows > 1 && (M + r.rows / 2 - 1LL) / (r.rows / 2) * r.ks <= sm_count) r.rows /= 2;
  return r;
}

// The shrink kernel on tcgen05: rows of a block, blocks that share the K extent, k-blocks in a slot of the ring (as many as leave three slots for tiles of one or two agents,
// every block two slots to fill, and one slot with all lanes of an accumulator), tensor-memory columns and shared memory.
struct ShrinkTcPlan { int tn = 0, ks = 1, kps = 4, tmem_cols = 32, ring = 0, smem = 0; };
inline ShrinkTcPlan plan_shrink_tc(int M, int nkb, int rank, int n_agents, bool q8, int sm_count, int max_smem) {
  ShrinkTcPlan r;
  const int rounds = (int)((M + sm_count * 256LL - 1) / (sm_count * 256LL));
  r.tn = (int)((M + (long long)sm_count * rounds - 1) / ((long long)sm_count * rounds) + 15) / 16 * 16;
  if (M <= 4096) r.tn = std::max(r.tn, std::min(32, (M + 15) / 16 * 16));
  const long long tiles = (M + (long long)r.tn - 1) / r.tn;
  while (r.ks < 8 && tiles * r.ks * 2 <= sm_count && nkb >= r.ks * 4) r.ks *= 2;
  // Up to 112 rows a block, twice the rows and half the K extent instead (measured at 4096 deep only): a tile with a second agent then costs half as much more, and A is read half as often
  // (4096 deep, bf16, eight agents' runs of rank 16 / 64, this kernel in us: 3000 rows 18.4 / 21.8 -> 14.1 / 16.6, 4096 19.1 / 22.2 -> 14.4 / 18.0, 8192 20.1 / 24.6 -> 18.8 / 23.4; but
  // 9472 with 128 rows a block 21.0 / 25.4 -> 20.4 / 26.3, 12000 24.5 / 27.5 -> 23.6 / 30.5, and in 8 bits 12000 18.4 / 21.8 -> 19.1 / 27.8).
  const int pair_tn = ((M + sm_count / 2 - 1) / (sm_count / 2) + 15) / 16 * 16;
  if (r.ks == 1 && pair_tn <= 112 && nkb >= 4) { r.tn = pair_tn; r.ks = 2; }
  const int slots = AS_LANES / rank, chunks = std::min(as_chunks(q8), (n_agents + slots - 1) / slots);
  while (r.tmem_cols < std::min(chunks * r.tn, 512)) r.tmem_cols <<= 1;
  // behind the ring: 64 rows of an accumulator, and the sums of a K slice
  const int tail = AS_TAIL_BYTES + (r.ks > 1 ? r.tn * rank * 4 : 0), ring = max_smem - STATIC_SMEM - tail;
  const int typical = r.tn * AP_ROW_BYTES + std::min(n_agents, 2) * rank * AP_ROW_BYTES * (q8 ? 2 : 1);
  const int whole = r.tn * AP_ROW_BYTES + as_chunk_bytes(q8);             // 64 KB at most, beside a tail of up to 97 KB
  while (r.kps > 1 && (3 * r.kps * typical > ring || r.kps * whole > ring || nkb < 2 * r.ks * r.kps)) r.kps /= 2;
  r.ring = ring;
  r.smem = ring + tail + 1024;
  return r;
}

}  // namespace precc
