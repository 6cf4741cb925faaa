// libprecc: the projection of a batch whose rows carry adapters of their own, in bf16 and in 8 bits, and the packing of 8-bit weights.
#include <cuda_fp16.h>

#include <algorithm>

#include "adapted_few.cuh"
#include "adapted_pair.cuh"
#include "adapted_shrink.cuh"
#include "adapted_turn.cuh"
#include "api_internal.h"

using namespace precc;

namespace {

// ------------------------------------------------------------------------------------------ 8-bit weights
// A block quantises 32 columns: their largest magnitudes first, then k-blocks of 128 through shared memory.  The scale of a
// column is the least power of two 2^s with max <= 448 * 2^s = 1.75 * 2^(8 + s), read off the bits of the maximum: e4m3 is a
// floating type, so a power of two costs it no precision, and B / scale is exact in bf16.
constexpr int PACK8_COLS = 32, PACK8_ROWS = 8;

__device__ __forceinline__ int e4m3_scale_exponent(float top) {
  const uint32_t b = __float_as_uint(top);
  const int s = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return top == 0.f || (b >> 23) == 255u ? 0 : max(s, -100);
}

__global__ void __launch_bounds__(PACK8_COLS * PACK8_ROWS)
pack_kmajor_e4m3_kernel(const __nv_bfloat16* __restrict__ src, int K, int N, uint8_t* __restrict__ dst, float* __restrict__ scale) {
  __shared__ float top_s[PACK8_ROWS][PACK8_COLS];
  __shared__ float inv_s[PACK8_COLS];
  __shared__ float tile[128][PACK8_COLS + 1];
  const int tx = threadIdx.x % PACK8_COLS, ty = threadIdx.x / PACK8_COLS;
  const int c0 = blockIdx.x * PACK8_COLS, c = c0 + tx;
  float top = 0.f;
  for (int k = ty; k < K; k += PACK8_ROWS) top = fmaxf(top, c < N ? fabsf(__bfloat162float(src[(size_t)k * N + c])) : 0.f);
  top_s[ty][tx] = top;
  __syncthreads();
  if (ty == 0) {
    for (int i = 1; i < PACK8_ROWS; ++i) top = fmaxf(top, top_s[i][tx]);
    const int s = e4m3_scale_exponent(top);
    inv_s[tx] = __uint_as_float((uint32_t)(127 - s) << 23);
    if (c < N) scale[c] = __uint_as_float((uint32_t)(127 + s) << 23);
  }
  __syncthreads();
  for (int k0 = 0; k0 < K; k0 += 128) {
    for (int k = ty; k < 128; k += PACK8_ROWS) tile[k][tx] = c < N ? __bfloat162float(src[(size_t)(k0 + k) * N + c]) * inv_s[tx] : 0.f;
    __syncthreads();
    for (int i = threadIdx.x; i < PACK8_COLS * 32; i += PACK8_COLS * PACK8_ROWS) {        // four values of K of a column
      const int cc = i / 32, k = i % 32 * 4;
      if (c0 + cc < N)
        *reinterpret_cast<uint32_t*>(dst + ((size_t)(k0 / 128) * N + c0 + cc) * 128 + k) =
            pack_e4m3x4(tile[k][cc], tile[k + 1][cc], tile[k + 2][cc], tile[k + 3][cc]);
    }
    __syncthreads();
  }
}

__global__ void pack_expand_e4m3_kernel(const __nv_bfloat16* __restrict__ B, long long n, int N, const float* __restrict__ scale,
                                        __nv_bfloat16* __restrict__ dst) {
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x)
    dst[i] = __float2bfloat16(__fdiv_rn(__bfloat162float(B[i]), scale[i % N]));
}

// A of one agent, [K][rank] -> two e4m3 matrices with one power of two per coordinate: hi = e4m3(a / scale) and lo = e4m3(a / scale - hi).  bf16 has eight
// significant bits and e4m3 four, so hi + lo is a / scale exactly where that is at
// least 1/4 (2^-9 of the coordinate's largest value), and off by at most half of the least step 2^-9 (2^-17 of the largest) below.
// dst [K/128][2][n_agents * rank][128].
__global__ void __launch_bounds__(256)
pack_adapter_e4m3_kernel(const __nv_bfloat16* __restrict__ src, int K, int rank, int agent, int rows, uint8_t* __restrict__ dst, float* __restrict__ scale) {
  __shared__ float top_s[8];
  const int c = blockIdx.x;                                          // the coordinate
  float top = 0.f;
  for (int k = threadIdx.x; k < K; k += 256) top = fmaxf(top, fabsf(__bfloat162float(src[(size_t)k * rank + c])));
  for (int m = 16; m > 0; m >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, m));
  if ((threadIdx.x & 31) == 0) top_s[threadIdx.x / 32] = top;
  __syncthreads();
  for (int i = 0; i < 8; ++i) top = fmaxf(top, top_s[i]);
  const int s = e4m3_scale_exponent(top);
  if (threadIdx.x == 0) scale[agent * rank + c] = __uint_as_float((uint32_t)(127 + s) << 23);
  const float inv = __uint_as_float((uint32_t)(127 - s) << 23);
  for (int k = threadIdx.x; k < K; k += 256) {
    const float v = __bfloat162float(src[(size_t)k * rank + c]) * inv;
    const uint32_t hi = pack_e4m3x4(v, 0.f, 0.f, 0.f) & 0xffu;
    uint32_t h2;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(h2) : "h"((uint16_t)hi));
    const float rest = v - __half2float(__ushort_as_half((uint16_t)h2));
    uint8_t* at = dst + ((size_t)(k / 128) * 2 * rows + agent * rank + c) * 128 + k % 128;
    at[0] = (uint8_t)hi;
    at[(size_t)rows * 128] = (uint8_t)pack_e4m3x4(rest, 0.f, 0.f, 0.f);
  }
}

// ------------------------------------------------------------------------------------------ tensor maps
int32_t encode(precc_ctx* ctx, CUtensorMap* map, CUtensorMapDataType type, int rank, const void* base, const cuuint64_t* dims,
               const cuuint64_t* strides, const cuuint32_t* box, CUtensorMapSwizzle swizzle) {
  const cuuint32_t one[3] = {1, 1, 1};
  const CUresult r = ctx->encode_tiled(map, type, rank, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                                       CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return fail(ctx, PRECC_ERR_CUDA, "cuTensorMapEncodeTiled (adapted projection) failed (%d)", (int)r);
  return PRECC_OK;
}
// Rows of X, and packed weights [K / step][N][step], as k-blocks of 128 bytes: a box is `box_rows` rows of one k-block (of
// X, also of several, one behind the other; those past K arrive as zeros).
int32_t map_rows(precc_ctx* ctx, CUtensorMap* map, const void* x, int M, int K, int box_rows, bool q8, int blocks = 1) {
  const cuuint32_t step = q8 ? 128 : 64;
  const cuuint64_t dims[3] = {step, (cuuint64_t)M, (cuuint64_t)K / step}, strides[2] = {(cuuint64_t)K * (q8 ? 1 : 2), 128};
  const cuuint32_t box[3] = {step, (cuuint32_t)box_rows, (cuuint32_t)blocks};
  return encode(ctx, map, q8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, x, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}
int32_t map_weights(precc_ctx* ctx, CUtensorMap* map, const void* w, int N, int K, int box_rows, bool q8) {
  const cuuint32_t step = q8 ? 128 : 64;
  const cuuint64_t dims[3] = {step, (cuuint64_t)N, (cuuint64_t)K / step}, strides[2] = {128, (cuuint64_t)N * 128};
  const cuuint32_t box[3] = {step, (cuuint32_t)box_rows, 1};
  return encode(ctx, map, q8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, w, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}
// B [agents][rank][N]: 64 columns x rank_pad coordinates of one agent (coordinates past the rank arrive as zeros).
int32_t map_expand(precc_ctx* ctx, CUtensorMap* map, const AdaptedParams& p) {
  const cuuint64_t dims[3] = {(cuuint64_t)p.N, (cuuint64_t)p.rank, (cuuint64_t)p.n_agents}, strides[2] = {(cuuint64_t)p.N * 2, (cuuint64_t)p.N * 2 * p.rank};
  const cuuint32_t box[3] = {64, (cuuint32_t)p.rank_pad, 1};
  return encode(ctx, map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, p.B, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

// ------------------------------------------------------------------------------------------ launches
struct Launch {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  Launch(dim3 grid, int threads, int smem, int cluster, cudaStream_t stream) {
    cfg.gridDim = grid; cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem; cfg.stream = stream;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = cluster > 1 ? 2 : 1;
  }
};

template <int MT, int NT, bool Q8>
int32_t launch_shrink(precc_ctx* ctx, AdaptedParams p, cudaStream_t stream) {
  const ShrinkPlan plan = plan_shrink(p.M, p.K, 8 * NT, ctx->sm_count);
  p.tile_rows = plan.rows;
  Launch l(dim3((unsigned)((p.M + plan.rows - 1LL) / plan.rows * plan.ks)), SHRINK_THREADS, 0, plan.ks, stream);
  PRECC_CUDA(ctx, cudaLaunchKernelEx(&l.cfg, adapted_shrink_kernel<MT, NT, Q8>, p));
  return PRECC_OK;
}

template <bool Q8>
int32_t launch_shrink_tc(precc_ctx* ctx, AdaptedParams p, cudaStream_t stream) {
  const ShrinkTcPlan plan = plan_shrink_tc(p.M, p.K / (Q8 ? 128 : 64), p.rank, p.n_agents, Q8, ctx->sm_count, ctx->max_smem_optin);
  p.BN = plan.tn; p.kps = plan.kps; p.tmem_cols = plan.tmem_cols;
  CUtensorMap map_x, map_a;
  int32_t rc = map_rows(ctx, &map_x, p.x, p.M, p.K, p.BN, Q8, p.kps);
  if (!rc) rc = map_weights(ctx, &map_a, p.A, p.n_agents * p.rank * (Q8 ? 2 : 1), p.K, p.rank, Q8);
  if (rc) return rc;
  PRECC_CUDA(ctx, raise_smem_limit(ctx, adapted_shrink_tc_kernel<Q8>, plan.smem));
  Launch l(dim3((unsigned)((p.M + (long long)p.BN - 1) / p.BN * plan.ks)), AS_THREADS, plan.smem, plan.ks, stream);
  PRECC_CUDA(ctx, cudaLaunchKernelEx(&l.cfg, adapted_shrink_tc_kernel<Q8>, map_x, map_a, p, plan.ring));
  return PRECC_OK;
}

template <bool Q8>
int32_t run_shrink(precc_ctx* ctx, const AdaptedParams& p, bool tc, cudaStream_t stream) {
  if (tc) return launch_shrink_tc<Q8>(ctx, p, stream);
  const bool few = p.M <= 64;
  switch (p.rank_pad) {
    case 16: return few ? launch_shrink<1, 1, Q8>(ctx, p, stream) : launch_shrink<1, 4, Q8>(ctx, p, stream);
    case 32: return few ? launch_shrink<2, 1, Q8>(ctx, p, stream) : launch_shrink<2, 4, Q8>(ctx, p, stream);
    default: return few ? launch_shrink<4, 1, Q8>(ctx, p, stream) : launch_shrink<4, 2, Q8>(ctx, p, stream);
  }
}

template <bool Q8>
int32_t run_pair(precc_ctx* ctx, AdaptedParams p, const void* W, const AdaptedPlan& plan, cudaStream_t stream) {
  p.BN = plan.bn; p.stages = plan.stages;
  p.tmem_cols = 32;
  while (p.tmem_cols < 2 * p.BN) p.tmem_cols <<= 1;
  CUtensorMap map_x, map_w, map_t, map_b;
  int32_t rc = map_rows(ctx, &map_x, p.x, p.M, p.K, GEMM_BM, Q8);
  if (!rc) rc = map_weights(ctx, &map_w, W, p.N, p.K, p.BN / 2, Q8);
  if (p.agent_id) {
    if (!rc) rc = make_map2(ctx, &map_t, p.T, p.M, p.rank_pad, GEMM_BM, p.rank_pad);
    if (!rc) rc = map_expand(ctx, &map_b, p);
  } else {
    map_t = map_b = map_x;
  }
  if (rc) return rc;
  const long long tiles = (p.M + AP_BM - 1LL) / AP_BM * ((p.N + p.BN - 1) / p.BN);
  const int smem = ap_smem_bytes(p.BN, p.stages);
  PRECC_CUDA(ctx, raise_smem_limit(ctx, adapted_pair_kernel<Q8>, smem));
  Launch l(dim3((unsigned)(2 * std::min<long long>(tiles, ctx->sm_count / 2))), AP_THREADS, smem, 2, stream);
  PRECC_CUDA(ctx, cudaLaunchKernelEx(&l.cfg, adapted_pair_kernel<Q8>, map_x, map_w, map_t, map_b, p));
  return PRECC_OK;
}

template <int NT, bool Q8>
int32_t launch_few(precc_ctx* ctx, const AdaptedParams& p, const void* W, cudaStream_t stream) {
  const int smem = af_smem_bytes(NT, p.agent_id ? p.rank_pad : 0);
  PRECC_CUDA(ctx, raise_smem_limit(ctx, adapted_few_kernel<NT, Q8>, smem));
  Launch l(dim3((unsigned)((p.N + AF_COLS - 1) / AF_COLS)), AF_THREADS, smem, 1, stream);
  PRECC_CUDA(ctx, cudaLaunchKernelEx(&l.cfg, adapted_few_kernel<NT, Q8>, p, (const uint8_t*)W));
  return PRECC_OK;
}
template <bool Q8>
int32_t run_few(precc_ctx* ctx, const AdaptedParams& p, const void* W, cudaStream_t stream) {
  return p.M <= 8 ? launch_few<1, Q8>(ctx, p, W, stream) : p.M <= 16 ? launch_few<2, Q8>(ctx, p, W, stream) : launch_few<4, Q8>(ctx, p, W, stream);
}

template <bool Q8>
int32_t run_turn(precc_ctx* ctx, AdaptedParams p, const void* W, const AdaptedPlan& plan, cudaStream_t stream) {
  p.BN = plan.tn; p.stages = plan.stages;
  p.tmem_cols = 32;
  while (p.tmem_cols < p.BN) p.tmem_cols <<= 1;
  const int smem = std::max(PT_MIN_SMEM, at_smem_bytes(p.BN, plan.ks, p.stages));
  CUtensorMap map_x, map_w;
  int32_t rc = map_rows(ctx, &map_x, p.x, p.M, p.K, p.BN, Q8);
  if (!rc) rc = map_weights(ctx, &map_w, W, p.N, p.K, PT_COLS, Q8);
  if (rc) return rc;
  PRECC_CUDA(ctx, raise_smem_limit(ctx, adapted_turn_kernel<Q8>, smem));
  Launch l(dim3((unsigned)plan.ks, (unsigned)((p.N + PT_COLS - 1) / PT_COLS), (unsigned)((p.M + p.BN - 1) / p.BN)), AT_THREADS, smem, plan.ks, stream);
  PRECC_CUDA(ctx, cudaLaunchKernelEx(&l.cfg, adapted_turn_kernel<Q8>, map_x, map_w, p));
  return PRECC_OK;
}

int32_t check_projection(precc_ctx* ctx, const precc_projection* d, int step) {
  if (!ctx) return PRECC_ERR_INVALID_ARG;
  if (!d) return fail(ctx, PRECC_ERR_INVALID_ARG, "projection descriptor is null");
  if (d->k_dim <= 0 || d->n_out <= 0 || d->n_agents < 0 || d->rank < 0) return fail(ctx, PRECC_ERR_INVALID_ARG, "non-positive size in projection descriptor");
  if (d->k_dim % step || d->n_out % 8) return fail(ctx, PRECC_ERR_UNSUPPORTED, "k_dim %d not a multiple of %d or n_out %d not of 8", d->k_dim, step, d->n_out);
  if (d->k_dim > 1 << 20 || d->n_out > 1 << 20) return fail(ctx, PRECC_ERR_UNSUPPORTED, "k_dim or n_out above 2^20");
  if (d->rank > 0 && !rank_ok(d->rank)) return fail(ctx, PRECC_ERR_UNSUPPORTED, "rank %d not in {0,8,16,32,64}", d->rank);
  if (d->rank > 0 && (d->n_agents < 1 || d->n_agents > AP_MAX_AGENTS)) return fail(ctx, PRECC_ERR_UNSUPPORTED, "n_agents %d outside [1,%d]", d->n_agents, AP_MAX_AGENTS);
  return PRECC_OK;
}

template <bool Q8>
int32_t project(precc_ctx* ctx, const precc_projection* d, const void* X, const float* x_scale, int32_t M, const void* W, const float* w_scale,
                const void* A, const float* a_scale, const void* B, const int32_t* agent_id, void* Y, void* ws, size_t ws_bytes, void* stream) {
  int32_t rc = check_projection(ctx, d, Q8 ? 128 : 64);
  if (rc) return rc;
  if (M < 0) return fail(ctx, PRECC_ERR_INVALID_ARG, "M < 0");
  if (M > 1 << 26) return fail(ctx, PRECC_ERR_UNSUPPORTED, "M above 2^26");
  if (M == 0) return PRECC_OK;
  if (!X || !W || !Y || (Q8 && (!x_scale || !w_scale))) return fail(ctx, PRECC_ERR_INVALID_ARG, "X / W / Y or a scale is null");
  const bool adapters = agent_id && d->rank > 0;
  if (adapters && (!A || !B || (Q8 && !a_scale))) return fail(ctx, PRECC_ERR_INVALID_ARG, "A, its scales or B is null");
  if (!aligned16(X) || !aligned16(W) || !aligned16(Y) || !aligned16(A) || !aligned16(B) || !aligned16(w_scale) || (reinterpret_cast<uintptr_t>(x_scale) & 3u) ||
      (reinterpret_cast<uintptr_t>(a_scale) & 3u) || (reinterpret_cast<uintptr_t>(agent_id) & 3u))
    return fail(ctx, PRECC_ERR_MISALIGNED, "X / W / Y / A / B / w_scale not 16-byte aligned (x_scale, a_scale, agent_id: 4)");
  AdaptedParams p = {};
  p.M = M; p.N = d->n_out; p.K = d->k_dim; p.rank = d->rank; p.rank_pad = std::max(16, d->rank); p.rank_shift = d->rank ? __builtin_ctz(d->rank) : 0; p.n_agents = d->n_agents;
  p.x = X; p.x_scale = x_scale; p.w_scale = w_scale; p.y = (__nv_bfloat16*)Y; p.s = d->lora_scale; p.status = ctx->status;
  if (adapters) {
    const size_t need = precc_adapted_ws_bytes(d, M);
    if (!ws || ws_bytes < need) return fail(ctx, PRECC_ERR_WORKSPACE, "workspace: need %zu bytes, got %zu", need, ws ? ws_bytes : (size_t)0);
    if (reinterpret_cast<uintptr_t>(ws) & 127u) return fail(ctx, PRECC_ERR_MISALIGNED, "workspace not 128-byte aligned");
    p.agent_id = agent_id; p.A = A; p.a_scale = a_scale; p.B = (const __nv_bfloat16*)B; p.T = (__nv_bfloat16*)ws;
  }
  rc = check_device(ctx);
  if (rc) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  const AdaptedPlan plan = plan_adapted(M, p.N, p.K, adapters ? p.rank : 0, Q8, ctx->sm_count, ctx->max_smem_optin, turn_clusters(ctx), ctx->adapted_kernel,
                                        ctx->adapted_shrink);
  if (adapters) {
    rc = run_shrink<Q8>(ctx, p, plan.shrink_tc, st);
    if (rc) return rc;
  }
  switch (plan.kernel) {
    case ADAPTED_FEW: return run_few<Q8>(ctx, p, W, st);
    case ADAPTED_TURN: return run_turn<Q8>(ctx, p, W, plan, st);
    default: return run_pair<Q8>(ctx, p, W, plan, st);
  }
}

}  // namespace

extern "C" {

int32_t precc_pack_kmajor_e4m3(precc_ctx* ctx, const void* src, int32_t k_dim, int32_t n_cols, void* dst, float* scale, void* stream) {
  if (!ctx) return PRECC_ERR_INVALID_ARG;
  if (!src || !dst || !scale || k_dim <= 0 || n_cols <= 0) return fail(ctx, PRECC_ERR_INVALID_ARG, "pack_kmajor_e4m3: bad arguments");
  if (k_dim % 128) return fail(ctx, PRECC_ERR_UNSUPPORTED, "pack_kmajor_e4m3: k_dim %% 128 != 0");
  if ((reinterpret_cast<uintptr_t>(src) & 1u) || !aligned16(dst) || (reinterpret_cast<uintptr_t>(scale) & 3u))
    return fail(ctx, PRECC_ERR_MISALIGNED, "pack_kmajor_e4m3: dst not 16-byte aligned (src: 2, scale: 4)");
  const int32_t rc = check_device(ctx);
  if (rc) return rc;
  pack_kmajor_e4m3_kernel<<<(n_cols + PACK8_COLS - 1) / PACK8_COLS, PACK8_COLS * PACK8_ROWS, 0, (cudaStream_t)stream>>>(
      (const __nv_bfloat16*)src, k_dim, n_cols, (uint8_t*)dst, scale);
  PRECC_CUDA(ctx, cudaGetLastError());
  return PRECC_OK;
}

int32_t precc_pack_adapter_e4m3(precc_ctx* ctx, const void* A, int32_t k_dim, int32_t rank, int32_t agent, int32_t n_agents, void* dst, float* scale,
                                void* stream) {
  if (!ctx) return PRECC_ERR_INVALID_ARG;
  if (!A || !dst || !scale || k_dim <= 0 || agent < 0 || agent >= n_agents) return fail(ctx, PRECC_ERR_INVALID_ARG, "pack_adapter_e4m3: bad arguments");
  if (k_dim % 128 || !rank_ok(rank) || n_agents > AP_MAX_AGENTS) return fail(ctx, PRECC_ERR_UNSUPPORTED, "pack_adapter_e4m3: k_dim, rank or n_agents outside the supported set");
  if ((reinterpret_cast<uintptr_t>(A) & 1u) || !aligned16(dst) || (reinterpret_cast<uintptr_t>(scale) & 3u))
    return fail(ctx, PRECC_ERR_MISALIGNED, "pack_adapter_e4m3: dst not 16-byte aligned (A: 2, scale: 4)");
  const int32_t rc = check_device(ctx);
  if (rc) return rc;
  pack_adapter_e4m3_kernel<<<rank, 256, 0, (cudaStream_t)stream>>>((const __nv_bfloat16*)A, k_dim, rank, agent, n_agents * rank, (uint8_t*)dst, scale);
  PRECC_CUDA(ctx, cudaGetLastError());
  return PRECC_OK;
}

int32_t precc_pack_expand_e4m3(precc_ctx* ctx, const void* B, int32_t rows, int32_t n_cols, const float* w_scale, void* dst, void* stream) {
  if (!ctx) return PRECC_ERR_INVALID_ARG;
  if (!B || !dst || !w_scale || rows <= 0 || n_cols <= 0) return fail(ctx, PRECC_ERR_INVALID_ARG, "pack_expand_e4m3: bad arguments");
  if (((reinterpret_cast<uintptr_t>(B) | reinterpret_cast<uintptr_t>(dst)) & 1u) || (reinterpret_cast<uintptr_t>(w_scale) & 3u))
    return fail(ctx, PRECC_ERR_MISALIGNED, "pack_expand_e4m3: misaligned pointer");
  const int32_t rc = check_device(ctx);
  if (rc) return rc;
  const long long n = (long long)rows * n_cols;
  pack_expand_e4m3_kernel<<<(unsigned)std::min<long long>((n + 255) / 256, 8LL * ctx->sm_count), 256, 0, (cudaStream_t)stream>>>(
      (const __nv_bfloat16*)B, n, n_cols, w_scale, (__nv_bfloat16*)dst);
  PRECC_CUDA(ctx, cudaGetLastError());
  return PRECC_OK;
}

size_t precc_adapted_ws_bytes(const precc_projection* proj, int32_t M) {
  if (!proj || M <= 0 || proj->rank <= 0) return 0;
  return ((size_t)M * std::max(16, proj->rank) * 2 + 255) / 256 * 256;
}

int32_t precc_adapted_project(precc_ctx* ctx, const precc_projection* proj, const void* X, int32_t M, const void* W_packed, const void* A_packed,
                              const void* B, const int32_t* agent_id, void* Y, void* ws, size_t ws_bytes, void* stream) {
  return project<false>(ctx, proj, X, nullptr, M, W_packed, nullptr, A_packed, nullptr, B, agent_id, Y, ws, ws_bytes, stream);
}

int32_t precc_adapted_project_e4m3(precc_ctx* ctx, const precc_projection* proj, const void* X, const float* x_scale, int32_t M,
                                   const void* W_packed, const float* w_scale, const void* A_packed, const float* a_scale, const void* B_packed,
                                   const int32_t* agent_id, void* Y, void* ws, size_t ws_bytes, void* stream) {
  return project<true>(ctx, proj, X, x_scale, M, W_packed, w_scale, A_packed, a_scale, B_packed, agent_id, Y, ws, ws_bytes, stream);
}

}  // extern "C"
