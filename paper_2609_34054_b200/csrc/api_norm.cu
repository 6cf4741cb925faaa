// libprecc: the norm of hidden states ahead of the projections.
#include "api_internal.h"
#include "norm.cuh"

using namespace precc;

namespace {

// Pieces of eight columns per thread (c), threads of a row, and whether several rows share a block.
// One row or a few: a piece a thread, for latency (1 x 4096: 1.7 us, 1.9 with two, 2.3 with four).  Many rows: what a thread has asked for at once has to cover the
// latency of memory, 64 bytes - two pieces with their residual, or four without.  32768 x 4096, 8-bit output, us with one / two / four pieces: with the
// residual 189 / 139 / 139, without 157 / 93 / 82 (16384 x 8192: 230 / 141 / 139 and 198 / 104 / 88; both outputs of
// 1337 x 3584 with it 10.4 / 8.8 / 9.7, without 8.9 / 6.6 / 7.7; eight pieces are slower everywhere).  Many short rows: a warp each, as blocks of one or two
// warps are bound by how fast blocks start (30000 x 512: 32 us in blocks of 64 threads, 12 with a warp a row).
struct NormPlan { int c, threads; bool shared_block; };
NormPlan plan_norm(int rows, int pieces, bool residual) {
  auto whole_warps = [&](int c) { return ((pieces + c - 1) / c + 31) / 32 * 32; };
  if (pieces <= 32) {
    int t = 1;
    while (t < pieces) t *= 2;
    return {1, t, true};
  }
  if (rows > 1024 && pieces <= 128) return {pieces <= 64 ? 2 : 4, 32, true};
  int c = rows <= 148 ? 1 : (residual ? pieces <= 512 : rows <= 4096) ? 2 : 4;
  if (whole_warps(c) > 1024) c = 4;
  return {c, whole_warps(c), false};
}

// Whether a_bytes from a on and b_bytes from b on share any.
inline bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return b && x < y + b_bytes && y < x + a_bytes;
}
// A thread reads its pieces of x and residual before it writes the same pieces of bf16, so those outputs may be x or residual as a whole.  Bytes of 8 bits lie
// on other rows' values, which their blocks may not have read, and two outputs on one place have no order.  (A decode step's call has two outputs: what
// is not given costs nothing here.)
bool outputs_apart(const void* x, const void* residual, const void* gain, size_t rows, size_t width, const void* residual_out, const void* out, const void* q,
                   const void* scale) {
  const size_t n = rows * width;
  auto meets_input = [&](const void* o, size_t bytes, bool may_be) {
    return (overlap(o, bytes, x, 2 * n) && !(may_be && o == x)) || (overlap(o, bytes, residual, 2 * n) && !(may_be && o == residual)) || overlap(o, bytes, gain, 2 * width);
  };
  if (residual_out && meets_input(residual_out, 2 * n, true)) return false;
  if (out && (meets_input(out, 2 * n, true) || overlap(out, 2 * n, residual_out, 2 * n))) return false;
  if (!q) return true;
  return !meets_input(q, n, false) && !meets_input(scale, 4 * rows, false) && !overlap(q, n, residual_out, 2 * n) && !overlap(q, n, out, 2 * n) && !overlap(q, n, scale, 4 * rows) &&
         !overlap(scale, 4 * rows, residual_out, 2 * n) && !overlap(scale, 4 * rows, out, 2 * n);
}

template <int C, bool SHORT>
int32_t norm_launch(precc_ctx* ctx, const NormParams& p, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  const int rows_per_block = SHORT ? NORM_SHORT_THREADS / p.T : 1;
  cfg.gridDim = dim3((unsigned)((p.rows + rows_per_block - 1LL) / rows_per_block));
  cfg.blockDim = dim3(SHORT ? NORM_SHORT_THREADS : p.T);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  PRECC_CUDA(ctx, p.residual ? cudaLaunchKernelEx(&cfg, rms_norm_kernel<C, SHORT, true>, p) : cudaLaunchKernelEx(&cfg, rms_norm_kernel<C, SHORT, false>, p));
  return PRECC_OK;
}

}  // namespace

extern "C" int32_t precc_rms_norm(precc_ctx* ctx, const void* x, const void* residual, const void* gain, int32_t rows,
                                  int32_t width, float eps, void* residual_out, void* out, void* out_e4m3, float* out_scale,
                                  void* stream) {
  if (!ctx) return PRECC_ERR_INVALID_ARG;
  if (rows < 0 || width <= 0) return fail(ctx, PRECC_ERR_INVALID_ARG, "rows < 0 or width <= 0");
  if (width % 8 || width > NORM_MAX_WIDTH) return fail(ctx, PRECC_ERR_UNSUPPORTED, "width %d not a multiple of 8 up to %d", width, NORM_MAX_WIDTH);
  if (!(eps >= 0.f)) return fail(ctx, PRECC_ERR_INVALID_ARG, "eps is negative or NaN");
  if (rows == 0) return PRECC_OK;
  if (!x || !gain) return fail(ctx, PRECC_ERR_INVALID_ARG, "x / gain is null");
  if (!out && !out_e4m3) return fail(ctx, PRECC_ERR_INVALID_ARG, "neither a bf16 nor an 8-bit output is given");
  if ((out_e4m3 != nullptr) != (out_scale != nullptr)) return fail(ctx, PRECC_ERR_INVALID_ARG, "the 8-bit output and its scales come together");
  if (!aligned16(x) || !aligned16(residual) || !aligned16(gain) || !aligned16(residual_out) || !aligned16(out) || !aligned16(out_e4m3) ||
      (reinterpret_cast<uintptr_t>(out_scale) & 3u))
    return fail(ctx, PRECC_ERR_MISALIGNED, "x / residual / gain / residual_out / out / out_e4m3 not 16-byte aligned (out_scale: 4)");
  if (!outputs_apart(x, residual, gain, rows, width, residual_out, out, out_e4m3, out_scale))
    return fail(ctx, PRECC_ERR_INVALID_ARG, "outputs overlap an input or one another (only residual_out and out may be x or residual themselves)");
  const int32_t rc = check_device(ctx);
  if (rc) return rc;
  NormParams p;
  p.x = (const __nv_bfloat16*)x; p.residual = (const __nv_bfloat16*)residual; p.gain = (const __nv_bfloat16*)gain;
  p.residual_out = (__nv_bfloat16*)residual_out; p.out = (__nv_bfloat16*)out; p.q = (uint8_t*)out_e4m3; p.q_scale = out_scale;
  p.rows = rows; p.pieces = width / 8; p.inv_width = 1.0f / width; p.eps = eps;
  cudaStream_t st = (cudaStream_t)stream;
  const NormPlan plan = plan_norm(rows, p.pieces, residual != nullptr);
  p.T = plan.threads;
  if (plan.shared_block) return plan.c == 1 ? norm_launch<1, true>(ctx, p, st) : plan.c == 2 ? norm_launch<2, true>(ctx, p, st) : norm_launch<4, true>(ctx, p, st);
  return plan.c == 1 ? norm_launch<1, false>(ctx, p, st) : plan.c == 2 ? norm_launch<2, false>(ctx, p, st) : norm_launch<4, false>(ctx, p, st);
}
