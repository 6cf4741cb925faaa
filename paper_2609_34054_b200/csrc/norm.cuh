// Root-mean-square norm of hidden states with the residual's addition, bf16 and / or 8-bit output:
//   s = x + residual,  residual_out = bf16(s),  y = s / sqrt(mean(s^2) + eps) * gain
//   bf16 output: bf16(y);  8-bit output: scale = max |y| / 448 of the row (1 for a row of zeros), q = e4m3(y / scale)
//
// HBM-bound: a row is read once, kept in registers as fp32 from the addition to the last rounding (the norm is of the unrounded
// sum; every output is rounded once, the 8-bit one behind a product with 1 / scale), and written once.  A thread holds C pieces of eight columns, piece i of the row
// at thread i % T, so that a warp's loads are 512 consecutive bytes.  Measured in graphs of calls over rotating inputs: 32768 x 4096 with residual and 8-bit output
// 136.5 .. 139.8 us, 6.7 .. 6.9 TB/s of what is read and written, the rate of a plain copy; without the residual 83.9 (4.8 TB/s: one block a row, and half the
// bytes in flight), with both outputs 104 (6.4 TB/s); both outputs of 1337 x 3584 with residual 8.5 us (6.2 from L2).  One row of 2048: 1.4 .. 1.6 us a call.
#pragma once
#include "common.cuh"

namespace precc {

constexpr int NORM_MAX_WIDTH = 32768;
constexpr int NORM_SHORT_THREADS = 128;      // block of rows that fit a warp or a part of one
constexpr float E4M3_MAX = 448.f;

struct NormParams {
  const __nv_bfloat16* x;
  const __nv_bfloat16* residual;             // RES
  const __nv_bfloat16* gain;
  __nv_bfloat16* residual_out;               // or null
  __nv_bfloat16* out;                        // or null
  uint8_t* q;                                // or null
  float* q_scale;
  int rows, pieces;                          // pieces of eight columns in a row
  int T;                                     // threads of a row
  float inv_width, eps;
};

// Sums, products and magnitudes that keep subnormal numbers, bf16's own among them (the library is built with flushing ones).
__device__ __forceinline__ float add_full(float a, float b) {
  float r;
  asm("add.rn.f32 %0, %1, %2;\n" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float mul_full(float a, float b) {
  float r;
  asm("mul.rn.f32 %0, %1, %2;\n" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float fma_full(float a, float b, float c) {
  float r;
  asm("fma.rn.f32 %0, %1, %2, %3;\n" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float abs_full(float a) {
  float r;
  asm("abs.f32 %0, %1;\n" : "=f"(r) : "f"(a));
  return r;
}
// max that lets a NaN through (fmaxf drops it): a row with a NaN gets a NaN scale, not a plausible one
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;\n" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint32_t pack_e4m3x4(float a, float b, float c, float d) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(hi) : "f"(d), "f"(c));
  return static_cast<uint32_t>(lo) | (static_cast<uint32_t>(hi) << 16);
}
__device__ __forceinline__ void unpack_bf16x8(const uint4& v, float (&f)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ uint4 pack_bf16x8(const float (&f)[8]) {
  return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
}

// C pieces per thread.  SHORT: several rows of T <= 32 threads (a power of two) in a block of NORM_SHORT_THREADS; else one row
// of blockDim.x = T threads.  RES: with a residual.
template <int C, bool SHORT, bool RES>
__global__ void __launch_bounds__(SHORT ? NORM_SHORT_THREADS : 1024)
rms_norm_kernel(const NormParams p) {
  __shared__ float part[3][32];
  const int t = SHORT ? threadIdx.x % p.T : threadIdx.x;
  const long long row = SHORT ? (long long)blockIdx.x * (NORM_SHORT_THREADS / p.T) + threadIdx.x / p.T : blockIdx.x;
  const bool live = !SHORT || row < p.rows;
  // over the threads of a row; every thread gets the result
  auto reduce = [&](float v, int slot, auto op) {
    for (int m = (SHORT ? p.T : 32) / 2; m > 0; m >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, m));
    if constexpr (!SHORT) {
      const int warps = p.T / 32;
      if ((threadIdx.x & 31) == 0) part[slot][threadIdx.x / 32] = v;
      __syncthreads();
      v = part[slot][0];
      for (int w = 1; w < warps; ++w) v = op(v, part[slot][w]);
    }
    return v;
  };
  pdl_wait();
  pdl_launch_dependents();
  const long long at = row * p.pieces;       // in pieces of eight columns
  // s[c][k]: x, or with a residual half of the sum, as the whole one may pass fp32's largest number (a power of two changes no rounding, and bf16's
  // least subnormal has a half in fp32).  The norm is the same with eps in these units, a quarter of it.
  float s[C][8];
  float sum = 0.f;
  uint4 xv[C], rv[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int i = t + c * p.T;
    xv[c] = rv[c] = make_uint4(0, 0, 0, 0);
    if (live && i < p.pieces) {
      xv[c] = reinterpret_cast<const uint4*>(p.x)[at + i];
      if (RES) rv[c] = reinterpret_cast<const uint4*>(p.residual)[at + i];
    }
  }
#pragma unroll
  for (int c = 0; c < C; ++c) {
    float r[8];
    unpack_bf16x8(xv[c], s[c]);
    unpack_bf16x8(rv[c], r);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      s[c][k] = RES ? fma_full(s[c][k], 0.5f, mul_full(r[k], 0.5f)) : add_full(s[c][k], 0.f);       // (-0 is 0)
      sum = fmaf(s[c][k], s[c][k], sum);
    }
  }
  if (p.residual_out) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int i = t + c * p.T;
      if (live && i < p.pieces) {
        float whole[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) whole[k] = RES ? add_full(s[c][k], s[c][k]) : s[c][k];
        reinterpret_cast<uint4*>(p.residual_out)[at + i] = pack_bf16x8(whole);
      }
    }
  }
  sum = reduce(sum, 0, [](float a, float b) { return a + b; });
  float mean = fmaf(sum, p.inv_width, RES ? 0.25f * p.eps : p.eps);
  // Squares past fp32's range (values above 2^56, such as a type's lowest one): the row, and eps with it, in units of 2^72, which leaves 32768 squares of the
  // largest values in range.  Squares that vanish (below 2^-126, so at most 2^-126 of the mean) where neither the others nor eps outweigh
  // them: in units of 2^-100, where the least subnormal's does not vanish and a mean of 2^-100 is in range.  y is the same.  (Rows that share a
  // warp go through it together, each with its own unit.)
  const bool over = isinf(sum), under = mean < 0x1p-100f;
  if (SHORT ? __any_sync(0xffffffffu, over || under) : over || under) {
    const float unit = over ? 0x1p-72f : under ? 0x1p100f : 1.f;
    sum = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int k = 0; k < 8; ++k) { s[c][k] = mul_full(s[c][k], unit); sum = fmaf(s[c][k], s[c][k], sum); }
    sum = reduce(sum, 2, [](float a, float b) { return a + b; });
    mean = fmaf(sum, p.inv_width, mul_full(mul_full(p.eps, unit), RES ? 0.25f * unit : unit));
  }
  const float inv = 1.0f / sqrtf(mean);
  float top = 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int i = t + c * p.T;
    if (live && i < p.pieces) {
      float g[8];
      unpack_bf16x8(__ldg(reinterpret_cast<const uint4*>(p.gain) + i), g);
#pragma unroll
      for (int k = 0; k < 8; ++k) { s[c][k] = mul_full(mul_full(s[c][k], inv), g[k]); top = max_nan(top, abs_full(s[c][k])); }
      if (p.out) reinterpret_cast<uint4*>(p.out)[at + i] = pack_bf16x8(s[c]);
    }
  }
  if (!p.q) return;
  top = reduce(top, 1, [](float a, float b) { return max_nan(a, b); });
  const float scale = __float_as_uint(top) == 0u ? 1.f : max_nan(top * (1.f / E4M3_MAX), 1.17549435e-38f);     // (a normal number, and so is its reciprocal)
  const float to_q = 1.0f / scale;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int i = t + c * p.T;
    if (live && i < p.pieces) {
#pragma unroll
      for (int k = 0; k < 8; ++k) s[c][k] = mul_full(s[c][k], to_q);
      reinterpret_cast<uint2*>(p.q)[at + i] = make_uint2(pack_e4m3x4(s[c][0], s[c][1], s[c][2], s[c][3]), pack_e4m3x4(s[c][4], s[c][5], s[c][6], s[c][7]));
    }
  }
  if (live && t == 0) p.q_scale[row] = scale;
}

}  // namespace precc
