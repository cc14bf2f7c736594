// Scales and values of the block-scaled float8 (e4m3) format of xshare_ops.h.
#pragma once

#include <cuda_fp8.h>

#include "f8_ptx.cuh"
#include "ops_internal.cuh"

namespace xs {

__device__ __forceinline__ float f8_scale(float amax) { return __fdiv_rn(fmaxf(amax, kTinyAmax), kE4m3Max); }

// x / s for many x of one block, correctly rounded, so that a value on the border
// between two e4m3 numbers falls on the side that the definition gives.  Markstein:
// with r the rounded reciprocal, one step of q += r (x - q s) makes q = x r faithful,
// a second one correct (both residuals are exact fused operations).  Five multiply-adds for
// two values (packed pairs) instead of a division each; scales near the ends of the
// exponent range, where a residual could underflow, take the division.  All of it with -x and -r: the
// residual of a zero is +0, and -0 + r 0 would be +0, where -0 - r 0 stays -0.
struct F8Divider {
  float s0, s1;        // of the first and the second of two values
  uint64_t nr2, s2;
  bool plain;
  // r0, r1: 1 / s0, 1 / s1, rounded.
  __device__ __forceinline__ F8Divider(float a, float b, float r0, float r1)
      : s0(a), s1(b), nr2(ptx::pack2(-r0, -r1)), s2(ptx::pack2(a, b)),
        plain(!(fminf(a, b) > 0x1p-60f && fmaxf(a, b) < 0x1p60f)) {}
  __device__ __forceinline__ F8Divider(float s, float r) : F8Divider(s, s, r, r) {}
  __device__ __forceinline__ explicit F8Divider(float s) : F8Divider(s, 1.f / s) {}
  // Two quotients; not for `plain`.
  __device__ __forceinline__ float2 operator()(float a, float b) const {
    const uint64_t nx = ptx::pack2(-a, -b);
    uint64_t q = ptx::mul2(nx, nr2);
    q = ptx::fma2(ptx::fma2(q, s2, nx), nr2, q);
    return ptx::unpack2(ptx::fma2(ptx::fma2(q, s2, nx), nr2, q));
  }
  __device__ __forceinline__ float2 slow(float a, float b) const {
    return make_float2(__fdiv_rn(a, s0), __fdiv_rn(b, s1));
  }
};

// silu(g) = g / (1 + e^-g) for activations that are rounded to e4m3 next: the
// exponential and the reciprocal of the special function unit, relative error below
// 2^-20 + |g| 2^-24 (the product g log2 e is rounded once); e^-g = infinity gives 0.
__device__ __forceinline__ float f8_silu(float g) {
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(g * -1.44269504f));
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
  return g * r;
}

// Two values as e4m3 bytes, the first in the lower one.
__device__ __forceinline__ uint32_t f8_pack2(float2 v) {
  return __nv_cvt_float2_to_fp8x2(v, __NV_SATFINITE, __NV_E4M3);
}

// kN (a multiple of four) values divided by the scale, as e4m3 bytes.
template <int kN>
__device__ __forceinline__ void f8_quantise(const float (&v)[kN], const F8Divider &div, uint32_t (&w)[kN / 4]) {
  if (div.plain) {
#pragma unroll
    for (int j = 0; j < kN / 4; ++j)
      w[j] = f8_pack2(div.slow(v[4 * j], v[4 * j + 1])) | f8_pack2(div.slow(v[4 * j + 2], v[4 * j + 3])) << 16;
  } else {
#pragma unroll
    for (int j = 0; j < kN / 4; ++j)
      w[j] = f8_pack2(div(v[4 * j], v[4 * j + 1])) | f8_pack2(div(v[4 * j + 2], v[4 * j + 3])) << 16;
  }
}

}  // namespace xs
