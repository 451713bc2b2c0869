// Exponentials and sigmoids of pairs of fp32 values on the fast units (conv.cu, scan*.cu).
#pragma once
#include "lm_ops.h"

namespace lsgd {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float ex2(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float2 ex2(float2 v) { return make_float2(ex2(v.x), ex2(v.y)); }
__device__ __forceinline__ float2 add2(float2 a, float2 b) { return __fadd2_rn(a, b); }
// 1 / v of a v >= 1; zero beyond 2^126, where it would be subnormal
__device__ __forceinline__ float rcp(float v) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float2 rcp(float2 v) { return make_float2(rcp(v.x), rcp(v.y)); }
// sigmoid(v): zero where exp(-v) passes 2^126 (v below -87.3), infinities included.  (Held at 2^-126 there, v sigmoid(v) of -1e38 was -1.2.)
__device__ __forceinline__ float2 sigmoid(float2 v) { return rcp(add2(ex2(mul2(v, both(-kLog2e))), both(1.f))); }
__device__ __forceinline__ float sigmoid(float v) { return sigmoid(both(v)).x; }

}  // namespace lsgd
