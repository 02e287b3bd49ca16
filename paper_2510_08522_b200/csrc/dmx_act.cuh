// dmx_act.cuh — the activations of the group norm and of the matrix product, and their slopes, in packed fp32.
//
// Exponentials and reciprocals are the approximate instructions (2 ulp). The normal distribution function is
// Hastings' approximation (Abramowitz and Stegun 7.1.26, |error| <= 1.5e-7 of erf): one reciprocal, five
// multiply-adds and the exponential, which the slope's density shares.
#pragma once
#include "dmx.h"
#include "dmx_f32x2.cuh"

namespace dmx_act {

using namespace dmx_f32x2;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float2 ex2_2(float2 x) { return make_float2(ex2(x.x), ex2(x.y)); }
__device__ __forceinline__ float2 rcp_2(float2 x) { return make_float2(rcp(x.x), rcp(x.y)); }

// 1 / (1 + exp(-u))
__device__ __forceinline__ float2 sigmoid(float2 u) { return rcp_2(add2(ex2_2(mul2(u, two(-1.4426950408889634f))), two(1.f))); }

// Phi(u), and e = exp(-u^2/2)
__device__ __forceinline__ float2 normal_cdf(float2 u, float2& e) {
  e = ex2_2(mul2(mul2(u, u), two(-0.72134752044448170f)));
  const float2 a = abs2(u);
  const float2 t = rcp_2(fma2(a, two(0.3275911f * 0.70710678118654752f), two(1.f)));
  float2 p = fma2(t, two(0.5f * 1.061405429f), two(0.5f * -1.453152027f));
  p = fma2(p, t, two(0.5f * 1.421413741f));
  p = fma2(p, t, two(0.5f * -0.284496736f));
  p = fma2(p, t, two(0.5f * 0.254829592f));
  p = mul2(mul2(p, t), e);                       // Phi(-|u|)
  const float2 q = sub2(two(1.f), p);
  return make_float2(u.x < 0.f ? p.x : q.x, u.y < 0.f ? p.y : q.y);
}

// max(u, 0) that keeps a NaN
__device__ __forceinline__ float relu(float u) {
  float y;
  asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(y) : "f"(u));
  return y;
}

template <int ACT>
__device__ __forceinline__ float2 apply(float2 u) {
  if constexpr (ACT == DMX_ACT_RELU) return make_float2(relu(u.x), relu(u.y));
  if constexpr (ACT == DMX_ACT_SILU) return mul2(u, sigmoid(u));
  if constexpr (ACT == DMX_ACT_GELU) {
    float2 e;
    return mul2(u, normal_cdf(u, e));
  }
  return u;
}

// g * act'(u)
template <int ACT>
__device__ __forceinline__ float2 times_slope(float2 g, float2 u) {
  if constexpr (ACT == DMX_ACT_RELU) return make_float2(u.x > 0.f ? g.x : 0.f, u.y > 0.f ? g.y : 0.f);
  if constexpr (ACT == DMX_ACT_SILU) {
    const float2 s = sigmoid(u);
    return mul2(g, fma2(mul2(u, s), sub2(two(1.f), s), s));
  }
  if constexpr (ACT == DMX_ACT_GELU) {
    float2 e;
    const float2 c = normal_cdf(u, e);
    return mul2(g, fma2(mul2(u, two(0.39894228040143268f)), e, c));
  }
  return g;
}

}  // namespace dmx_act
