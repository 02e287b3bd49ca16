// dmx_act.cuh — the activations of the group norm and of the matrix product, and their slopes, in fp32.
#pragma once
#include "dmx.h"

namespace dmx_act {

__device__ __forceinline__ float sigmoid(float u) { return __fdividef(1.f, 1.f + __expf(-u)); }

// Distribution function and density of the standard normal.
__device__ __forceinline__ float phi_cdf(float u) { return 0.5f * (1.f + erff(u * 0.70710678118654752f)); }
__device__ __forceinline__ float phi_pdf(float u) { return 0.39894228040143268f * __expf(-0.5f * u * u); }

// max(u, 0) that keeps a NaN
__device__ __forceinline__ float relu(float u) { return u < 0.f ? 0.f : u; }

template <int V>
__device__ __forceinline__ void apply(float (&u)[V], int act) {
  if (act == DMX_ACT_RELU) {
#pragma unroll
    for (int v = 0; v < V; ++v) u[v] = relu(u[v]);
  } else if (act == DMX_ACT_SILU) {
#pragma unroll
    for (int v = 0; v < V; ++v) u[v] *= sigmoid(u[v]);
  } else if (act == DMX_ACT_GELU) {
#pragma unroll
    for (int v = 0; v < V; ++v) u[v] *= phi_cdf(u[v]);
  }
}

// g *= act'(u)
template <int V>
__device__ __forceinline__ void times_slope(float (&g)[V], const float (&u)[V], int act) {
  if (act == DMX_ACT_RELU) {
#pragma unroll
    for (int v = 0; v < V; ++v) g[v] = u[v] > 0.f ? g[v] : 0.f;
  } else if (act == DMX_ACT_SILU) {
#pragma unroll
    for (int v = 0; v < V; ++v) { const float s = sigmoid(u[v]); g[v] *= fmaf(u[v] * s, 1.f - s, s); }
  } else if (act == DMX_ACT_GELU) {
#pragma unroll
    for (int v = 0; v < V; ++v) g[v] *= fmaf(u[v], phi_pdf(u[v]), phi_cdf(u[v]));
  }
}

}  // namespace dmx_act
