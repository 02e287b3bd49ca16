// dmx_f32x2.cuh — the packed fp32 instructions of sm_100 on float2.
#pragma once

namespace dmx_f32x2 {

// Pairs of elements go through the packed fp32 instructions of sm_100 (each half IEEE fp32, round to nearest
// unless named otherwise): half the issue slots.
// A packed product that feeds a packed sum is contracted to one rounding even where both name theirs (seen in
// results); where two are wanted the sum is an fma with a factor of 1 that only the launch knows.
__device__ __forceinline__ unsigned long long bits2(float2 x) {
  unsigned long long r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x.x), "f"(x.y));
  return r;
}
__device__ __forceinline__ float2 float2_of(unsigned long long b) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(b));
  return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits2(a)), "l"(bits2(b)));
  return float2_of(r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  unsigned long long r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits2(a)), "l"(bits2(b)));
  return float2_of(r);
}
__device__ __forceinline__ float2 add2_down(float2 a, float2 b) {
  unsigned long long r;
  asm("add.rm.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits2(a)), "l"(bits2(b)));
  return float2_of(r);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(bits2(a)), "l"(bits2(b)), "l"(bits2(c)));
  return float2_of(r);
}
__device__ __forceinline__ float2 two(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 sub2(float2 a, float2 b) { return fma2(b, make_float2(-1.f, -1.f), a); }
__device__ __forceinline__ float2 neg2(float2 x) { return make_float2(-x.x, -x.y); }
__device__ __forceinline__ float2 abs2(float2 x) { return make_float2(fabsf(x.x), fabsf(x.y)); }
// two bf16 in a word
__device__ __forceinline__ float2 widen2(unsigned w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }

}  // namespace dmx_f32x2
