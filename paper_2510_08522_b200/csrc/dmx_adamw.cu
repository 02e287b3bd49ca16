// dmx_adamw.cu — AdamW over many tensors in one launch, with the moments held in fp32 or in 8-bit
// block codes, and the global gradient norm that clips it.
//
// Per element, with s the optional device-side gradient factor (decoupled weight decay, Loshchilov &
// Hutter 2019, on the bias-corrected update of Kingma & Ba 2015):
//   g = s*grad        m' = b1 m + (1-b1) g        v' = b2 v + (1-b2) g^2
//   p' = p (1 - lr wd) - lr/(1-b1^t) * m' / (sqrt(v') / sqrt(1-b2^t) + eps)
// 8-bit moments: a block of 256 elements shares a scale per moment. First moment: m = S sgn(c) (c/127)^2,
// c in [-127,127], S = max|m| of the block. Second moment: sqrt(v) = R (c/255)^2, c in [0,255], R = max
// sqrt(v). The square law spends the codes where small values are (relative spacing 1.6 % at the top of
// m's range, 0.8 % of sqrt(v)'s, range 6e-5 of S and 1.5e-5 of R) and costs one square root to write and
// one multiplication to read. A nonzero v never gets code 0, so a denominator never vanishes by rounding.
// With a seed the codes are dithered (floor(x + u), u from a hash of the element's index and the seed):
// to nearest, a second moment that decays by 0.1 % a step would never leave its code.
// Everything between reading and writing the codes is fp32.
//
// Bound: HBM. A step moves 8 + grad + states (16, or 4 with 8-bit codes) + copy bytes per element. Measured on
// B200: 138 M parameters, all fp32: 566 us = 6.85 TB/s (measured copy rate 6.55); 340 M parameters, bf16
// gradients and copies, 8-bit moments: 938 us = 5.8 TB/s, where some 75 instructions per element (a third of them the
// dither) keep the issue slots nearly as busy as the memory (under the power limit, where the clock falls: 1056 us). A warp owns one block of 256 elements (its scales need a maximum over the block:
// one redux instruction), eight per lane as two groups of four neighbours, so every access of an aligned
// tensor is 16 bytes of fp32, 8 of bf16 or 4 of codes per lane and a warp's lines are full. A tensor whose
// start is not so aligned (a segment of a flat vector) takes its parameters and gradients element by element,
// 32 neighbours per access; the state is the library's own layout and stays aligned.
#include "dmx.h"

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <float.h>
#include <math.h>
#include <new>
#include <string.h>
#include <type_traits>
#include <vector>

#include "dmx_f32x2.cuh"
#include "dmx_host.h"

namespace {

using namespace dmx_f32x2;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
// A step's CTAs. With 8-bit moments a CTA is one warp with eight blocks, 32 CTAs per SM at 64 registers: the long
// arithmetic makes warps drift apart, and a CTA of several holds its slot until the last one is done (340 M
// parameters: 8 warps 1077 us, 4 warps 975 us, 2 warps 927 us, 1 warp 919-927 us). With fp32 moments there is
// little arithmetic, and eight warps that sweep 32 neighbouring blocks do better (138 M: 566 us against 590).
template <int BITS>
constexpr int kStepThreads = BITS == 8 ? 32 : 256;
template <int BITS>
constexpr int kStepCtas = BITS == 8 ? 32 : 3;
constexpr int kBlock = DMX_ADAMW_BLOCK;
static_assert(kBlock == 256, "a lane holds eight elements of a block");

struct Tensor {
  void* p;
  const void* g;          // null: the tensor has no gradient this step and is left alone
  __nv_bfloat16* copy;    // null: no bf16 copy is kept
  int64_t n;
  int64_t block0;         // first block of the tensor in the state arrays
  int decay;              // weight decay applies
  int vec;                // p, g and copy allow the grouped accesses
};

struct Chunk {            // consecutive blocks of one tensor
  int tensor;
  int nblocks;
  int64_t first;          // first block, counted within the tensor
};

struct StepArgs {
  const Tensor* tensors;
  const Chunk* chunks;
  void *m, *v;
  float *m_scale, *v_scale;
  const float* grad_scale;
  float b1, omb1, b2, omb2, eps, keep, rs_bc2, step, one;
  float quick_from;       // sum of a lane's second moments from which root2 serves
  unsigned key;
};

__device__ __forceinline__ float wide(float x) { return x; }
__device__ __forceinline__ float wide(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void narrow(float x, float* y) { *y = x; }
__device__ __forceinline__ void narrow(float x, __nv_bfloat16* y) { *y = __float2bfloat16_rn(x); }

__device__ __forceinline__ float bf_lo(unsigned x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float bf_hi(unsigned x) { return __uint_as_float(x & 0xffff0000u); }
__device__ __forceinline__ unsigned bf_pack(float a, float b) {
  __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<unsigned*>(&t);
}

// four neighbours, streamed (each byte of a step is used once)
__device__ __forceinline__ void load4(const float* p, float* x) {
  const float4 t = __ldcs(reinterpret_cast<const float4*>(p));
  x[0] = t.x; x[1] = t.y; x[2] = t.z; x[3] = t.w;
}
__device__ __forceinline__ void load4(const __nv_bfloat16* p, float* x) {
  const uint2 t = __ldcs(reinterpret_cast<const uint2*>(p));
  x[0] = bf_lo(t.x); x[1] = bf_hi(t.x); x[2] = bf_lo(t.y); x[3] = bf_hi(t.y);
}
__device__ __forceinline__ void store4(float* p, const float* x) {
  __stcs(reinterpret_cast<float4*>(p), make_float4(x[0], x[1], x[2], x[3]));
}
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float* x) {
  __stcs(reinterpret_cast<uint2*>(p), make_uint2(bf_pack(x[0], x[1]), bf_pack(x[2], x[3])));
}

// A lane's eight elements of a block: slot j holds element at<VEC>(j, lane). VEC: two groups of four neighbours;
// otherwise neighbours go to neighbouring lanes and `left` elements exist.
template <bool VEC>
__device__ __forceinline__ int at(int j, int lane) {
  return VEC ? (j >> 2) * 128 + lane * 4 + (j & 3) : j * 32 + lane;
}
template <bool VEC, typename T>
__device__ __forceinline__ void load8(const T* p, float* x, int lane, int left) {
  if constexpr (VEC) {
    load4(p + lane * 4, x);
    load4(p + 128 + lane * 4, x + 4);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = at<false>(j, lane) < left ? wide(p[at<false>(j, lane)]) : 0.f;
  }
}
template <bool VEC, typename T>
__device__ __forceinline__ void store8(T* p, const float* x, int lane, int left) {
  if constexpr (VEC) {
    store4(p + lane * 4, x);
    store4(p + 128 + lane * 4, x + 4);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (at<false>(j, lane) < left) narrow(x[j], p + at<false>(j, lane));
  }
}

// A lane's eight codes as two words, slot j in byte j & 3 of word j >> 2. With VEC they lie so in memory. Otherwise
// a slot's codes lie across the lanes: lane 4a + r of a quad takes the word of elements 4a..4a+3 of slot
// 4q + r, and the quad transposes its four words of four bytes (an involution, so it serves both ways).
__device__ __forceinline__ unsigned transpose4(unsigned w, int lane) {
  unsigned p = __shfl_xor_sync(0xffffffffu, w, 1);
  w = __byte_perm(w, p, lane & 1 ? 0x3715 : 0x6240);
  p = __shfl_xor_sync(0xffffffffu, w, 2);
  return __byte_perm(w, p, lane & 2 ? 0x3276 : 0x5410);
}
template <bool VEC>
__device__ __forceinline__ int word_of(int q, int lane) {
  return VEC ? q * 32 + lane : (q * 4 + (lane & 3)) * 8 + (lane >> 2);
}
template <bool VEC>
__device__ __forceinline__ void load_codes(const void* p, unsigned* w, int lane) {
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    w[q] = __ldcs(static_cast<const unsigned*>(p) + word_of<VEC>(q, lane));
    if constexpr (!VEC) w[q] = transpose4(w[q], lane);
  }
}
template <bool VEC>
__device__ __forceinline__ void store_codes(void* p, const unsigned* w, int lane) {
#pragma unroll
  for (int q = 0; q < 2; ++q)
    __stcs(static_cast<unsigned*>(p) + word_of<VEC>(q, lane), VEC ? w[q] : transpose4(w[q], lane));
}

// Codes as floats and back without the conversion unit (a quarter as fast as the multipliers, and busy with
// the roots): a byte in the low mantissa bits of 2^23 is that number plus 2^23, and an addition to 2^23 that
// rounds down leaves the floor in those bits.
constexpr float kMagic = 8388608.f;   // 2^23
template <int J>
__device__ __forceinline__ float2 byte_floats(unsigned w) {   // bytes J and J+1 of w, plus 2^23
  return make_float2(__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7440 + J)), __uint_as_float(__byte_perm(w, 0x4b000000u, 0x7440 + J + 1)));
}
// two codes of the first moment: S a |a|, a = c/127 (c is held as c + 128 by the xor)
template <int J>
__device__ __forceinline__ float2 decode_m(unsigned w, float S) {
  const float2 a = mul2(add2(byte_floats<J>(w ^ 0x80808080u), two(-kMagic - 128.f)), two(1.f / 127.f));
  return mul2(mul2(a, abs2(a)), two(S));
}
// two codes of the second: (R a^2)^2, a = c/255
template <int J>
__device__ __forceinline__ float2 decode_v(unsigned w, float R) {
  const float2 a = mul2(add2(byte_floats<J>(w), two(-kMagic)), two(1.f / 255.f));
  const float2 r = mul2(mul2(a, a), two(R));
  return mul2(r, r);
}
__device__ __forceinline__ unsigned pack4(const unsigned* c) {     // the low bytes of four words
  return __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
}
// Root and quotient to nearest: an approximation and one correction by its exact remainder (Markstein, "Computation
// of elementary functions on the IBM RISC System/6000 processor", 1990), for what decides a code. A code is
// read again in the next step, so a last bit there would grow into the parameters; the values that the codes
// come from are therefore rounded operation by operation, as the formulas are written, and the codes are
// those of plain fp32 arithmetic. The root is right to a unit in the last place from 5e-35 on (the guard's share of the
// approximation's error, squared by the correction); below that it comes out too small.
__device__ __forceinline__ float rsqrt_near(float x) {
  float y;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float2 root2(float2 x) {
  const float2 z = add2(x, two(1.2e-38f));    // nothing but a guard: x itself from 2e-31 on
  const float2 y = make_float2(rsqrt_near(z.x), rsqrt_near(z.y));
  const float2 s = mul2(x, y);
  const float2 e = fma2(make_float2(-s.x, -s.y), s, x);
  return fma2(e, mul2(y, two(0.5f)), s);
}
// The root of any second moment. An infinite one (a finite gradient above 1.8e19) has an infinite root, and its update is
// zero. Small ones are taken 2^96 times as large, where the remainder is exact.
__device__ __forceinline__ float2 any_root2(float2 x) {
  const float2 up = make_float2(x.x < 0x1p-60f ? 0x1p96f : 1.f, x.y < 0x1p-60f ? 0x1p96f : 1.f);
  const float2 down = make_float2(x.x < 0x1p-60f ? 0x1p-48f : 1.f, x.y < 0x1p-60f ? 0x1p-48f : 1.f);
  const float2 r = mul2(root2(mul2(x, up)), down);
  return make_float2(x.x == INFINITY ? INFINITY : r.x, x.y == INFINITY ? INFINITY : r.y);
}
__device__ __forceinline__ float2 quotient2(float2 a, float b, float rcp_b) {
  const float2 q = mul2(a, two(rcp_b));
  return fma2(fma2(q, two(-b), a), two(rcp_b), q);
}
__device__ __forceinline__ float rcp_near(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The dither hash: Murmur3's 32-bit finaliser (Appleby) but for its last exchange, which only the low half sees:
// the two uniforms are the halves of h ^ (h >> 16).
__device__ __forceinline__ unsigned mix(unsigned h) {
  h ^= h >> 16; h *= 0x85ebca6bu;
  h ^= h >> 13; h *= 0xc2b2ae35u;
  return h;
}
__device__ __forceinline__ float half_float(unsigned w, unsigned sel) {   // 16 bits of w, plus 2^23
  return __uint_as_float(__byte_perm(w, 0x4b000000u, sel));
}

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float block_max(float x) {   // over the warp, of non-negative values; a NaN wins
  return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(x)));
}

constexpr float kTiny = 1.1754944e-38f;   // below it a reciprocal overflows: such a block is held as zeros
constexpr float kMostRoot = 1.8446742e19f;   // its square is finite: where a second moment is not, codes hold it as this one

// What a lane reads of a block.
template <typename P, typename G, int BITS>
struct Raw {
  float p[8], g[8], m[BITS == 32 ? 8 : 1], v[BITS == 32 ? 8 : 1];
  unsigned wm[2], wv[2];
  float S, R;
};

// A chunk's places in memory; block i lies i*256 elements (i scales) further.
template <typename P, typename G, int BITS>
struct Place {
  using S = typename std::conditional<BITS == 32, float, uint8_t>::type;
  P* p;
  const G* g;
  __nv_bfloat16* copy;
  S *m, *v;
  float *ms, *vs;
  unsigned s0;               // state index of its first element (low bits)
};

template <bool VEC, typename P, typename G, int BITS>
__device__ __forceinline__ void fetch(Raw<P, G, BITS>& x, const Place<P, G, BITS>& at, int i, int left, int lane) {
  const int e = i * kBlock;
  load8<VEC>(at.g + e, x.g, lane, left);
  load8<VEC>(at.p + e, x.p, lane, left);
  if constexpr (BITS == 32) {
    load8<VEC>(at.m + e, x.m, lane, kBlock);
    load8<VEC>(at.v + e, x.v, lane, kBlock);
  } else {
    load_codes<VEC>(at.m + e, x.wm, lane);
    load_codes<VEC>(at.v + e, x.wv, lane);
    x.S = at.ms[i];
    x.R = at.vs[i];
  }
}

template <bool VEC, typename P, typename G, int BITS, bool DITHER>
__device__ __forceinline__ void finish(const Raw<P, G, BITS>& x, const StepArgs& A, const Place<P, G, BITS>& to, int i, int left, float s, float keep, int lane) {
  const int e = i * kBlock;
  float p[8], m[8], v[8];
  const float* g = x.g;
#pragma unroll
  for (int j = 0; j < 8; ++j) p[j] = x.p[j];
  if constexpr (BITS == 32) {
#pragma unroll
    for (int j = 0; j < 8; ++j) { m[j] = x.m[j]; v[j] = x.v[j]; }
  } else {
    float2 *m2 = reinterpret_cast<float2*>(m), *v2 = reinterpret_cast<float2*>(v);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      m2[2 * q] = decode_m<0>(x.wm[q], x.S); m2[2 * q + 1] = decode_m<2>(x.wm[q], x.S);
      v2[2 * q] = decode_v<0>(x.wv[q], x.R); v2[2 * q + 1] = decode_v<2>(x.wv[q], x.R);
    }
  }
  float2 m2[4], v2[4], g2[4], root[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    g2[j] = mul2(make_float2(g[2 * j], g[2 * j + 1]), two(s));
    v2[j] = fma2(mul2(make_float2(v[2 * j], v[2 * j + 1]), two(A.b2)), two(A.one), mul2(mul2(g2[j], g2[j]), two(A.omb2)));
  }
  auto update = [&](auto root_of) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      m2[j] = fma2(mul2(make_float2(m[2 * j], m[2 * j + 1]), two(A.b1)), two(A.one), mul2(g2[j], two(A.omb1)));
      root[j] = root_of(v2[j]);
      const float2 den = fma2(root[j], two(A.rs_bc2), two(A.eps));
      const float2 u = mul2(m2[j], make_float2(rcp_near(den.x), rcp_near(den.y)));
      const float2 q = fma2(u, two(-A.step), mul2(make_float2(p[2 * j], p[2 * j + 1]), two(keep)));
      p[2 * j] = q.x; p[2 * j + 1] = q.y;
      m[2 * j] = m2[j].x; m[2 * j + 1] = m2[j].y;
      v[2 * j] = v2[j].x; v[2 * j + 1] = v2[j].y;
    }
  };
  // The sum of a lane's second moments tells whether one is infinite, and whether all are so small that their codes would
  // show the quick root's error (a small one beside larger ones has a code of a few units at most): half an instruction per element.
  const float2 pair = add2(add2(v2[0], v2[1]), add2(v2[2], v2[3]));
  const float sum = pair.x + pair.y;
  if (__builtin_expect((sum <= FLT_MAX && sum >= A.quick_from) || sum == 0.f, 1)) update([](float2 x) { return root2(x); });
  else update([](float2 x) { return any_root2(x); });
  store8<VEC>(to.p + e, p, lane, left);
  if (to.copy) store8<VEC>(to.copy + e, p, lane, left);
  if constexpr (BITS == 32) {
    store8<VEC>(to.m + e, m, lane, kBlock);
    store8<VEC>(to.v + e, v, lane, kBlock);
  } else {
    // elements past the tensor's end were read as zero gradients and zero codes: they stay zero
    float S = 0.f, R = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      S = max_nan(S, max_nan(fabsf(m2[j].x), fabsf(m2[j].y)));
      R = max_nan(R, max_nan(root[j].x, root[j].y));
    }
    S = block_max(S); R = block_max(R);
    S = S < kTiny ? 0.f : S;
    R = R < kTiny ? 0.f : R;
    if (R > kMostRoot) {
      R = kMostRoot;
#pragma unroll
      for (int j = 0; j < 4; ++j) root[j] = make_float2(fminf(root[j].x, kMostRoot), fminf(root[j].y, kMostRoot));
    }
    const float is = S == 0.f ? 0.f : 1.f / S, ir = R == 0.f ? 0.f : 1.f / R;
    const unsigned h0 = (to.s0 + (unsigned)(e + at<VEC>(0, lane))) * 0x9e3779b1u + A.key;
    unsigned wm[2], wv[2], cm[4], cv[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float2 um = two(0.5f), uv = two(0.5f);
      if constexpr (DITHER) {
        const unsigned a = mix(h0 + (unsigned)at<VEC>(2 * j, 0) * 0x9e3779b1u), b = mix(h0 + (unsigned)at<VEC>(2 * j + 1, 0) * 0x9e3779b1u);
        um = mul2(add2(make_float2(half_float(a ^ (a >> 16), 0x7410), half_float(b ^ (b >> 16), 0x7410)), two(-kMagic)), two(0x1p-16f));
        uv = mul2(add2(make_float2(half_float(a, 0x7432), half_float(b, 0x7432)), two(-kMagic)), two(0x1p-16f));
      }
      const float2 x = root2(quotient2(abs2(m2[j]), S, is)), y = root2(quotient2(root[j], R, ir));
      float2 a = fma2(mul2(x, two(127.f)), two(A.one), um);
      a = add2_down(a, two(kMagic));       // x <= 1 and u <= 1 - 2^-16: never above 127 (255)
      a = add2(a, two(-kMagic));     // the code as a float; then its sign, and into the low bits as two's complement
      a = add2(make_float2(copysignf(a.x, m2[j].x), copysignf(a.y, m2[j].y)), two(1.5f * kMagic));
      float2 b = fma2(mul2(y, two(255.f)), two(A.one), uv);
      // any nonzero y keeps a code of 1 at least
      b.x = fmaxf(b.x, __saturatef(y.x * 1e38f));
      b.y = fmaxf(b.y, __saturatef(y.y * 1e38f));
      b = add2_down(b, two(kMagic));
      cm[(2 * j) & 3] = __float_as_uint(a.x); cm[(2 * j + 1) & 3] = __float_as_uint(a.y);
      cv[(2 * j) & 3] = __float_as_uint(b.x); cv[(2 * j + 1) & 3] = __float_as_uint(b.y);
      if (j & 1) { wm[j >> 1] = pack4(cm); wv[j >> 1] = pack4(cv); }
    }
    store_codes<VEC>(to.m + e, wm, lane);
    store_codes<VEC>(to.v + e, wv, lane);
    if (lane == 0) {
      to.ms[i] = S;
      to.vs[i] = R;
    }
  }
}

// Blocks k, k + kWarps, ... below nb of a chunk that has `rest` elements, by one warp. With 8-bit moments a block's
// loads are issued before the block ahead of it is computed: the arithmetic is long enough to idle the
// memory otherwise. With fp32 moments the loads alone fill the
// registers, and the SM's other warps hide them.
template <bool VEC, typename P, typename G, int BITS, bool DITHER>
__device__ __forceinline__ void run(const StepArgs& A, const Place<P, G, BITS>& at, int k, int nb, int64_t rest, float s, float keep, int lane) {
  constexpr int kW = kStepThreads<BITS> / 32;
  auto left = [&](int i) { return VEC || rest >= (i + 1) * kBlock ? kBlock : (int)(rest - i * kBlock); };
  if (k >= nb) return;
  Raw<P, G, BITS> x;
  fetch<VEC>(x, at, k, left(k), lane);
  for (; k < nb; k += kW) {
    const int kn = k + kW;
    if constexpr (BITS == 8) {
      Raw<P, G, BITS> y;
      if (kn < nb) fetch<VEC>(y, at, kn, left(kn), lane);
      finish<VEC, P, G, BITS, DITHER>(x, A, at, k, left(k), s, keep, lane);
      x = y;
    } else {
      finish<VEC, P, G, BITS, DITHER>(x, A, at, k, left(k), s, keep, lane);
      if (kn < nb) fetch<VEC>(x, at, kn, left(kn), lane);
    }
  }
}

template <typename P, typename G, int BITS, bool DITHER>
__global__ void __launch_bounds__(kStepThreads<BITS>, kStepCtas<BITS>) adamw_kernel(const __grid_constant__ StepArgs A) {
  asm volatile("griddepcontrol.launch_dependents;\n\tgriddepcontrol.wait;" ::: "memory");
  const float s = A.grad_scale ? __ldcg(A.grad_scale) : 1.f;
  if (s != s) return;                       // the factor says: skip this step
  const Chunk c = A.chunks[blockIdx.x];
  const Tensor T = A.tensors[c.tensor];
  if (!T.g) return;
  const int lane = threadIdx.x & 31;
  const float keep = T.decay ? A.keep : 1.f;
  constexpr int kW = kStepThreads<BITS> / 32;
  const int w = threadIdx.x >> 5;
  const int64_t e0 = c.first * kBlock, rest = T.n - e0, sb = T.block0 + c.first;
  Place<P, G, BITS> at;
  at.p = static_cast<P*>(T.p) + e0;
  at.g = static_cast<const G*>(T.g) + e0;
  at.copy = T.copy ? T.copy + e0 : nullptr;
  at.m = static_cast<typename Place<P, G, BITS>::S*>(A.m) + sb * kBlock;
  at.v = static_cast<typename Place<P, G, BITS>::S*>(A.v) + sb * kBlock;
  at.ms = A.m_scale + sb;
  at.vs = A.v_scale + sb;
  at.s0 = (unsigned)(sb * kBlock);
  if (T.vec) {
    const int full = rest >= c.nblocks * kBlock ? c.nblocks : c.nblocks - 1;
    run<true, P, G, BITS, DITHER>(A, at, w, full, rest, s, keep, lane);
    if (full < c.nblocks && w == (full & (kW - 1)))       // the tensor's last block is a part
      run<false, P, G, BITS, DITHER>(A, at, full, c.nblocks, rest, s, keep, lane);
  } else {
    run<false, P, G, BITS, DITHER>(A, at, w, c.nblocks, rest, s, keep, lane);
  }
}

// Values of 8-bit moments, for checkpoints and inspection: eight codes of each moment per thread.
__device__ __forceinline__ void store8_flat(float* p, const float2* x) {
  __stcs(reinterpret_cast<float4*>(p), make_float4(x[0].x, x[0].y, x[1].x, x[1].y));
  __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(x[2].x, x[2].y, x[3].x, x[3].y));
}
__device__ __forceinline__ void store8_flat(__nv_bfloat16* p, const float2* x) {
  __stcs(reinterpret_cast<uint4*>(p), make_uint4(bf_pack(x[0].x, x[0].y), bf_pack(x[1].x, x[1].y), bf_pack(x[2].x, x[2].y), bf_pack(x[3].x, x[3].y)));
}
template <typename O>
__global__ void __launch_bounds__(kThreads) moments_kernel(const uint2* __restrict__ m, const uint2* __restrict__ v,
                                                           const float* __restrict__ ms, const float* __restrict__ vs,
                                                           O* __restrict__ om, O* __restrict__ ov, int64_t n8) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= n8) return;
  const uint2 a = __ldcs(m + i), b = __ldcs(v + i);
  const float S = ms[i / (kBlock / 8)], R = vs[i / (kBlock / 8)];
  const float2 x[4] = {decode_m<0>(a.x, S), decode_m<2>(a.x, S), decode_m<0>(a.y, S), decode_m<2>(a.y, S)};
  const float2 y[4] = {decode_v<0>(b.x, R), decode_v<2>(b.x, R), decode_v<0>(b.y, R), decode_v<2>(b.y, R)};
  store8_flat(om + i * 8, x);
  store8_flat(ov + i * 8, y);
}

// Global norm: a CTA's chunks by the grid's stride, squares summed eight at a time in fp32 and from there
// in fp64; the CTA that finishes last adds the CTAs' sums in CTA order, so the result does not depend on
// which one that is.
template <typename G>
__global__ void __launch_bounds__(kThreads) norm_kernel(const Tensor* __restrict__ tensors, const Chunk* __restrict__ chunks,
                                                        int nchunks, float max_norm, double* __restrict__ part,
                                                        unsigned* __restrict__ ticket, float* __restrict__ out) {
  __shared__ double sh[kWarps];
  __shared__ bool last;
  asm volatile("griddepcontrol.launch_dependents;\n\tgriddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  double sum = 0.0;
  for (int ci = blockIdx.x; ci < nchunks; ci += gridDim.x) {
    const Chunk c = chunks[ci];
    const Tensor T = tensors[c.tensor];
    if (!T.g) continue;
    for (int k = wid; k < c.nblocks; k += kWarps) {
      const int64_t e0 = (c.first + k) * kBlock, rest = T.n - e0;
      float g[8];
      if (T.vec && rest >= kBlock) load8<true>(static_cast<const G*>(T.g) + e0, g, lane, kBlock);
      else load8<false>(static_cast<const G*>(T.g) + e0, g, lane, rest < kBlock ? (int)rest : kBlock);
      float q = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) q = fmaf(g[j], g[j], q);
      sum += (double)q;
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) sh[wid] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0.0;
    for (int w = 0; w < kWarps; ++w) t += sh[w];
    part[blockIdx.x] = t;
    __threadfence();
    last = atomicAdd(ticket, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  double t = 0.0;
  for (int i = threadIdx.x; i < (int)gridDim.x; i += kThreads) t += __ldcg(part + i);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
  if (lane == 0) sh[wid] = t;
  __syncthreads();
  if (threadIdx.x == 0) {
    t = 0.0;
    for (int w = 0; w < kWarps; ++w) t += sh[w];
    const float norm = (float)sqrt(t);
    const double coef = (double)max_norm / (sqrt(t) + 1e-6);
    out[0] = norm;
    out[1] = isfinite(norm) ? (float)(coef < 1.0 ? coef : 1.0) : __int_as_float(0x7fc00000);
    *ticket = 0u;
  }
}

}  // namespace

struct dmx_adamw {
  int device = 0, n = 0, param_dtype = 0, grad_dtype = 0, bits = 0;
  int nchunks = 0, norm_grid = 0;
  int64_t blocks = 0;
  bool bound = false;
  std::vector<Tensor> host;        // the table as last bound; the device copy is read by the kernels
  Tensor* tensors = nullptr;
  Chunk* chunks = nullptr;
  double* part = nullptr;
  unsigned* ticket = nullptr;
};

namespace {

bool live(const dmx_adamw* h) { return dmxh::live_has(h, dmxh::kAdamwHandle); }

void release(dmx_adamw* h) {
  cudaFree(h->tensors); cudaFree(h->chunks); cudaFree(h->part); cudaFree(h->ticket);
  (void)cudaGetLastError();
  delete h;
}

// As programmatic dependents: a step behind its gradient norm is resident when that ends (the kernels' first act is to
// wait for it; 1 Mi parameters: 2 us less for the two).
template <typename... K, typename... V>
int start(int grid, int threads, cudaStream_t st, void (*kernel)(K...), V... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return dmxh::cuda_ok(cudaLaunchKernelEx(&cfg, kernel, static_cast<K>(args)...)) ? DMX_OK : DMX_ERR_CUDA;
}

template <typename P, typename G>
int launch_step(const dmx_adamw* h, const StepArgs& A, bool dither, cudaStream_t st) {
  if (h->bits == 32) return start(h->nchunks, kStepThreads<32>, st, adamw_kernel<P, G, 32, false>, A);
  if (dither) return start(h->nchunks, kStepThreads<8>, st, adamw_kernel<P, G, 8, true>, A);
  return start(h->nchunks, kStepThreads<8>, st, adamw_kernel<P, G, 8, false>, A);
}

bool aligned(const void* p, unsigned a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// 8-bit moments need their scales, fp32 moments take none
int check_state(const dmx_adamw* h, const void* m, const void* v, const float* ms, const float* vs) {
  const bool some = h->blocks > 0;         // (empty arrays need no address)
  if (some && (!m || !v || m == v)) return DMX_ERR_ARG;
  if (some && h->bits == 8 && (!ms || !vs || ms == vs)) return DMX_ERR_ARG;
  if (h->bits == 32 && (ms || vs)) return DMX_ERR_ARG;
  if (!aligned(m, 16) || !aligned(v, 16) || !aligned(ms, 4) || !aligned(vs, 4)) return DMX_ERR_ALIGN;
  return DMX_OK;
}

}  // namespace

extern "C" {

int dmx_adamw_create(int n, const int64_t* sizes, const uint8_t* decay, int param_dtype, int grad_dtype, int state_bits,
                     dmx_adamw** out) {
  if (!out) return DMX_ERR_ARG;
  *out = nullptr;
  if (n < 1 || n > DMX_ADAMW_MAX_TENSORS || !sizes) return DMX_ERR_ARG;
  if (param_dtype != DMX_F32 && param_dtype != DMX_BF16) return DMX_ERR_ARG;
  if (grad_dtype != DMX_F32 && grad_dtype != DMX_BF16) return DMX_ERR_ARG;
  if (state_bits != 8 && state_bits != 32) return DMX_ERR_ARG;
  int64_t blocks = 0;
  for (int i = 0; i < n; ++i) {
    if (sizes[i] < 0 || sizes[i] >= DMX_MAX_PARAMS) return DMX_ERR_ARG;
    blocks += (sizes[i] + kBlock - 1) / kBlock;
    if (blocks > DMX_MAX_PARAMS / kBlock) return DMX_ERR_ARG;
  }
  dmxh::alloc_begin();
  dmx_adamw* h = dmxh::alloc_host_ok() ? new (std::nothrow) dmx_adamw : nullptr;
  if (!h) return DMX_ERR_NOMEM;
  std::vector<Chunk> chunks;
  bool ok = dmxh::cuda_ok(cudaGetDevice(&h->device));
  int sms = 0;
  ok = ok && dmxh::cuda_ok(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, h->device));
  if (!ok) { release(h); return DMX_ERR_CUDA; }
  // fp32 moments: four blocks per warp where that still gives every SM several CTAs; a small model is cut finer,
  // one block per warp, so that all SMs have work (1 Mi parameters: 8.0 us cut finely, 9.0 us with twice the
  // blocks). 8-bit moments: eight blocks for a CTA's one warp; 16 gain 1 % on 340 M and cost 10 % on 25 M.
  const int per = state_bits == 8 || blocks < (int64_t)sms * 256 ? 8 : 32;
  try {
    h->host.resize(n);
    int64_t b0 = 0;
    for (int i = 0; i < n; ++i) {
      const int64_t nb = (sizes[i] + kBlock - 1) / kBlock;
      Tensor t;
      memset(&t, 0, sizeof t);
      t.n = sizes[i]; t.block0 = b0; t.decay = decay ? decay[i] != 0 : 1;
      h->host[i] = t;
      for (int64_t f = 0; f < nb; f += per) {
        Chunk c;
        c.tensor = i; c.first = f; c.nblocks = (int)(nb - f < per ? nb - f : per);
        chunks.push_back(c);
      }
      b0 += nb;
    }
  } catch (...) {
    release(h);
    return DMX_ERR_NOMEM;
  }
  if (chunks.size() > 0x7fffffffu) { release(h); return DMX_ERR_ARG; }
  h->n = n; h->param_dtype = param_dtype; h->grad_dtype = grad_dtype; h->bits = state_bits;
  h->blocks = blocks; h->nchunks = (int)chunks.size();
  h->norm_grid = h->nchunks < sms * 8 ? (h->nchunks > 0 ? h->nchunks : 1) : sms * 8;
  ok = dmxh::dev_alloc((void**)&h->tensors, sizeof(Tensor) * n) &&
       dmxh::dev_alloc((void**)&h->chunks, sizeof(Chunk) * (chunks.empty() ? 1 : chunks.size())) &&
       dmxh::dev_alloc((void**)&h->part, sizeof(double) * h->norm_grid) &&
       dmxh::dev_alloc((void**)&h->ticket, sizeof(unsigned));
  if (!ok) { release(h); return DMX_ERR_NOMEM; }
  ok = (chunks.empty() || dmxh::cuda_ok(cudaMemcpy(h->chunks, chunks.data(), sizeof(Chunk) * chunks.size(), cudaMemcpyHostToDevice))) &&
       dmxh::cuda_ok(cudaMemset(h->ticket, 0, sizeof(unsigned))) && dmxh::cuda_ok(cudaDeviceSynchronize());
  if (!ok) { release(h); return DMX_ERR_CUDA; }
  try {
    dmxh::live_add(h, dmxh::kAdamwHandle);
  } catch (...) {
    release(h);
    return DMX_ERR_NOMEM;
  }
  *out = h;
  return DMX_OK;
}

int64_t dmx_adamw_blocks(const dmx_adamw* h) { return live(h) ? h->blocks : DMX_ERR_HANDLE; }

int64_t dmx_adamw_first_block(const dmx_adamw* h, int i) {
  if (!live(h)) return DMX_ERR_HANDLE;
  if (i < 0 || i >= h->n) return DMX_ERR_ARG;
  return h->host[i].block0;
}

int dmx_adamw_bind(dmx_adamw* h, void* const* params, const void* const* grads, void* const* copies, void* cuda_stream) {
  if (!live(h)) return DMX_ERR_HANDLE;
  if (!params || !grads) return DMX_ERR_ARG;
  const int rc = dmxh::check_current_device(h->device);
  if (rc != DMX_OK) return rc;
  const unsigned pe = h->param_dtype == DMX_F32 ? 4 : 2, ge = h->grad_dtype == DMX_F32 ? 4 : 2;
  for (int i = 0; i < h->n; ++i) {
    if (h->host[i].n == 0) continue;
    if (!params[i] || params[i] == grads[i]) return DMX_ERR_ARG;
    if (!aligned(params[i], pe) || !aligned(grads[i], ge) || (copies && !aligned(copies[i], 2))) return DMX_ERR_ALIGN;
  }
  for (int i = 0; i < h->n; ++i) {
    Tensor& t = h->host[i];
    t.p = params[i];
    t.g = grads[i];
    t.copy = copies ? static_cast<__nv_bfloat16*>(copies[i]) : nullptr;
    t.vec = aligned(t.p, 4 * pe) && aligned(t.g, 4 * ge) && aligned(t.copy, 8);
  }
  if (!dmxh::cuda_ok(cudaMemcpyAsync(h->tensors, h->host.data(), sizeof(Tensor) * h->n, cudaMemcpyHostToDevice,
                                     static_cast<cudaStream_t>(cuda_stream)))) return DMX_ERR_CUDA;
  h->bound = true;
  return DMX_OK;
}

int dmx_adamw_grad_norm(dmx_adamw* h, float max_norm, float* out, void* cuda_stream) {
  if (!live(h)) return DMX_ERR_HANDLE;
  if (!h->bound || !out || !(max_norm > 0.f)) return DMX_ERR_ARG;
  if (!aligned(out, 4)) return DMX_ERR_ALIGN;
  const int rc = dmxh::check_current_device(h->device);
  if (rc != DMX_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  return start(h->norm_grid, kThreads, st, h->grad_dtype == DMX_F32 ? norm_kernel<float> : norm_kernel<__nv_bfloat16>, (const Tensor*)h->tensors,
               (const Chunk*)h->chunks, h->nchunks, max_norm, h->part, h->ticket, out);
}

int dmx_adamw_step(dmx_adamw* h, void* m, void* v, float* m_scale, float* v_scale, const float* grad_scale, double lr,
                   double beta1, double beta2, double eps, double weight_decay, int64_t t, int dither, uint32_t seed,
                   void* cuda_stream) {
  if (!live(h)) return DMX_ERR_HANDLE;
  if (!h->bound) return DMX_ERR_ARG;
  if (!(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1) || !(eps >= 0) || !(weight_decay >= 0) || t < 1) return DMX_ERR_ARG;
  if (!isfinite(lr) || !isfinite(eps) || !isfinite(weight_decay)) return DMX_ERR_ARG;
  int rc = check_state(h, m, v, m_scale, v_scale);
  if (rc != DMX_OK) return rc;
  if (!aligned(grad_scale, 4)) return DMX_ERR_ALIGN;
  rc = dmxh::check_current_device(h->device);
  if (rc != DMX_OK) return rc;
  if (h->nchunks == 0) return DMX_OK;
  StepArgs A;
  A.tensors = h->tensors; A.chunks = h->chunks;
  A.m = m; A.v = v; A.m_scale = m_scale; A.v_scale = v_scale; A.grad_scale = grad_scale;
  A.b1 = (float)beta1; A.omb1 = (float)(1.0 - beta1);
  A.b2 = (float)beta2; A.omb2 = (float)(1.0 - beta2);
  A.eps = (float)eps; A.one = 1.f;
  A.keep = (float)(1.0 - lr * weight_decay);
  A.rs_bc2 = (float)(1.0 / sqrt(1.0 - pow(beta2, (double)t)));
  A.step = (float)(lr / (1.0 - pow(beta1, (double)t)));
  // Where v' < 5e-35 the quick root is off by up to 7e-18, which eps hides in the denominator if half its last place is more
  // than that; otherwise every root is taken with care.
  A.quick_from = (double)A.eps >= 7e-18 * 0x1p25 * (double)A.rs_bc2 ? 1e-26f : INFINITY;
  A.key = seed * 0x85ebca6bu + 0x1b873593u;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const bool pf = h->param_dtype == DMX_F32, gf = h->grad_dtype == DMX_F32;
  if (pf && gf) return launch_step<float, float>(h, A, dither != 0, st);
  if (pf) return launch_step<float, __nv_bfloat16>(h, A, dither != 0, st);
  return gf ? launch_step<__nv_bfloat16, float>(h, A, dither != 0, st)
            : launch_step<__nv_bfloat16, __nv_bfloat16>(h, A, dither != 0, st);
}

int dmx_adamw_moments(dmx_adamw* h, const void* m, const void* v, const float* m_scale, const float* v_scale, int out_dtype,
                      void* out_m, void* out_v, void* cuda_stream) {
  if (!live(h)) return DMX_ERR_HANDLE;
  if (h->bits != 8 || (h->blocks > 0 && (!out_m || !out_v || out_m == out_v)) || (out_dtype != DMX_F32 && out_dtype != DMX_BF16)) return DMX_ERR_ARG;
  int rc = check_state(h, m, v, m_scale, v_scale);
  if (rc != DMX_OK) return rc;
  if (!aligned(out_m, 16) || !aligned(out_v, 16)) return DMX_ERR_ALIGN;
  rc = dmxh::check_current_device(h->device);
  if (rc != DMX_OK) return rc;
  const int64_t n8 = h->blocks * (kBlock / 8);
  if (n8 == 0) return DMX_OK;
  const int grid = (int)((n8 + kThreads - 1) / kThreads);      // at most 2^40 / 8 / kThreads < 2^31
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const uint2 *cm = static_cast<const uint2*>(m), *cv = static_cast<const uint2*>(v);
  if (out_dtype == DMX_F32)
    moments_kernel<float><<<grid, kThreads, 0, st>>>(cm, cv, m_scale, v_scale, static_cast<float*>(out_m), static_cast<float*>(out_v), n8);
  else
    moments_kernel<__nv_bfloat16><<<grid, kThreads, 0, st>>>(cm, cv, m_scale, v_scale, static_cast<__nv_bfloat16*>(out_m),
                                                             static_cast<__nv_bfloat16*>(out_v), n8);
  return dmxh::cuda_ok(cudaGetLastError()) ? DMX_OK : DMX_ERR_CUDA;
}

int dmx_adamw_destroy(dmx_adamw* h) {
  if (!h) return DMX_OK;
  if (!dmxh::live_remove(h, dmxh::kAdamwHandle)) return DMX_ERR_HANDLE;
  release(h);
  return DMX_OK;
}

}  // extern "C"
