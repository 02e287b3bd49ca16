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
// Bound: HBM. A step moves 8 + grad + states (16, or 4 with 8-bit codes) + copy bytes per element and does
// ~40 operations on them. A warp owns one block of 256 elements (its scales need a maximum over the block:
// one redux instruction), eight per lane as two groups of four neighbours, so every access of an aligned
// tensor is 16 bytes of fp32, 8 of bf16 or 4 of codes per lane and a warp's lines are full. A tensor whose
// start is not so aligned (a segment of a flat vector) takes its parameters and gradients element by element,
// 32 neighbours per access; the state is the library's own layout and stays aligned.
#include "dmx.h"

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <new>
#include <string.h>
#include <vector>

#include "dmx_host.h"

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
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
  float b1, omb1, b2, omb2, eps, keep, rs_bc2, step;
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

// Eight elements of a lane: element e of the block is at slot j with e = at(j, lane, vec).
// vec: two groups of four neighbours; otherwise neighbours go to neighbouring lanes.
__device__ __forceinline__ int at(int j, int lane, bool vec) {
  return vec ? (j >> 2) * 128 + lane * 4 + (j & 3) : j * 32 + lane;
}

template <typename T>
__device__ __forceinline__ void load8(const T* p, float* x, int lane, bool vec, int left) {
  if (vec && left >= kBlock) {
    load4(p + lane * 4, x);
    load4(p + 128 + lane * 4, x + 4);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = at(j, lane, vec);
      x[j] = e < left ? wide(p[e]) : 0.f;
    }
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float* x, int lane, bool vec, int left) {
  if (vec && left >= kBlock) {
    store4(p + lane * 4, x);
    store4(p + 128 + lane * 4, x + 4);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = at(j, lane, vec);
      if (e < left) narrow(x[j], p + e);
    }
  }
}

// Codes as floats and back without the conversion unit (a quarter as fast as the multipliers, and busy with
// the roots): a byte in the low mantissa bits of 2^23 is that number plus 2^23, and an addition to 2^23 that
// rounds down leaves the floor in those bits.
constexpr float kMagic = 8388608.f;   // 2^23
__device__ __forceinline__ float byte_float(unsigned w, int j) {   // byte j of w, plus 2^23
  return __uint_as_float(__byte_perm(w, 0x4b000000u, 0x7440 + j));
}
__device__ __forceinline__ unsigned floor_bits(float x) {          // floor(x) in the low bits, x >= 0
  return __float_as_uint(__fadd_rd(x, kMagic));
}
// four codes of the first moment: S a |a|, a = c/127 (c is held as c + 128 by the xor)
__device__ __forceinline__ void decode_m(unsigned w, float S, float* x) {
  w ^= 0x80808080u;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float a = (byte_float(w, j) - (kMagic + 128.f)) * (1.f / 127.f);
    x[j] = a * fabsf(a) * S;
  }
}
// four codes of the second: (R a^2)^2, a = c/255
__device__ __forceinline__ void decode_v(unsigned w, float R, float* x) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float a = (byte_float(w, j) - kMagic) * (1.f / 255.f);
    const float r = a * a * R;
    x[j] = r * r;
  }
}
// Two words of four codes per lane: aligned tensors take their own; the others' elements lie across the
// lanes, so a lane fetches each element's byte.
__device__ __forceinline__ void load_codes(const void* p, unsigned* w, int lane, bool vec) {
  if (vec) {
    w[0] = __ldcs(static_cast<const unsigned*>(p) + lane);
    w[1] = __ldcs(static_cast<const unsigned*>(p) + 32 + lane);
  } else {
    const uint8_t* b = static_cast<const uint8_t*>(p) + lane;
    w[0] = w[1] = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j >> 2] |= (unsigned)b[j * 32] << (8 * (j & 3));
  }
}
__device__ __forceinline__ void store_codes(void* p, const unsigned* w, int lane, bool vec) {
  if (vec) {
    __stcs(static_cast<unsigned*>(p) + lane, w[0]);
    __stcs(static_cast<unsigned*>(p) + 32 + lane, w[1]);
  } else {
    uint8_t* b = static_cast<uint8_t*>(p) + lane;
#pragma unroll
    for (int j = 0; j < 8; ++j) b[j * 32] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
  }
}
__device__ __forceinline__ unsigned pack4(const unsigned* c) {     // the low bytes of four words
  return __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
}
// Root and quotient to nearest: an approximation and one correction by its exact remainder (Markstein, "Computation
// of elementary functions on the IBM RISC System/6000 processor", 1990), for what decides a code. A code is
// read again in the next step, so a last bit there would grow into the parameters; the values that the codes
// come from are therefore rounded operation by operation, as the formulas are written, and the codes are
// those of plain fp32 arithmetic. Under 1.2e-38 the root loses accuracy, not its sign.
__device__ __forceinline__ float root_of(float x) {
  float y;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(fmaxf(x, 1.1754944e-38f)));
  const float s = x * y;
  return fmaf(fmaf(-s, s, x), 0.5f * y, s);
}
__device__ __forceinline__ float quotient(float a, float b, float rcp_b) {
  const float q = a * rcp_b;
  return fmaf(fmaf(-q, b, a), rcp_b, q);
}

__device__ __forceinline__ unsigned mix(unsigned h) {   // Murmur3's 32-bit finaliser (Appleby)
  h ^= h >> 16; h *= 0x85ebca6bu;
  h ^= h >> 13; h *= 0xc2b2ae35u;
  return h ^ (h >> 16);
}

template <bool ABS>
__device__ __forceinline__ float block_max(const float* x) {   // of |x| or of non-negative x; a NaN wins
  unsigned u = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) u = max(u, __float_as_uint(ABS ? fabsf(x[j]) : x[j]));
  return __uint_as_float(__reduce_max_sync(0xffffffffu, u));
}

constexpr float kTiny = 1.1754944e-38f;   // below it a reciprocal overflows: such a block is held as zeros

template <typename P, typename G, int BITS, bool DITHER>
__global__ void __launch_bounds__(kThreads, 3) adamw_kernel(const __grid_constant__ StepArgs A) {
  const float s = A.grad_scale ? __ldg(A.grad_scale) : 1.f;
  if (s != s) return;                       // the factor says: skip this step
  const Chunk c = A.chunks[blockIdx.x];
  const Tensor T = A.tensors[c.tensor];
  if (!T.g) return;
  const int lane = threadIdx.x & 31;
  const bool vec = T.vec != 0;
  const float keep = T.decay ? A.keep : 1.f;
  for (int k = threadIdx.x >> 5; k < c.nblocks; k += kWarps) {
    const int64_t blk = c.first + k;
    const int64_t e0 = blk * kBlock, rest = T.n - e0;
    const int left = rest < kBlock ? (int)rest : kBlock;
    const int64_t sb = T.block0 + blk, s0 = sb * kBlock;
    float p[8], g[8], m[8], v[8];
    P* pp = static_cast<P*>(T.p) + e0;
    load8(static_cast<const G*>(T.g) + e0, g, lane, vec, left);
    load8(static_cast<const P*>(pp), p, lane, vec, left);
    if constexpr (BITS == 32) {
      load8(static_cast<const float*>(A.m) + s0, m, lane, vec, kBlock);
      load8(static_cast<const float*>(A.v) + s0, v, lane, vec, kBlock);
    } else {
      unsigned wm[2], wv[2];
      load_codes(static_cast<const uint8_t*>(A.m) + s0, wm, lane, vec);
      load_codes(static_cast<const uint8_t*>(A.v) + s0, wv, lane, vec);
      const float S = A.m_scale[sb], R = A.v_scale[sb];
      decode_m(wm[0], S, m); decode_m(wm[1], S, m + 4);
      decode_v(wv[0], R, v); decode_v(wv[1], R, v + 4);
    }
    float root[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float gj = g[j] * s;
      m[j] = __fadd_rn(__fmul_rn(m[j], A.b1), __fmul_rn(gj, A.omb1));
      v[j] = __fadd_rn(__fmul_rn(v[j], A.b2), __fmul_rn(__fmul_rn(gj, gj), A.omb2));
      root[j] = root_of(v[j]);
      const float u = __fdividef(m[j], fmaf(root[j], A.rs_bc2, A.eps));
      p[j] = fmaf(-A.step, u, p[j] * keep);
    }
    store8(pp, p, lane, vec, left);
    if (T.copy) store8(T.copy + e0, p, lane, vec, left);
    if constexpr (BITS == 32) {
      store8(static_cast<float*>(A.m) + s0, m, lane, vec, kBlock);
      store8(static_cast<float*>(A.v) + s0, v, lane, vec, kBlock);
    } else {
      // elements past the tensor's end were read as zero gradients and zero codes: they stay zero
      float S = block_max<true>(m), R = block_max<false>(root);
      S = S < kTiny ? 0.f : S;
      R = R < kTiny ? 0.f : R;
      const float is = S == 0.f ? 0.f : 1.f / S, ir = R == 0.f ? 0.f : 1.f / R;
      unsigned cm[8], cv[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float um = 0.5f, uv = 0.5f;
        if (DITHER) {
          const unsigned h = mix((unsigned)(s0 + at(j, lane, vec)) * 0x9e3779b1u + A.key);
          um = __uint_as_float(0x3f800000u | (h & 0xffffu) << 7) - 1.f;
          uv = __uint_as_float(0x3f800000u | (h >> 16) << 7) - 1.f;
        }
        const float x = root_of(quotient(fabsf(m[j]), S, is)), y = root_of(quotient(root[j], R, ir));
        const unsigned a = floor_bits(fminf(__fadd_rn(__fmul_rn(x, 127.f), um), 127.5f));
        const unsigned neg = (unsigned)(__float_as_int(m[j]) >> 31);
        cm[j] = (a ^ neg) - neg;
        // any nonzero y keeps a code of 1 at least
        cv[j] = floor_bits(fminf(fmaxf(__fadd_rn(__fmul_rn(y, 255.f), uv), __saturatef(y * 1e38f)), 255.5f));
      }
      unsigned wm[2] = {pack4(cm), pack4(cm + 4)}, wv[2] = {pack4(cv), pack4(cv + 4)};
      store_codes(static_cast<uint8_t*>(A.m) + s0, wm, lane, vec);
      store_codes(static_cast<uint8_t*>(A.v) + s0, wv, lane, vec);
      if (lane == 0) {
        A.m_scale[sb] = S;
        A.v_scale[sb] = R;
      }
    }
  }
}

// Values of 8-bit moments, for checkpoints and inspection: four codes of each moment per thread.
template <typename O>
__global__ void __launch_bounds__(kThreads) moments_kernel(const int8_t* __restrict__ m, const uint8_t* __restrict__ v,
                                                           const float* __restrict__ ms, const float* __restrict__ vs,
                                                           O* __restrict__ om, O* __restrict__ ov, int64_t quads) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < quads; i += (int64_t)gridDim.x * kThreads) {
    const unsigned a = __ldcs(reinterpret_cast<const unsigned*>(m) + i);
    const unsigned b = __ldcs(reinterpret_cast<const unsigned*>(v) + i);
    const float S = ms[i / (kBlock / 4)], R = vs[i / (kBlock / 4)];
    float x[4], y[4];
    decode_m(a, S, x);
    decode_v(b, R, y);
    store4(om + i * 4, x);
    store4(ov + i * 4, y);
  }
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
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  double sum = 0.0;
  for (int ci = blockIdx.x; ci < nchunks; ci += gridDim.x) {
    const Chunk c = chunks[ci];
    const Tensor T = tensors[c.tensor];
    if (!T.g) continue;
    for (int k = wid; k < c.nblocks; k += kWarps) {
      const int64_t e0 = (c.first + k) * kBlock, rest = T.n - e0;
      float g[8];
      load8(static_cast<const G*>(T.g) + e0, g, lane, T.vec != 0, rest < kBlock ? (int)rest : kBlock);
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

template <typename P, typename G>
void launch_step(const dmx_adamw* h, const StepArgs& A, bool dither, cudaStream_t st) {
  if (h->bits == 32) adamw_kernel<P, G, 32, false><<<h->nchunks, kThreads, 0, st>>>(A);
  else if (dither) adamw_kernel<P, G, 8, true><<<h->nchunks, kThreads, 0, st>>>(A);
  else adamw_kernel<P, G, 8, false><<<h->nchunks, kThreads, 0, st>>>(A);
}

bool aligned(const void* p, unsigned a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// 8-bit moments need their scales, fp32 moments take none
int check_state(const dmx_adamw* h, const void* m, const void* v, const float* ms, const float* vs) {
  if (!m || !v || m == v) return DMX_ERR_ARG;
  if (h->bits == 8 && (!ms || !vs || ms == vs)) return DMX_ERR_ARG;
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
  // A CTA takes four blocks per warp where that still gives every SM several CTAs; a small model is cut
  // finer, one block per warp, so that all SMs have work.
  const int per = blocks >= (int64_t)sms * 256 ? 4 * kWarps : kWarps;
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
  if (h->grad_dtype == DMX_F32)
    norm_kernel<float><<<h->norm_grid, kThreads, 0, st>>>(h->tensors, h->chunks, h->nchunks, max_norm, h->part, h->ticket, out);
  else
    norm_kernel<__nv_bfloat16><<<h->norm_grid, kThreads, 0, st>>>(h->tensors, h->chunks, h->nchunks, max_norm, h->part, h->ticket, out);
  return dmxh::cuda_ok(cudaGetLastError()) ? DMX_OK : DMX_ERR_CUDA;
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
  A.eps = (float)eps;
  A.keep = (float)(1.0 - lr * weight_decay);
  A.rs_bc2 = (float)(1.0 / sqrt(1.0 - pow(beta2, (double)t)));
  A.step = (float)(lr / (1.0 - pow(beta1, (double)t)));
  A.key = seed * 0x85ebca6bu + 0x1b873593u;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const bool pf = h->param_dtype == DMX_F32, gf = h->grad_dtype == DMX_F32;
  if (pf && gf) launch_step<float, float>(h, A, dither != 0, st);
  else if (pf) launch_step<float, __nv_bfloat16>(h, A, dither != 0, st);
  else if (gf) launch_step<__nv_bfloat16, float>(h, A, dither != 0, st);
  else launch_step<__nv_bfloat16, __nv_bfloat16>(h, A, dither != 0, st);
  return dmxh::cuda_ok(cudaGetLastError()) ? DMX_OK : DMX_ERR_CUDA;
}

int dmx_adamw_moments(dmx_adamw* h, const void* m, const void* v, const float* m_scale, const float* v_scale, int out_dtype,
                      void* out_m, void* out_v, void* cuda_stream) {
  if (!live(h)) return DMX_ERR_HANDLE;
  if (h->bits != 8 || !out_m || !out_v || out_m == out_v || (out_dtype != DMX_F32 && out_dtype != DMX_BF16)) return DMX_ERR_ARG;
  int rc = check_state(h, m, v, m_scale, v_scale);
  if (rc != DMX_OK) return rc;
  if (!aligned(out_m, 16) || !aligned(out_v, 16)) return DMX_ERR_ALIGN;
  rc = dmxh::check_current_device(h->device);
  if (rc != DMX_OK) return rc;
  const int64_t quads = h->blocks * (kBlock / 4);
  if (quads == 0) return DMX_OK;
  const int64_t want = (quads + kThreads - 1) / kThreads;
  const int grid = want > 148 * 64 ? 148 * 64 : (int)want;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const int8_t* cm = static_cast<const int8_t*>(m);
  const uint8_t* cv = static_cast<const uint8_t*>(v);
  if (out_dtype == DMX_F32)
    moments_kernel<float><<<grid, kThreads, 0, st>>>(cm, cv, m_scale, v_scale, static_cast<float*>(out_m), static_cast<float*>(out_v), quads);
  else
    moments_kernel<__nv_bfloat16><<<grid, kThreads, 0, st>>>(cm, cv, m_scale, v_scale, static_cast<__nv_bfloat16*>(out_m),
                                                             static_cast<__nv_bfloat16*>(out_v), quads);
  return dmxh::cuda_ok(cudaGetLastError()) ? DMX_OK : DMX_ERR_CUDA;
}

int dmx_adamw_destroy(dmx_adamw* h) {
  if (!h) return DMX_OK;
  if (!dmxh::live_remove(h, dmxh::kAdamwHandle)) return DMX_ERR_HANDLE;
  release(h);
  return DMX_OK;
}

}  // extern "C"
