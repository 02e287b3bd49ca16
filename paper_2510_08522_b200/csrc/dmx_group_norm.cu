// dmx_group_norm.cu — group norm with an activation on channels-last data, and its gradient.
//
// forward    per image and group: mean and variance over L positions x C/G channels, then
//            y = act((x - mean) rstd w + b)
// backward   du = dy act'(u), xh = (x - mean) rstd; per image and channel A_c = sum du xh, B_c = sum du over the
//            positions; dx = rstd (w du - (sum_c w B_c + xh sum_c w A_c) / n); dweight, dbias = sums of A, B over images
//
// Bound: HBM. The sums have to be known before the first result, so x (and dy) is either read twice or kept
// on the chip. Here it is kept: a CTA takes a slab of neighbouring whole groups and a range of positions, each
// thread a fixed column of 16 bytes (or one element, where alignment allows no more) and every R-th position,
// in shared memory slots of its own that asynchronous copies fill (no barrier between copy and use). Up to eight CTAs of
// a cluster share an image's slab and exchange their sums through distributed shared memory. The CTAs stay and
// take slab after slab; a slot is refilled for the next slab as soon as its result is out, so loads run while
// sums are exchanged and results stored. One read, one write. An image too large for that is cut into chunks:
// one launch for the chunks' sums, a small one that joins them, one that reads again, mostly from L2.
// Variances: a thread sums deviations from its own first value, s = sum d, q = sum d^2, and takes q - s^2/n. That
// cancels only if the first value is far off, and then the group's variance contains that distance itself:
// the error stays within n (at most 128) roundings of the result. From there on deviations of means are added
// (Chan, Golub, LeVeque 1983), each mean held as a float and what its rounding lost, and deviations taken from a rough mean whose own
// deviation is summed beside them: a mean a million deviations away costs the variance nothing (with means in one float, rstd was
// off by 1e-7 times mean over deviation where the spread lies between channels). Nothing is added atomically; the order of all sums is fixed by the shape.
// Measured on B200, bf16: forward on 1024 x 32x32 x 64 55 us (4.9 TB/s of algorithmic bytes; 41 us at the measured copy
// rate), backward on 64 x 56x56 x 256 with SiLU 104 us (3.0 TB/s; 47 us); what keeps them from it is what each slab costs
// besides its data (reductions, exchange, parameters: a third of a slab's time) at two or three CTAs per SM.
#include "dmx.h"

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <float.h>
#include <math.h>
#include <stdint.h>
#include <atomic>

#include "dmx_act.cuh"
#include "dmx_host.h"

namespace {

using namespace dmx_f32x2;

constexpr int kMaxCluster = 8;

struct Operand {
  void* p;
  int64_t image, row;    // strides in elements
};

struct Args {
  Operand x, dy, out;    // out: y or dx
  const float *weight, *bias;
  float *mean, *rstd;    // forward: outputs; backward: inputs
  float* part;           // partial sums (workspace)
  int64_t items;         // image slabs (and chunks)
  int L, N, C, G, cpg, W, gW, slabs, R, cols, rows;   // W channels (gW groups) per slab, R positions at a time, cols columns of V, rows positions per CTA
  int parts;             // CTAs (or chunks) per image and slab
  int slots;             // positions per thread
  int fold;              // neighbouring channels of a column that surely share a group (a power of two)
  int lanes;             // lanes of a warp that hold different columns, if that divides 32, else 0
  float eps;
};

template <typename T, int V>
struct Vec;                                            // V elements as one access
template <> struct Vec<float, 4> { using type = uint4; };
template <> struct Vec<float, 1> { using type = unsigned; };
template <> struct Vec<__nv_bfloat16, 8> { using type = uint4; };
template <> struct Vec<__nv_bfloat16, 1> { using type = unsigned short; };

// A thread computes on pairs: neighbouring channels of a column, or, where a column is one element, the elements of two
// positions.
template <int V> constexpr int kPairs = V > 1 ? V / 2 : 1;
template <int V> constexpr int kSlots = V > 1 ? 1 : 2;

__device__ __forceinline__ void widen(const uint4* s, bool, int, float2, float2 (&x)[2]) {
  const uint4 r = *s;
  x[0] = make_float2(__uint_as_float(r.x), __uint_as_float(r.y));
  x[1] = make_float2(__uint_as_float(r.z), __uint_as_float(r.w));
}
__device__ __forceinline__ void widen(const uint4* s, bool, int, float2, float2 (&x)[4]) {
  const uint4 r = *s;
  x[0] = widen2(r.x); x[1] = widen2(r.y); x[2] = widen2(r.z); x[3] = widen2(r.w);
}
// `second`: the next position exists (`step` slots further); otherwise `fill` stands for its value
__device__ __forceinline__ void widen(const unsigned* s, bool second, int step, float2 fill, float2 (&x)[1]) {
  x[0] = make_float2(__uint_as_float(*s), second ? __uint_as_float(s[step]) : fill.y);
}
__device__ __forceinline__ void widen(const unsigned short* s, bool second, int step, float2 fill, float2 (&x)[1]) {
  x[0] = make_float2(__uint_as_float((unsigned)*s << 16), second ? __uint_as_float((unsigned)s[step] << 16) : fill.y);
}
__device__ __forceinline__ unsigned pack2(float2 x) {
  __nv_bfloat162 t = __floats2bfloat162_rn(x.x, x.y);
  return *reinterpret_cast<unsigned*>(&t);
}
__device__ __forceinline__ void put(float* p, bool, int64_t, const float2 (&x)[2]) { __stcs(reinterpret_cast<float4*>(p), make_float4(x[0].x, x[0].y, x[1].x, x[1].y)); }
__device__ __forceinline__ void put(__nv_bfloat16* p, bool, int64_t, const float2 (&x)[4]) {
  __stcs(reinterpret_cast<uint4*>(p), make_uint4(pack2(x[0]), pack2(x[1]), pack2(x[2]), pack2(x[3])));
}
__device__ __forceinline__ void put(float* p, bool second, int64_t step, const float2 (&x)[1]) {
  __stcs(p, x[0].x);
  if (second) __stcs(p + step, x[0].y);
}
__device__ __forceinline__ void put(__nv_bfloat16* p, bool second, int64_t step, const float2 (&x)[1]) {
  *p = __float2bfloat16_rn(x[0].x);
  if (second) p[step] = __float2bfloat16_rn(x[0].y);
}
// a channel's value for pair j, from per-channel reads: f(v) for channel v of the column
template <int V, typename F>
__device__ __forceinline__ void per_channel(float2 (&x)[kPairs<V>], F f) {
  if constexpr (V == 1) {
    const float t = f(0);
    x[0] = make_float2(t, t);
  } else {
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
      x[j].x = f(2 * j);
      x[j].y = f(2 * j + 1);
    }
  }
}

// ... from an array in shared memory with an entry per channel (p: the column's first)
__device__ __forceinline__ void channels(const float* p, float2 (&x)[4]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  x[0] = make_float2(a.x, a.y); x[1] = make_float2(a.z, a.w); x[2] = make_float2(b.x, b.y); x[3] = make_float2(b.z, b.w);
}
__device__ __forceinline__ void channels(const float* p, float2 (&x)[2]) {
  const float4 a = *reinterpret_cast<const float4*>(p);
  x[0] = make_float2(a.x, a.y); x[1] = make_float2(a.z, a.w);
}
__device__ __forceinline__ void channels(const float* p, float2 (&x)[1]) { x[0] = two(*p); }
__device__ __forceinline__ void to_channels(float* p, const float2 (&x)[4]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0].x, x[0].y, x[1].x, x[1].y);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[2].x, x[2].y, x[3].x, x[3].y);
}
__device__ __forceinline__ void to_channels(float* p, const float2 (&x)[2]) { *reinterpret_cast<float4*>(p) = make_float4(x[0].x, x[0].y, x[1].x, x[1].y); }
__device__ __forceinline__ void to_channels(float* p, const float2 (&x)[1]) { *p = x[0].x + x[0].y; }
// ... from one with an entry per group; `one`: the whole column lies in group g
template <int V>
__device__ __forceinline__ void groups_of(const float* p, int g, int rem, int cpg, bool one, float2 (&x)[kPairs<V>]) {
  if (one) {
    const float t = p[g];
#pragma unroll
    for (int j = 0; j < kPairs<V>; ++j) x[j] = two(t);
  } else if ((cpg & 1) == 0) {      // a pair's channels share a group
#pragma unroll
    for (int j = 0; j < kPairs<V>; ++j) {
      x[j] = two(p[g]);
      if ((rem += 2) == cpg) { rem = 0; ++g; }
    }
  } else {
    per_channel<V>(x, [&](int) {
      const float t = p[g];
      if (++rem == cpg) { rem = 0; ++g; }
      return t;
    });
  }
}

// One element or column into the thread's own slot. Two bytes are below what an asynchronous copy takes.
__device__ __forceinline__ void bring(uint4* slot, const void* p) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16;" ::"r"((unsigned)__cvta_generic_to_shared(slot)), "l"(p));
}
__device__ __forceinline__ void bring(unsigned* slot, const void* p) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"((unsigned)__cvta_generic_to_shared(slot)), "l"(p));
}
__device__ __forceinline__ void bring(unsigned short* slot, const void* p) { *slot = __ldcs(static_cast<const unsigned short*>(p)); }
__device__ __forceinline__ void bring_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// The arrays in shared memory start on 16 bytes, whatever their length.
__host__ __device__ constexpr int padded(int n) { return (n + 3) & ~3; }

// RESIDENT: the whole job, the CTAs of an image's slab being one cluster. STATS: the chunks' sums only.
// APPLY: the results, from the chunks' sums.
enum Mode { RESIDENT, STATS, APPLY };

// Threads per CTA and CTAs per SM the registers are cut for. Resident: every warp repeats what a slab costs besides its data, so
// few warps with much data each, and unrolled loops in place of more warps (backward on 64 x 56x56 x 256 bf16 with SiLU:
// 256 threads 145 us, 128 threads 120 us, and 104 us with the registers of two CTAs per SM instead of three; where the
// slope is cheap three are better, 114 against 125 us on 1024 x 32x32 x 64). The chunked modes stream: 256 threads.
constexpr int kResidentThreads = 128, kChunkThreads = 256;
template <int V, Mode M>
constexpr int kMostThreads = V == 1 ? 1024 : M == RESIDENT ? kResidentThreads : kChunkThreads;
template <int V, Mode M, int ACT>
constexpr int kCtas = V == 1 ? 1 : M != RESIDENT || ACT == DMX_ACT_SILU || ACT == DMX_ACT_GELU ? 2 : 3;

// Forward: four for fp32, whose columns take half the registers (1024 x 8x8 x 64 with SiLU: 8.3 us, with three 10.4 us).
template <int V, Mode M>
constexpr int kForwardCtas = V == 1 ? 1 : M != RESIDENT ? 2 : V == 4 ? 4 : 3;

// A CTA's place in one item, and a thread's in that.
struct Here {
  int n, part, c0, g0, Wl, groups, rows, r0;
  int cnt;               // positions of this thread
  bool on;               // its column exists
};
template <int V, Mode M>
__device__ __forceinline__ Here place(const Args& A, int64_t item, int rl, int col) {
  Here h;
  unsigned b = (unsigned)item;
  if constexpr (M == RESIDENT) {
    h.part = A.parts > 1 ? blockIdx.x & (A.parts - 1) : 0;   // a power of two
  } else {
    h.part = b % (unsigned)A.parts;
    b /= (unsigned)A.parts;
  }
  const int slab = A.slabs > 1 ? b % (unsigned)A.slabs : 0;
  h.n = A.slabs > 1 ? b / (unsigned)A.slabs : b;
  h.c0 = slab * A.W;
  h.g0 = slab * A.gW;
  h.Wl = min(A.W, A.C - h.c0);
  h.groups = min(A.gW, A.G - h.g0);
  h.r0 = min((int64_t)h.part * A.rows, (int64_t)A.L);
  h.rows = min(A.rows, A.L - h.r0);
  h.on = rl < A.R && col * V < h.Wl;
  h.cnt = h.on && rl < h.rows ? (h.rows - rl + A.R - 1) / A.R : 0;
  return h;
}
template <typename T, int V>
__device__ __forceinline__ T* start(const Operand& o, const Here& h, int rl, int col) {
  return static_cast<T*>(o.p) + h.n * o.image + (int64_t)(h.r0 + rl) * o.row + h.c0 + col * V;
}

__device__ __forceinline__ int lanes_for(int total) {
  return total >= 32 ? 32 : total <= 1 ? 1 : 1 << (32 - __clz(total - 1));
}
// Sums over groups of an array [R][width], `per` neighbouring entries of a row being a group's. `each` lanes (a
// power of two) take a group, in a fixed order; they all get its sum.
struct Lanes {
  int each, l, g1, gstep;      // lane within the group, group within a round, groups per round
  int R, per, width, i0, r0, c0, dr, dc;
};
__device__ __forceinline__ Lanes lanes(int R, int per, int width) {
  Lanes q;
  q.each = lanes_for(R * per);
  q.l = threadIdx.x & (q.each - 1);
  const int sh = 31 - __clz(q.each);
  q.g1 = threadIdx.x >> sh;
  q.gstep = blockDim.x >> sh;
  q.R = R; q.per = per; q.width = width;
  q.r0 = q.l / per;
  q.c0 = q.l - q.r0 * per;
  q.dr = q.each / per;
  q.dc = q.each - q.dr * per;
  return q;
}
template <typename F>
__device__ __forceinline__ float lane_sum(const Lanes& q, bool on, int g, F term) {    // term(i, r, c): entry i = r*width + c
  float s = 0.f;
  if (on) {
    int r = q.r0, c = q.c0;
    while (r < q.R) {
      const int at = g * q.per + c;
      s += term(r * q.width + at, r, at);
      r += q.dr;
      c += q.dc;
      if (c >= q.per) { c -= q.per; ++r; }
    }
  }
  for (int o = q.each >> 1; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}

// ... of two terms at once
template <typename F>
__device__ __forceinline__ float2 lane_sums(const Lanes& q, bool on, int g, F term) {
  float2 s = make_float2(0.f, 0.f);
  if (on) {
    int r = q.r0, c = q.c0;
    while (r < q.R) {
      const int at = g * q.per + c;
      s = add2(s, term(r * q.width + at, r));
      r += q.dr;
      c += q.dc;
      if (c >= q.per) { c -= q.per; ++r; }
    }
  }
  for (int o = q.each >> 1; o > 0; o >>= 1) s = add2(s, make_float2(__shfl_xor_sync(0xffffffffu, s.x, o), __shfl_xor_sync(0xffffffffu, s.y, o)));
  return s;
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
// into the same place of another CTA's shared memory
__device__ __forceinline__ void send(float* p, int rank, float v) {
  unsigned a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((unsigned)__cvta_generic_to_shared(p)), "r"(rank));
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(a), "f"(v) : "memory");
}
// weight and bias of an item's channels and, backward, its groups' statistics, into shared memory beside the data
struct Params {
  float *w, *b, *mean, *rstd;
};
__device__ __forceinline__ Params params_at(float* base, int W, int groups) {
  Params p;
  p.w = base;
  p.b = p.w + padded(W);
  p.mean = p.b + padded(W);
  p.rstd = p.mean + padded(groups);
  return p;
}
__host__ __device__ constexpr int params_size(int W, int groups) { return 2 * padded(W) + 2 * padded(groups); }
template <bool STATISTICS>
__device__ __forceinline__ void bring_params(const Args& A, const Here& h, const Params& p) {
  for (int c = threadIdx.x; c < h.Wl; c += blockDim.x) {
    if (A.weight) bring(reinterpret_cast<unsigned*>(p.w + c), A.weight + h.c0 + c);
    else p.w[c] = 1.f;
    if (A.bias) bring(reinterpret_cast<unsigned*>(p.b + c), A.bias + h.c0 + c);
    else p.b[c] = 0.f;
  }
  if (STATISTICS)
    for (int g = threadIdx.x; g < h.groups; g += blockDim.x) {
      const int64_t at = (int64_t)h.n * A.G + h.g0 + g;
      bring(reinterpret_cast<unsigned*>(p.mean + g), A.mean + at);
      bring(reinterpret_cast<unsigned*>(p.rstd + g), A.rstd + at);
    }
}

// A mean and what its rounding to a float lost. The sum of n values' deviations from a rough mean is c = n times what the rough one
// lacks, that of their squares m2' = m2 + c^2/n.
struct Mean {
  float hi, lo;
};
__device__ __forceinline__ Mean corrected(float rough, float by) {
  by = fabsf(by) <= FLT_MAX ? by : 0.f;             // (an infinite mean stays infinite)
  const float hi = rough + by;
  return {hi, (rough - hi) + by};
}
__device__ __forceinline__ float squares(float m2, float c, float by) { return dmx_act::relu(fmaf(-c, by, m2)); }   // by = c/n; a NaN stays one

// Over `lanes` lanes: parts' means, squared deviations pm and `have` positions of cpg values each -> the mean and variance
// of all L positions.
__device__ __forceinline__ float2 join(Mean part, float pm, float have, float cpg, float L, int lanes) {
  float rough = have > 0.f ? part.hi * have : 0.f;
  for (int o = lanes >> 1; o > 0; o >>= 1) rough += __shfl_xor_sync(0xffffffffu, rough, o);
  rough /= L;
  const float d = have > 0.f ? (part.hi - rough) + part.lo : 0.f;
  float2 s = make_float2(have * d, have > 0.f ? fmaf(have * cpg * d, d, pm) : 0.f);
  for (int o = lanes >> 1; o > 0; o >>= 1) s = add2(s, make_float2(__shfl_xor_sync(0xffffffffu, s.x, o), __shfl_xor_sync(0xffffffffu, s.y, o)));
  const float by = s.x / L;
  return make_float2(corrected(rough, by).hi, squares(s.y, s.x * cpg, by) / (L * cpg));
}

template <typename T, int V, Mode M, int ACT>
__global__ void __launch_bounds__(kMostThreads<V, M>, kForwardCtas<V, M>) forward_kernel(const __grid_constant__ Args A) {
  using U = typename Vec<T, V>::type;
  constexpr int NP = kPairs<V>, SL = kSlots<V>;
  extern __shared__ __align__(16) float sm[];
  const int W = A.W, cpg = A.cpg, R = A.R, threads = blockDim.x;
  const int tid = threadIdx.x, rl = tid / A.cols, col = tid - rl * A.cols;
  // entries: per column V/fold values; rows of them: the warps where a warp's lanes can be added up, else all R
  const int vals = V / A.fold, width = A.cols * vals, per = cpg / A.fold;
  const int rows = A.lanes ? threads >> 5 : R;
  U* slot = reinterpret_cast<U*>(sm) + tid;
  float* emean = sm + (size_t)A.slots * threads * sizeof(U) / sizeof(float);
  float* elo = emean + padded(rows * width);
  float* em2 = elo + padded(rows * width);
  float* en = em2 + padded(rows * width);
  // per group: every part's mean (two floats) and squared deviations, in turn for one item and the next (the cluster's CTAs write to
  // one another's: whoever writes for an item has seen all others' sums of the item before, so the buffer of two
  // items ago is free); then mean and rstd
  const int pG = padded(A.gW), gparts = M == RESIDENT ? A.parts : 1;
  float* got = en + padded(rows);
  float* gmean = got + 6 * gparts * pG;
  float* grstd = gmean + pG;
  float* par = grstd + pG;
  int turn = 0;
  const Lanes Q = lanes(rows, per, width);
  int grp0 = 0, rem0 = 0;                          // group of the column's first channel, and its place there
  if (rl < R) { grp0 = col * V / cpg; rem0 = col * V - grp0 * cpg; }

  const int64_t first = M == RESIDENT ? blockIdx.x / (unsigned)A.parts : blockIdx.x;
  const int64_t stride = M == RESIDENT ? gridDim.x / (unsigned)A.parts : gridDim.x;
  if (first >= A.items) return;                    // the whole cluster
  asm volatile("griddepcontrol.launch_dependents;\n\tgriddepcontrol.wait;" ::: "memory");
  Here h = place<V, M>(A, first, rl, col);
  {
    const T* p = start<T, V>(A.x, h, rl, col);
    for (int i = 0; i < h.cnt; ++i) bring(slot + i * threads, p + (int64_t)i * R * A.x.row);
    if (M != STATS) bring_params<M == APPLY>(A, h, params_at(par, W, A.gW));
  }
  if (M == RESIDENT && A.parts > 1) cluster_sync();      // all of the cluster runs: its memory may be written
  for (int64_t item = first; item < A.items; item += stride) {
    const Params P = params_at(par + turn * params_size(W, A.gW), W, A.gW);
    float* mine = got + turn * 3 * gparts * pG;
    if constexpr (M != APPLY) {
      bring_wait();
      float2 p0[NP], ps[NP], pq[NP];
#pragma unroll
      for (int j = 0; j < NP; ++j) p0[j] = ps[j] = pq[j] = two(0.f);
      if (h.cnt > 0) widen(slot, false, 0, two(0.f), p0);
      if (V == 1) p0[0].y = p0[0].x;
#pragma unroll 4
      for (int i = 0; i < h.cnt; i += SL) {
        float2 x[NP];
        widen(slot + i * threads, i + 1 < h.cnt, threads, p0[0], x);
#pragma unroll
        for (int j = 0; j < NP; ++j) {
          const float2 d = sub2(x[j], p0[j]);
          ps[j] = add2(ps[j], d);
          pq[j] = fma2(d, d, pq[j]);
        }
      }
      float x0[V], s[V], q[V], lo[V];
      if constexpr (V == 1) {
        x0[0] = p0[0].x; s[0] = ps[0].x + ps[0].y; q[0] = pq[0].x + pq[0].y;
      } else {
#pragma unroll
        for (int j = 0; j < NP; ++j) {
          x0[2 * j] = p0[j].x; x0[2 * j + 1] = p0[j].y;
          s[2 * j] = ps[j].x; s[2 * j + 1] = ps[j].y;
          q[2 * j] = pq[j].x; q[2 * j + 1] = pq[j].y;
        }
      }
      // per value: mean and squared deviations of this thread's n entries, neighbours joined while they share a group
      float n = (float)h.cnt;
      const float inv = h.cnt > 0 ? __frcp_rn(n) : 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float d = s[v] * inv;
        q[v] = fmaxf(fmaf(-s[v], d, q[v]), 0.f) + 0.f * d;      // (a NaN or infinity stays one)
        s[v] = x0[v] + d;
        lo[v] = (x0[v] - s[v]) + d;
      }
#pragma unroll
      for (int f = 1; f < V; f *= 2) {
        if (A.fold <= f) break;
#pragma unroll
        for (int j = 0; j < V / (2 * f); ++j) {
          const float b = s[2 * j + 1], d = (s[2 * j] - b) + (lo[2 * j] - lo[2 * j + 1]);
          q[j] = q[2 * j] + q[2 * j + 1] + 0.5f * n * d * d;
          s[j] = b + 0.5f * d;
          lo[j] = ((b - s[j]) + 0.5f * d) + lo[2 * j + 1];
        }
        n *= 2.f;
      }
      if (A.lanes) {                               // lanes that hold the same column
        float N = n;
        for (int o = A.lanes; o < 32; o <<= 1) N += __shfl_xor_sync(0xffffffffu, N, o);
        const float iN = N > 0.f ? __frcp_rn(N) : 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
          if (j >= vals) break;
          float t = s[j] * n;
          for (int o = A.lanes; o < 32; o <<= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
          t *= iN;
          const float d = n > 0.f ? (s[j] - t) + lo[j] : 0.f;
          float2 c = make_float2(n * d, n > 0.f ? fmaf(n * d, d, q[j]) : 0.f);
          for (int o = A.lanes; o < 32; o <<= 1) c = add2(c, make_float2(__shfl_xor_sync(0xffffffffu, c.x, o), __shfl_xor_sync(0xffffffffu, c.y, o)));
          const float by = c.x * iN;
          const Mean mean = corrected(t, by);
          s[j] = mean.hi; lo[j] = mean.lo; q[j] = squares(c.y, c.x, by);
        }
        const int lane = tid & 31, wid = tid >> 5;
        if (lane < A.lanes) {
#pragma unroll
          for (int j = 0; j < V; ++j) {
            if (j >= vals) break;
            emean[wid * width + col * vals + j] = s[j];
            elo[wid * width + col * vals + j] = lo[j];
            em2[wid * width + col * vals + j] = q[j];
          }
          if (lane == 0) en[wid] = N;
        }
      } else if (rl < R) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          if (j >= vals) break;
          emean[rl * width + col * vals + j] = s[j];
          elo[rl * width + col * vals + j] = lo[j];
          em2[rl * width + col * vals + j] = q[j];
        }
        if (col == 0) en[rl] = n;
      }
      __syncthreads();
      const float cnt = (float)h.rows * (float)cpg, icnt = h.rows > 0 ? 1.f / cnt : 0.f;
      for (int gb = 0; gb < h.groups; gb += Q.gstep) {
        const int g = gb + Q.g1;
        const bool mineg = g < h.groups;
        const float sum = lane_sum(Q, mineg, g, [&](int i, int r, int) { return en[r] > 0.f ? emean[i] * en[r] : 0.f; });
        const float rough = sum * icnt;
        const float2 c = lane_sums(Q, mineg, g, [&](int i, int r) {
          const float d = (emean[i] - rough) + elo[i];
          return en[r] > 0.f ? make_float2(en[r] * d, fmaf(en[r] * d, d, em2[i])) : make_float2(0.f, 0.f);
        });
        const Mean mean = corrected(rough, c.x * icnt);
        const float m2 = squares(c.y, c.x, c.x * icnt);
        if (M == STATS) {
          if (mineg && Q.l == 0) {
            float* to = A.part + 3 * (((int64_t)h.n * A.parts + h.part) * A.G + h.g0 + g);
            to[0] = mean.hi; to[1] = mean.lo; to[2] = m2;
          }
        } else if (A.parts > 1) {
          if (mineg)
            for (int k = Q.l; k < 3 * A.parts; k += Q.each) {
              const int to = k / 3, which = k - 3 * to;
              send(mine + (3 * h.part + which) * pG + g, to, which == 0 ? mean.hi : which == 1 ? mean.lo : m2);
            }
        } else if (mineg && Q.l == 0) {              // nothing to join
          const float rstd = 1.f / sqrtf(m2 * icnt + A.eps);
          gmean[g] = mean.hi;
          grstd[g] = rstd;
          A.mean[(int64_t)h.n * A.G + h.g0 + g] = mean.hi;
          A.rstd[(int64_t)h.n * A.G + h.g0 + g] = rstd;
        }
      }
      if (M == RESIDENT && A.parts > 1) cluster_arrive();
    }
    // the next item's place and parameters, while the others arrive
    const Here now = h;
    const int64_t next = item + stride;
    const T* np = nullptr;
    int ncnt = 0;
    if (next < A.items) {
      h = place<V, M>(A, next, rl, col);
      np = start<T, V>(A.x, h, rl, col);
      ncnt = h.cnt;
      if (M != STATS) bring_params<M == APPLY>(A, h, params_at(par + (turn ^ 1) * params_size(W, A.gW), W, A.gW));
    }
    turn ^= 1;
    if constexpr (M != APPLY) {
      if (M == RESIDENT && A.parts > 1) cluster_wait();
      else __syncthreads();
    }
    if (M == APPLY || (M == RESIDENT && A.parts > 1)) {
      if constexpr (M == RESIDENT) {
        // join the parts of each group: a lane per part, added in a fixed order
        const int kl = lanes_for(A.parts), k0 = tid & (kl - 1);
        const int64_t gat = (int64_t)now.n * A.G + now.g0;
        for (int gb = 0; gb < now.groups; gb += threads / kl) {
          const int g = gb + tid / kl;
          const float have = (float)(min((int64_t)(k0 + 1) * A.rows, (int64_t)A.L) - min((int64_t)k0 * A.rows, (int64_t)A.L));
          Mean part = {0.f, 0.f};
          float pm = 0.f;
          if (g < now.groups) {
            part = {mine[3 * k0 * pG + g], mine[(3 * k0 + 1) * pG + g]};
            pm = mine[(3 * k0 + 2) * pG + g];
          }
          float2 t = join(part, pm, have, (float)cpg, (float)A.L, kl);
          if (g < now.groups && k0 == 0) {
            t.y = 1.f / sqrtf(t.y + A.eps);
            gmean[g] = t.x;
            grstd[g] = t.y;
            if (now.part == 0) {
              A.mean[gat + g] = t.x;
              A.rstd[gat + g] = t.y;
            }
          }
        }
      }
      if (M == APPLY) bring_wait();          // (the others have waited for their copies above)
      __syncthreads();
    }
    // results, each slot refilled for the next item behind its last use
    const int64_t in_step = (int64_t)R * A.x.row;
    if constexpr (M != STATS) {
      float2 mu[NP], a[NP], b[NP];
      if (now.on) {
        groups_of<V>(M == APPLY ? P.mean : gmean, grp0, rem0, cpg, A.fold == V, mu);
        groups_of<V>(M == APPLY ? P.rstd : grstd, grp0, rem0, cpg, A.fold == V, a);
        channels(P.w + col * V, b);
#pragma unroll
        for (int j = 0; j < NP; ++j) a[j] = mul2(a[j], b[j]);
        channels(P.b + col * V, b);
      }
      T* out = start<T, V>(A.out, now, rl, col);
      const int64_t out_step = (int64_t)R * A.out.row;
#pragma unroll 4
      for (int i = 0; i < now.cnt; i += SL) {
        float2 x[NP];
        const bool second = i + 1 < now.cnt;
        widen(slot + i * threads, second, threads, two(0.f), x);
#pragma unroll
        for (int j = 0; j < NP; ++j) x[j] = dmx_act::apply<ACT>(fma2(sub2(x[j], mu[j]), a[j], b[j]));
        put(out, second, out_step, x);
        out += SL * out_step;
#pragma unroll
        for (int k = 0; k < SL; ++k)
          if (i + k < ncnt) { bring(slot + (i + k) * threads, np); np += in_step; }
      }
      for (int i = (now.cnt + SL - 1) / SL * SL; i < ncnt; ++i) { bring(slot + i * threads, np); np += in_step; }
      if (M == APPLY) __syncthreads();                         // (the other modes pass a barrier before they write means)
    } else {
      for (int i = 0; i < ncnt; ++i) { bring(slot + i * threads, np); np += in_step; }
    }
  }
}

// du = dy act'(u) is kept between the two sweeps of a resident backward pass where it costs an exponential and fits where dy
// was: in fp32. (For bf16, 32 bytes more per slot of eight made the slabs narrower, and cost more than they saved.)
template <typename T>
__host__ __device__ constexpr bool keeps(int act) { return (act == DMX_ACT_SILU || act == DMX_ACT_GELU) && sizeof(T) == 4; }
__device__ __forceinline__ void keep(uint4* g, bool, int, const float2 (&x)[2]) {
  *g = make_uint4(__float_as_uint(x[0].x), __float_as_uint(x[0].y), __float_as_uint(x[1].x), __float_as_uint(x[1].y));
}
__device__ __forceinline__ void keep(unsigned* g, bool second, int step, const float2 (&x)[1]) {
  *g = __float_as_uint(x[0].x);
  if (second) g[step] = __float_as_uint(x[0].y);
}

// Backward. Workspace: A and B per image (and chunk) and channel, [2][N*chunks][C].
template <typename T, int V, Mode M, int ACT>
__global__ void __launch_bounds__(kMostThreads<V, M>, kCtas<V, M, ACT>) backward_kernel(const __grid_constant__ Args A) {
  using U = typename Vec<T, V>::type;
  constexpr int NP = kPairs<V>, SL = kSlots<V>;
  extern __shared__ __align__(16) float sm[];
  const int W = A.W, cpg = A.cpg, R = A.R, threads = blockDim.x;
  const int tid = threadIdx.x, rl = tid / A.cols, col = tid - rl * A.cols;
  const int rows = A.lanes ? threads >> 5 : R;
  U* xs = reinterpret_cast<U*>(sm) + tid;
  U* gs = xs + (size_t)A.slots * threads;
  constexpr bool KEEP = M == RESIDENT && keeps<T>(ACT);
  const size_t ends = (size_t)2 * A.slots * threads * sizeof(U);
  float* red = reinterpret_cast<float*>(reinterpret_cast<char*>(sm) + ends);     // rows of A, rows of B
  // every part's channel sums A, B, in turn as in the forward kernel; then per group the two factors that the
  // sums of w A and w B give
  const int pW = padded(W), pG = padded(A.gW), gparts = M == RESIDENT ? A.parts : 1;
  float* got = red + padded(2 * rows * W);
  float* grp = got + 4 * gparts * pW;
  float* par = grp + 2 * pG;
  int turn = 0;
  const Lanes Q = lanes(gparts, cpg, 2 * pW);
  int grp0 = 0, rem0 = 0;
  if (rl < R) { grp0 = col * V / cpg; rem0 = col * V - grp0 * cpg; }
  const int64_t plane = (int64_t)A.N * (M == RESIDENT ? 1 : A.parts) * A.C;

  const int64_t first = M == RESIDENT ? blockIdx.x / (unsigned)A.parts : blockIdx.x;
  const int64_t stride = M == RESIDENT ? gridDim.x / (unsigned)A.parts : gridDim.x;
  if (first >= A.items) return;
  asm volatile("griddepcontrol.launch_dependents;\n\tgriddepcontrol.wait;" ::: "memory");
  Here h = place<V, M>(A, first, rl, col);
  {
    const T *p = start<T, V>(A.x, h, rl, col), *g = start<T, V>(A.dy, h, rl, col);
    for (int i = 0; i < h.cnt; ++i) {
      bring(xs + i * threads, p + (int64_t)i * R * A.x.row);
      bring(gs + i * threads, g + (int64_t)i * R * A.dy.row);
    }
    bring_params<true>(A, h, params_at(par, W, A.gW));
  }
  if (M == RESIDENT && A.parts > 1) cluster_sync();      // all of the cluster runs: its memory may be written
  for (int64_t item = first; item < A.items; item += stride) {
    const Params P = params_at(par + turn * params_size(W, A.gW), W, A.gW);
    float* mine = got + turn * 2 * gparts * pW;
    bring_wait();
    __syncthreads();                 // the parameters are other threads' copies
    // u = (x - mu) a + b with a = rstd weight
    float2 mu[NP], a[NP], b[NP];
    if (h.on) {
      groups_of<V>(P.mean, grp0, rem0, cpg, A.fold == V, mu);
      groups_of<V>(P.rstd, grp0, rem0, cpg, A.fold == V, a);
      channels(P.w + col * V, b);
#pragma unroll
      for (int j = 0; j < NP; ++j) a[j] = mul2(a[j], b[j]);
      channels(P.b + col * V, b);
    }
    if constexpr (M != APPLY) {
      float2 pa[NP], pb[NP];
#pragma unroll
      for (int j = 0; j < NP; ++j) pa[j] = pb[j] = two(0.f);
#pragma unroll 4
      for (int i = 0; i < h.cnt; i += SL) {
        float2 x[NP], g[NP];
        widen(xs + i * threads, i + 1 < h.cnt, threads, mu[0], x);
        widen(gs + i * threads, i + 1 < h.cnt, threads, two(0.f), g);
#pragma unroll
        for (int j = 0; j < NP; ++j) {
          x[j] = sub2(x[j], mu[j]);
          g[j] = dmx_act::times_slope<ACT>(g[j], fma2(x[j], a[j], b[j]));
          pa[j] = fma2(g[j], x[j], pa[j]);
          pb[j] = add2(pb[j], g[j]);
        }
        if constexpr (KEEP) keep(gs + i * threads, i + 1 < h.cnt, threads, g);
      }
      // (the sums of A without their factor rstd)
      const int lane = tid & 31, row = A.lanes ? tid >> 5 : rl;
      if (A.lanes)
        for (int o = A.lanes; o < 32; o <<= 1)
#pragma unroll
          for (int j = 0; j < NP; ++j) {
            pa[j] = add2(pa[j], make_float2(__shfl_xor_sync(0xffffffffu, pa[j].x, o), __shfl_xor_sync(0xffffffffu, pa[j].y, o)));
            pb[j] = add2(pb[j], make_float2(__shfl_xor_sync(0xffffffffu, pb[j].x, o), __shfl_xor_sync(0xffffffffu, pb[j].y, o)));
          }
      if (A.lanes ? lane < A.lanes : rl < R) {
        to_channels(red + row * W + col * V, pa);
        to_channels(red + (rows + row) * W + col * V, pb);
      }
      __syncthreads();
      for (int c = tid; c < 2 * W; c += threads) {
        const int k = c < W ? c : c - W;
        const float* p = red + (c < W ? 0 : rows * W) + k;
        float t = 0.f;
#pragma unroll 8
        for (int r = 0; r < rows; ++r) t += p[r * W];
        if (M == STATS) {
          if (k < h.Wl) A.part[(c < W ? 0 : plane) + ((int64_t)h.n * A.parts + h.part) * A.C + h.c0 + k] = t;
        } else if (A.parts > 1) {
          for (int q = 0; q < A.parts; ++q) send(mine + (2 * h.part + (c < W ? 0 : 1)) * pW + k, q, t);
        } else {
          mine[(c < W ? 0 : pW) + k] = t;
        }
      }
      if (M == RESIDENT && A.parts > 1) cluster_arrive();
    }
    // the next item's place and parameters, while the others arrive
    const Here now = h;
    const int64_t next = item + stride;
    const T *nx = nullptr, *ng = nullptr;
    int ncnt = 0;
    if (next < A.items) {
      h = place<V, M>(A, next, rl, col);
      nx = start<T, V>(A.x, h, rl, col);
      ng = start<T, V>(A.dy, h, rl, col);
      ncnt = h.cnt;
      bring_params<true>(A, h, params_at(par + (turn ^ 1) * params_size(W, A.gW), W, A.gW));
    }
    turn ^= 1;
    if constexpr (M != APPLY) {
      if (M == RESIDENT && A.parts > 1) cluster_wait();
      else __syncthreads();
    }
    if constexpr (M == APPLY) {      // the image's sums
      for (int c = tid; c < 2 * W; c += threads) {
        const int k = c < W ? c : c - W;
        if (k < now.Wl) mine[(c < W ? 0 : pW) + k] = A.part[2 * plane + ((c < W ? 0 : (int64_t)A.N) + now.n) * A.C + now.c0 + k];
      }
      __syncthreads();
    }
    if constexpr (M != STATS) {
      // the groups' weighted sums over parts and channels: rows 2k (A) and 2k + 1 (B) are part k's
      for (int gb = 0; gb < now.groups; gb += Q.gstep) {
        const int g = gb + Q.g1;
        const bool mineg = g < now.groups;
        const float ta = lane_sum(Q, mineg, g, [&](int i, int, int c) { return mine[i] * P.w[c]; });
        const float tb = lane_sum(Q, mineg, g, [&](int i, int, int c) { return mine[i + pW] * P.w[c]; });
        if (mineg && Q.l == 0) {
          const float r = P.rstd[g], n = -1.f / ((float)A.L * (float)cpg);
          grp[g] = ta * n * r * r * r;
          grp[pG + g] = tb * n * r;
        }
      }
      __syncthreads();
      if (M == RESIDENT && now.part == 0)          // what dweight and dbias are summed from
        for (int c = tid; c < 2 * W; c += threads) {
          const int k = c < W ? c : c - W;
          float t = 0.f;
          for (int q = 0; q < gparts; ++q) t += mine[(2 * q + (c < W ? 0 : 1)) * pW + k];
          if (k < now.Wl) A.part[(c < W ? 0 : plane) + (int64_t)now.n * A.C + now.c0 + k] = t;
        }
    }
    const int64_t xstep = (int64_t)R * A.x.row, gstep2 = (int64_t)R * A.dy.row;
    if constexpr (M != STATS) {
      // the sums A lack their factor rstd: dx = a du - rstd s1 / n - (x - mu) rstd^3 s2 / n
      float2 k1[NP], k2[NP];
      if (now.on) {
        groups_of<V>(grp + pG, grp0, rem0, cpg, A.fold == V, k1);
        groups_of<V>(grp, grp0, rem0, cpg, A.fold == V, k2);
      }
      T* out = start<T, V>(A.out, now, rl, col);
      const int64_t out_step = (int64_t)R * A.out.row;
#pragma unroll 4
      for (int i = 0; i < now.cnt; i += SL) {
        float2 x[NP], gr[NP];
        const bool second = i + 1 < now.cnt;
        widen(xs + i * threads, second, threads, mu[0], x);
        widen(gs + i * threads, second, threads, two(0.f), gr);
#pragma unroll
        for (int j = 0; j < NP; ++j) {
          x[j] = sub2(x[j], mu[j]);
          if constexpr (!KEEP) gr[j] = dmx_act::times_slope<ACT>(gr[j], fma2(x[j], a[j], b[j]));
          x[j] = fma2(gr[j], a[j], fma2(x[j], k2[j], k1[j]));
        }
        put(out, second, out_step, x);
        out += SL * out_step;
#pragma unroll
        for (int k = 0; k < SL; ++k)
          if (i + k < ncnt) {
            bring(xs + (i + k) * threads, nx);
            bring(gs + (i + k) * threads, ng);
            nx += xstep; ng += gstep2;
          }
      }
    }
    for (int i = M == STATS ? 0 : (now.cnt + SL - 1) / SL * SL; i < ncnt; ++i) {
      bring(xs + i * threads, nx);
      bring(gs + i * threads, ng);
      nx += xstep; ng += gstep2;
    }
  }
}

// The chunks' sums of an image, joined between the two launches that read it. Forward: a warp per image and group.
__global__ void __launch_bounds__(256) join_groups_kernel(const float* part, int64_t groups, int parts, int rows, int L, int G, int cpg,
                                                          float eps, float* mean, float* rstd) {
  asm volatile("griddepcontrol.launch_dependents;\n\tgriddepcontrol.wait;" ::: "memory");
  const int64_t i = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);       // image * G + group
  const int lane = threadIdx.x & 31;
  if (i >= groups) return;
  const float* src = part + 3 * (i / G * parts * G + i % G);
  auto positions = [&](int k) { return (float)(min((int64_t)(k + 1) * rows, (int64_t)L) - (int64_t)k * rows); };
  // 32nd parts by lane: each lane joins its own first
  float sum = 0.f, have = 0.f;
  for (int k = lane; k < parts; k += 32) {
    sum = fmaf(src[(int64_t)k * 3 * G], positions(k), sum);
    have += positions(k);
  }
  const float mu = have > 0.f ? sum / have : 0.f;
  float c = 0.f, m2 = 0.f;
  for (int k = lane; k < parts; k += 32) {
    const float* p = src + (int64_t)k * 3 * G;
    const float n = positions(k), d = (p[0] - mu) + p[1];
    c = fmaf(n, d, c);
    m2 += fmaf(n * (float)cpg * d, d, p[2]);
  }
  const float by = have > 0.f ? c / have : 0.f;
  const float2 t = join(corrected(mu, by), squares(m2, c * (float)cpg, by), have, (float)cpg, (float)L, 32);
  if (lane == 0) {
    mean[i] = t.x;
    rstd[i] = 1.f / sqrtf(t.y + eps);
  }
}
// Backward: the rows of an image's chunks to one row, for A and for B. 32 channels and eight row lanes per CTA.
__global__ void __launch_bounds__(256) join_rows_kernel(const float* part, float* out, int N, int parts, int C) {
  __shared__ float sh[8][33];
  asm volatile("griddepcontrol.launch_dependents;\n\tgriddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31, r = threadIdx.x >> 5, blocks = (C + 31) / 32;
  const int64_t row = blockIdx.x / blocks;                               // [2][N]
  const int c = (blockIdx.x % blocks) * 32 + lane;
  float s = 0.f;
  if (c < C) {
    const float* p = part + row * parts * C + c;
#pragma unroll 8
    for (int i = r; i < parts; i += 8) s += p[(int64_t)i * C];
  }
  sh[r][lane] = s;
  __syncthreads();
  if (r == 0 && c < C) {
    for (int k = 1; k < 8; ++k) s += sh[k][lane];
    out[row * C + c] = s;
  }
}

// dweight and dbias: sums of the images' rows, those of A times their group's rstd. 32 channels and 32 row lanes per CTA.
__global__ void __launch_bounds__(1024) columns_kernel(const float* part, int64_t rows, int C, int G, int cpg,
                                                      const float* rstd, float* dw, float* db) {
  __shared__ float sh[32][33];
  const int lane = threadIdx.x & 31, r = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  const float* p = part + (int64_t)blockIdx.y * rows * C;
  float* out = blockIdx.y ? db : dw;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (!out) return;
  float s = 0.f;
  if (c < C) {
    const float* q = rstd + c / cpg;
    if (blockIdx.y) {
#pragma unroll 8
      for (int64_t i = r; i < rows; i += 32) s += p[i * C + c];
    } else {
#pragma unroll 8
      for (int64_t i = r; i < rows; i += 32) s = fmaf(p[i * C + c], q[i * G], s);
    }
  }
  sh[r][lane] = s;
  __syncthreads();
  if (r == 0 && c < C) {
    for (int k = 1; k < 32; ++k) s += sh[k][lane];
    out[c] = s;
  }
}

// ---------------------------------------------------------------------------------------------- host

struct Plan {
  int V, W, slabs, parts, rows, R, cols, threads, slots, fold, lanes;
  bool resident;
  size_t smem;
};

int lcm(int a, int b) {
  int x = a, y = b;
  while (y) { const int t = x % y; x = y; y = t; }
  return a / x * b;
}

constexpr int kMostSlots = 128;               // what the error bound of a thread's sums is taken for
constexpr size_t kMostData = 100 * 1024;     // two CTAs per SM
constexpr int64_t kChunkData = 64 * 1024;    // chunks of a larger image: three
constexpr size_t kMostShared = 200 * 1024;   // of a plan, with its sums and parameters

// The rest of a plan whose slab width and parts are chosen; false if its slots need more than `most` bytes.
bool settle(Plan& p, int64_t L, int C, int cpg, int e, bool backward, int64_t rows, size_t most) {
  p.slabs = (C + p.W - 1) / p.W;
  p.cols = (p.W + p.V - 1) / p.V;
  p.threads = p.V > 1 ? (p.resident ? kResidentThreads : kChunkThreads) : p.cols <= 256 ? 256 : 1024;
  p.R = p.threads / p.cols;
  p.lanes = p.cols <= 32 && 32 % p.cols == 0 ? p.cols : 0;
  p.fold = 1;
  while (p.fold < p.V && cpg % (2 * p.fold) == 0) p.fold *= 2;
  const int64_t slots = (rows + p.R - 1) / p.R;
  const int erows = p.lanes ? p.threads / 32 : p.R;
  const size_t f = sizeof(float), data = (size_t)slots * p.threads * p.V * e * (backward ? 2 : 1);
  if (slots > kMostSlots || data > most) return false;
  p.rows = (int)rows;
  p.slots = (int)slots;
  const int groups = p.W / cpg;
  const int sums = p.resident ? p.parts : 1;
  if (backward) p.smem = data + f * (padded(2 * erows * p.W) + 4 * sums * padded(p.W) + 2 * padded(groups));
  else p.smem = data + f * (3 * padded(erows * p.cols * (p.V / p.fold)) + padded(erows) + (6 * sums + 2) * padded(groups));
  p.smem += 2 * f * params_size(p.W, groups);
  if (p.smem > kMostShared) return false;
  return true;
}


// Slab width, CTAs per image and slab, and positions per thread. Slabs are multiples of whole groups and of
// whole columns. Of the splits that keep an image's slab in one cluster's shared memory, the one of least
// cost: a cluster of more CTAs waits longer for its slowest, and rows of 32 bytes (a DRAM sector) take L1 twice the
// lines that 64 do. Measured, bf16 backward: 64 x 56x56 x 256 with 32 bytes and two CTAs 104 us, 64 bytes and four 112 us; 1024 x
// 32x32 x 64 with 32 bytes and one CTA 114 us, 64 bytes and two 107 us. Where the problem is too small to give every
// SM two CTAs, more CTAs count more than that (37 x 27x27 x 90 fp32, single elements: 17 us against 34).
Plan plan(int64_t N, int64_t L, int C, int cpg, int dtype, bool vec, bool backward) {
  Plan p, best;
  const int e = dtype == DMX_F32 ? 4 : 2;
  p.V = vec ? 16 / e : 1;
  const int unit = lcm(cpg, p.V);
  const int want[5] = {512, 256, 128, 64, 32};
  p.resident = true;
  best.resident = false;
  float least = 0.f;
  for (int k = 0, last = 0; k < 5; ++k) {
    p.W = (want[k] / e) / unit * unit;
    if (p.W < unit) p.W = unit;
    if (p.W > C) p.W = C;
    if (p.W == last) continue;
    last = p.W;
    for (p.parts = 1; p.parts <= kMaxCluster; p.parts *= 2) {
      if (!settle(p, L, C, cpg, e, backward, (L + p.parts - 1) / p.parts, kMostData)) continue;
      if (p.parts > 1 && p.rows < p.R) break;
      float cost = p.parts == 1 ? 1.f : p.parts == 2 ? 1.2f : p.parts == 4 ? 1.55f : 2.f;
      if (p.V > 1 && p.W * e < 64) cost *= 1.25f;
      const float ctas = (float)N * p.slabs * p.parts;
      if (ctas < 2 * 148) cost *= 2 * 148 / ctas;
      if (!best.resident || cost < least) { best = p; least = cost; }
      if (ctas >= 2 * 148) break;                  // more CTAs per slab would only cost more
    }
  }
  if (best.resident) return best;
  p.resident = false;
  p.parts = 1;
  p.W = (256 / e) / unit * unit;
  if (p.W < unit) p.W = unit;
  if (p.W > C) p.W = C;
  settle(p, L, C, cpg, e, backward, 1, kMostData);
  int64_t slots = kChunkData / ((int64_t)p.threads * p.V * e * (backward ? 2 : 1));
  slots = slots < 1 ? 1 : slots > kMostSlots ? kMostSlots : slots;
  const int64_t rows = p.R * slots;
  settle(p, L, C, cpg, e, backward, rows, ~(size_t)0);
  p.parts = (int)((L + rows - 1) / rows);
  return p;
}

// A kernel's limit of shared memory belongs to the kernel, not to a launch, and host threads share it: it is raised once per
// device, to the most that any plan takes.
template <auto kernel>
int launch(const Plan& p, const Args& A, bool cluster, cudaStream_t st) {
  static std::atomic<uint64_t> raised{0};
  int device = 0;
  if (!dmxh::cuda_ok(cudaGetDevice(&device))) return DMX_ERR_CUDA;
  const uint64_t bit = (uint64_t)1 << (device & 63);
  if (device > 63 || !(raised.load(std::memory_order_relaxed) & bit)) {
    if (!dmxh::cuda_ok(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared))) return DMX_ERR_CUDA;
    raised.fetch_or(bit, std::memory_order_relaxed);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(p.threads);
  cfg.dynamicSmemBytes = p.smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  const int per = cluster ? p.parts : 1;
  attr[1].val.clusterDim.x = per;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = per > 1 ? 2 : 1;
  // as many clusters as run at once; each takes item after item
  int64_t clusters = A.items;
  if (clusters * per > 148) {
    int at_once = 0;
    cfg.gridDim = dim3((unsigned)per);
    if (per > 1) {
      if (!dmxh::cuda_ok(cudaOccupancyMaxActiveClusters(&at_once, kernel, &cfg))) return DMX_ERR_CUDA;
    } else {
      if (!dmxh::cuda_ok(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&at_once, kernel, p.threads, p.smem))) return DMX_ERR_CUDA;
      at_once *= 148;
    }
    if (at_once < 1) return DMX_ERR_CUDA;
    // an even share: with 4.3 items each, five rounds of fewer CTAs
    const int64_t rounds = (clusters + at_once - 1) / at_once;
    clusters = (clusters + rounds - 1) / rounds;
  }
  cfg.gridDim = dim3((unsigned)(clusters * per));
  return dmxh::cuda_ok(cudaLaunchKernelEx(&cfg, kernel, A)) ? DMX_OK : DMX_ERR_CUDA;
}

template <typename... P, typename... V>
int start(int64_t ctas, int rows, int threads, cudaStream_t st, void (*kernel)(P...), V... args) {     // a dependent of the launch before
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas, rows);
  cfg.blockDim = dim3(threads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return dmxh::cuda_ok(cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...)) ? DMX_OK : DMX_ERR_CUDA;
}

template <typename T, int V, int ACT>
int run_act(bool backward, const Plan& p, const Args& A, cudaStream_t st) {
  if (backward) {
    if (p.resident) return launch<backward_kernel<T, V, RESIDENT, ACT>>(p, A, true, st);
    int rc = launch<backward_kernel<T, V, STATS, ACT>>(p, A, false, st);
    if (rc != DMX_OK) return rc;
    rc = start((int64_t)2 * A.N * ((A.C + 31) / 32), 1, 256, st, join_rows_kernel, A.part, A.part + 2 * (int64_t)A.N * A.parts * A.C, A.N, A.parts, A.C);
    return rc != DMX_OK ? rc : launch<backward_kernel<T, V, APPLY, ACT>>(p, A, false, st);
  }
  if (p.resident) return launch<forward_kernel<T, V, RESIDENT, ACT>>(p, A, true, st);
  int rc = launch<forward_kernel<T, V, STATS, DMX_ACT_NONE>>(p, A, false, st);
  if (rc != DMX_OK) return rc;
  const int64_t groups = (int64_t)A.N * A.G;
  rc = start((groups + 7) / 8, 1, 256, st, join_groups_kernel, (const float*)A.part, groups, A.parts, A.rows, A.L, A.G, A.cpg, A.eps,
             A.mean, A.rstd);
  return rc != DMX_OK ? rc : launch<forward_kernel<T, V, APPLY, ACT>>(p, A, false, st);
}

template <typename T, int V>
int run_typed(bool backward, int act, const Plan& p, const Args& A, cudaStream_t st) {
  switch (act) {
    case DMX_ACT_RELU: return run_act<T, V, DMX_ACT_RELU>(backward, p, A, st);
    case DMX_ACT_SILU: return run_act<T, V, DMX_ACT_SILU>(backward, p, A, st);
    case DMX_ACT_GELU: return run_act<T, V, DMX_ACT_GELU>(backward, p, A, st);
    default: return run_act<T, V, DMX_ACT_NONE>(backward, p, A, st);
  }
}

int run(bool backward, int act, int dtype, bool vec, const Plan& p, const Args& A, cudaStream_t st) {
  if (dtype == DMX_F32) return vec ? run_typed<float, 4>(backward, act, p, A, st) : run_typed<float, 1>(backward, act, p, A, st);
  return vec ? run_typed<__nv_bfloat16, 8>(backward, act, p, A, st) : run_typed<__nv_bfloat16, 1>(backward, act, p, A, st);
}

void fill(Args& A, const Plan& p, int64_t N, int64_t L, int C, int G) {
  A.L = (int)L; A.C = C; A.G = G; A.cpg = C / G; A.W = p.W; A.gW = p.W / A.cpg; A.slabs = p.slabs; A.R = p.R; A.cols = p.cols; A.rows = p.rows;
  A.parts = p.parts; A.slots = p.slots; A.fold = p.fold; A.lanes = p.lanes; A.N = (int)N;
  A.items = N * p.slabs * (p.resident ? 1 : p.parts);
}

bool shape_ok(int64_t N, int64_t L, int C, int G, int dtype) {
  if (N < 0 || L < 0 || C < 1 || G < 1 || C % G != 0 || C / G > DMX_GN_MAX_GROUP) return false;
  if (C > DMX_GN_MAX_CHANNELS || N > 0x7fffffff || L > 0x7fffffff) return false;
  return dtype == DMX_F32 || dtype == DMX_BF16;
}

// what is only read may repeat rows or images (stride 0); what is written has every element in a place of its own: image
// after image, or the images' rows in turn
bool strides_ok(int64_t N, int64_t L, int C, int64_t image, int64_t row, bool written) {
  if (row < 0 || image < 0) return false;
  if (!written || N == 0 || L == 0) return true;
  if (L > 1 && row < C) return false;
  return N <= 1 || image >= (L - 1) * row + C || (image >= C && row >= (N - 1) * image + C);
}

// 16-byte columns need every one of them to start on 16 bytes
bool wide(const void* p, int64_t N, int64_t L, int C, int64_t image, int64_t row, int e) {
  const int V = 16 / e;
  return p && (reinterpret_cast<uintptr_t>(p) & 15) == 0 && C % V == 0 && (L <= 1 || row % V == 0) && (N <= 1 || image % V == 0);
}

bool element_aligned(const void* p, int e) { return (reinterpret_cast<uintptr_t>(p) & (e - 1)) == 0; }

// ... and the narrowest slab of whole columns and whole groups has to fit a CTA's threads
bool columns_fit(int C, int cpg, int e) { return C % (16 / e) == 0 && lcm(cpg, 16 / e) / (16 / e) <= kResidentThreads; }

int64_t workspace_of(const Plan& p, int64_t N, int C, int G, bool backward) {
  if (backward) return 2 * N * (p.resident ? 1 : p.parts + 1) * C * (int64_t)sizeof(float);
  return p.resident ? 0 : 3 * N * p.parts * G * (int64_t)sizeof(float);
}

}  // namespace

extern "C" {

// the caller's pointers are not known here: the larger of what the two access widths need
int64_t dmx_group_norm_workspace(int64_t N, int64_t L, int C, int G, int dtype, int backward) {
  if (!shape_ok(N, L, C, G, dtype)) return DMX_ERR_ARG;
  if (N == 0 || L == 0) return 0;
  const int64_t one = workspace_of(plan(N, L, C, C / G, dtype, false, backward != 0), N, C, G, backward != 0);
  if (!columns_fit(C, C / G, dtype == DMX_F32 ? 4 : 2)) return one;
  const int64_t two = workspace_of(plan(N, L, C, C / G, dtype, true, backward != 0), N, C, G, backward != 0);
  return one > two ? one : two;
}

int dmx_group_norm_plan(int64_t N, int64_t L, int C, int G, int dtype, int wide_access, int backward, int64_t* out) {
  if (!shape_ok(N, L, C, G, dtype) || N < 1 || L < 1 || !out) return DMX_ERR_ARG;
  const Plan p = plan(N, L, C, C / G, dtype, wide_access && columns_fit(C, C / G, dtype == DMX_F32 ? 4 : 2), backward != 0);
  out[0] = p.V; out[1] = p.resident; out[2] = p.parts; out[3] = N * p.slabs * (p.resident ? 1 : p.parts); out[4] = p.threads; out[5] = (int64_t)p.smem;
  return DMX_OK;
}

int dmx_group_norm_forward(int64_t N, int64_t L, int C, int G, int dtype, const void* x, int64_t x_image, int64_t x_row,
                           const float* weight, const float* bias, float eps, int act, void* y, int64_t y_image,
                           int64_t y_row, float* mean, float* rstd, void* workspace, int64_t workspace_bytes,
                           void* cuda_stream) {
  if (!shape_ok(N, L, C, G, dtype) || act < DMX_ACT_NONE || act > DMX_ACT_GELU || !(eps >= 0.f)) return DMX_ERR_ARG;
  if (!strides_ok(N, L, C, x_image, x_row, false) || !strides_ok(N, L, C, y_image, y_row, true)) return DMX_ERR_ARG;
  if (N == 0) return DMX_OK;
  if (!element_aligned(mean, 4) || !element_aligned(rstd, 4)) return DMX_ERR_ALIGN;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (L == 0) {                    // nothing over nothing: bytes of ones are a NaN
    for (float* p : {mean, rstd})
      if (p && !dmxh::cuda_ok(cudaMemsetAsync(p, 0xff, sizeof(float) * N * G, st))) return DMX_ERR_CUDA;
    return DMX_OK;
  }
  if (!x || !y || !mean || !rstd) return DMX_ERR_ARG;
  const int e = dtype == DMX_F32 ? 4 : 2;
  if (!element_aligned(x, e) || !element_aligned(y, e) || !element_aligned(weight, 4) || !element_aligned(bias, 4) || !element_aligned(workspace, 16))
    return DMX_ERR_ALIGN;
  const bool vec = columns_fit(C, C / G, e) && wide(x, N, L, C, x_image, x_row, e) && wide(y, N, L, C, y_image, y_row, e);
  const Plan p = plan(N, L, C, C / G, dtype, vec, false);
  const int64_t need = workspace_of(p, N, C, G, false);
  if (workspace_bytes < need || (need > 0 && !workspace)) return DMX_ERR_ARG;
  if (N * p.slabs * (int64_t)p.parts > 0x7fffffff || 2 * N * ((C + 31) / 32) > 0x7fffffff) return DMX_ERR_ARG;
  Args A = {};
  A.x = {const_cast<void*>(x), x_image, x_row};
  A.out = {y, y_image, y_row};
  A.weight = weight; A.bias = bias; A.mean = mean; A.rstd = rstd; A.part = static_cast<float*>(workspace);
  fill(A, p, N, L, C, G);
  A.eps = eps;
  return run(false, act, dtype, vec, p, A, st);
}

int dmx_group_norm_backward(int64_t N, int64_t L, int C, int G, int dtype, const void* dy, int64_t dy_image,
                            int64_t dy_row, const void* x, int64_t x_image, int64_t x_row, const float* mean,
                            const float* rstd, const float* weight, const float* bias, int act, void* dx,
                            int64_t dx_image, int64_t dx_row, float* dweight, float* dbias, void* workspace,
                            int64_t workspace_bytes, void* cuda_stream) {
  if (!shape_ok(N, L, C, G, dtype) || act < DMX_ACT_NONE || act > DMX_ACT_GELU) return DMX_ERR_ARG;
  if (!strides_ok(N, L, C, x_image, x_row, false) || !strides_ok(N, L, C, dy_image, dy_row, false) || !strides_ok(N, L, C, dx_image, dx_row, true)) return DMX_ERR_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (!element_aligned(dweight, 4) || !element_aligned(dbias, 4)) return DMX_ERR_ALIGN;
  if (N == 0 || L == 0) {
    if (dweight && !dmxh::cuda_ok(cudaMemsetAsync(dweight, 0, sizeof(float) * C, st))) return DMX_ERR_CUDA;
    if (dbias && !dmxh::cuda_ok(cudaMemsetAsync(dbias, 0, sizeof(float) * C, st))) return DMX_ERR_CUDA;
    return DMX_OK;
  }
  if (!dy || !x || !dx || !mean || !rstd) return DMX_ERR_ARG;
  const int e = dtype == DMX_F32 ? 4 : 2;
  if (!element_aligned(x, e) || !element_aligned(dy, e) || !element_aligned(dx, e) || !element_aligned(mean, 4) || !element_aligned(rstd, 4) ||
      !element_aligned(weight, 4) || !element_aligned(bias, 4) || !element_aligned(workspace, 16)) return DMX_ERR_ALIGN;
  const bool vec = columns_fit(C, C / G, e) && wide(x, N, L, C, x_image, x_row, e) && wide(dy, N, L, C, dy_image, dy_row, e) && wide(dx, N, L, C, dx_image, dx_row, e);
  const Plan p = plan(N, L, C, C / G, dtype, vec, true);
  if (workspace_bytes < workspace_of(p, N, C, G, true) || !workspace) return DMX_ERR_ARG;
  if (N * p.slabs * (int64_t)p.parts > 0x7fffffff || 2 * N * ((C + 31) / 32) > 0x7fffffff) return DMX_ERR_ARG;
  Args A = {};
  A.x = {const_cast<void*>(x), x_image, x_row};
  A.dy = {const_cast<void*>(dy), dy_image, dy_row};
  A.out = {dx, dx_image, dx_row};
  A.weight = weight; A.bias = bias; A.mean = const_cast<float*>(mean); A.rstd = const_cast<float*>(rstd); A.part = static_cast<float*>(workspace);
  fill(A, p, N, L, C, G);
  const int rc = run(true, act, dtype, vec, p, A, st);
  if (rc != DMX_OK || (!dweight && !dbias)) return rc;
  return start((C + 31) / 32, 2, 1024, st, columns_kernel, A.part + (p.resident ? 0 : 2 * N * p.parts * C), N, C, G, C / G, rstd, dweight, dbias);
}

}  // extern "C"
