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
// one launch for the chunks' sums, one that reads again, mostly from L2.
// Variances: a thread sums deviations from its own first value, s = sum d, q = sum d^2, and takes q - s^2/n. That
// cancels only if the first value is far off, and then the group's variance contains that distance itself:
// the error stays within n (at most 40 or so) roundings of the result. From there on deviations of means are added
// (Chan, Golub, LeVeque 1983). Nothing is added atomically; the order of all sums is fixed by the shape.
#include "dmx.h"

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "dmx_act.cuh"
#include "dmx_host.h"

namespace {

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
  int L, N, C, G, cpg, W, slabs, R, cols, rows;   // W channels per slab, R positions at a time, cols columns of V, rows positions per CTA
  int parts;             // CTAs (or chunks) per image and slab
  int slots;             // positions per thread
  int fold;              // neighbouring channels of a column that surely share a group (a power of two)
  int lanes;             // lanes of a warp that hold different columns, if that divides 32, else 0
  float eps;
  int act;
};

template <typename T, int V>
struct Vec;                                            // V elements as one access
template <> struct Vec<float, 4> { using type = uint4; };
template <> struct Vec<float, 1> { using type = unsigned; };
template <> struct Vec<__nv_bfloat16, 8> { using type = uint4; };
template <> struct Vec<__nv_bfloat16, 1> { using type = unsigned short; };

__device__ __forceinline__ void widen(uint4 r, float (&x)[4]) {
  x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y); x[2] = __uint_as_float(r.z); x[3] = __uint_as_float(r.w);
}
__device__ __forceinline__ void widen(unsigned r, float (&x)[1]) { x[0] = __uint_as_float(r); }
__device__ __forceinline__ void widen(unsigned short r, float (&x)[1]) { x[0] = __uint_as_float((unsigned)r << 16); }
__device__ __forceinline__ void widen(uint4 r, float (&x)[8]) {
  const unsigned w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) { x[2 * j] = __uint_as_float(w[j] << 16); x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u); }
}
__device__ __forceinline__ unsigned pack2(float a, float b) {
  __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<unsigned*>(&t);
}
__device__ __forceinline__ void put(float* p, const float (&x)[4]) { __stcs(reinterpret_cast<float4*>(p), make_float4(x[0], x[1], x[2], x[3])); }
__device__ __forceinline__ void put(float* p, const float (&x)[1]) { __stcs(p, x[0]); }
__device__ __forceinline__ void put(__nv_bfloat16* p, const float (&x)[8]) {
  __stcs(reinterpret_cast<uint4*>(p), make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])));
}
__device__ __forceinline__ void put(__nv_bfloat16* p, const float (&x)[1]) { *p = __float2bfloat16_rn(x[0]); }

// One element or column into the thread's own slot. Two bytes are below what an asynchronous copy takes.
__device__ __forceinline__ void bring(uint4* slot, const void* p) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((unsigned)__cvta_generic_to_shared(slot)), "l"(p));
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

// A CTA's place in one item, and a thread's in that.
struct Here {
  int n, part, c0, Wl, groups, rows, r0;
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
  h.Wl = min(A.W, A.C - h.c0);
  h.groups = h.Wl == A.W ? A.W / A.cpg : h.Wl / A.cpg;
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

// Sums over groups of red[R][width], `per` neighbouring entries of a row being a group's: term(i, r, g) for
// entry i in row r. `each` lanes (a power of two) take a group, in a fixed order.
template <typename F>
__device__ __forceinline__ float group_sum(int g, int groups, int per, int R, int width, int each, int l, F term) {
  float s = 0.f;
  if (g < groups) {
    int r = l / per, c = l - r * per;
    const int dr = each / per, dc = each - dr * per;
    for (; r < R;) {
      s += term(r * width + g * per + c, r, g);
      r += dr; c += dc;
      if (c >= per) { c -= per; ++r; }
    }
  }
  for (int o = each >> 1; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}
__device__ __forceinline__ int lanes_for(int total) {
  return total >= 32 ? 32 : total <= 1 ? 1 : 1 << (32 - __clz(total - 1));
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ float remote(const float* p, int rank) {
  unsigned a;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((unsigned)__cvta_generic_to_shared(p)), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}

template <typename T, int V, Mode M>
__global__ void __launch_bounds__(V == 1 ? 1024 : 256) forward_kernel(const __grid_constant__ Args A) {
  using U = typename Vec<T, V>::type;
  extern __shared__ __align__(16) float sm[];
  const int W = A.W, cpg = A.cpg, R = A.R, threads = blockDim.x;
  const int tid = threadIdx.x, rl = tid / A.cols, col = tid - rl * A.cols;
  // entries: per column V/fold values; rows of them: the warps where a warp's lanes can be added up, else all R
  const int vals = V / A.fold, width = A.cols * vals, per = cpg / A.fold;
  const int rows = A.lanes ? threads >> 5 : R;
  U* slot = reinterpret_cast<U*>(sm) + tid;
  float* emean = sm + (size_t)A.slots * threads * sizeof(U) / sizeof(float);
  float* em2 = emean + padded(rows * width);
  float* en = em2 + padded(rows * width);
  float* gsum = en + padded(rows);                 // per group: this CTA's sum and squared deviations (read by the cluster)
  float* gm2 = gsum + padded(W / cpg);
  float* gmean = gm2 + padded(W / cpg);            // per group: mean, rstd
  float* grstd = gmean + padded(W / cpg);
  const int each = lanes_for(rows * per), gl = tid & (each - 1), g1 = tid / each, gstep = threads / each;
  int grp0 = 0, rem0 = 0;                          // group of the column's first channel, and its place there
  if (rl < R) { grp0 = col * V / cpg; rem0 = col * V - grp0 * cpg; }

  const int64_t first = M == RESIDENT ? blockIdx.x / (unsigned)A.parts : blockIdx.x;
  const int64_t stride = M == RESIDENT ? gridDim.x / (unsigned)A.parts : gridDim.x;
  if (first >= A.items) return;                    // the whole cluster
  Here h = place<V, M>(A, first, rl, col);
  {
    const T* p = start<T, V>(A.x, h, rl, col);
    for (int i = 0; i < h.cnt; ++i) bring(slot + i * threads, p + (int64_t)i * R * A.x.row);
  }
  for (int64_t item = first; item < A.items; item += stride) {
    float w[V], b[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      w[v] = h.on && A.weight ? __ldg(A.weight + h.c0 + col * V + v) : 1.f;
      b[v] = h.on && A.bias ? __ldg(A.bias + h.c0 + col * V + v) : 0.f;
    }
    bring_wait();
    if constexpr (M != APPLY) {
      float x0[V], s[V], q[V];
#pragma unroll
      for (int v = 0; v < V; ++v) { x0[v] = 0.f; s[v] = 0.f; q[v] = 0.f; }
      if (h.cnt > 0) widen(*slot, x0);
#pragma unroll 4
      for (int i = 1; i < h.cnt; ++i) {
        float x[V];
        widen(slot[i * threads], x);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const float d = x[v] - x0[v];
          s[v] += d;
          q[v] = fmaf(d, d, q[v]);
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
      }
#pragma unroll
      for (int f = 1; f < V; f *= 2) {
        if (A.fold <= f) break;
#pragma unroll
        for (int j = 0; j < V / (2 * f); ++j) {
          const float d = s[2 * j] - s[2 * j + 1];
          q[j] = q[2 * j] + q[2 * j + 1] + 0.5f * n * d * d;
          s[j] = 0.5f * (s[2 * j] + s[2 * j + 1]);
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
          const float d = s[j] - t;
          float m = n > 0.f ? fmaf(n * d, d, q[j]) : 0.f;
          for (int o = A.lanes; o < 32; o <<= 1) m += __shfl_xor_sync(0xffffffffu, m, o);
          s[j] = t; q[j] = m;
        }
        const int lane = tid & 31, wid = tid >> 5;
        if (lane < A.lanes) {
#pragma unroll
          for (int j = 0; j < V; ++j) {
            if (j >= vals) break;
            emean[wid * width + col * vals + j] = s[j];
            em2[wid * width + col * vals + j] = q[j];
          }
          if (lane == 0) en[wid] = N;
        }
      } else if (rl < R) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          if (j >= vals) break;
          emean[rl * width + col * vals + j] = s[j];
          em2[rl * width + col * vals + j] = q[j];
        }
        if (col == 0) en[rl] = n;
      }
      __syncthreads();
      const float cnt = (float)h.rows * (float)cpg, icnt = h.rows > 0 ? 1.f / cnt : 0.f;
      for (int g0 = 0; g0 < h.groups; g0 += gstep) {
        const int g = g0 + g1;
        const float sum = group_sum(g, h.groups, per, rows, width, each, gl, [&](int i, int r, int) { return en[r] > 0.f ? emean[i] * en[r] : 0.f; });
        const float mean = sum * icnt;
        const float m2 = group_sum(g, h.groups, per, rows, width, each, gl, [&](int i, int r, int) {
          const float d = emean[i] - mean;
          return en[r] > 0.f ? fmaf(en[r] * d, d, em2[i]) : 0.f;
        });
        if (g < h.groups && gl == 0) {
          gsum[g] = mean * (float)h.rows;          // times channels below: keeps the product in range
          gm2[g] = m2;
        }
      }
      if constexpr (M == STATS) {
        __syncthreads();
        float2* out = reinterpret_cast<float2*>(A.part) + ((int64_t)h.n * A.parts + h.part) * A.G + h.c0 / cpg;
        for (int g = tid; g < h.groups; g += threads) out[g] = make_float2(gsum[g], gm2[g]);
      } else if (A.parts > 1) {
        cluster_sync();
      } else {
        __syncthreads();
      }
    }
    if constexpr (M != STATS) {
      // join the parts of each group, in their order
      for (int g = tid; g < h.groups; g += threads) {
        const float2* src = reinterpret_cast<const float2*>(A.part) + (int64_t)h.n * A.parts * A.G + h.c0 / cpg + g;
        float sum = 0.f, m2 = 0.f;
        for (int k = 0; k < A.parts; ++k) {
          if constexpr (M == RESIDENT) sum += A.parts > 1 ? remote(gsum + g, k) : gsum[g];
          else sum += __ldg(&src[(int64_t)k * A.G]).x;
        }
        const float mean = sum / (float)A.L;
        for (int k = 0; k < A.parts; ++k) {
          const float have = (float)(min((int64_t)(k + 1) * A.rows, (int64_t)A.L) - min((int64_t)k * A.rows, (int64_t)A.L));
          float ps, pm;
          if constexpr (M == RESIDENT) {
            ps = A.parts > 1 ? remote(gsum + g, k) : gsum[g];
            pm = A.parts > 1 ? remote(gm2 + g, k) : gm2[g];
          } else {
            const float2 t = __ldg(&src[(int64_t)k * A.G]);
            ps = t.x; pm = t.y;
          }
          if (have > 0.f) {
            const float d = ps / have - mean;
            m2 += fmaf(have * (float)cpg * d, d, pm);
          }
        }
        const float rstd = 1.f / sqrtf(m2 / ((float)A.L * (float)cpg) + A.eps);
        gmean[g] = mean;
        grstd[g] = rstd;
        if (h.part == 0) {
          const int64_t at = (int64_t)h.n * A.G + h.c0 / cpg + g;
          A.mean[at] = mean;
          A.rstd[at] = rstd;
        }
      }
      if (M == RESIDENT && A.parts > 1) cluster_arrive();
      __syncthreads();
    }
    // results, each slot refilled for the next item behind its last use
    const Here now = h;
    const int64_t next = item + stride;
    const bool more = next < A.items;
    const T* np = nullptr;
    int ncnt = 0;
    if (more) {
      h = place<V, M>(A, next, rl, col);
      np = start<T, V>(A.x, h, rl, col);
      ncnt = h.cnt;
    }
    const int64_t in_step = (int64_t)R * A.x.row;
    if constexpr (M != STATS) {
      float mu[V];
      int g = grp0, rem = rem0;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (now.on) { mu[v] = gmean[g]; w[v] *= grstd[g]; }
        if (++rem == cpg) { rem = 0; ++g; }
      }
      T* out = start<T, V>(A.out, now, rl, col);
      const int64_t out_step = (int64_t)R * A.out.row;
#pragma unroll 2
      for (int i = 0; i < now.cnt; ++i) {
        float x[V];
        widen(slot[i * threads], x);
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = fmaf(x[v] - mu[v], w[v], b[v]);
        dmx_act::apply<V>(x, A.act);
        put(out, x);
        out += out_step;
        if (i < ncnt) { bring(slot + i * threads, np); np += in_step; }
      }
      for (int i = now.cnt; i < ncnt; ++i) { bring(slot + i * threads, np); np += in_step; }
      if (M == RESIDENT && A.parts > 1) cluster_wait();        // the sums may be overwritten from here on
      if (M == APPLY) __syncthreads();                         // (the other modes pass a barrier before they write means)
    } else {
      for (int i = 0; i < ncnt; ++i) { bring(slot + i * threads, np); np += in_step; }
    }
  }
}

// Backward. Workspace: A and B per image (and chunk) and channel, [2][N*chunks][C].
template <typename T, int V, Mode M>
__global__ void __launch_bounds__(V == 1 ? 1024 : 256) backward_kernel(const __grid_constant__ Args A) {
  using U = typename Vec<T, V>::type;
  extern __shared__ __align__(16) float sm[];
  const int W = A.W, cpg = A.cpg, R = A.R, threads = blockDim.x;
  const int tid = threadIdx.x, rl = tid / A.cols, col = tid - rl * A.cols;
  const int rows = A.lanes ? threads >> 5 : R;
  U* xs = reinterpret_cast<U*>(sm) + tid;
  U* gs = xs + (size_t)A.slots * threads;
  float* red = sm + (size_t)2 * A.slots * threads * sizeof(U) / sizeof(float);   // rows of A, rows of B
  float* ch = red + padded(2 * rows * W);          // this CTA's channel sums A, B (read by the cluster)
  float* wch = ch + padded(2 * W);                 // their totals times weight
  float* grp = wch + padded(2 * W);                // per group: sum w A, sum w B
  const int groups_all = W / cpg;
  const int each = lanes_for(cpg), gl = tid & (each - 1), g1 = tid / each, gstep = threads / each;
  int grp0 = 0, rem0 = 0;
  if (rl < R) { grp0 = col * V / cpg; rem0 = col * V - grp0 * cpg; }
  const int64_t plane = (int64_t)A.N * (M == RESIDENT ? 1 : A.parts) * A.C;

  const int64_t first = M == RESIDENT ? blockIdx.x / (unsigned)A.parts : blockIdx.x;
  const int64_t stride = M == RESIDENT ? gridDim.x / (unsigned)A.parts : gridDim.x;
  if (first >= A.items) return;
  Here h = place<V, M>(A, first, rl, col);
  {
    const T *p = start<T, V>(A.x, h, rl, col), *g = start<T, V>(A.dy, h, rl, col);
    for (int i = 0; i < h.cnt; ++i) {
      bring(xs + i * threads, p + (int64_t)i * R * A.x.row);
      bring(gs + i * threads, g + (int64_t)i * R * A.dy.row);
    }
  }
  for (int64_t item = first; item < A.items; item += stride) {
    float w[V], b[V], mu[V], rs[V];
    {
      const int64_t sidx = (int64_t)h.n * A.G + h.c0 / cpg;
      int g = grp0, rem = rem0;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        w[v] = h.on && A.weight ? __ldg(A.weight + h.c0 + col * V + v) : 1.f;
        b[v] = h.on && A.bias ? __ldg(A.bias + h.c0 + col * V + v) : 0.f;
        mu[v] = h.on ? __ldg(A.mean + sidx + g) : 0.f;
        rs[v] = h.on ? __ldg(A.rstd + sidx + g) : 0.f;
        if (++rem == cpg) { rem = 0; ++g; }
      }
    }
    bring_wait();
    if constexpr (M != APPLY) {
      float sa[V], sb[V];
#pragma unroll
      for (int v = 0; v < V; ++v) sa[v] = sb[v] = 0.f;
#pragma unroll 2
      for (int i = 0; i < h.cnt; ++i) {
        float x[V], g[V], u[V];
        widen(xs[i * threads], x);
        widen(gs[i * threads], g);
#pragma unroll
        for (int v = 0; v < V; ++v) { x[v] = (x[v] - mu[v]) * rs[v]; u[v] = fmaf(x[v], w[v], b[v]); }
        dmx_act::times_slope<V>(g, u, A.act);
#pragma unroll
        for (int v = 0; v < V; ++v) { sa[v] = fmaf(g[v], x[v], sa[v]); sb[v] += g[v]; }
      }
      if (A.lanes) {
        const int lane = tid & 31, wid = tid >> 5;
        for (int o = A.lanes; o < 32; o <<= 1)
#pragma unroll
          for (int v = 0; v < V; ++v) {
            sa[v] += __shfl_xor_sync(0xffffffffu, sa[v], o);
            sb[v] += __shfl_xor_sync(0xffffffffu, sb[v], o);
          }
        if (lane < A.lanes)
#pragma unroll
          for (int v = 0; v < V; ++v) {
            red[wid * W + col * V + v] = sa[v];
            red[(rows + wid) * W + col * V + v] = sb[v];
          }
      } else if (rl < R) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
          red[rl * W + col * V + v] = sa[v];
          red[(rows + rl) * W + col * V + v] = sb[v];
        }
      }
      __syncthreads();
      for (int c = tid; c < 2 * W; c += threads) {
        const float* p = c < W ? red + c : red + rows * W + (c - W);
        float t = 0.f;
        for (int r = 0; r < rows; ++r) t += p[r * W];
        ch[c] = t;
      }
      if constexpr (M == STATS) {
        __syncthreads();
        float* out = A.part + ((int64_t)h.n * A.parts + h.part) * A.C + h.c0;
        for (int c = tid; c < h.Wl; c += threads) { out[c] = ch[c]; out[plane + c] = ch[W + c]; }
      } else if (A.parts > 1) {
        cluster_sync();
      } else {
        __syncthreads();
      }
    }
    if constexpr (M != STATS) {
      // channel totals over the parts, in their order; then the groups' weighted sums
      for (int c = tid; c < 2 * W; c += threads) {
        const int k = c < W ? c : c - W;
        if (k >= h.Wl) continue;
        float t = 0.f;
        if constexpr (M == RESIDENT) {
          if (A.parts > 1) for (int p = 0; p < A.parts; ++p) t += remote(ch + c, p);
          else t = ch[c];
          if (h.part == 0) A.part[(c < W ? 0 : plane) + (int64_t)h.n * A.C + h.c0 + k] = t;
        } else {
          const float* src = A.part + (c < W ? 0 : plane) + (int64_t)h.n * A.parts * A.C + h.c0 + k;
          for (int p = 0; p < A.parts; ++p) t += __ldg(src + (int64_t)p * A.C);
        }
        wch[c] = A.weight ? t * __ldg(A.weight + h.c0 + k) : t;
      }
      if (M == RESIDENT && A.parts > 1) cluster_arrive();
      __syncthreads();
      for (int g0 = 0; g0 < 2 * groups_all; g0 += gstep) {
        const int g = g0 + g1;                       // the B half's groups follow the A half's: W / cpg whole groups
        const float t = group_sum(g, 2 * groups_all, cpg, 1, 0, each, gl, [&](int i, int, int) { return wch[i]; });
        if (g < 2 * groups_all && gl == 0) grp[g] = t;
      }
      __syncthreads();
    }
    const Here now = h;
    const int64_t next = item + stride;
    const T *nx = nullptr, *ng = nullptr;
    int ncnt = 0;
    if (next < A.items) {
      h = place<V, M>(A, next, rl, col);
      nx = start<T, V>(A.x, h, rl, col);
      ng = start<T, V>(A.dy, h, rl, col);
      ncnt = h.cnt;
    }
    const int64_t xstep = (int64_t)R * A.x.row, gstep2 = (int64_t)R * A.dy.row;
    if constexpr (M != STATS) {
      float s1[V], s2[V];
      const float n = 1.f / ((float)A.L * (float)cpg);
      int g = grp0, rem = rem0;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (now.on) { s2[v] = grp[g] * n; s1[v] = grp[groups_all + g] * n; }
        if (++rem == cpg) { rem = 0; ++g; }
      }
      T* out = start<T, V>(A.out, now, rl, col);
      const int64_t out_step = (int64_t)R * A.out.row;
#pragma unroll 2
      for (int i = 0; i < now.cnt; ++i) {
        float x[V], gr[V], u[V];
        widen(xs[i * threads], x);
        widen(gs[i * threads], gr);
#pragma unroll
        for (int v = 0; v < V; ++v) { x[v] = (x[v] - mu[v]) * rs[v]; u[v] = fmaf(x[v], w[v], b[v]); }
        dmx_act::times_slope<V>(gr, u, A.act);
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = rs[v] * (fmaf(gr[v], w[v], -s1[v]) - x[v] * s2[v]);
        put(out, x);
        out += out_step;
        if (i < ncnt) {
          bring(xs + i * threads, nx);
          bring(gs + i * threads, ng);
          nx += xstep; ng += gstep2;
        }
      }
    }
    for (int i = M == STATS ? 0 : min(now.cnt, ncnt); i < ncnt; ++i) {
      bring(xs + i * threads, nx);
      bring(gs + i * threads, ng);
      nx += xstep; ng += gstep2;
    }
    if (M == RESIDENT && A.parts > 1) cluster_wait();
    if (M == APPLY) __syncthreads();
  }
}

// dweight and dbias: sums of the images' (and chunks') rows. 32 channels and eight row lanes per CTA.
__global__ void __launch_bounds__(256) columns_kernel(const float* __restrict__ part, int64_t rows, int C, float* __restrict__ dw,
                                                      float* __restrict__ db) {
  __shared__ float sh[8][33];
  const int lane = threadIdx.x & 31, r = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  const float* p = part + (int64_t)blockIdx.y * rows * C;
  float* out = blockIdx.y ? db : dw;
  if (!out) return;
  float s = 0.f;
  if (c < C)
    for (int64_t i = r; i < rows; i += 8) s += __ldg(p + i * C + c);
  sh[r][lane] = s;
  __syncthreads();
  if (r == 0 && c < C) {
    for (int k = 1; k < 8; ++k) s += sh[k][lane];
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

// The rest of a plan whose slab width and parts are chosen; false if its slots need more than `most` bytes.
bool settle(Plan& p, int64_t L, int C, int cpg, int e, bool backward, int64_t rows, size_t most) {
  p.slabs = (C + p.W - 1) / p.W;
  p.cols = (p.W + p.V - 1) / p.V;
  p.threads = p.cols <= 256 ? 256 : 1024;
  p.R = p.threads / p.cols;
  p.lanes = p.cols <= 32 && 32 % p.cols == 0 ? p.cols : 0;
  p.fold = 1;
  while (p.fold < p.V && cpg % (2 * p.fold) == 0) p.fold *= 2;
  const int64_t slots = (rows + p.R - 1) / p.R;
  const int erows = p.lanes ? p.threads / 32 : p.R;
  const size_t f = sizeof(float), data = (size_t)slots * p.threads * p.V * e * (backward ? 2 : 1);
  if (slots > 64 || data > most) return false;
  p.rows = (int)rows;
  p.slots = (int)slots;
  const int groups = p.W / cpg;
  if (backward) p.smem = data + f * (padded(2 * erows * p.W) + 2 * padded(2 * p.W) + padded(2 * groups));
  else p.smem = data + f * (2 * padded(erows * p.cols * (p.V / p.fold)) + padded(erows) + 4 * padded(groups));
  return true;
}

constexpr size_t kMostData = 96 * 1024;      // two CTAs per SM

// Slab width, CTAs per image and slab, and positions per thread. Slabs are multiples of whole groups and of
// whole columns. Among the splits that keep an image's slab in one cluster's shared memory: segments of up to 512
// bytes, then 128, 64, 32 (a DRAM sector); within a width the fewest CTAs per slab. Where the problem is too
// small to give every SM two CTAs, narrow slabs come first (no exchange needed), then more CTAs per slab.
Plan plan(int64_t N, int64_t L, int C, int cpg, int dtype, bool vec, bool backward) {
  Plan p;
  const int e = dtype == DMX_F32 ? 4 : 2;
  p.V = vec ? 16 / e : 1;
  const int unit = lcm(cpg, p.V);
  const int want[4] = {512, 128, 64, 32};
  for (int k = 0; k < 4; ++k) {
    p.W = (want[k] / e) / unit * unit;
    if (p.W < unit) p.W = unit;
    if (p.W > C) p.W = C;
    if (k == 0 && p.W * e < 512 && p.W < C) continue;
    for (p.parts = 1; p.parts <= kMaxCluster; p.parts *= 2) {
      if (!settle(p, L, C, cpg, e, backward, (L + p.parts - 1) / p.parts, kMostData)) continue;
      if (N * p.slabs * p.parts < 2 * 148) {
        if (k < 2 && unit * e < want[k]) break;                     // more CTAs from narrower slabs first
        if (p.parts < kMaxCluster && p.slots > 1) continue;         // then from more of them per slab
      }
      p.resident = true;
      return p;
    }
  }
  p.resident = false;
  p.W = (256 / e) / unit * unit;
  if (p.W < unit) p.W = unit;
  if (p.W > C) p.W = C;
  settle(p, L, C, cpg, e, backward, 1, kMostData);
  const int64_t rows = (int64_t)p.R * 8;
  settle(p, L, C, cpg, e, backward, rows, ~(size_t)0);
  p.parts = (int)((L + rows - 1) / rows);
  return p;
}

template <typename K>
int launch(K kernel, const Plan& p, const Args& A, bool cluster, cudaStream_t st) {
  if (p.smem > 48 * 1024 && !dmxh::cuda_ok(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)p.smem))) return DMX_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(p.threads);
  cfg.dynamicSmemBytes = p.smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1] = {};
  attr[0].id = cudaLaunchAttributeClusterDimension;
  const int per = cluster ? p.parts : 1;
  attr[0].val.clusterDim.x = per;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
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

template <typename T, int V>
int run_forward(const Plan& p, const Args& A, cudaStream_t st) {
  if (p.resident) return launch(forward_kernel<T, V, RESIDENT>, p, A, true, st);
  const int rc = launch(forward_kernel<T, V, STATS>, p, A, false, st);
  return rc != DMX_OK ? rc : launch(forward_kernel<T, V, APPLY>, p, A, false, st);
}

template <typename T, int V>
int run_backward(const Plan& p, const Args& A, cudaStream_t st) {
  if (p.resident) return launch(backward_kernel<T, V, RESIDENT>, p, A, true, st);
  const int rc = launch(backward_kernel<T, V, STATS>, p, A, false, st);
  return rc != DMX_OK ? rc : launch(backward_kernel<T, V, APPLY>, p, A, false, st);
}

void fill(Args& A, const Plan& p, int64_t N, int64_t L, int C, int G) {
  A.L = (int)L; A.C = C; A.G = G; A.cpg = C / G; A.W = p.W; A.slabs = p.slabs; A.R = p.R; A.cols = p.cols; A.rows = p.rows;
  A.parts = p.parts; A.slots = p.slots; A.fold = p.fold; A.lanes = p.lanes; A.N = (int)N;
  A.items = N * p.slabs * (p.resident ? 1 : p.parts);
}

bool shape_ok(int64_t N, int64_t L, int C, int G, int dtype) {
  if (N < 0 || L < 0 || C < 1 || G < 1 || C % G != 0 || C / G > DMX_GN_MAX_GROUP) return false;
  if (C > DMX_GN_MAX_CHANNELS || N > 0x7fffffff || L > 0x7fffffff) return false;
  return dtype == DMX_F32 || dtype == DMX_BF16;
}

bool strides_ok(int64_t N, int64_t L, int C, int64_t image, int64_t row) {
  return (L <= 1 || row >= C) && (N <= 1 || image >= 0) && row >= 0 && image >= 0;
}

// 16-byte columns need every one of them to start on 16 bytes
bool wide(const void* p, int64_t N, int64_t L, int C, int64_t image, int64_t row, int e) {
  const int V = 16 / e;
  return p && (reinterpret_cast<uintptr_t>(p) & 15) == 0 && C % V == 0 && (L <= 1 || row % V == 0) && (N <= 1 || image % V == 0);
}

bool element_aligned(const void* p, int e) { return (reinterpret_cast<uintptr_t>(p) & (e - 1)) == 0; }

// ... and the narrowest slab of whole columns and whole groups has to fit a CTA's threads
bool columns_fit(int C, int cpg, int e) { return C % (16 / e) == 0 && lcm(cpg, 16 / e) / (16 / e) <= 256; }

int64_t workspace_for(int64_t N, int64_t L, int C, int G, int dtype, bool vec, bool backward) {
  const Plan p = plan(N, L, C, C / G, dtype, vec, backward);
  if (backward) return 2 * N * (p.resident ? 1 : p.parts) * C * (int64_t)sizeof(float);
  return p.resident ? 0 : N * p.parts * G * (int64_t)sizeof(float2);
}

}  // namespace

extern "C" {

// the caller's pointers are not known here: the larger of what the two access widths need
int64_t dmx_group_norm_workspace(int64_t N, int64_t L, int C, int G, int dtype, int backward) {
  if (!shape_ok(N, L, C, G, dtype)) return DMX_ERR_ARG;
  if (N == 0 || L == 0) return 0;
  const int64_t one = workspace_for(N, L, C, G, dtype, false, backward != 0);
  const int64_t two = columns_fit(C, C / G, dtype == DMX_F32 ? 4 : 2) ? workspace_for(N, L, C, G, dtype, true, backward != 0) : 0;
  return one > two ? one : two;
}

int dmx_group_norm_forward(int64_t N, int64_t L, int C, int G, int dtype, const void* x, int64_t x_image, int64_t x_row,
                           const float* weight, const float* bias, float eps, int act, void* y, int64_t y_image,
                           int64_t y_row, float* mean, float* rstd, void* workspace, int64_t workspace_bytes,
                           void* cuda_stream) {
  if (!shape_ok(N, L, C, G, dtype) || act < DMX_ACT_NONE || act > DMX_ACT_GELU || !(eps >= 0.f)) return DMX_ERR_ARG;
  if (!strides_ok(N, L, C, x_image, x_row) || !strides_ok(N, L, C, y_image, y_row)) return DMX_ERR_ARG;
  if (N == 0 || L == 0) return DMX_OK;
  if (!x || !y || !mean || !rstd) return DMX_ERR_ARG;
  const int e = dtype == DMX_F32 ? 4 : 2;
  if (!element_aligned(x, e) || !element_aligned(y, e) || !element_aligned(mean, 4) || !element_aligned(rstd, 4) ||
      !element_aligned(weight, 4) || !element_aligned(bias, 4) || !element_aligned(workspace, 16)) return DMX_ERR_ALIGN;
  const bool vec = columns_fit(C, C / G, e) && wide(x, N, L, C, x_image, x_row, e) && wide(y, N, L, C, y_image, y_row, e);
  const int64_t need = workspace_for(N, L, C, G, dtype, vec, false);
  if (workspace_bytes < need || (need > 0 && !workspace)) return DMX_ERR_ARG;
  const Plan p = plan(N, L, C, C / G, dtype, vec, false);
  if (N * p.slabs * (int64_t)p.parts > 0x7fffffff) return DMX_ERR_ARG;
  Args A = {};
  A.x = {const_cast<void*>(x), x_image, x_row};
  A.out = {y, y_image, y_row};
  A.weight = weight; A.bias = bias; A.mean = mean; A.rstd = rstd; A.part = static_cast<float*>(workspace);
  fill(A, p, N, L, C, G);
  A.eps = eps; A.act = act;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (dtype == DMX_F32) return vec ? run_forward<float, 4>(p, A, st) : run_forward<float, 1>(p, A, st);
  return vec ? run_forward<__nv_bfloat16, 8>(p, A, st) : run_forward<__nv_bfloat16, 1>(p, A, st);
}

int dmx_group_norm_backward(int64_t N, int64_t L, int C, int G, int dtype, const void* dy, int64_t dy_image,
                            int64_t dy_row, const void* x, int64_t x_image, int64_t x_row, const float* mean,
                            const float* rstd, const float* weight, const float* bias, int act, void* dx,
                            int64_t dx_image, int64_t dx_row, float* dweight, float* dbias, void* workspace,
                            int64_t workspace_bytes, void* cuda_stream) {
  if (!shape_ok(N, L, C, G, dtype) || act < DMX_ACT_NONE || act > DMX_ACT_GELU) return DMX_ERR_ARG;
  if (!strides_ok(N, L, C, x_image, x_row) || !strides_ok(N, L, C, dy_image, dy_row) || !strides_ok(N, L, C, dx_image, dx_row)) return DMX_ERR_ARG;
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
  const int64_t need = workspace_for(N, L, C, G, dtype, vec, true);
  if (workspace_bytes < need || !workspace) return DMX_ERR_ARG;
  const Plan p = plan(N, L, C, C / G, dtype, vec, true);
  if (N * p.slabs * (int64_t)p.parts > 0x7fffffff) return DMX_ERR_ARG;
  Args A = {};
  A.x = {const_cast<void*>(x), x_image, x_row};
  A.dy = {const_cast<void*>(dy), dy_image, dy_row};
  A.out = {dx, dx_image, dx_row};
  A.weight = weight; A.bias = bias; A.mean = const_cast<float*>(mean); A.rstd = const_cast<float*>(rstd); A.part = static_cast<float*>(workspace);
  fill(A, p, N, L, C, G);
  A.act = act;
  int rc;
  if (dtype == DMX_F32) rc = vec ? run_backward<float, 4>(p, A, st) : run_backward<float, 1>(p, A, st);
  else rc = vec ? run_backward<__nv_bfloat16, 8>(p, A, st) : run_backward<__nv_bfloat16, 1>(p, A, st);
  if (rc != DMX_OK || (!dweight && !dbias)) return rc;
  columns_kernel<<<dim3((C + 31) / 32, 2), 256, 0, st>>>(A.part, N * (p.resident ? 1 : p.parts), C, dweight, dbias);
  return dmxh::cuda_ok(cudaGetLastError()) ? DMX_OK : DMX_ERR_CUDA;
}

}  // extern "C"
