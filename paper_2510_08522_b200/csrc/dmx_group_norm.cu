// dmx_group_norm.cu — group norm with an activation on channels-last data, and its gradient.
//
// forward    per image and group: mean and variance over L positions x C/G channels, then
//            y = act((x - mean) rstd w + b)
// backward   du = dy act'(u), xh = (x - mean) rstd; per image and channel A_c = sum du xh, B_c = sum du over the
//            positions; dx = rstd (w du - (sum_c w B_c + xh sum_c w A_c) / n); dweight, dbias = sums of A, B over images
//
// Bound: HBM. The values have to be known before the first result, so x (and dy) is either read twice or kept
// on the chip. Here it is kept, in registers: a CTA takes a slab of neighbouring whole groups and a range of
// positions, each thread a fixed column of 16 bytes (or one element, where alignment allows no more) and every
// R-th position, all its loads in flight at once; up to eight CTAs of a cluster share an image's slab and
// exchange their groups' sums through distributed shared memory. One read, one write. An image too large for
// that (512 KB per slab of 64 bytes forward, half of it backward) is cut into chunks: one launch for the chunks' sums, one that
// reads again, mostly from L2.
// Variances come from deviations: a CTA's from the mean of its own values, the CTAs' joined by the
// difference of their means (Chan, Golub, LeVeque 1983). Nothing is added atomically; the order of all sums is
// fixed by the shape.
#include "dmx.h"

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "dmx_act.cuh"
#include "dmx_host.h"

namespace {

namespace cg = cooperative_groups;

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
  int64_t L;
  int C, G, cpg, W, slabs, R, cols, rows;   // W channels per slab, R positions at a time, cols columns of V, rows positions per CTA
  int parts;             // CTAs (or chunks) per image and slab
  float eps;
  int act;
  int N;
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

// The arrays in shared memory start on 16 bytes, whatever their length.
__host__ __device__ constexpr int padded(int n) { return (n + 3) & ~3; }

template <int V>
__device__ __forceinline__ void from_shared(const float* p, float (&x)[V]) {
#pragma unroll
  for (int v = 0; v < V; ++v) x[v] = p[v];
}

// Sums over a slab's groups of red[R][width], width = a value per channel, or per column where a column lies in
// one group. `each` lanes add a group's values, in a fixed order.
__device__ __forceinline__ void group_sums(const float* red, float* out, int groups, int per, int R, int width) {
  const int total = R * per;
  int each = 1;
  while (each < 32 && each < total) each <<= 1;
  const int l = threadIdx.x & (each - 1);
  const int dr = each / per, dc = each - dr * per;
  for (int g0 = 0; g0 < groups; g0 += blockDim.x / each) {
    const int g = g0 + threadIdx.x / each;
    float s = 0.f;
    if (g < groups) {
      int r = l / per, c = l - r * per;
      for (int k = l; k < total; k += each) {
        s += red[r * width + g * per + c];
        r += dr; c += dc;
        if (c >= per) { c -= per; ++r; }
      }
    }
    for (int o = each >> 1; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (g < groups && l == 0) out[g] = s;
  }
}

// What every mode starts with: the CTA's place, and its values in registers.
struct Here {
  int n, slab, part, c0, Wl, groups, col, rl;
  int64_t r0, rows;
  bool on;
};
__device__ __forceinline__ Here here(const Args& A, int V) {
  Here h;
  int b = blockIdx.x;
  h.part = b % A.parts; b /= A.parts;
  h.slab = b % A.slabs;
  h.n = b / A.slabs;
  h.c0 = h.slab * A.W;
  h.Wl = min(A.W, A.C - h.c0);
  h.groups = h.Wl / A.cpg;
  h.rl = threadIdx.x / A.cols;
  h.col = threadIdx.x - h.rl * A.cols;
  h.r0 = (int64_t)h.part * A.rows;
  h.rows = min((int64_t)A.rows, A.L - h.r0);
  if (h.rows < 0) h.rows = 0;
  h.on = h.rl < A.R && h.col * V < h.Wl;
  return h;
}
template <typename T, int V, int NV>
__device__ __forceinline__ void read(const Operand& o, const Here& h, int R, typename Vec<T, V>::type (&raw)[NV]) {
  using U = typename Vec<T, V>::type;
  const T* p = static_cast<const T*>(o.p) + h.n * o.image + (h.r0 + h.rl) * o.row + h.c0 + h.col * V;
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (h.on && h.rl + i * R < h.rows) raw[i] = __ldcs(reinterpret_cast<const U*>(p + (int64_t)i * R * o.row));
}

// RESIDENT: the whole job, the CTAs of an image's slab being one cluster. STATS: the chunks' sums only.
// APPLY: the results, from the chunks' sums.
enum Mode { RESIDENT, STATS, APPLY };

template <typename T, int V, int NV, Mode M>
__global__ void __launch_bounds__(V == 1 ? 1024 : 256) forward_kernel(const __grid_constant__ Args A) {
  extern __shared__ __align__(16) float sm[];
  const Here h = here(A, V);
  const int W = A.W, cpg = A.cpg, R = A.R;
  typename Vec<T, V>::type raw[NV];
  read<T, V, NV>(A.x, h, R, raw);
  float* cmean = sm;               // per channel
  float* ca = cmean + padded(W);   // rstd * weight
  float* cb = ca + padded(W);      // bias
  float2* gst = reinterpret_cast<float2*>(cb + padded(W));   // per group: sum, sum of squared deviations
  float* red = reinterpret_cast<float*>(gst) + padded(2 * (W / cpg));
  const bool inner = cpg % V == 0;                   // a column lies in one group
  const int width = inner ? A.cols : W, per = inner ? cpg / V : cpg;
  cg::cluster_group cluster = cg::this_cluster();

  if constexpr (M != APPLY) {
    float acc[V];
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
      float mu[V];
      if (pass == 1 && h.on) from_shared<V>(cmean + h.col * V, mu);
#pragma unroll
      for (int v = 0; v < V; ++v) acc[v] = 0.f;
      if (h.on) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          if (h.rl + i * R >= h.rows) continue;
          float x[V];
          widen(raw[i], x);
#pragma unroll
          for (int v = 0; v < V; ++v) {
            if (pass == 0) acc[v] += x[v];
            else { const float d = x[v] - mu[v]; acc[v] = fmaf(d, d, acc[v]); }
          }
        }
      }
      if (h.rl < R) {
        if (inner) {
          float s = acc[0];
#pragma unroll
          for (int v = 1; v < V; ++v) s += acc[v];
          red[h.rl * width + h.col] = s;
        } else {
#pragma unroll
          for (int v = 0; v < V; ++v) red[h.rl * width + h.col * V + v] = acc[v];
        }
      }
      __syncthreads();
      float* gs = reinterpret_cast<float*>(red) + R * width;
      group_sums(red, gs, h.groups, per, R, width);
      __syncthreads();
      const float inv = h.rows > 0 ? 1.f / ((float)h.rows * (float)cpg) : 0.f;
      for (int g = threadIdx.x; g < h.groups; g += blockDim.x) {
        if (pass == 0) gst[g].x = gs[g];
        else gst[g].y = gs[g];
      }
      if (pass == 0)
        for (int c = threadIdx.x; c < h.Wl; c += blockDim.x) cmean[c] = gs[c / cpg] * inv;
      __syncthreads();
    }
    if constexpr (M == STATS) {
      float2* out = reinterpret_cast<float2*>(A.part) + ((int64_t)h.n * A.parts + h.part) * A.G + h.c0 / cpg;
      for (int g = threadIdx.x; g < h.groups; g += blockDim.x) out[g] = gst[g];
      return;
    } else if (A.parts > 1) {
      cluster.sync();
    }
  }
  // join the parts of each group, in their order
  float2* tot = reinterpret_cast<float2*>(red);       // per group: mean, rstd (red is not needed any more)
  for (int g = threadIdx.x; g < h.groups; g += blockDim.x) {
    const float n = (float)A.L * (float)cpg;
    float2 st[kMaxCluster];
    float sum = 0.f, m2 = 0.f;
    const float2* src = reinterpret_cast<const float2*>(A.part) + (int64_t)h.n * A.parts * A.G + h.c0 / cpg + g;
    if constexpr (M == RESIDENT) {
      for (int k = 0; k < A.parts; ++k) {
        st[k] = A.parts > 1 ? cluster.map_shared_rank(gst, k)[g] : gst[g];
        sum += st[k].x;
      }
    } else {
      for (int k = 0; k < A.parts; ++k) sum += __ldg(&src[(int64_t)k * A.G]).x;
    }
    const float mean = sum / n;
    for (int k = 0; k < A.parts; ++k) {
      const float2 s = M == RESIDENT ? st[k] : __ldg(&src[(int64_t)k * A.G]);
      const float rows = (float)(min((int64_t)(k + 1) * A.rows, A.L) - min((int64_t)k * A.rows, A.L)) * (float)cpg;
      if (rows > 0.f) {
        const float d = s.x / rows - mean;
        m2 += fmaf(rows * d, d, s.y);
      }
    }
    const float rstd = 1.f / sqrtf(m2 / n + A.eps);
    tot[g] = make_float2(mean, rstd);
    if (h.part == 0) {
      const int64_t at = (int64_t)h.n * A.G + h.c0 / cpg + g;
      A.mean[at] = mean;
      A.rstd[at] = rstd;
    }
  }
  if (M == RESIDENT && A.parts > 1) cg::this_cluster().barrier_arrive();
  __syncthreads();
  for (int c = threadIdx.x; c < h.Wl; c += blockDim.x) {
    const float2 t = tot[c / cpg];
    cmean[c] = t.x;
    ca[c] = A.weight ? t.y * __ldg(A.weight + h.c0 + c) : t.y;
    cb[c] = A.bias ? __ldg(A.bias + h.c0 + c) : 0.f;
  }
  __syncthreads();
  if (h.on) {
    float mu[V], a[V], b[V];
    from_shared<V>(cmean + h.col * V, mu);
    from_shared<V>(ca + h.col * V, a);
    from_shared<V>(cb + h.col * V, b);
    T* out = static_cast<T*>(A.out.p) + h.n * A.out.image + (h.r0 + h.rl) * A.out.row + h.c0 + h.col * V;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (h.rl + i * R >= h.rows) continue;
      float x[V];
      widen(raw[i], x);
#pragma unroll
      for (int v = 0; v < V; ++v) x[v] = fmaf(x[v] - mu[v], a[v], b[v]);
      dmx_act::apply<V>(x, A.act);
      put(out + (int64_t)i * R * A.out.row, x);
    }
  }
  if (M == RESIDENT && A.parts > 1) cg::this_cluster().barrier_wait();     // its sums may still be read until here
}

// Backward. Workspace: A and B per image (and chunk) and channel, [2][N*chunks][C]; `part` rows.
template <typename T, int V, int NV, Mode M>
__global__ void __launch_bounds__(V == 1 ? 1024 : 256) backward_kernel(const __grid_constant__ Args A) {
  extern __shared__ __align__(16) float sm[];
  const Here h = here(A, V);
  const int W = A.W, cpg = A.cpg, R = A.R;
  typename Vec<T, V>::type rx[NV], rg[NV];
  read<T, V, NV>(A.x, h, R, rx);
  read<T, V, NV>(A.dy, h, R, rg);
  float* cmean = sm;
  float* crs = cmean + W;
  float* cw = crs + W;
  float* cb = cw + W;
  float* chA = cb + W;             // this CTA's channel sums (read by the cluster)
  float* chB = chA + W;
  float* red = chB + W;            // two of R*W
  const int64_t sidx = (int64_t)h.n * A.G + h.c0 / cpg;
  for (int c = threadIdx.x; c < h.Wl; c += blockDim.x) {
    cmean[c] = __ldg(A.mean + sidx + c / cpg);
    crs[c] = __ldg(A.rstd + sidx + c / cpg);
    cw[c] = A.weight ? __ldg(A.weight + h.c0 + c) : 1.f;
    cb[c] = A.bias ? __ldg(A.bias + h.c0 + c) : 0.f;
  }
  __syncthreads();
  float mu[V], rs[V], w[V], b[V];
  if (h.on) {
    from_shared<V>(cmean + h.col * V, mu);
    from_shared<V>(crs + h.col * V, rs);
    from_shared<V>(cw + h.col * V, w);
    from_shared<V>(cb + h.col * V, b);
  }
  cg::cluster_group cluster = cg::this_cluster();
  const int64_t plane = (int64_t)A.N * (M == RESIDENT ? 1 : A.parts) * A.C;
  if constexpr (M != APPLY) {
    float sa[V], sb[V];
#pragma unroll
    for (int v = 0; v < V; ++v) sa[v] = sb[v] = 0.f;
    if (h.on) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (h.rl + i * R >= h.rows) continue;
        float x[V], g[V], u[V];
        widen(rx[i], x);
        widen(rg[i], g);
#pragma unroll
        for (int v = 0; v < V; ++v) { x[v] = (x[v] - mu[v]) * rs[v]; u[v] = fmaf(x[v], w[v], b[v]); }
        dmx_act::times_slope<V>(g, u, A.act);
#pragma unroll
        for (int v = 0; v < V; ++v) { sa[v] = fmaf(g[v], x[v], sa[v]); sb[v] += g[v]; }
      }
    }
    if (h.rl < R) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        red[h.rl * W + h.col * V + v] = sa[v];
        red[(R + h.rl) * W + h.col * V + v] = sb[v];
      }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < h.Wl; c += blockDim.x) {
      float a = 0.f, bb = 0.f;
      for (int r = 0; r < R; ++r) { a += red[r * W + c]; bb += red[(R + r) * W + c]; }
      chA[c] = a;
      chB[c] = bb;
    }
    __syncthreads();
    if constexpr (M == STATS) {
      float* out = A.part + ((int64_t)h.n * A.parts + h.part) * A.C + h.c0;
      for (int c = threadIdx.x; c < h.Wl; c += blockDim.x) { out[c] = chA[c]; out[plane + c] = chB[c]; }
      return;
    } else if (A.parts > 1) {
      cluster.sync();
    }
  }
  // channel totals over the parts, in their order; then the groups' weighted sums
  for (int c = threadIdx.x; c < h.Wl; c += blockDim.x) {
    float a = 0.f, bb = 0.f;
    if constexpr (M == RESIDENT) {
      for (int k = 0; k < A.parts; ++k) {
        a += A.parts > 1 ? cluster.map_shared_rank(chA, k)[c] : chA[c];
        bb += A.parts > 1 ? cluster.map_shared_rank(chB, k)[c] : chB[c];
      }
      if (h.part == 0 && A.part) {
        float* out = A.part + (int64_t)h.n * A.C + h.c0;
        out[c] = a;
        out[plane + c] = bb;
      }
    } else {
      const float* src = A.part + (int64_t)h.n * A.parts * A.C + h.c0 + c;
      for (int k = 0; k < A.parts; ++k) { a += __ldg(src + (int64_t)k * A.C); bb += __ldg(src + plane + (int64_t)k * A.C); }
    }
    red[c] = a * cw[c];
    red[W + c] = bb * cw[c];
  }
  if (M == RESIDENT && A.parts > 1) cg::this_cluster().barrier_arrive();
  __syncthreads();
  float* gs = red + 2 * W;
  group_sums(red, gs, h.groups, cpg, 1, W);
  group_sums(red + W, gs + h.groups, h.groups, cpg, 1, W);
  __syncthreads();
  if (h.on) {
    float s1[V], s2[V];
    const float n = 1.f / ((float)A.L * (float)cpg);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int g = (h.col * V + v) / cpg;
      s2[v] = gs[g] * n;
      s1[v] = gs[h.groups + g] * n;
    }
    T* out = static_cast<T*>(A.out.p) + h.n * A.out.image + (h.r0 + h.rl) * A.out.row + h.c0 + h.col * V;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (h.rl + i * R >= h.rows) continue;
      float x[V], g[V], u[V];
      widen(rx[i], x);
      widen(rg[i], g);
#pragma unroll
      for (int v = 0; v < V; ++v) { x[v] = (x[v] - mu[v]) * rs[v]; u[v] = fmaf(x[v], w[v], b[v]); }
      dmx_act::times_slope<V>(g, u, A.act);
#pragma unroll
      for (int v = 0; v < V; ++v) x[v] = rs[v] * (fmaf(g[v], w[v], -s1[v]) - x[v] * s2[v]);
      put(out + (int64_t)i * R * A.out.row, x);
    }
  }
  if (M == RESIDENT && A.parts > 1) cg::this_cluster().barrier_wait();
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
  int V, W, slabs, parts, rows, R, cols, threads, nv;
  bool resident;
  size_t smem;
};

int lcm(int a, int b) {
  int x = a, y = b;
  while (y) { const int t = x % y; x = y; y = t; }
  return a / x * b;
}

// Slab width, CTAs per image and slab, and positions per thread. Slabs are multiples of whole groups and of
// whole columns. Among the splits that keep an image's slab in one cluster's registers: segments of at least
// 128 bytes, then 64, then 32 (a DRAM sector); within a width the fewest CTAs per slab that still make
// two for every SM. Where the problem is too small for that, narrow slabs come first (no exchange needed).
Plan plan(int64_t N, int64_t L, int C, int cpg, int dtype, bool vec, bool backward) {
  Plan p;
  const int e = dtype == DMX_F32 ? 4 : 2;
  p.V = vec ? 16 / e : 1;
  const int unit = lcm(cpg, p.V);
  const int nvmax = p.V == 1 ? 16 : backward ? 8 : 16;
  const int tmax = 256;
  bool found = false;
  const int want[4] = {512, 128, 64, 32};
  for (int k = 0; k < 4 && !found; ++k) {
    int W = (want[k] / e) / unit * unit;
    if (W < unit) W = unit;
    if (W > C) W = C;
    if (k == 0 && W * e < 512 && W < C) continue;
    p.W = W;
    p.slabs = (C + W - 1) / W;
    p.cols = (W + p.V - 1) / p.V;
    p.threads = p.cols <= tmax ? tmax : p.V == 1 ? 1024 : tmax;
    p.R = p.threads / p.cols;
    for (p.parts = 1; p.parts <= kMaxCluster; p.parts *= 2) {
      const int64_t rows = (L + p.parts - 1) / p.parts;
      const int64_t nv = (rows + p.R - 1) / p.R;
      if (nv > nvmax) continue;
      const bool narrower = k < 3 && unit * e < want[k];
      if (N * p.slabs * p.parts < 2 * 148) {
        if (narrower && k < 2) break;                       // more CTAs from narrower slabs first
        if (p.parts < kMaxCluster && nv > 1) continue;      // then from more of them per slab
      }
      p.rows = (int)rows;
      p.nv = (int)nv;
      found = true;
      break;
    }
  }
  p.resident = found;
  if (!found) {
    int W = (256 / e) / unit * unit;
    if (W < unit) W = unit;
    if (W > C) W = C;
    p.W = W;
    p.slabs = (C + W - 1) / W;
    p.cols = (W + p.V - 1) / p.V;
    p.threads = p.cols <= tmax ? tmax : p.V == 1 ? 1024 : tmax;
    p.R = p.threads / p.cols;
    p.nv = 8;
    const int64_t rows = (int64_t)p.R * p.nv;
    p.rows = (int)rows;
    p.parts = (int)((L + rows - 1) / rows);
  }
  int nv = 1;
  while (nv < p.nv) nv *= 2;
  p.nv = nv;
  const size_t f = sizeof(float);
  const size_t groups = p.W / cpg;
  if (backward) p.smem = f * (6 * (size_t)p.W + (size_t)(2 * p.R > 2 ? 2 * p.R : 2) * p.W + 2 * groups);
  else p.smem = f * (3 * (size_t)padded(p.W) + padded(2 * (int)groups) + (size_t)p.R * p.cols * p.V + 2 * groups);
  return p;
}

template <typename K>
int launch(K kernel, const Plan& p, const Args& A, int64_t ctas, bool cluster, cudaStream_t st) {
  if (p.smem > 48 * 1024 && !dmxh::cuda_ok(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)p.smem))) return DMX_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(p.threads);
  cfg.dynamicSmemBytes = p.smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1] = {};
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster ? p.parts : 1;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return dmxh::cuda_ok(cudaLaunchKernelEx(&cfg, kernel, A)) ? DMX_OK : DMX_ERR_CUDA;
}

template <typename T, int V>
int run_forward(const Plan& p, const Args& A, int64_t ctas, cudaStream_t st) {
  if (!p.resident) {
    const int rc = launch(forward_kernel<T, V, 8, STATS>, p, A, ctas, false, st);
    return rc != DMX_OK ? rc : launch(forward_kernel<T, V, 8, APPLY>, p, A, ctas, false, st);
  }
  switch (p.nv) {
    case 1: return launch(forward_kernel<T, V, 1, RESIDENT>, p, A, ctas, true, st);
    case 2: return launch(forward_kernel<T, V, 2, RESIDENT>, p, A, ctas, true, st);
    case 4: return launch(forward_kernel<T, V, 4, RESIDENT>, p, A, ctas, true, st);
    case 8: return launch(forward_kernel<T, V, 8, RESIDENT>, p, A, ctas, true, st);
    default: return launch(forward_kernel<T, V, 16, RESIDENT>, p, A, ctas, true, st);
  }
}

template <typename T, int V>
int run_backward(const Plan& p, const Args& A, int64_t ctas, cudaStream_t st) {
  if (!p.resident) {
    const int rc = launch(backward_kernel<T, V, 8, STATS>, p, A, ctas, false, st);
    return rc != DMX_OK ? rc : launch(backward_kernel<T, V, 8, APPLY>, p, A, ctas, false, st);
  }
  switch (p.nv) {
    case 1: return launch(backward_kernel<T, V, 1, RESIDENT>, p, A, ctas, true, st);
    case 2: return launch(backward_kernel<T, V, 2, RESIDENT>, p, A, ctas, true, st);
    case 4: return launch(backward_kernel<T, V, 4, RESIDENT>, p, A, ctas, true, st);
    case 8: return launch(backward_kernel<T, V, 8, RESIDENT>, p, A, ctas, true, st);
    default:
      if constexpr (V == 1) return launch(backward_kernel<T, V, 16, RESIDENT>, p, A, ctas, true, st);
      return DMX_ERR_ARG;
  }
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
  const int64_t ctas = N * p.slabs * p.parts;
  if (ctas > 0x7fffffff) return DMX_ERR_ARG;
  Args A = {};
  A.x = {const_cast<void*>(x), x_image, x_row};
  A.out = {y, y_image, y_row};
  A.weight = weight; A.bias = bias; A.mean = mean; A.rstd = rstd; A.part = static_cast<float*>(workspace);
  A.L = L; A.C = C; A.G = G; A.cpg = C / G; A.W = p.W; A.slabs = p.slabs; A.R = p.R; A.cols = p.cols; A.rows = p.rows;
  A.parts = p.parts; A.eps = eps; A.act = act; A.N = (int)N;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (dtype == DMX_F32) return vec ? run_forward<float, 4>(p, A, ctas, st) : run_forward<float, 1>(p, A, ctas, st);
  return vec ? run_forward<__nv_bfloat16, 8>(p, A, ctas, st) : run_forward<__nv_bfloat16, 1>(p, A, ctas, st);
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
  const int64_t ctas = N * p.slabs * p.parts;
  if (ctas > 0x7fffffff) return DMX_ERR_ARG;
  Args A = {};
  A.x = {const_cast<void*>(x), x_image, x_row};
  A.dy = {const_cast<void*>(dy), dy_image, dy_row};
  A.out = {dx, dx_image, dx_row};
  A.weight = weight; A.bias = bias; A.mean = const_cast<float*>(mean); A.rstd = const_cast<float*>(rstd); A.part = static_cast<float*>(workspace);
  A.L = L; A.C = C; A.G = G; A.cpg = C / G; A.W = p.W; A.slabs = p.slabs; A.R = p.R; A.cols = p.cols; A.rows = p.rows;
  A.parts = p.parts; A.act = act; A.N = (int)N;
  int rc;
  if (dtype == DMX_F32) rc = vec ? run_backward<float, 4>(p, A, ctas, st) : run_backward<float, 1>(p, A, ctas, st);
  else rc = vec ? run_backward<__nv_bfloat16, 8>(p, A, ctas, st) : run_backward<__nv_bfloat16, 1>(p, A, ctas, st);
  if (rc != DMX_OK || (!dweight && !dbias)) return rc;
  columns_kernel<<<dim3((C + 31) / 32, 2), 256, 0, st>>>(A.part, N * (p.resident ? 1 : p.parts), C, dweight, dbias);
  return dmxh::cuda_ok(cudaGetLastError()) ? DMX_OK : DMX_ERR_CUDA;
}

}  // extern "C"
