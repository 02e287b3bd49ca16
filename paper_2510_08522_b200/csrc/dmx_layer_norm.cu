// dmx_layer_norm.cu — layer norm over rows, and its gradient.
//
// forward    mean and variance of a row's D values, y = (x - mean) rstd w + b
// backward   xh = (x - mean) rstd, g = w dy; dx = rstd (g - (sum g + xh sum g xh) / D) + add; dw = sum of dy xh over the rows, db = sum of dy
//
// Bound: HBM. A team of threads (8 lanes, a warp, a CTA, or a cluster of CTAs, by the row's width) holds a row in registers, up to
// 32 values a thread, so that everything is read once; teams stay and take row after row. Rows to come are on their way into shared
// memory by asynchronous copies, every thread its own columns into slots of its own (no barrier between copy and use). In backward a
// thread's columns are the same in every row: it sums its share of dw and db in registers, a CTA's teams join theirs in shared memory, and a
// small second launch adds the CTAs' in a fixed order.
// Variance: deviations from the rounded mean are summed beside their squares, and what that mean was off is taken out again:
// a mean a million deviations away costs the variance nothing.
// Measured on B200 (replayed in graphs, data mostly in L2): 16384 x 1024 bf16 forward 12 us (10.4 at the measured copy rate; 14 us a call among others), fp32 24 us (20.9),
// gradient 22 us (15.6), fp32 36 (31.3), without dw and db 17 and 31, with a residual 28 us (20.9): about 550 instructions a row and warp at eight warps per SM, of which two fifths issue.
// 2999 x 771 fp32, a slice of wider rows, gradient 13 us (4.3): three rows a warp, and 4.5 us for the second launch. A third CTA per SM in backward spilled (37 us), five warps a CTA too (40 us),
// weights loaded anew for every row cost 8 us, halves kept packed over the row's loop saved no instruction.
#include <atomic>

#include "dmx_f32x2.cuh"
#include "dmx_rows.cuh"

namespace {

using namespace dmx_rows;
using namespace dmx_f32x2;

constexpr int kMaxCluster = 8, kMaxWarps = 16;      // of a CTA that is one team
// Rows on their way to a team: with the warps there are, more than the 40 KB that an SM has to have on its way
constexpr int kForwardStages = 4;
__host__ __device__ constexpr int backward_stages(int bytes) { return bytes == 2 ? 3 : 2; }
// CTAs on an SM, for their registers (a thread of backward holds its sums, 2 N, and a row's values, 2 N)
constexpr int forward_ctas(int values, bool wide) { return values == 32 ? 3 + wide : values == 16 ? 4 + wide : 6; }
constexpr int backward_ctas(int values) { return values == 32 ? 2 : values == 16 ? 4 : 6; }

struct Args {
  const void *x, *dy, *add;
  void* out;                                       // y or dx
  int64_t ldx, lddy, ldadd, ldout, M;
  const float *weight, *bias;
  float *mean, *rstd;                              // forward: outputs; backward: inputs
  float* part;                                     // backward: [CTAs of a cluster's rows][2][D]
  int D, wvec;                                     // wvec: weight and bias in 16-byte accesses
  float eps;
};

// How a row is held. TEAM: lanes of a warp that share a row, 0 a CTA, -1 a cluster. N values per thread, in accesses of V neighbours: 16 bytes,
// or single elements where alignment allows no more. Rows to come are copied 16 bytes at a time in either case: with single elements a
// team's threads copy what covers the row from one 16-byte border to the next (the bytes before its start lie in the same 16, and are not used).
template <typename T, int V, int TEAM, int N>
struct Held {
  static constexpr int kAccesses = N / V, kThreads = TEAM > 0 ? 128 : 8192 / N;
  typedef typename Vec<T, V>::type Raw;

  int t, size;          // access i has the columns from (i * size + t) * V on
  int own, first, D;    // this thread among its team's in this CTA; this CTA's first column
  int threads;          // of the team in this CTA
  int64_t row, step, group;      // the team's first row, the rows between its rows; the CTA (or cluster)

  __device__ __forceinline__ explicit Held(int D_) : D(D_) {
    first = 0;
    if constexpr (TEAM > 0) {
      const int teams = blockDim.x / TEAM;
      own = threadIdx.x % TEAM; threads = size = TEAM;
      group = blockIdx.x;
      row = group * teams + threadIdx.x / TEAM; step = (int64_t)gridDim.x * teams;
      t = own;
    } else {
      unsigned rank = 0, n = 1;
      if constexpr (TEAM < 0) {
        asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
        asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
      }
      own = threadIdx.x; threads = blockDim.x;
      row = group = blockIdx.x / n; step = gridDim.x / n;
      if constexpr (V > 1) { t = rank * blockDim.x + own; size = n * blockDim.x; }          // all CTAs' accesses in turn
      else { first = rank * N * blockDim.x; t = first + own; size = blockDim.x; }           // each CTA a range
    }
  }
  __device__ __forceinline__ int column(int i) const { return (i * size + t) * V; }
  // bytes that one row of one input takes in a stage, of all teams of the CTA
  static __host__ __device__ constexpr int stage_bytes(int ctaThreads) { return ctaThreads * N * (int)sizeof(T) + (V > 1 ? 0 : 32 * (TEAM > 0 ? ctaThreads / (TEAM > 0 ? TEAM : 1) : 1)); }
  // where this thread (V > 1) or its team (V = 1) finds its part of a stage
  __device__ __forceinline__ unsigned char* slot(unsigned char* stage) const {
    if constexpr (V > 1) return stage + threadIdx.x * sizeof(Raw);
    else return stage + threadIdx.x / threads * (threads * N * (int)sizeof(T) + 32);
  }
  __device__ __forceinline__ void send(unsigned char* to, const void* p, int64_t ld, int64_t r) const {
    const unsigned dst = (unsigned)__cvta_generic_to_shared(to);
    if constexpr (V > 1) {
      const T* q = static_cast<const T*>(p) + r * ld + t * V;
      const unsigned apart = blockDim.x * sizeof(Raw);
      if (D == N * size) {
#pragma unroll
        for (int i = 0; i < kAccesses; ++i) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + i * apart), "l"(q + i * size * V) : "memory");
      } else {
#pragma unroll
        for (int i = 0; i < kAccesses; ++i) {
          const bool in = column(i) < D;                   // behind the row's end: zeros
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + i * apart), "l"(in ? q + i * size * V : static_cast<const T*>(p)), "r"(in ? 16 : 0) : "memory");
        }
      }
    } else {
      const T* q = static_cast<const T*>(p) + r * ld + first;
      const int count = min(D - first, N * threads), shift = (int)(reinterpret_cast<uintptr_t>(q) & 15);
      const unsigned char* from = reinterpret_cast<const unsigned char*>(q) - shift;
      const int bytes = count > 0 ? shift + count * (int)sizeof(T) : 0;
      const unsigned char* nothing = reinterpret_cast<const unsigned char*>(reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)15);
#pragma unroll
      for (int i = 0; i <= N * (int)sizeof(T) / 16; ++i) {
        const int at = (i * threads + own) * 16, left = bytes - at;
        if (at >= threads * N * (int)sizeof(T) + 32) continue;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + at), "l"(left > 0 ? from + at : nothing), "r"(left > 16 ? 16 : left > 0 ? left : 0)
                     : "memory");
      }
    }
  }
  // (With single elements they come from other threads' copies: the team meets before it takes them.)
  static __device__ __forceinline__ void meet() {
    if constexpr (V == 1) {
      if constexpr (TEAM > 0) __syncwarp();
      else __syncthreads();
    }
  }
  // access i of row r out of the slot
  __device__ __forceinline__ void take(int i, const unsigned char* slot, const void* p, int64_t ld, int64_t r, float* x) const {
    if constexpr (V > 1) {
      widen<T>(*reinterpret_cast<const Raw*>(slot + i * blockDim.x * sizeof(Raw)), x);
    } else {
      const int shift = (int)(reinterpret_cast<uintptr_t>(static_cast<const T*>(p) + r * ld + first) & 15);
      widen<T>(*reinterpret_cast<const Raw*>(slot + shift + (i * threads + own) * sizeof(T)), x);
    }
  }
  __device__ __forceinline__ void store(void* p, int64_t ld, int64_t r, const float (&x)[N]) const {
    T* q = static_cast<T*>(p) + r * ld;
#pragma unroll
    for (int i = 0; i < kAccesses; ++i)
      if (column(i) < D) *reinterpret_cast<Raw*>(q + column(i)) = narrow<T, V>(x + i * V);
  }
  // an fp32 vector's values at this thread's columns; `otherwise` where there is no vector
  __device__ __forceinline__ void vector(const float* w, int wvec, float otherwise, float (&x)[N]) const {
#pragma unroll
    for (int i = 0; i < kAccesses; ++i) {
      const int c = column(i);
      if (V > 1 && w && wvec) {
#pragma unroll
        for (int k = 0; k < V; k += 4) {
          const float4 v = c < D ? *reinterpret_cast<const float4*>(w + c + k) : make_float4(0.f, 0.f, 0.f, 0.f);
          x[i * V + k] = v.x; x[(i * V + k + 1) % N] = v.y; x[(i * V + k + 2) % N] = v.z; x[(i * V + k + 3) % N] = v.w;
        }
      } else {
#pragma unroll
        for (int k = 0; k < V; ++k) x[i * V + k] = w ? (c < D ? w[c + k] : 0.f) : otherwise;
      }
    }
  }
  // The vector in shared memory, [N / 4][threads] float4 or [N][threads] floats: a thread reads what it (and others alike) wrote.
  __device__ __forceinline__ void keep(float* held, const float (&x)[N]) const {
#pragma unroll
    for (int j = 0; j < N; j += V > 1 ? 4 : 1) {
      if constexpr (V > 1) reinterpret_cast<float4*>(held)[j / 4 * threads + own] = make_float4(x[j], x[(j + 1) % N], x[(j + 2) % N], x[(j + 3) % N]);
      else held[j * threads + own] = x[j];
    }
  }
  __device__ __forceinline__ void kept(const float* held, int i, float (&x)[V]) const {
    if constexpr (V > 1) {
#pragma unroll
      for (int k = 0; k < V; k += 4) {
        const float4 v = reinterpret_cast<const float4*>(held)[(i * V + k) / 4 * threads + own];
        x[k] = v.x; x[(k + 1) % V] = v.y; x[(k + 2) % V] = v.z; x[(k + 3) % V] = v.w;
      }
    } else {
      x[0] = held[i * threads + own];
    }
  }
  // zeros behind the row's end
  __device__ __forceinline__ void cut(float (&x)[N]) const {
#pragma unroll
    for (int i = 0; i < kAccesses; ++i) {
      if (first + (i + 1) * size * V <= D) continue;       // (the same for all)
#pragma unroll
      for (int k = 0; k < V; ++k) x[i * V + k] = column(i) < D ? x[i * V + k] : 0.f;
    }
  }
};

template <int STAGES>
__device__ __forceinline__ void copies_landed() { asm volatile("cp.async.wait_group %0;" ::"n"(STAGES) : "memory"); }
__device__ __forceinline__ void copies_sent() { asm volatile("cp.async.commit_group;" ::: "memory"); }

__device__ __forceinline__ float2 pair(const float* x, int i) { return make_float2(x[2 * i], x[2 * i + 1]); }
__device__ __forceinline__ void set_pair(float* x, int i, float2 v) { x[2 * i] = v.x; x[2 * i + 1] = v.y; }

// Sums of two values over a team. `red`: two buffers of kMaxCluster x kMaxWarps pairs, used in turn (`turn` flips).
template <int TEAM>
__device__ __forceinline__ float2 team_sum(float2 v, float2 (*red)[kMaxCluster * kMaxWarps], int& turn) {
#pragma unroll
  for (int o = (TEAM > 0 ? TEAM : 32) / 2; o > 0; o >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
  }
  if constexpr (TEAM > 0) return v;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  int count = warps;
  if constexpr (TEAM == 0) {
    if (lane == 0) red[turn][warp] = v;
    __syncthreads();
  } else {
    unsigned rank, n;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
    count = warps * n;
    if (lane < n) {
      unsigned to;
      asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"((unsigned)__cvta_generic_to_shared(&red[turn][rank * warps + warp])), "r"(lane));
      asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(v.x), "f"(v.y) : "memory");
    }
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
  }
  v = make_float2(0.f, 0.f);
  for (int i = 0; i < count; ++i) {
    const float2 u = red[turn][i];
    v.x += u.x; v.y += u.y;
  }
  turn ^= 1;
  return v;
}

template <int TEAM>
__device__ __forceinline__ float team_sum(float v, float2 (*red)[kMaxCluster * kMaxWarps], int& turn) {
  if constexpr (TEAM > 0) {
#pragma unroll
    for (int o = TEAM / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
  }
  return team_sum<TEAM>(make_float2(v, 0.f), red, turn).x;
}

// (A warp's lanes stay together: those of a team without a row left take part in its sums and store nothing.)
template <typename T, int V, int TEAM, int N>
__global__ void __launch_bounds__(Held<T, V, TEAM, N>::kThreads, (TEAM > 0 ? forward_ctas(N, V > 1) : 2)) forward_kernel(const __grid_constant__ Args A) {
  extern __shared__ __align__(16) unsigned char raw[];
  __shared__ float2 red[2][kMaxCluster * kMaxWarps];
  typedef Held<T, V, TEAM, N> H;
  const H held(A.D);
  const int stage = H::stage_bytes(blockDim.x);
  unsigned char* slot = held.slot(raw);
  int turn = 0;
  int64_t row = held.row;
  start_dependents();
  if constexpr (TEAM < 0) asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");   // all of it is there
  wait_for_previous();
  auto send = [&](int s, int64_t r) {
    if (r < A.M) held.send(slot + s * stage, A.x, A.ldx, r);
    copies_sent();
  };
#pragma unroll
  for (int s = 0; s < kForwardStages; ++s) send(s, row + s * held.step);
  float w[N], b[N];
  held.vector(A.weight, A.wvec, 1.f, w);
  held.vector(A.bias, A.wvec, 0.f, b);
  const float per = 1.f / (float)A.D;
  int s = 0;
  for (int64_t base = row - (TEAM > 0 ? threadIdx.x % 32 / (TEAM > 0 ? TEAM : 1) : 0); base < A.M; base += held.step, row += held.step) {
    const bool live = TEAM != 8 || row < A.M;
    float x[N];
    copies_landed<kForwardStages - 1>();
    H::meet();
#pragma unroll
    for (int i = 0; i < H::kAccesses; ++i) held.take(i, slot + s * stage, A.x, A.ldx, row, x + i * V);
    float2 a = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) a = add2(a, pair(x, i));
    const float rough = team_sum<TEAM>(a.x + a.y, red, turn) * per;
    send(s, row + kForwardStages * held.step);             // (its values are in registers by now, the whole team's)
    if (++s == kForwardStages) s = 0;
    float2 q = make_float2(0.f, 0.f);
    a = q;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) set_pair(x, i, add2(pair(x, i), two(-rough)));
    held.cut(x);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) { a = add2(a, pair(x, i)); q = fma2(pair(x, i), pair(x, i), q); }
    const float2 sum = team_sum<TEAM>(make_float2(a.x + a.y, q.x + q.y), red, turn);
    const float off = sum.x * per, var = fmaf(-off, off, sum.y * per), rstd = rsqrtf((var < 0.f ? 0.f : var) + A.eps);   // (a NaN stays)
#pragma unroll
    for (int i = 0; i < N / 2; ++i) set_pair(x, i, fma2(fma2(pair(x, i), two(rstd), two(-off * rstd)), pair(w, i), pair(b, i)));
    if (!live) continue;
    held.store(A.out, A.ldout, row, x);
    if (held.t == 0) { A.mean[row] = rough + off; A.rstd[row] = rstd; }
  }
  copies_landed<0>();
}

template <typename T, int V, int TEAM, int N>
__global__ void __launch_bounds__(Held<T, V, TEAM, N>::kThreads, (TEAM > 0 ? backward_ctas(N) : 1)) backward_kernel(const __grid_constant__ Args A) {
  constexpr int kStages = backward_stages(sizeof(T));
  extern __shared__ __align__(16) unsigned char raw[];     // weights, then the stages
  __shared__ float2 red[2][kMaxCluster * kMaxWarps];
  typedef Held<T, V, TEAM, N> H;
  const H held(A.D);
  const int part = H::stage_bytes(blockDim.x), stage = part * (A.add ? 3 : 2);      // from input to input, from stage to stage
  float* weights = reinterpret_cast<float*>(raw);
  unsigned char* slot = held.slot(raw + held.threads * N * sizeof(float));
  int turn = 0;
  int64_t row = held.row;
  start_dependents();
  if constexpr (TEAM < 0) asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
  wait_for_previous();
  auto send = [&](int s, int64_t r) {
    if (r < A.M) {
      held.send(slot + s * stage, A.x, A.ldx, r);
      held.send(slot + s * stage + part, A.dy, A.lddy, r);
      if (A.add) held.send(slot + s * stage + 2 * part, A.add, A.ldadd, r);
    }
    copies_sent();
  };
#pragma unroll
  for (int s = 0; s < kStages; ++s) send(s, row + s * held.step);
  const float per = 1.f / (float)A.D;
  float dw[N], db[N];
  held.vector(A.weight, A.wvec, 1.f, dw);
  held.keep(weights, dw);
#pragma unroll
  for (int i = 0; i < N; ++i) dw[i] = db[i] = 0.f;
  float next_mean = 0.f, next_rstd = 0.f;
  if (row < A.M) { next_mean = A.mean[row]; next_rstd = A.rstd[row]; }
  int s = 0;
  for (int64_t base = row - (TEAM > 0 ? threadIdx.x % 32 / (TEAM > 0 ? TEAM : 1) : 0); base < A.M; base += held.step, row += held.step) {
    const bool live = TEAM != 8 || row < A.M;
    const float mean = next_mean, rstd = next_rstd;
    if (row + held.step < A.M) { next_mean = A.mean[row + held.step]; next_rstd = A.rstd[row + held.step]; }
    float h[N], g[N];
    const unsigned char* from = slot + s * stage;
    copies_landed<kStages - 1>();
    H::meet();
    float2 a = make_float2(0.f, 0.f), q = a;
#pragma unroll
    for (int i = 0; i < H::kAccesses; ++i) {               // (behind the row's end dy is 0)
      float w[V];
      held.kept(weights, i, w);
      held.take(i, from, A.x, A.ldx, row, h + i * V);
      held.take(i, from + part, A.dy, A.lddy, row, g + i * V);
      if constexpr (V > 1) {
#pragma unroll
        for (int j = 0; j < V / 2; ++j) {
          const int k = i * V / 2 + j;
          const float2 u = mul2(add2(pair(h, k), two(-mean)), two(rstd)), v = pair(g, k), x = mul2(v, pair(w, j));
          if (live) {
            set_pair(dw, k, fma2(v, u, pair(dw, k)));
            set_pair(db, k, add2(pair(db, k), v));
          }
          a = add2(a, x);
          q = fma2(x, u, q);
          set_pair(h, k, u);
          set_pair(g, k, x);
        }
      } else {
        const float u = (h[i] - mean) * rstd, v = g[i], x = v * w[0];
        if (live) { dw[i] = fmaf(v, u, dw[i]); db[i] += v; }
        a.x += x;
        q.x = fmaf(x, u, q.x);
        h[i] = u;
        g[i] = x;
      }
    }
    const float2 sum = team_sum<TEAM>(make_float2(a.x + a.y, q.x + q.y), red, turn);
    const float c1 = -sum.x * per * rstd, c2 = -sum.y * per * rstd;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) set_pair(g, i, fma2(pair(g, i), two(rstd), fma2(pair(h, i), two(c2), two(c1))));
    if (A.add) {
#pragma unroll
      for (int i = 0; i < H::kAccesses; ++i) held.take(i, from + 2 * part, A.add, A.ldadd, row, h + i * V);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) set_pair(g, i, add2(pair(g, i), pair(h, i)));
      if constexpr (V == 1) H::meet();                     // the whole team has its values
    }
    if (live) held.store(A.out, A.ldout, row, g);
    send(s, row + kStages * held.step);
    if (++s == kStages) s = 0;
  }
  copies_landed<0>();
  if (!A.part) return;
  float* part_of = A.part + held.group * 2 * A.D;
  if constexpr (TEAM > 0) {
    // the lanes of a warp that hold the same columns, then the warps
    __syncthreads();                                       // the stages are free
    float* joined = reinterpret_cast<float*>(raw);         // [warps][2][N][32]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 16; o >= TEAM; o >>= 1) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        dw[i] += __shfl_xor_sync(0xffffffffu, dw[i], o);
        db[i] += __shfl_xor_sync(0xffffffffu, db[i], o);
      }
    }
    if (lane < TEAM) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        joined[(warp * 2 * N + i) * 32 + lane] = dw[i];
        joined[((warp * 2 + 1) * N + i) * 32 + lane] = db[i];
      }
    }
    __syncthreads();
    const int warps = blockDim.x >> 5;
    for (int j = threadIdx.x; j < 2 * N * 32; j += blockDim.x) {
      const int l = j & 31, i = (j >> 5) % N, which = (j >> 5) / N;
      const int c = (i / V * TEAM + l) * V + i % V;
      if (l >= TEAM || c >= A.D) continue;
      float v = 0.f;
      for (int k = 0; k < warps; ++k) v += joined[((k * 2 + which) * N + i) * 32 + l];
      part_of[which * (int64_t)A.D + c] = v;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = held.column(i / V) + i % V;
      if (c < A.D) { part_of[c] = dw[i]; part_of[(int64_t)A.D + c] = db[i]; }
    }
  }
}

// dweight and dbias from the CTAs' sums: 32 columns a CTA, its warps take every 32nd row of sums
__global__ void __launch_bounds__(1024) columns_kernel(const float* part, int64_t rows, int D, float* dweight, float* dbias) {
  __shared__ float sh[32][33];
  start_dependents();
  wait_for_previous();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, which = blockIdx.y;
  float* out = which ? dbias : dweight;
  if (!out) return;
  float s = 0.f;
  if (c < D) {
#pragma unroll 8
    for (int64_t r = warp; r < rows; r += 32) s += part[(r * 2 + which) * D + c];
  }
  sh[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < D) {
    s = 0.f;
    for (int k = 0; k < 32; ++k) s += sh[k][lane];
    out[c] = s;
  }
}

// ---------------------------------------------------------------------------------------------- host

constexpr int kMostShared = 225 * 1024;

// A row's team by its width: 8 lanes to 64 values, a warp to 1024, a CTA to 8192, a cluster above. (Wider teams leave fewer
// values to a thread and add a barrier to every sum.)
struct Plan {
  int team, values, threads, cluster;
  int64_t groups;            // CTAs, or clusters of them
};
Plan plan_of(int64_t M, int D, int dtype, int backward, bool wide) {      // (backward's does not go by `wide`: its workspace is asked for without)
  Plan p = {};
  p.cluster = 1;
  p.threads = 128;
  p.team = D <= 64 ? 8 : D <= 1024 ? 32 : D <= 8192 ? 0 : -1;
  // (backward's teams of several warps hold 16 values a thread: with 32 the two CTAs on an SM, a barrier a row, were too few warps: 4000 x 4096 bf16
  // 44 us, with 16 33 us)
  p.values = D <= 256 ? 8 : D <= 512 || (backward && D > 1024) ? 16 : 32;
  if (D > 1024) {
    while (p.cluster * 8192 < D) p.cluster *= 2;
    const int share = (D + p.cluster - 1) / p.cluster;
    p.threads = ((share + p.values - 1) / p.values + 31) / 32 * 32;
  }
  const int bytes = element_size(dtype), values = p.threads * p.values;              // a CTA's of one input
  const int slots = backward ? backward_stages(bytes) * 3 * values * bytes + 4 * (p.team > 0 ? p.team * p.values : values) : kForwardStages * values * bytes;
  int at_once = p.team > 0 ? (backward ? backward_ctas(p.values) : forward_ctas(p.values, wide)) : 512 / p.threads;
  const int fit = 224 * 1024 / (slots + 2048);
  at_once = fit < 1 ? 1 : at_once > fit ? fit : at_once;
  const int rows = p.team > 0 ? 128 / p.team : 1;
  const int64_t want = (M + rows - 1) / rows, most = 148 * at_once / p.cluster;
  p.groups = want < most ? want : most;
  return p;
}

template <typename T, int V, int TEAM, int N, bool BACK>
int launch(const Args& A, const Plan& p, cudaStream_t st) {
  typedef Held<T, V, TEAM, N> H;
  const dim3 grid((unsigned)(p.groups * p.cluster));
  int shared = kForwardStages * H::stage_bytes(p.threads);
  void (*kernel)(const Args);
  if constexpr (BACK) {
    kernel = backward_kernel<T, V, TEAM, N>;
    shared = backward_stages(sizeof(T)) * (A.add ? 3 : 2) * H::stage_bytes(p.threads) + 4 * N * (TEAM > 0 ? TEAM : p.threads);
    if (TEAM > 0 && shared < 4 * 2 * N * 32 * 4) shared = 4 * 2 * N * 32 * 4;        // the warps' sums
  } else {
    kernel = forward_kernel<T, V, TEAM, N>;
  }
  static std::atomic<uint64_t> set{0};                    // devices on which the kernel may use that much
  int device = 0;
  if (!dmxh::cuda_ok(cudaGetDevice(&device))) return DMX_ERR_CUDA;
  const uint64_t bit = (uint64_t)1 << (device & 63);
  if (!(set.load(std::memory_order_relaxed) & bit) || device > 63) {
    if (!dmxh::cuda_ok(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared))) return DMX_ERR_CUDA;
    set.fetch_or(bit, std::memory_order_relaxed);
  }
  return start(grid, p.threads, p.cluster, shared, st, kernel, A);
}
template <typename T, int V, bool BACK>
int launch(const Args& A, const Plan& p, cudaStream_t st) {
  constexpr int kTeamValues = BACK ? 16 : 32;
  if (p.team == 8) return launch<T, V, 8, 8, BACK>(A, p, st);
  if (p.team < 0) return launch<T, V, -1, kTeamValues, BACK>(A, p, st);
  if (p.team == 0) return launch<T, V, 0, kTeamValues, BACK>(A, p, st);
  if (p.values == 8) return launch<T, V, 32, 8, BACK>(A, p, st);
  return p.values == 16 ? launch<T, V, 32, 16, BACK>(A, p, st) : launch<T, V, 32, 32, BACK>(A, p, st);
}
template <typename T, int V>
int launch(const Args& A, const Plan& p, int backward, cudaStream_t st) { return backward ? launch<T, V, true>(A, p, st) : launch<T, V, false>(A, p, st); }
int launch(const Args& A, const Plan& p, int dtype, bool wide, int backward, cudaStream_t st) {
  if (dtype == DMX_F32) return wide ? launch<float, 4>(A, p, backward, st) : launch<float, 1>(A, p, backward, st);
  return wide ? launch<bf16, 8>(A, p, backward, st) : launch<bf16, 1>(A, p, backward, st);
}

bool shape_ok(int64_t M, int D, int dtype) { return M >= 0 && M < ((int64_t)1 << 40) && D >= 1 && D <= DMX_LN_MAX_WIDTH && (dtype == DMX_F32 || dtype == DMX_BF16); }

}  // namespace

extern "C" {

int64_t dmx_layer_norm_workspace(int64_t M, int D, int dtype) {
  if (!shape_ok(M, D, dtype)) return DMX_ERR_ARG;
  return M == 0 ? 0 : pad256(plan_of(M, D, dtype, 1, true).groups * 2 * D * (int64_t)sizeof(float));
}

int dmx_layer_norm_forward(int64_t M, int D, int dtype, const void* x, int64_t ldx, const float* weight, const float* bias, float eps, void* y,
                           int64_t ldy, float* mean, float* rstd, void* cuda_stream) {
  if (!shape_ok(M, D, dtype) || !(eps >= 0.f) || (M > 1 && (ldx < 0 || ldy < D))) return DMX_ERR_ARG;
  if (M == 0) return DMX_OK;
  if (!x || !y || !mean || !rstd) return DMX_ERR_ARG;
  const unsigned e = element_size(dtype);
  if (!aligned(x, e) || !aligned(y, e) || !aligned(weight, 4) || !aligned(bias, 4) || !aligned(mean, 4) || !aligned(rstd, 4)) return DMX_ERR_ALIGN;
  Args A = {};
  A.x = x; A.out = y; A.ldx = M > 1 ? ldx : D; A.ldout = M > 1 ? ldy : D; A.M = M; A.D = D;
  A.weight = weight; A.bias = bias; A.mean = mean; A.rstd = rstd; A.eps = eps;
  A.wvec = aligned(weight, 16) && aligned(bias, 16);
  const bool wide = wide_rows(x, M, ldx, D, dtype) && wide_rows(y, M, ldy, D, dtype);
  return launch(A, plan_of(M, D, dtype, 0, wide), dtype, wide, 0, static_cast<cudaStream_t>(cuda_stream));
}

int dmx_layer_norm_backward(int64_t M, int D, int dtype, const void* dy, int64_t lddy, const void* x, int64_t ldx, const float* mean, const float* rstd,
                            const float* weight, const void* add, int64_t ldadd, void* dx, int64_t lddx, float* dweight, float* dbias,
                            void* workspace, int64_t workspace_bytes, void* cuda_stream) {
  if (!shape_ok(M, D, dtype) || (M > 1 && (lddy < 0 || ldx < 0 || (add && ldadd < 0) || lddx < D))) return DMX_ERR_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (!aligned(dweight, 4) || !aligned(dbias, 4)) return DMX_ERR_ALIGN;
  if (M == 0) {              // empty sums
    if (dweight && !dmxh::cuda_ok(cudaMemsetAsync(dweight, 0, sizeof(float) * D, st))) return DMX_ERR_CUDA;
    if (dbias && !dmxh::cuda_ok(cudaMemsetAsync(dbias, 0, sizeof(float) * D, st))) return DMX_ERR_CUDA;
    return DMX_OK;
  }
  if (!dy || !x || !mean || !rstd || !dx) return DMX_ERR_ARG;
  const bool sums = dweight || dbias;
  if (sums && (workspace_bytes < dmx_layer_norm_workspace(M, D, dtype) || !workspace)) return DMX_ERR_ARG;
  const unsigned e = element_size(dtype);
  if (!aligned(dy, e) || !aligned(x, e) || !aligned(add, e) || !aligned(dx, e) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(weight, 4) ||
      !aligned(workspace, 16)) return DMX_ERR_ALIGN;
  Args A = {};
  A.x = x; A.dy = dy; A.add = add; A.out = dx; A.M = M; A.D = D;
  A.ldx = M > 1 ? ldx : D; A.lddy = M > 1 ? lddy : D; A.ldadd = M > 1 ? ldadd : D; A.ldout = M > 1 ? lddx : D;
  A.weight = weight; A.mean = const_cast<float*>(mean); A.rstd = const_cast<float*>(rstd);
  A.part = sums ? static_cast<float*>(workspace) : nullptr;
  A.wvec = aligned(weight, 16);
  const Plan p = plan_of(M, D, dtype, 1, true);
  const bool wide = wide_rows(x, M, ldx, D, dtype) && wide_rows(dy, M, lddy, D, dtype) && wide_rows(dx, M, lddx, D, dtype) && (!add || wide_rows(add, M, ldadd, D, dtype));
  const int rc = launch(A, p, dtype, wide, 1, st);
  if (rc != DMX_OK || !sums) return rc;
  return start(dim3((D + 31) / 32, 2), 1024, 1, 0, st, columns_kernel, (const float*)A.part, p.groups, D, dweight, dbias);
}

}  // extern "C"
