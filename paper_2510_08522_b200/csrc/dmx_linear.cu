// dmx_linear.cu — matrix product with bias, activation and residual in its epilogue, and its gradient (bf16
// operands, fp32 accumulation).
//
//   forward    z = x W^T + b, y = act(z) + r
//   backward   dz = dy act'(z) (one elementwise pass, which also sums its columns for db), dx = dz W, dW = dz^T x
//
// All three products are D[i, j] = sum_k A[i, k] B[j, k], by the kernel of dmx_gemm.cuh. W in dx, and both operands of dW, run across k (MN-major).
// Few rows (M <= 64): the operands change places, so that W's rows fill the 128 lanes and the few rows of x are the narrow
// side. Few tiles: k is split over the CTAs of a cluster.
// Bound: the tensor cores for large products, what an SM fetches from L2 (64 bytes a cycle) for narrow tiles, HBM for few rows.
// Measured on B200 in bursts at full clock / back to back for seconds under the power limit: 8192^3 714 / 833 us = 1.54 / 1.32 PFLOP/s
// (the library's 669 / 774 us); 8192 x 4096 x 1024 with GELU, y and z written, 65 / 77 us = 1.06 / 0.89 PFLOP/s (the library's bare product
// 56 / 60 us); its gradient 132 / 151 us; one row x 4096 x 4096 7.9 / 7.6 us = 4.3 TB/s.
#include "dmx.h"

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <mutex>

#include "dmx_act.cuh"
#include "dmx_gemm.cuh"

namespace {

using namespace dmx_gemm;

struct GemmArgs : GemmShape {
  const bf16 *bias, *residual;
  bf16 *y, *z;
  int64_t ldr, ldy, ldz;
  int act;
  int vecy, vecz, vecr;                       // 16-byte rows
  const float* unit;                          // of one operand, if it is held in units of something
};

// ---------------------------------------------------------------------------------------------- epilogue

template <int NC>
__device__ __forceinline__ void activate(float (&v)[NC], int act) {
  auto all = [&](auto f) {
#pragma unroll
    for (int i = 0; i < NC / 2; ++i) {
      const float2 t = f(make_float2(v[2 * i], v[2 * i + 1]));
      v[2 * i] = t.x; v[2 * i + 1] = t.y;
    }
  };
  if (act == DMX_ACT_RELU) all([](float2 u) { return dmx_act::apply<DMX_ACT_RELU>(u); });
  else if (act == DMX_ACT_SILU) all([](float2 u) { return dmx_act::apply<DMX_ACT_SILU>(u); });
  else if (act == DMX_ACT_GELU) all([](float2 u) { return dmx_act::apply<DMX_ACT_GELU>(u); });
}

// One warp's 32 rows x NC columns of D, a row per lane.
template <int NC>
__device__ __forceinline__ void finish(const GemmArgs& A, float (&v)[NC], uint4* stage, int r0, int c0, int lane) {
  auto to_stage = [&] {
#pragma unroll
    for (int u = 0; u < NC / 8; ++u)
      *unit(stage, lane, u) = make_uint4(pack2(v[8 * u], v[8 * u + 1]), pack2(v[8 * u + 2], v[8 * u + 3]), pack2(v[8 * u + 4], v[8 * u + 5]),
                                         pack2(v[8 * u + 6], v[8 * u + 7]));
  };
  auto add8 = [&](int u, uint4 b) {
    const unsigned w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 t = widen2(w[k]);
      v[8 * u + 2 * k] += t.x; v[8 * u + 2 * k + 1] += t.y;
    }
  };
  if (A.bias) {
    if (c0 + NC <= A.rowsB && (reinterpret_cast<uintptr_t>(A.bias) & 15) == 0) {
#pragma unroll
      for (int u = 0; u < NC / 8; ++u) add8(u, reinterpret_cast<const uint4*>(A.bias + c0)[u]);
    } else {
#pragma unroll
      for (int i = 0; i < NC; ++i)
        if (c0 + i < A.rowsB) v[i] += bf_value(reinterpret_cast<const unsigned short*>(A.bias)[c0 + i]);
    }
  }
  if (A.z) {
    to_stage();
    store_tile<32, NC>(A.z, A.ldz, A.vecz, stage, r0, A.rowsA, c0, A.rowsB, lane);
  }
  activate(v, A.act);
  if (A.residual) {
    load_tile<32, NC>(A.residual, A.ldr, A.vecr, stage, r0, A.rowsA, c0, A.rowsB, lane);
#pragma unroll
    for (int u = 0; u < NC / 8; ++u) add8(u, *unit(stage, lane, u));
    __syncwarp();
  }
  to_stage();
  store_tile<32, NC>(A.y, A.ldy, A.vecy, stage, r0, A.rowsA, c0, A.rowsB, lane);
}

// The same with the operands exchanged: a lane holds one column of y (a row of W) for NC rows of x from t0; the
// staging buffer turns them.
template <int NC>
__device__ __forceinline__ void finish_swapped(const GemmArgs& A, float (&v)[NC], uint4* stage, int f0, int t0, float bias, int lane) {
  unsigned short* at[4];         // this lane's column in rows of each exchange pattern
#pragma unroll
  for (int k = 0; k < 4; ++k) at[k] = reinterpret_cast<unsigned short*>(stage + ((lane >> 3) ^ k)) + (lane & 7);
  auto to_stage = [&] {
#pragma unroll
    for (int i = 0; i < NC; ++i) at[(i >> 1) & 3][i * 32] = __bfloat16_as_ushort(__float2bfloat16_rn(v[i]));
  };
#pragma unroll
  for (int i = 0; i < NC; ++i) v[i] += bias;
  if (A.z) {
    to_stage();
    store_tile<NC, 32>(A.z, A.ldz, A.vecz, stage, t0, A.rowsB, f0, A.rowsA, lane);
  }
  activate(v, A.act);
  if (A.residual) {
    load_tile<NC, 32>(A.residual, A.ldr, A.vecr, stage, t0, A.rowsB, f0, A.rowsA, lane);
#pragma unroll
    for (int i = 0; i < NC; ++i) v[i] += bf_value(at[(i >> 1) & 3][i * 32]);
    __syncwarp();
  }
  to_stage();
  store_tile<NC, 32>(A.y, A.ldy, A.vecy, stage, t0, A.rowsB, f0, A.rowsA, lane);
}
// D, or with the operands exchanged its transpose. UNIT: times *A.unit.
template <bool SWAP, bool UNIT>
struct LinearEpilogue {
  typedef GemmArgs Args;
  static constexpr int kStaging = 2048, kOwnShared = 0;
  static constexpr bool kRanged = false;
  float bias, unit;
  __device__ __forceinline__ void fetch(const Args&, int, int) {}
  __device__ __forceinline__ void begin(const Args& A, int r0, int c0, int lane) {
    bias = 0.f;
    if (UNIT) unit = *A.unit;                  // (here: read for each chunk it would be waited for, 64 x 30522 x 1024's dW 8 us)
    if (SWAP && A.bias && r0 + lane < A.rowsA) bias = bf_value(reinterpret_cast<const unsigned short*>(A.bias)[r0 + lane]);
    if (!SWAP && A.bias && c0 < A.rowsB) asm volatile("prefetch.global.L1 [%0];" ::"l"(A.bias + c0));
  }
  template <int NC>
  __device__ __forceinline__ void chunk(const Args& A, float (&v)[NC], uint4* stage, int r0, int c0, int lane) {
    if constexpr (UNIT) {
#pragma unroll
      for (int i = 0; i < NC; ++i) v[i] *= unit;
    }
    if constexpr (SWAP) finish_swapped<NC>(A, v, stage, r0, c0, bias, lane);
    else finish<NC>(A, v, stage, r0, c0, lane);
  }
  static __device__ __forceinline__ void setup() {}
  __device__ __forceinline__ bool end(const Args&, int, int, int, int, int, unsigned) { return true; }
};

// ---------------------------------------------------------------------------------------------- elementwise parts

// Row-wise jobs, up to three to a launch (blockIdx.z): dz = dy act'(z) as bf16 rows of `ldo` elements with, per chunk of
// rows, the column sums of the unrounded dz; and the laying out of an operand whose rows TMA cannot take. Bound: HBM (dz
// reads two matrices and writes one: 8192 x 4096, 201 MB).
template <int V, int ACT>
__device__ __forceinline__ void row_job(const Job& J, float* sh) {
  constexpr int NP = (V + 1) / 2;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = (blockIdx.x * 32 + lane) * V;
  if (blockIdx.x * 32 * V >= J.cols) return;
  const int64_t r0 = (int64_t)blockIdx.y * kChunkRows + warp, r1 = min((int64_t)(blockIdx.y + 1) * kChunkRows, J.rows);
  float2 acc[NP];
#pragma unroll
  for (int j = 0; j < NP; ++j) acc[j] = two(0.f);
  if (c < J.cols) {
#pragma unroll
    for (int i = 0; i < kChunkRows / 8; ++i) {
      const int64_t r = r0 + 8 * i;
      if (r >= r1) continue;
      float2 g[NP], u[NP];
      if constexpr (V == 8) {
        const uint4 a = __ldcs(reinterpret_cast<const uint4*>(J.in + r * J.ldi + c));
        g[0] = widen2(a.x); g[1] = widen2(a.y); g[2] = widen2(a.z); g[3] = widen2(a.w);
        if constexpr (ACT != DMX_ACT_NONE) {
          const uint4 b = __ldcs(reinterpret_cast<const uint4*>(J.z + r * J.ldz + c));
          u[0] = widen2(b.x); u[1] = widen2(b.y); u[2] = widen2(b.z); u[3] = widen2(b.w);
        }
      } else {
        g[0] = make_float2(__bfloat162float(J.in[r * J.ldi + c]), 0.f);
        if constexpr (ACT != DMX_ACT_NONE) u[0] = make_float2(__bfloat162float(J.z[r * J.ldz + c]), 0.f);
      }
#pragma unroll
      for (int j = 0; j < NP; ++j) {
        if constexpr (ACT != DMX_ACT_NONE) g[j] = dmx_act::times_slope<ACT>(g[j], u[j]);
        acc[j] = add2(acc[j], g[j]);
      }
      if (J.out) {
        if constexpr (V == 8) *reinterpret_cast<uint4*>(J.out + r * J.ldo + c) = make_uint4(pack2(g[0].x, g[0].y), pack2(g[1].x, g[1].y), pack2(g[2].x, g[2].y), pack2(g[3].x, g[3].y));
        else J.out[r * J.ldo + c] = __float2bfloat16_rn(g[0].x);
      }
    }
  }
  if (!J.sums) return;
  float* mine = sh + (warp * 32 + lane) * V;
#pragma unroll
  for (int j = 0; j < NP; ++j) {
    mine[2 * j] = acc[j].x;
    if (V > 1) mine[(2 * j + 1) % V] = acc[j].y;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 32 * V; i += 256) {
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) t += sh[w * 32 * V + i];
    if (blockIdx.x * 32 * V + i < J.cols) J.sums[(int64_t)blockIdx.y * J.cols + blockIdx.x * 32 * V + i] = t;
  }
}

// ACT: of the first job; the others are copies. Six CTAs per SM hide the loads better than more rows in flight per thread:
// dz of 8192 x 4096 with GELU takes 33 us (6.1 TB/s), with two rows ahead and four CTAs 40 us, four rows and three 49 us.
template <int ACT>
__global__ void __launch_bounds__(256, 6) rows_kernel(const __grid_constant__ Jobs all) {
  __shared__ __align__(16) float sh[8 * 32 * 8];
  start_dependents();
  wait_for_previous();
  const Job& J = all.job[blockIdx.z];
  if ((int64_t)blockIdx.y * kChunkRows >= J.rows) return;
  if (blockIdx.z == 0) {
    if (J.vec) row_job<8, ACT>(J, sh);
    else row_job<1, ACT>(J, sh);
  } else {
    row_job<1, DMX_ACT_NONE>(J, sh);
  }
}

// dbias from the chunks' sums: 32 columns and eight lanes of chunks per CTA
__global__ void __launch_bounds__(256) columns_kernel(const float* sums, int64_t chunks, int cols, bf16* out) {
  __shared__ float sh[8][33];
  start_dependents();
  wait_for_previous();
  const int lane = threadIdx.x & 31, r = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  float s = 0.f;
  if (c < cols) {
#pragma unroll 8
    for (int64_t i = r; i < chunks; i += 8) s += sums[i * cols + c];
  }
  sh[r][lane] = s;
  __syncthreads();
  if (r == 0 && c < cols) {
    for (int k = 1; k < 8; ++k) s += sh[k][lane];
    out[c] = __float2bfloat16_rn(s);
  }
}

// K = 0: y = act(bias) + residual
__global__ void __launch_bounds__(256) bias_kernel(const __grid_constant__ GemmArgs A) {
  start_dependents();
  wait_for_previous();
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)A.rowsA * A.rowsB; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / A.rowsB;
    const int c = (int)(i - r * A.rowsB);
    float v[2] = {};
    v[0] = A.bias ? __bfloat162float(A.bias[c]) : 0.f;
    if (A.z) A.z[r * A.ldz + c] = __float2bfloat16_rn(v[0]);
    activate(v, A.act);
    if (A.residual) v[0] += __bfloat162float(A.residual[r * A.ldr + c]);
    A.y[r * A.ldy + c] = __float2bfloat16_rn(v[0]);
  }
}
// ---------------------------------------------------------------------------------------------- host

// 64 rows or fewer: b's rows take the 128 lanes (b keeps whichever way it lies; a, the narrow side, has to be K-major)
struct Form {
  bool exchanged;
  Choice choice;
};
Form form_of(int64_t rowsA, int64_t rowsB, int kblocks, int mnA, bool unit = false) {
  const bool exchanged = rowsA <= 64 && !mnA;
  if (unit) return {exchanged, exchanged ? choose_by_tiles(rowsB, rowsA, kblocks, true, true, 1.2f) : choose_by_tiles(rowsA, rowsB, kblocks, false, true, 1.2f)};
  return {exchanged, exchanged ? choose(rowsB, rowsA, kblocks, true) : choose(rowsA, rowsB, kblocks, false)};
}

// D = A B^T with the epilogue in E (bias, residual, outputs, act). mn: the operand's rows run along D's extent.
template <bool UNIT>
int product(const Matrix& a, int mnA, const Matrix& b, int mnB, int64_t k, const GemmArgs& E, cudaStream_t st) {
  GemmArgs A = E;
  const int64_t rowsA = mnA ? a.cols : a.rows, rowsB = mnB ? b.cols : b.rows;
  A.kblocks = (int)((k + kBK - 1) / kBK);
  A.vecy = aligned(A.y, 16) && (rowsA <= 1 || A.ldy % 8 == 0);
  A.vecz = A.z && aligned(A.z, 16) && (rowsA <= 1 || A.ldz % 8 == 0);
  A.vecr = A.residual && aligned(A.residual, 16) && (rowsA <= 1 || A.ldr % 8 == 0);
  const Form f = form_of(rowsA, rowsB, A.kblocks, mnA, UNIT);
  const Choice& c = f.choice;
  if (f.exchanged) {
    A.rowsA = (int)rowsB; A.rowsB = (int)rowsA;
    A.mnA = mnB; A.mnB = mnA;
    if (c.bn == 32) {
      if (c.split == 4) return launch_gemm<32, false, 4, LinearEpilogue<true, UNIT>>(b, a, A, st);
      return c.split == 2 ? launch_gemm<32, false, 2, LinearEpilogue<true, UNIT>>(b, a, A, st) : launch_gemm<32, false, 1, LinearEpilogue<true, UNIT>>(b, a, A, st);
    }
    if (c.split == 4) return launch_gemm<64, false, 4, LinearEpilogue<true, UNIT>>(b, a, A, st);
    return c.split == 2 ? launch_gemm<64, false, 2, LinearEpilogue<true, UNIT>>(b, a, A, st) : launch_gemm<64, false, 1, LinearEpilogue<true, UNIT>>(b, a, A, st);
  }
  A.rowsA = (int)rowsA; A.rowsB = (int)rowsB;
  A.mnA = mnA; A.mnB = mnB;
  if (c.pair) return c.bn == 256 ? launch_gemm<256, true, 1, LinearEpilogue<false, UNIT>>(a, b, A, st) : launch_gemm<128, true, 1, LinearEpilogue<false, UNIT>>(a, b, A, st);
  if (c.bn == 256) return launch_gemm<256, false, 1, LinearEpilogue<false, UNIT>>(a, b, A, st);
  if (c.bn == 128) return c.split == 2 ? launch_gemm<128, false, 2, LinearEpilogue<false, UNIT>>(a, b, A, st) : launch_gemm<128, false, 1, LinearEpilogue<false, UNIT>>(a, b, A, st);
  return c.split == 2 ? launch_gemm<64, false, 2, LinearEpilogue<false, UNIT>>(a, b, A, st) : launch_gemm<64, false, 1, LinearEpilogue<false, UNIT>>(a, b, A, st);
}

}  // namespace

namespace dmx_gemm {

int run_jobs(const Jobs& jobs, int n, int act, cudaStream_t st) {
  int64_t columns = 0, chunks = 0;
  for (int i = 0; i < n; ++i) {
    const Job& j = jobs.job[i];
    const int64_t c = (j.cols + (j.vec ? 255 : 31)) / (j.vec ? 256 : 32), r = (j.rows + kChunkRows - 1) / kChunkRows;
    columns = c > columns ? c : columns;
    chunks = r > chunks ? r : chunks;
  }
  const dim3 grid((unsigned)columns, (unsigned)chunks, (unsigned)n);
  switch (act) {
    case DMX_ACT_RELU: return start(grid, st, rows_kernel<DMX_ACT_RELU>, jobs);
    case DMX_ACT_SILU: return start(grid, st, rows_kernel<DMX_ACT_SILU>, jobs);
    case DMX_ACT_GELU: return start(grid, st, rows_kernel<DMX_ACT_GELU>, jobs);
    default: return start(grid, st, rows_kernel<DMX_ACT_NONE>, jobs);
  }
}

// m's copy at *ws (which moves on), if it needs one
void lay_out(Matrix& m, unsigned char*& ws, Jobs& jobs, int& n) {
  const int64_t bytes = laid_out_bytes(m);
  if (bytes == 0) return;
  Job& j = jobs.job[n++];
  j = Job();
  j.in = m.p; j.ldi = m.ld; j.rows = m.rows; j.cols = (int)m.cols;
  j.out = reinterpret_cast<bf16*>(ws);
  j.ldo = pad8(m.cols);
  ws += bytes;
  m.p = j.out;
  m.ld = j.ldo;
}

int plain_product(const Matrix& a, int mnA, const Matrix& b, int mnB, int64_t k, const float* unit, bf16* y, int64_t ldy, cudaStream_t st) {
  GemmArgs E = {};
  E.act = DMX_ACT_NONE;
  E.y = y; E.ldy = ldy; E.unit = unit;
  return unit ? product<true>(a, mnA, b, mnB, k, E, st) : product<false>(a, mnA, b, mnB, k, E, st);
}

float plain_product_ns(int64_t rowsA, int64_t rowsB, int64_t k, int mnA) { return form_of(rowsA, rowsB, (int)((k + kBK - 1) / kBK), mnA, true).choice.ns; }

}  // namespace dmx_gemm

namespace {

bool extents_ok(int64_t M, int64_t N, int64_t K) {
  const int64_t most = DMX_LINEAR_MAX_EXTENT;
  return M >= 0 && N >= 0 && K >= 0 && M <= most && N <= most && K <= most;
}
// what is only read may repeat rows (0) or overlap them; what is written may not
bool in_ok(int64_t rows, int64_t ld) { return rows <= 1 || ld >= 0; }
bool out_ok(int64_t rows, int64_t cols, int64_t ld) { return rows <= 1 || ld >= cols; }

struct BackPlan {
  bool needs_dz;            // dz is written to the workspace
  int64_t dz, sums, x, w, total;
};
BackPlan back_plan(const Matrix& dy, const Matrix& x, const Matrix& w, int act) {
  BackPlan p;
  p.needs_dz = act != DMX_ACT_NONE || !tma_ready(dy);
  p.dz = p.needs_dz ? pad256(dy.rows * pad8(dy.cols) * 2) : 0;
  p.sums = pad256((dy.rows + kChunkRows - 1) / kChunkRows * dy.cols * 4);
  p.x = laid_out_bytes(x);
  p.w = laid_out_bytes(w);
  p.total = p.dz + p.sums + p.x + p.w;
  return p;
}

}  // namespace

extern "C" {

int64_t dmx_linear_workspace(int64_t M, int64_t N, int64_t K, const void* x, int64_t ldx, const void* w, int64_t ldw) {
  if (!extents_ok(M, N, K)) return DMX_ERR_ARG;
  if (M == 0 || N == 0 || K == 0) return 0;
  return laid_out_bytes({static_cast<const bf16*>(x), M, K, ldx}) + laid_out_bytes({static_cast<const bf16*>(w), N, K, ldw});
}

int dmx_linear_forward(int64_t M, int64_t N, int64_t K, const void* x, int64_t ldx, const void* w, int64_t ldw, const void* bias,
                       int act, const void* residual, int64_t ldr, void* y, int64_t ldy, void* z, int64_t ldz, void* workspace,
                       int64_t workspace_bytes, void* cuda_stream) {
  if (!extents_ok(M, N, K) || act < DMX_ACT_NONE || act > DMX_ACT_GELU) return DMX_ERR_ARG;
  if (!in_ok(M, ldx) || !in_ok(N, ldw) || !out_ok(M, N, ldy) || (residual && !in_ok(M, ldr)) || (z && !out_ok(M, N, ldz))) return DMX_ERR_ARG;
  if (M == 0 || N == 0) return DMX_OK;
  if (!y || (K > 0 && (!x || !w))) return DMX_ERR_ARG;
  if (!aligned(x, 2) || !aligned(w, 2) || !aligned(bias, 2) || !aligned(residual, 2) || !aligned(y, 2) || !aligned(z, 2) || !aligned(workspace, 256)) return DMX_ERR_ALIGN;
  const int64_t need = dmx_linear_workspace(M, N, K, x, ldx, w, ldw);
  if (need > workspace_bytes || (need > 0 && !workspace)) return DMX_ERR_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  GemmArgs E = {};
  E.bias = static_cast<const bf16*>(bias); E.residual = static_cast<const bf16*>(residual);
  E.y = static_cast<bf16*>(y); E.z = static_cast<bf16*>(z);
  E.ldr = M > 1 ? ldr : N; E.ldy = M > 1 ? ldy : N; E.ldz = M > 1 ? ldz : N; E.act = act;
  if (K == 0) {
    E.rowsA = (int)M; E.rowsB = (int)N;
    const int64_t want = (M * N + 255) / 256;
    return start(dim3((unsigned)(want < 148 * 8 ? want : 148 * 8)), st, bias_kernel, E);
  }
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  Matrix a = {static_cast<const bf16*>(x), M, K, M > 1 ? ldx : K}, b = {static_cast<const bf16*>(w), N, K, N > 1 ? ldw : K};
  Jobs jobs;
  int n = 0;
  lay_out(a, ws, jobs, n);
  lay_out(b, ws, jobs, n);
  const int rc = n > 0 ? run_jobs(jobs, n, DMX_ACT_NONE, st) : DMX_OK;
  return rc != DMX_OK ? rc : product<false>(a, 0, b, 0, K, E, st);
}

int64_t dmx_linear_backward_workspace(int64_t M, int64_t N, int64_t K, const void* dy, int64_t lddy, const void* x, int64_t ldx,
                                      const void* w, int64_t ldw, int act) {
  if (!extents_ok(M, N, K) || act < DMX_ACT_NONE || act > DMX_ACT_GELU) return DMX_ERR_ARG;
  if (M == 0 || N == 0) return 0;
  return back_plan({static_cast<const bf16*>(dy), M, N, lddy}, {static_cast<const bf16*>(x), M, K, ldx}, {static_cast<const bf16*>(w), N, K, ldw}, act).total;
}

int dmx_linear_backward(int64_t M, int64_t N, int64_t K, const void* dy, int64_t lddy, const void* x, int64_t ldx, const void* w, int64_t ldw,
                        const void* z, int64_t ldz, int act, void* dx, int64_t lddx, void* dw, int64_t lddw, void* dbias, void* workspace,
                        int64_t workspace_bytes, void* cuda_stream) {
  if (!extents_ok(M, N, K) || act < DMX_ACT_NONE || act > DMX_ACT_GELU) return DMX_ERR_ARG;
  if (!in_ok(M, lddy) || !in_ok(M, ldx) || !in_ok(N, ldw) || (z && !in_ok(M, ldz)) || (dx && !out_ok(M, K, lddx)) || (dw && !out_ok(N, K, lddw))) return DMX_ERR_ARG;
  if (!aligned(dy, 2) || !aligned(x, 2) || !aligned(w, 2) || !aligned(z, 2) || !aligned(dx, 2) || !aligned(dw, 2) || !aligned(dbias, 2) || !aligned(workspace, 256)) return DMX_ERR_ALIGN;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (M == 0 || N == 0) {          // empty sums
    if (dw && N > 0 && K > 0 && !dmxh::cuda_ok(cudaMemset2DAsync(dw, (N > 1 ? lddw : K) * 2, 0, K * 2, N, st))) return DMX_ERR_CUDA;
    if (dbias && N > 0 && !dmxh::cuda_ok(cudaMemsetAsync(dbias, 0, N * 2, st))) return DMX_ERR_CUDA;
    if (dx && M > 0 && K > 0 && !dmxh::cuda_ok(cudaMemset2DAsync(dx, (M > 1 ? lddx : K) * 2, 0, K * 2, M, st))) return DMX_ERR_CUDA;
    return DMX_OK;
  }
  if (!dy || (K > 0 && ((dx && !w) || (dw && !x))) || (act != DMX_ACT_NONE && !z)) return DMX_ERR_ARG;
  Matrix g = {static_cast<const bf16*>(dy), M, N, M > 1 ? lddy : N};
  Matrix a = {static_cast<const bf16*>(x), M, K, M > 1 ? ldx : K}, b = {static_cast<const bf16*>(w), N, K, N > 1 ? ldw : K};
  const BackPlan p = back_plan(g, a, b, act);
  if (p.total > workspace_bytes || !workspace) return DMX_ERR_ARG;
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  float* sums = reinterpret_cast<float*>(ws);
  ws += p.sums;
  Jobs jobs;
  int n = 0, rc = DMX_OK;
  const bool products = K > 0 && (dx || dw);
  if ((p.needs_dz && products) || dbias) {
    Job& j = jobs.job[n++];
    j = Job();
    j.in = g.p; j.ldi = g.ld; j.rows = M; j.cols = (int)N;
    j.z = act != DMX_ACT_NONE ? static_cast<const bf16*>(z) : nullptr;
    j.ldz = M > 1 ? ldz : N;
    j.sums = dbias ? sums : nullptr;
    j.vec = aligned(g.p, 16) && (M <= 1 || g.ld % 8 == 0) && N % 8 == 0 && (!j.z || (aligned(j.z, 16) && (M <= 1 || j.ldz % 8 == 0)));
    if (p.needs_dz && products) {
      g.p = j.out = reinterpret_cast<bf16*>(ws);
      g.ld = j.ldo = pad8(N);
    }
  } else {                         // (only the first job takes the activation)
    act = DMX_ACT_NONE;
  }
  ws += p.dz;
  if (K > 0 && dx) lay_out(b, ws, jobs, n);
  if (K > 0 && dw) lay_out(a, ws, jobs, n);
  if (n > 0) rc = run_jobs(jobs, n, act, st);
  if (rc == DMX_OK && dbias)
    rc = start(dim3((unsigned)((N + 31) / 32)), st, columns_kernel, (const float*)sums, (M + kChunkRows - 1) / kChunkRows, (int)N, static_cast<bf16*>(dbias));
  if (products && dx && rc == DMX_OK)          // dx[m, k] = sum_n dz[m, n] w[n, k]
    rc = plain_product(g, 0, b, 1, N, nullptr, static_cast<bf16*>(dx), M > 1 ? lddx : K, st);
  if (products && dw && rc == DMX_OK)          // dw[n, k] = sum_m dz[m, n] x[m, k]
    rc = plain_product(g, 1, a, 1, M, nullptr, static_cast<bf16*>(dw), N > 1 ? lddw : K, st);
  return rc;
}

int dmx_linear_plan(int64_t rows, int64_t cols, int64_t k, int rows_across, int64_t* plan) {
  if (!extents_ok(rows, cols, k) || rows < 1 || cols < 1 || k < 1 || !plan) return DMX_ERR_ARG;
  const Form f = form_of(rows, cols, (int)((k + kBK - 1) / kBK), rows_across);
  const int64_t r = f.exchanged ? cols : rows, c = f.exchanged ? rows : cols, high = f.choice.pair ? 2 * kBM : kBM, at_once = f.choice.pair ? 74 : 148;
  const int64_t tiles = ((r + high - 1) / high) * ((c + f.choice.bn - 1) / f.choice.bn);
  plan[0] = f.choice.bn; plan[1] = f.choice.pair; plan[2] = f.choice.split; plan[3] = f.exchanged;
  plan[4] = f.choice.split > 1 ? 1 : (tiles + at_once - 1) / at_once;
  return DMX_OK;
}

int dmx_linear_status(int* errors) {
  if (!errors) return DMX_ERR_ARG;
  // The kernels' count only grows, so nothing is lost between a read and a reset; what was reported is kept here.
  static std::mutex one_at_a_time;
  static unsigned reported[256] = {};
  int device = 0;
  if (!dmxh::cuda_ok(cudaGetDevice(&device)) || !dmxh::cuda_ok(cudaDeviceSynchronize())) return DMX_ERR_CUDA;
  const std::lock_guard<std::mutex> lock(one_at_a_time);
  unsigned n = 0, more = 0;
  if (!dmxh::cuda_ok(cudaMemcpyFromSymbol(&n, g_gave_up, sizeof n)) || !loss_gave_up(&more)) return DMX_ERR_CUDA;
  n += more;
  unsigned& before = reported[device & 255];
  *errors = (int)(n >= before ? n - before : n);       // (below it: the device was reset)
  before = n;
  return DMX_OK;
}

}  // extern "C"
