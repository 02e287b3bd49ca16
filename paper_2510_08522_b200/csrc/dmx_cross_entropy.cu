// dmx_cross_entropy.cu — softmax cross entropy of a linear layer over a vocabulary, logits never kept, and its gradient.
//
//   forward    z = x W^T + b, lse[n] = log sum_v exp z[n, v], loss[n] = lse[n] - z[n, t_n]
//   backward   G = (exp(z - lse) - [v = t_n]) dloss[n], dx = G W, dW = G^T x, db = column sums of G
//
// forward is one product (dmx_gemm.cuh) whose epilogue keeps, of a row's 32-column chunks, the running maximum and the sum of exponentials
// of the distances from it, in one pass; a small launch joins the tiles' pairs. Distances are taken before they go to units of log2 e: the maximum's own
// term is 1, the loss is log(sum) + (maximum - z[n, t_n]), never below 0, and 0 where the others' terms vanish. (One fma from logit to exponent, against
// a maximum in those units, left -4e-6 at logits of 60; it takes 1 % less of 8192 x 30522 x 1024 and 3 % less at D = 256.) backward goes through the vocabulary in pieces: a product as forward's whose epilogue
// makes a piece of G, bf16, then the two products that take it. dx is summed over the pieces in fp32.
// G is rounded to bf16 because the tensor cores take 16-bit operands; everything else up to a store is fp32. It is held in units of
// the significand of the largest |dloss|, by which the products' epilogues multiply: where all rows that count have one dloss (a mean), a
// target's entry is 1 - p times a power of two. (Units with the exponent would let rows of far smaller dloss underflow.)
// With dloss inside, the entries near -dloss of all rows were rounded the same way: dx and dW were off by 0.33 % in the mean square, with
// the unit 0.17 to 0.20 %, where one rounding of the result alone gives 0.17 %. (Few rows or words: a result may be off by two roundings, 0.2 to 0.3 % in the mean square.)
// Bound: the tensor cores, 2 N V D operations forward and 6 N V D backward (the logits are computed again). With D up to some hundred the epilogues: a
// pair's tile of 65536 logits takes about 2.5 us whatever D is (taking them out of TMEM alone 1.5), one CTA's of 32768 2.1 us, two at a time.
// Measured on B200, 8192 x 30522 x 1024 with bias: forward 315 us in bursts at full clock (1.6 PFLOP/s; floor 299 at the measured 1715), 374 us back to back under
// the power limit; backward 1120 / 1316 us (896 / 1062 at the measured 1715 / 1447; storing G takes 58 us, db 46, dx's last wave of tiles 40). 128 x 10 x 64 forward 3.5 us,
// 777 x 1000 x 513 backward 25 us, 8192 x 30522 x 256 without bias forward 115, backward 428 us (with bias and dbias 131 to 150, 490 to 520).
#include "dmx.h"

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "dmx_act.cuh"
#include "dmx_gemm.cuh"

namespace {

using namespace dmx_gemm;
using dmx_act::ex2;
using dmx_act::ex2_2;

constexpr int kFewRows = 2048;          // whose largest dloss every warp finds while the first tile is on its way; a launch of its own takes 2.5 us
constexpr float kLog2e = 1.4426950408889634f;

// ---------------------------------------------------------------------------------------------- forward

__device__ __forceinline__ int64_t target_at(const void* targets, int wide, int n) {
  return wide ? static_cast<const long long*>(targets)[n] : (int64_t)static_cast<const int*>(targets)[n];
}

template <int NC>
__device__ __forceinline__ void add_bias(const bf16* bias, int cols, float (&v)[NC], int c0) {
  if (!bias) return;
  if (c0 + NC <= cols && (reinterpret_cast<uintptr_t>(bias + c0) & 15) == 0) {
#pragma unroll
    for (int u = 0; u < NC / 8; ++u) {
      const uint4 b = reinterpret_cast<const uint4*>(bias + c0)[u];
      const unsigned w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 t = widen2(w[k]);
        v[8 * u + 2 * k] += t.x; v[8 * u + 2 * k + 1] += t.y;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < NC; ++i)
      if (c0 + i < cols) v[i] += bf_value(reinterpret_cast<const unsigned short*>(bias)[c0 + i]);
  }
}

struct SumArgs : GemmShape {
  const bf16* bias;
  const void* target;
  int wide_target;
  float* hit;                     // the targets' logits
  float2* part;                   // [tiles across][rows]: maximum, sum of exponentials of the distances from it
  float *loss, *lse;              // written here where one tile has the whole vocabulary
};

__device__ __forceinline__ float2 joined(float2 a, float2 b) {
  const float most = fmaxf(a.x, b.x), from = most == -INFINITY ? 0.f : most;         // (nothing but -inf so far)
  return make_float2(most, a.y * ex2((a.x - from) * kLog2e) + b.y * ex2((b.x - from) * kLog2e));
}
// The sum has a 1 for the maximum itself: its logarithm is not below 0, and a loss made of it and of the maximum's lead over the target neither.
__device__ __forceinline__ float lse_of(float2 v) { return v.x + logf(v.y); }
__device__ __forceinline__ float loss_of(float2 v, float hit) { return logf(v.y) + (v.x - hit); }

struct SumEpilogue {
  typedef SumArgs Args;
  static constexpr int kStaging = 0, kOwnShared = 64 + 2 * 4 * 3 * 32 * 12;
  static constexpr bool kRanged = false;
  float2 all;                     // of the row so far
  float hit;                      // its target's logit, if that is among them, else -inf
  int target;                     // -1: none (extents fit an int)
  int64_t next_target;
  __device__ __forceinline__ void fetch(const Args& A, int r0, int lane) { next_target = r0 + lane < A.rowsA ? target_at(A.target, A.wide_target, r0 + lane) : -1; }
  __device__ __forceinline__ void begin(const Args& A, int, int c0, int) {
    all = make_float2(-INFINITY, 0.f);
    hit = -INFINITY;
    target = next_target >= 0 && next_target < A.rowsB ? (int)next_target : -1;
    if (A.bias && c0 < A.rowsB) asm volatile("prefetch.global.L1 [%0];" ::"l"(A.bias + c0));
  }
  template <int NC>
  __device__ __forceinline__ void chunk(const Args& A, float (&v)[NC], uint4*, int r0, int c0, int lane) {
    add_bias(A.bias, A.rowsB, v, c0);
    if (c0 + NC > A.rowsB) {
#pragma unroll
      for (int i = 0; i < NC; ++i)
        if (c0 + i >= A.rowsB) v[i] = -INFINITY;
    }
    const unsigned place = (unsigned)((int)target - c0);
    if (__any_sync(0xffffffffu, place < (unsigned)NC)) {
#pragma unroll
      for (int i = 0; i < NC; ++i) hit = place == (unsigned)i ? v[i] : hit;
      if (place < (unsigned)NC && !A.loss) A.hit[r0 + lane] = hit;
    }
    float m[4];                   // several chains: the epilogue's latency is what short products wait for
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      m[j] = v[j * (NC / 4)];
#pragma unroll
      for (int i = 1; i + 1 < NC / 4; i += 2) m[j] = fmaxf(fmaxf(m[j], v[j * (NC / 4) + i]), v[j * (NC / 4) + i + 1]);
      m[j] = fmaxf(m[j], v[(j + 1) * (NC / 4) - 1]);
    }
    const float most = fmaxf(all.x, fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])));
    const float from = most == -INFINITY ? 0.f : most;         // (nothing but -inf so far)
    float2 e[2] = {make_float2(all.y * ex2((all.x - from) * kLog2e), 0.f), two(0.f)};
#pragma unroll
    for (int i = 0; i < NC / 2; ++i) e[i & 1] = add2(e[i & 1], ex2_2(mul2(add2(make_float2(v[2 * i], v[2 * i + 1]), two(-from)), two(kLog2e))));
    const float2 s = add2(e[0], e[1]);
    all = make_float2(most, s.x + s.y);
  }
  // The four warps that share rows meet in shared memory, in two places by turns; the accumulators are handed back afterwards, so that
  // nobody is so far ahead that it writes where the first still reads.
  struct Meeting {
    uint64_t here[2][4];
    float2 pair[2][4][3][32];
    float hit[2][4][3][32];
  };
  static_assert(sizeof(Meeting) <= kOwnShared, "what the launch leaves room for");
  static __device__ __forceinline__ Meeting& meeting() {
    __shared__ Meeting m;
    return m;
  }
  static __device__ __forceinline__ void setup() {
    for (int i = 0; i < 8; ++i) bar_init(smem_addr(&meeting().here[i / 4][i % 4]), 3);
  }
  __device__ __forceinline__ bool end(const Args& A, int r0, int tb, int group, int lane, int turn, unsigned parity) {
    Meeting& m = meeting();
    const int quarter = (r0 >> 5) & 3;
    if (group > 0) {
      m.pair[turn][quarter][group - 1][lane] = all;
      if (A.loss) m.hit[turn][quarter][group - 1][lane] = hit;
      __syncwarp();
      if (lane == 0) bar_arrive(smem_addr(&m.here[turn][quarter]));
      return true;
    }
    if (!warp_wait(smem_addr(&m.here[turn][quarter]), parity)) return false;
#pragma unroll
    for (int g = 0; g < 3; ++g) all = joined(all, m.pair[turn][quarter][g][lane]);
    if (r0 + lane >= A.rowsA) return true;
    if (A.loss) {
      if (target >= 0) {
        const int g = target / 32 % 4;                    // which warp had it: chunks go to them in turn
        if (g > 0) hit = m.hit[turn][quarter][g - 1][lane];
      }
      A.lse[r0 + lane] = lse_of(all);
      A.loss[r0 + lane] = target >= 0 ? loss_of(all, hit) : 0.f;
    } else {
      A.part[(int64_t)tb * A.rowsA + r0 + lane] = all;
    }
    return true;
  }
};

// 32 rows a CTA, its warps take every eighth pair
__global__ void __launch_bounds__(256) join_kernel(const float2* part, int parts, int N, int V, const float* hit, const void* target, int wide_target, float* loss, float* lse) {
  __shared__ float2 sh[8][32];
  start_dependents();
  wait_for_previous();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n = blockIdx.x * 32 + lane;
  float2 v = make_float2(-INFINITY, 0.f);
  if (n < N) {
#pragma unroll 8
    for (int i = warp; i < parts; i += 8) v = joined(v, part[(int64_t)i * N + n]);
  }
  sh[warp][lane] = v;
  __syncthreads();
  if (warp > 0 || n >= N) return;
  for (int w = 1; w < 8; ++w) v = joined(v, sh[w][lane]);
  const int64_t t = target_at(target, wide_target, n);
  lse[n] = lse_of(v);
  loss[n] = t >= 0 && t < V ? loss_of(v, hit[n]) : 0.f;
}

// ---------------------------------------------------------------------------------------------- backward

struct SlopeArgs : GemmShape {
  const bf16* bias;               // of the piece
  const void* target;
  int wide_target, first, vocabulary, vec;    // first: the piece's first word
  const float *lse, *dloss;
  float* unit;                    // there already, or (few rows) found by every warp on its own while the first tile is on its way
  int find_unit;
  int64_t stride;                 // of dloss: 1 or 0
  bf16* g;                        // or NULL: the columns' sums alone
  int64_t ldg;
  float* columns;                 // [rows / 32][piece]: sums over 32 rows, or NULL
};

__device__ __forceinline__ float finite_size(float d) {
  d = fabsf(d);
  return d <= 3.402823466e38f ? d : 0.f;
}
__device__ __forceinline__ float unit_of(float most) {
  int e;
  return most == 0.f ? 1.f : 2.f * frexpf(most, &e);
}

struct SlopeEpilogue {
  typedef SlopeArgs Args;
  static constexpr int kStaging = 2048, kOwnShared = 0;
  static constexpr bool kRanged = false;
  float lse, scale, units = 0.f;
  bool every;                     // all of the warp's rows have a slope
  int target;                     // in the piece; outside of it where it lies elsewhere, far below where there is none
  int64_t next_target;
  float next_lse, next_dloss;
  __device__ __forceinline__ void fetch(const Args& A, int r0, int lane) {
    const int n = r0 + lane;
    next_target = -1;
    next_lse = next_dloss = 0.f;
    if (n >= A.rowsA) return;
    next_target = target_at(A.target, A.wide_target, n);
    next_lse = A.lse[n];
    next_dloss = A.dloss[n * A.stride];
  }
  __device__ __forceinline__ void begin(const Args& A, int r0, int c0, int lane) {
    if (units == 0.f) {
      if (A.find_unit) {
        float most = 0.f;
#pragma unroll 8
        for (int n = lane; n < A.rowsA; n += 32) most = fmaxf(most, finite_size(A.dloss[n * A.stride]));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        units = unit_of(most);
        if (r0 == 0 && c0 == 0 && lane == 0) *A.unit = units;
      } else {
        units = *A.unit;
      }
    }
    if (A.bias && c0 < A.rowsB) asm volatile("prefetch.global.L1 [%0];" ::"l"(A.bias + c0));
    const bool live = next_target >= 0 && next_target < A.vocabulary;
    lse = next_lse;
    scale = live ? next_dloss / units : 0.f;
    target = live ? (int)next_target - A.first : -0x40000000;
    every = __all_sync(0xffffffffu, scale != 0.f);
  }
  template <int NC>
  __device__ __forceinline__ void chunk(const Args& A, float (&v)[NC], uint4* stage, int r0, int c0, int lane) {
    add_bias(A.bias, A.rowsB, v, c0);
#pragma unroll
    for (int i = 0; i < NC / 2; ++i) {
      const float2 p = mul2(ex2_2(mul2(add2(make_float2(v[2 * i], v[2 * i + 1]), two(-lse)), two(kLog2e))), two(scale));
      v[2 * i] = p.x; v[2 * i + 1] = p.y;
    }
    if (!every) {                 // a row without a target has scale 0: its values are zeros whatever its logits are
#pragma unroll
      for (int i = 0; i < NC; ++i) v[i] = scale == 0.f ? 0.f : v[i];
    }
    const unsigned place = (unsigned)((int)target - c0);
    if (__any_sync(0xffffffffu, place < (unsigned)NC)) {
#pragma unroll
      for (int i = 0; i < NC; ++i) v[i] -= place == (unsigned)i ? scale : 0.f;
    }
    if (A.g) {
#pragma unroll
      for (int u = 0; u < NC / 8; ++u)
        *unit(stage, lane, u) = make_uint4(pack2(v[8 * u], v[8 * u + 1]), pack2(v[8 * u + 2], v[8 * u + 3]), pack2(v[8 * u + 4], v[8 * u + 5]),
                                           pack2(v[8 * u + 6], v[8 * u + 7]));
      store_tile<32, NC>(A.g, A.ldg, A.vec, stage, r0, A.rowsA, c0, A.rowsB, lane);
    }
    if (A.columns) {
      // lane i ends with column i's sum: in every step half of the columns go to the lane across
      static_assert(NC == 32, "a column per lane");
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        const bool high = lane & o;
#pragma unroll
        for (int i = 0; i < o; ++i) {
          const float keep = high ? v[i + o] : v[i], give = high ? v[i] : v[i + o];
          v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
      }
      if (r0 < A.rowsA && c0 + lane < A.rowsB) A.columns[(int64_t)(r0 >> 5) * A.rowsB + c0 + lane] = v[0];      // (in units)
    }
  }
  static __device__ __forceinline__ void setup() {}
  __device__ __forceinline__ bool end(const Args&, int, int, int, int, int, unsigned) { return true; }
};

// dx over several pieces: sums in fp32, in an order of their own (a warp's 32 rows x 32 columns after one another, a column of lanes at a time)
struct AddArgs : GemmShape {
  float* unit;
  float* sums;
  bf16* y;
  int64_t ldy;
  int first, last, vec;
};

template <int BN>
struct AddEpilogue {
  typedef AddArgs Args;
  static constexpr int kStaging = 2048, kOwnShared = 0;
  static constexpr bool kRanged = false;
  float times;
  __device__ __forceinline__ void fetch(const Args&, int, int) {}
  __device__ __forceinline__ void begin(const Args& A, int, int, int) { times = A.last ? *A.unit : 1.f; }
  template <int NC>
  __device__ __forceinline__ void chunk(const Args& A, float (&v)[NC], uint4* stage, int r0, int c0, int lane) {
    float* at = A.sums + ((int64_t)(r0 >> 5) * (A.tilesB * (BN / 32)) + (c0 >> 5)) * 1024 + lane;
    if (!A.first) {
#pragma unroll
      for (int i = 0; i < NC; ++i) v[i] += __ldcs(at + i * 32);
    }
    if (!A.last) {
#pragma unroll
      for (int i = 0; i < NC; ++i) __stcs(at + i * 32, v[i]);
      return;
    }
#pragma unroll
    for (int i = 0; i < NC; ++i) v[i] *= times;
#pragma unroll
    for (int u = 0; u < NC / 8; ++u)
      *unit(stage, lane, u) = make_uint4(pack2(v[8 * u], v[8 * u + 1]), pack2(v[8 * u + 2], v[8 * u + 3]), pack2(v[8 * u + 4], v[8 * u + 5]),
                                         pack2(v[8 * u + 6], v[8 * u + 7]));
    store_tile<32, NC>(A.y, A.ldy, A.vec, stage, r0, A.rowsA, c0, A.rowsB, lane);
  }
  static __device__ __forceinline__ void setup() {}
  __device__ __forceinline__ bool end(const Args&, int, int, int, int, int, unsigned) { return true; }
};

// the significand (1 to 2) of the largest finite |dloss|, 1 if that is zero: many rows
__global__ void __launch_bounds__(1024) unit_kernel(const float* dloss, int64_t stride, int N, float* unit) {
  __shared__ float sh[32];
  start_dependents();
  wait_for_previous();
  float most = 0.f;
#pragma unroll 8
  for (int n = threadIdx.x; n < N; n += 1024) most = fmaxf(most, finite_size(dloss[n * stride]));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = most;
  __syncthreads();
  if (threadIdx.x >= 32) return;
  most = sh[threadIdx.x];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
  if (threadIdx.x == 0) *unit = unit_of(most);
}

// A product of few tiles over a long k: every range's part in fp32, in the order of AddEpilogue, and a launch that adds them.
struct PartArgs : GemmShape {
  float* parts;
};

template <int BN>
struct PartEpilogue {
  typedef PartArgs Args;
  static constexpr int kStaging = 0, kOwnShared = 0;
  static constexpr bool kRanged = true;
  int range;
  __device__ __forceinline__ void fetch(const Args&, int, int) {}
  __device__ __forceinline__ void begin(const Args&, int, int, int) {}
  template <int NC>
  __device__ __forceinline__ void chunk(const Args& A, float (&v)[NC], uint4*, int r0, int c0, int lane) {
    const int64_t blocks = (A.rowsA + 31) / 32, across = (A.rowsB + 31) / 32;
    float* at = A.parts + ((range * blocks + (r0 >> 5)) * across + (c0 >> 5)) * 1024 + lane;
    if (r0 + lane < A.rowsA) {
#pragma unroll
      for (int i = 0; i < NC; ++i) at[i * 32] = v[i];
    }
    __syncwarp();
  }
  static __device__ __forceinline__ void setup() {}
  __device__ __forceinline__ bool end(const Args&, int, int, int, int, int, unsigned) { return true; }
};

// a warp: 32 rows (a lane each) x four columns
__global__ void __launch_bounds__(256) add_parts_kernel(const float* parts, int ranges, int rows, int cols, const float* unit, bf16* y, int64_t ldy) {
  start_dependents();
  wait_for_previous();
  const int lane = threadIdx.x & 31;
  const int64_t blocks = (rows + 31) / 32, across = (cols + 31) / 32, job = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (job >= blocks * across * 8) return;
  const int64_t block = job / 8;
  const int r = (int)(block / across) * 32 + lane, c = (int)(block % across) * 32 + (int)(job % 8) * 4;
  if (r >= rows || c >= cols) return;
  const float* at = parts + block * 1024 + job % 8 * 128 + lane;
  float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int k = 0; k < ranges; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] += at[k * blocks * across * 1024 + i * 32];
  const float times = *unit;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (c + i < cols) y[(int64_t)r * ldy + c + i] = __float2bfloat16_rn(s[i] * times);
}

// db from the sums over 32 rows each: 32 columns a CTA
__global__ void __launch_bounds__(1024) columns_kernel(const float* sums, int rows, int cols, const float* unit, bf16* out) {
  __shared__ float sh[32][33];
  start_dependents();
  wait_for_previous();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  float s = 0.f;
  if (c < cols) {
#pragma unroll 4
    for (int r = warp; r < rows; r += 32) s += sums[(int64_t)r * cols + c];
  }
  sh[warp][lane] = s;
  __syncthreads();
  if (warp > 0 || c >= cols) return;
  for (int w = 1; w < 32; ++w) s += sh[w][lane];
  out[c] = __float2bfloat16_rn(s * *unit);
}

// ---------------------------------------------------------------------------------------------- host

template <class E>
int product_rows(const Matrix& a, const Matrix& b, typename E::Args& A, const Choice& c, cudaStream_t st) {      // D's rows are a's
  if (c.pair) return c.bn == 256 ? launch_gemm<256, true, 1, E>(a, b, A, st) : launch_gemm<128, true, 1, E>(a, b, A, st);
  if (c.bn == 256) return launch_gemm<256, false, 1, E>(a, b, A, st);
  return c.bn == 128 ? launch_gemm<128, false, 1, E>(a, b, A, st) : launch_gemm<64, false, 1, E>(a, b, A, st);
}
Choice choose_rows(int64_t N, int64_t V, int64_t D, float weight) { return choose_by_tiles(N, V, (int)((D + kBK - 1) / kBK), false, false, weight); }
constexpr float kSumWeight = 1.f, kSlopeWeight = 1.3f;        // of their epilogues (1.5 leaves 8192 x 30522 x 512 to single CTAs: slopes 290 us, in pairs 272)

bool sizes_ok(int64_t N, int64_t V, int64_t D) {
  const int64_t most = DMX_LINEAR_MAX_EXTENT;
  return N >= 0 && V >= 1 && D >= 1 && N <= most && V <= most && D <= most;
}
bool in_ok(int64_t rows, int64_t ld) { return rows <= 1 || ld >= 0; }
bool out_ok(int64_t rows, int64_t cols, int64_t ld) { return rows <= 1 || ld >= cols; }
Matrix matrix(const void* p, int64_t rows, int64_t cols, int64_t ld) { return {static_cast<const bf16*>(p), rows, cols, rows > 1 ? ld : cols}; }

struct ForwardPlan {
  Choice choice;
  int64_t parts, part, hit, total;
};
ForwardPlan forward_plan(const Matrix& x, const Matrix& w) {
  ForwardPlan p;
  p.choice = choose_rows(x.rows, w.rows, x.cols, kSumWeight);
  p.parts = (w.rows + p.choice.bn - 1) / p.choice.bn;
  p.part = pad256(p.parts * x.rows * 8);
  p.hit = pad256(x.rows * 4);
  p.total = p.part + p.hit + laid_out_bytes(x) + laid_out_bytes(w);
  return p;
}

// A product with few tiles: tiles x ranges of k fill the card once. ranges 0: as plain_product does it, unless ranges take a fifth off its time
// (a stage's time as `choose_by_tiles` has it, 3.5 us for the launch that adds, the parts' traffic at 4 TB/s). 16000 x 64 into 300 words: dW 21 -> 9 us.
struct Cut {
  int bn, ranges;
  int64_t bytes;
};
Cut cut_of(int64_t rows, int64_t cols, int64_t k, int mnA) {
  const int kblocks = (int)((k + kBK - 1) / kBK);
  const int64_t area = (rows + 31) / 32 * ((cols + 31) / 32) * 4096;
  Cut best = {0, 0, 0};
  float least = 0.8f * plain_product_ns(rows, cols, k, mnA);
  const struct { int bn; float stage; } forms[2] = {{128, 290.f}, {64, 245.f}};
  for (const auto& f : forms) {
    const int64_t tiles = (rows + kBM - 1) / kBM * ((cols + f.bn - 1) / f.bn);
    int64_t ranges = 148 / tiles < kblocks ? 148 / tiles : kblocks;
    if (ranges < 2) continue;
    const float t = (float)((kblocks + ranges - 1) / ranges) * f.stage + 8.f * f.bn + 3500.f + (float)(ranges * area) * 2 / 4000.f;
    if (t < least) { least = t; best = {f.bn, (int)ranges, pad256(ranges * area)}; }
  }
  return best;
}
int product_of(const Cut& cut, const Matrix& a, int mnA, const Matrix& b, int mnB, int64_t k, const float* unit, float* parts, bf16* y, int64_t ldy, cudaStream_t st) {
  if (cut.ranges == 0) return plain_product(a, mnA, b, mnB, k, unit, y, ldy, st);
  const int64_t rows = mnA ? a.cols : a.rows, cols = mnB ? b.cols : b.rows;
  PartArgs A = {};
  A.rowsA = (int)rows; A.rowsB = (int)cols; A.kblocks = (int)((k + kBK - 1) / kBK); A.mnA = mnA; A.mnB = mnB;
  A.ranges = cut.ranges; A.parts = parts;
  const int rc = cut.bn == 128 ? launch_gemm<128, false, 1, PartEpilogue<128>>(a, b, A, st) : launch_gemm<64, false, 1, PartEpilogue<64>>(a, b, A, st);
  if (rc != DMX_OK) return rc;
  const int64_t jobs = (rows + 31) / 32 * ((cols + 31) / 32) * 8;
  return start(dim3((unsigned)((jobs + 7) / 8)), st, add_parts_kernel, (const float*)parts, cut.ranges, (int)rows, (int)cols, unit, y, ldy);
}

// Pieces of the vocabulary: G of a piece takes 512 MB at most (but 256 words at least).
struct BackPlan {
  int64_t pieces, words, g, columns, sums, total;      // sums: of dx over the pieces, or a cut product's parts
  Cut dx, dw;                                          // with one piece
};
enum { kDx = 1, kDw = 2, kDbias = 4 };                 // outputs
BackPlan back_plan(const Matrix& x, const Matrix& w, int outputs) {
  const int64_t N = x.rows, V = w.rows, D = x.cols;
  BackPlan p;
  int64_t most = ((int64_t)1 << 29) / (2 * N) / 256 * 256;
  if (most < 256) most = 256;
  p.pieces = (V + most - 1) / most;
  p.words = ((V + p.pieces - 1) / p.pieces + 255) / 256 * 256;
  p.pieces = (V + p.words - 1) / p.words;
  const int64_t cols = p.words < V ? p.words : V;
  p.g = outputs & (kDx | kDw) ? pad256(N * pad8(cols) * 2) : 0;
  p.columns = outputs & kDbias ? pad256((N + 31) / 32 * cols * 4) : 0;
  p.dx = p.dw = Cut{0, 0, 0};
  if (p.pieces == 1) {
    if (outputs & kDx) p.dx = cut_of(N, D, V, 0);
    if (outputs & kDw) p.dw = cut_of(V, D, N, 1);
  }
  p.sums = p.pieces == 1 ? (p.dx.bytes > p.dw.bytes ? p.dx.bytes : p.dw.bytes) : outputs & kDx ? ((N + 255) / 256 * 256) * ((D + 255) / 256 * 256) * 4 : 0;
  p.total = 256 + p.g + p.columns + p.sums + laid_out_bytes(x) + laid_out_bytes(w);
  return p;
}

}  // namespace

namespace dmx_gemm {

bool loss_gave_up(unsigned* n) { return dmxh::cuda_ok(cudaMemcpyFromSymbol(n, g_gave_up, sizeof *n)); }

}  // namespace dmx_gemm

extern "C" {

int64_t dmx_cross_entropy_workspace(int64_t N, int64_t V, int64_t D, const void* x, int64_t ldx, const void* w, int64_t ldw) {
  if (!sizes_ok(N, V, D)) return DMX_ERR_ARG;
  return N == 0 ? 0 : forward_plan(matrix(x, N, D, ldx), matrix(w, V, D, ldw)).total;
}

int dmx_cross_entropy_forward(int64_t N, int64_t V, int64_t D, const void* x, int64_t ldx, const void* w, int64_t ldw, const void* bias, int target_bytes,
                              const void* target, float* loss, float* lse, void* workspace, int64_t workspace_bytes, void* cuda_stream) {
  if (!sizes_ok(N, V, D) || !in_ok(N, ldx) || !in_ok(V, ldw) || (target_bytes != 4 && target_bytes != 8)) return DMX_ERR_ARG;
  if (N == 0) return DMX_OK;
  if (!x || !w || !target || !loss || !lse) return DMX_ERR_ARG;
  if (!aligned(x, 2) || !aligned(w, 2) || !aligned(bias, 2) || !aligned(target, target_bytes) || !aligned(loss, 4) || !aligned(lse, 4) || !aligned(workspace, 256)) return DMX_ERR_ALIGN;
  Matrix a = matrix(x, N, D, ldx), b = matrix(w, V, D, ldw);
  const ForwardPlan p = forward_plan(a, b);
  if (workspace_bytes < p.total || !workspace) return DMX_ERR_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  SumArgs A = {};
  A.rowsA = (int)N; A.rowsB = (int)V; A.kblocks = (int)((D + kBK - 1) / kBK);
  A.bias = static_cast<const bf16*>(bias); A.target = target; A.wide_target = target_bytes == 8;
  A.part = reinterpret_cast<float2*>(ws);
  A.hit = reinterpret_cast<float*>(ws + p.part);
  if (p.parts == 1) { A.loss = loss; A.lse = lse; }
  ws += p.part + p.hit;
  Jobs jobs;
  int n = 0;
  lay_out(a, ws, jobs, n);
  lay_out(b, ws, jobs, n);
  int rc = n > 0 ? run_jobs(jobs, n, DMX_ACT_NONE, st) : DMX_OK;
  if (rc == DMX_OK) rc = product_rows<SumEpilogue>(a, b, A, p.choice, st);
  if (rc != DMX_OK || p.parts == 1) return rc;
  return start(dim3((unsigned)((N + 31) / 32)), st, join_kernel, (const float2*)A.part, (int)p.parts, (int)N, (int)V, (const float*)A.hit, target, A.wide_target, loss, lse);
}

int64_t dmx_cross_entropy_backward_workspace_for(int64_t N, int64_t V, int64_t D, const void* x, int64_t ldx, const void* w, int64_t ldw, int outputs) {
  if (!sizes_ok(N, V, D) || outputs < 0 || outputs > (kDx | kDw | kDbias)) return DMX_ERR_ARG;
  return N == 0 || outputs == 0 ? 0 : back_plan(matrix(x, N, D, ldx), matrix(w, V, D, ldw), outputs).total;
}

int64_t dmx_cross_entropy_backward_workspace(int64_t N, int64_t V, int64_t D, const void* x, int64_t ldx, const void* w, int64_t ldw) {
  return dmx_cross_entropy_backward_workspace_for(N, V, D, x, ldx, w, ldw, kDx | kDw | kDbias);
}

int dmx_cross_entropy_backward(int64_t N, int64_t V, int64_t D, const float* dloss, int64_t dloss_stride, const void* x, int64_t ldx, const void* w, int64_t ldw,
                               const void* bias, int target_bytes, const void* target, const float* lse, void* dx, int64_t lddx, void* dw, int64_t lddw, void* dbias,
                               void* workspace, int64_t workspace_bytes, void* cuda_stream) {
  if (!sizes_ok(N, V, D) || !in_ok(N, ldx) || !in_ok(V, ldw) || (N > 1 && dloss_stride < 0) || (target_bytes != 4 && target_bytes != 8) || (dx && !out_ok(N, D, lddx)) ||
      (dw && !out_ok(V, D, lddw))) return DMX_ERR_ARG;
  if (!aligned(x, 2) || !aligned(w, 2) || !aligned(bias, 2) || !aligned(target, target_bytes) || !aligned(dloss, 4) || !aligned(lse, 4) || !aligned(dx, 2) || !aligned(dw, 2) ||
      !aligned(dbias, 2) || !aligned(workspace, 256)) return DMX_ERR_ALIGN;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (N == 0) {                                // empty sums
    if (dw && !dmxh::cuda_ok(cudaMemset2DAsync(dw, (V > 1 ? lddw : D) * 2, 0, D * 2, V, st))) return DMX_ERR_CUDA;
    if (dbias && !dmxh::cuda_ok(cudaMemsetAsync(dbias, 0, V * 2, st))) return DMX_ERR_CUDA;
    return DMX_OK;
  }
  if (!dx && !dw && !dbias) return DMX_OK;
  if (!x || !w || !target || !lse || !dloss) return DMX_ERR_ARG;
  Matrix a = matrix(x, N, D, ldx), b = matrix(w, V, D, ldw);
  const BackPlan p = back_plan(a, b, (dx ? kDx : 0) | (dw ? kDw : 0) | (dbias ? kDbias : 0));
  if (workspace_bytes < p.total || !workspace) return DMX_ERR_ARG;
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  float* unit = reinterpret_cast<float*>(ws);
  ws += 256;
  bf16* g = reinterpret_cast<bf16*>(ws);
  float* columns = reinterpret_cast<float*>(ws + p.g);
  float* sums = reinterpret_cast<float*>(ws + p.g + p.columns);
  ws += p.g + p.columns + p.sums;
  Jobs jobs;
  int n = 0;
  lay_out(a, ws, jobs, n);
  lay_out(b, ws, jobs, n);
  int rc = n > 0 ? run_jobs(jobs, n, DMX_ACT_NONE, st) : DMX_OK;
  const bool find_unit = N <= kFewRows;
  if (rc == DMX_OK && !find_unit) rc = start(dim3(1), 1024, st, unit_kernel, dloss, dloss_stride, dloss_stride == 0 ? 1 : (int)N, unit);
  for (int64_t first = 0; first < V && rc == DMX_OK; first += p.words) {
    const int64_t words = V - first < p.words ? V - first : p.words;
    const Matrix piece = {b.p + first * b.ld, words, D, b.ld};
    SlopeArgs A = {};
    A.rowsA = (int)N; A.rowsB = (int)words; A.kblocks = (int)((D + kBK - 1) / kBK);
    A.bias = bias ? static_cast<const bf16*>(bias) + first : nullptr; A.target = target; A.wide_target = target_bytes == 8;
    A.first = (int)first; A.vocabulary = (int)V; A.lse = lse; A.dloss = dloss; A.unit = unit; A.find_unit = find_unit && first == 0; A.stride = N > 1 ? dloss_stride : 0;
    A.g = dx || dw ? g : nullptr; A.ldg = pad8(words); A.vec = 1; A.columns = dbias ? columns : nullptr;
    rc = product_rows<SlopeEpilogue>(a, piece, A, choose_rows(N, words, D, kSlopeWeight), st);
    if (rc == DMX_OK && dbias)
      rc = start(dim3((unsigned)((words + 31) / 32)), 1024, st, columns_kernel, (const float*)columns, (int)((N + 31) / 32), (int)words, (const float*)unit, static_cast<bf16*>(dbias) + first);
    const Matrix G = {g, N, words, A.ldg};
    if (rc == DMX_OK && dw) rc = product_of(p.dw, G, 1, a, 1, N, unit, sums, static_cast<bf16*>(dw) + first * (V > 1 ? lddw : D), V > 1 ? lddw : D, st);
    if (rc != DMX_OK || !dx) continue;
    if (p.pieces == 1) {
      rc = product_of(p.dx, G, 0, piece, 1, words, unit, sums, static_cast<bf16*>(dx), N > 1 ? lddx : D, st);
      continue;
    }
    AddArgs E = {};
    E.rowsA = (int)N; E.rowsB = (int)D; E.kblocks = (int)((words + kBK - 1) / kBK); E.mnB = 1;
    E.unit = unit; E.sums = sums; E.y = static_cast<bf16*>(dx); E.ldy = N > 1 ? lddx : D; E.first = first == 0; E.last = first + words >= V;
    E.vec = aligned(dx, 16) && (N <= 1 || E.ldy % 8 == 0);
    rc = launch_gemm<256, true, 1, AddEpilogue<256>>(G, piece, E, st);
  }
  return rc;
}

int dmx_cross_entropy_plan(int64_t N, int64_t V, int64_t D, int64_t* plan) {
  if (!sizes_ok(N, V, D) || N < 1 || !plan) return DMX_ERR_ARG;
  const Matrix x = {nullptr, N, D, D}, w = {nullptr, V, D, D};
  const ForwardPlan f = forward_plan(x, w);
  const BackPlan b = back_plan(x, w, kDx | kDw | kDbias);
  const Choice s = choose_rows(N, b.words < V ? b.words : V, D, kSlopeWeight);
  const int64_t values[11] = {f.choice.bn, f.choice.pair, f.parts, b.pieces, b.words, s.bn, s.pair, b.dx.bn, b.dx.ranges, b.dw.bn, b.dw.ranges};
  for (int i = 0; i < 11; ++i) plan[i] = values[i];
  return DMX_OK;
}

}  // extern "C"
