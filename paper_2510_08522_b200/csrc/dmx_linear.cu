// dmx_linear.cu — matrix product with bias, activation and residual in its epilogue, and its gradient (bf16
// operands, fp32 accumulation).
//
//   forward    z = x W^T + b, y = act(z) + r
//   backward   dz = dy act'(z) (one elementwise pass, which also sums its columns for db), dx = dz W, dW = dz^T x
//
// All three products are D[i, j] = sum_k A[i, k] B[j, k] on the 5th-generation tensor cores, by one kernel: a
// producer warp moves tiles of A (128 rows) and B (32 to 256) of 64 k with TMA into a ring of shared memory
// stages, one thread issues tcgen05.mma on them into accumulators in TMEM, and sixteen warps take finished accumulators out
// (tcgen05.ld), apply the epilogue and store, while the next tile accumulates in the other half of TMEM. An
// operand whose rows run along k is K-major; W in dx, and both operands of dW, run across it (MN-major) and are
// multiplied as they lie: only the descriptors differ, nothing is transposed in memory.
// Few rows (M <= 64): the operands change places, so that W's rows fill the 128 lanes and the few rows of x are the narrow
// side. Few tiles: k is split over the CTAs of a cluster, whose partial sums meet in distributed shared memory and
// are added in a fixed order.
// Every wait is bounded; a warp that gives up counts itself in a device word (dmx_linear_status), and its CTA lets its
// copies land, frees its TMEM and returns.
// Bound: the tensor cores for large products, what an SM fetches from L2 (64 bytes a cycle) for narrow tiles, HBM for few rows.
// Measured on B200 in bursts at full clock / back to back for seconds under the power limit: 8192^3 714 / 833 us = 1.54 / 1.32 PFLOP/s
// (the library's 669 / 774 us); 8192 x 4096 x 1024 with GELU, y and z written, 65 / 77 us = 1.06 / 0.89 PFLOP/s (the library's bare product
// 56 / 60 us); its gradient 132 / 151 us; one row x 4096 x 4096 7.9 / 7.6 us = 4.3 TB/s.
#include "dmx.h"

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <atomic>
#include <mutex>

#include "dmx_act.cuh"
#include "dmx_host.h"

namespace {

using namespace dmx_f32x2;
typedef __nv_bfloat16 bf16;

constexpr int kBM = 128, kBK = 64;            // tile rows of A; k per stage (128 bytes: one swizzle row)
constexpr int kEpiWarps = 16;                 // four per scheduler: with two a GELU epilogue took longer than 1024 k
constexpr int kGemmThreads = 64 + 32 * kEpiWarps;
constexpr int kMaxStages = 8;
constexpr int kSmemMost = 226 * 1024;
constexpr unsigned kPolls = 1u << 18;         // about a second

__device__ unsigned g_gave_up;                // warps whose waits ran out

struct GemmArgs {
  int rowsA, rowsB, kblocks;                  // rows of D, columns of D, ceil(k / 64)
  int tilesA, tilesB, stages;
  int mnA, mnB;                               // operand is MN-major
  const bf16 *bias, *residual;
  bf16 *y, *z;
  int64_t ldr, ldy, ldz;
  int act;
  int vecy, vecz, vecr;                       // 16-byte rows
};

// ---------------------------------------------------------------------------------------------- PTX

__device__ __forceinline__ unsigned smem_addr(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }
// One lane of a converged warp, chosen so that the compiler knows it is one (tensor core and copy instructions take
// warp-uniform operands).
__device__ __forceinline__ bool elect() {
  unsigned p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ void bar_init(unsigned bar, unsigned count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(unsigned bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void bar_expect(unsigned bar, unsigned bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// false if the barrier did not complete in time
__device__ __forceinline__ bool bar_wait(unsigned bar, unsigned parity) {
  for (unsigned n = 0; n < kPolls; ++n) {
    unsigned done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    if (done) return true;
  }
  return false;
}
__device__ __forceinline__ bool warp_wait(unsigned bar, unsigned parity) { return __all_sync(0xffffffffu, bar_wait(bar, parity)); }
__device__ __forceinline__ void tma_load(unsigned dst, const CUtensorMap* map, int c0, int c1, unsigned bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(bar) : "memory");
}
// In a pair of CTAs the loads of both count on the first one's barrier.
__device__ __forceinline__ void tma_load_pair(unsigned dst, const CUtensorMap* map, int c0, int c1, unsigned bar) {
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(bar) : "memory");
}
__device__ __forceinline__ unsigned in_cta(unsigned addr, int rank) {     // the same place in another CTA of the cluster
  unsigned a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
  return a;
}
__device__ __forceinline__ void bar_arrive_cluster(unsigned bar) { asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void mma_pair(unsigned d, uint64_t a, uint64_t b, unsigned idesc, unsigned accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_commit_pair(unsigned bar) {           // to that barrier of both CTAs
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((unsigned short)3) : "memory");
}
__device__ __forceinline__ void mma(unsigned d, uint64_t a, uint64_t b, unsigned idesc, unsigned accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_commit(unsigned bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_load32(unsigned addr, float (&v)[32]) {
  unsigned r[32];
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
               "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
               "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                 "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
                 "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
                 "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]) : "r"(addr));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}

// Shared memory descriptor of a 128-byte swizzled operand. K-major: rows of 128 bytes, groups of eight 1024 bytes apart.
// MN-major: rows (one per k) of 64 elements; eight k 1024 bytes apart, the next 64 elements 64 rows further.
__device__ __forceinline__ uint64_t descriptor(unsigned addr, int mn) {
  const uint64_t lead = mn ? (kBK * 128) >> 4 : 1, stride = 1024 >> 4;
  return (uint64_t)((addr >> 4) & 0x3fff) | lead << 16 | stride << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

// Launched as programmatic dependents: what needs no data is set up while the kernel before still runs; then all of its
// (and earlier) writes are waited for. The kernel after may begin likewise.
__device__ __forceinline__ void start_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ __forceinline__ float bf_value(unsigned short u) { return __uint_as_float((unsigned)u << 16); }
__device__ __forceinline__ unsigned pack2(float a, float b) {
  __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<unsigned*>(&t);
}

// ---------------------------------------------------------------------------------------------- epilogue

// A warp's staging buffer: 32 rows of 64 bytes, 16-byte units exchanged by the row so that both a row per lane
// and eight rows at a time are free of bank conflicts.
__device__ __forceinline__ uint4* unit(uint4* stage, int row, int u) { return stage + row * 4 + (u ^ ((row >> 1) & 3)); }

// ROWS rows from r0 and COLS (8 to 32) columns from c0 of a matrix, out of and into the staging buffer
template <int ROWS, int COLS>
__device__ __forceinline__ void store_tile(bf16* p, int64_t ld, int vec, uint4* stage, int r0, int rows, int c0, int cols, int lane) {
  constexpr int kUnits = COLS / 8, kAtOnce = 32 / kUnits;
  __syncwarp();
  if (vec) {
#pragma unroll
    for (int i = 0; i < (ROWS + kAtOnce - 1) / kAtOnce; ++i) {
      const int r = i * kAtOnce + lane / kUnits, u = lane % kUnits, c = c0 + u * 8;
      if (r >= ROWS || r0 + r >= rows || c >= cols) continue;
      const uint4 v = *unit(stage, r, u);
      bf16* q = p + (int64_t)(r0 + r) * ld + c;
      if (c + 8 <= cols) {
        *reinterpret_cast<uint4*>(q) = v;
      } else {
        const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (c + k < cols) reinterpret_cast<unsigned short*>(q)[k] = (unsigned short)(w[k >> 1] >> (16 * (k & 1)));
      }
    }
  } else if (lane < COLS && c0 + lane < cols) {
    const int n = min(ROWS, rows - r0);
#pragma unroll 8
    for (int r = 0; r < n; ++r)
      reinterpret_cast<unsigned short*>(p)[(int64_t)(r0 + r) * ld + c0 + lane] = reinterpret_cast<const unsigned short*>(unit(stage, r, lane >> 3))[lane & 7];
  }
  __syncwarp();
}
template <int ROWS, int COLS>
__device__ __forceinline__ void load_tile(const bf16* p, int64_t ld, int vec, uint4* stage, int r0, int rows, int c0, int cols, int lane) {
  constexpr int kUnits = COLS / 8, kAtOnce = 32 / kUnits;
  if (vec) {
#pragma unroll
    for (int i = 0; i < (ROWS + kAtOnce - 1) / kAtOnce; ++i) {
      const int r = i * kAtOnce + lane / kUnits, u = lane % kUnits, c = c0 + u * 8;
      if (r >= ROWS || r0 + r >= rows || c >= cols) continue;
      const bf16* q = p + (int64_t)(r0 + r) * ld + c;
      if (c + 8 <= cols) {
        *unit(stage, r, u) = *reinterpret_cast<const uint4*>(q);
      } else {
        unsigned short* d = reinterpret_cast<unsigned short*>(unit(stage, r, u));
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (c + k < cols) d[k] = reinterpret_cast<const unsigned short*>(q)[k];
      }
    }
  } else if (lane < COLS && c0 + lane < cols) {
    const int n = min(ROWS, rows - r0);
#pragma unroll 8
    for (int r = 0; r < n; ++r)
      reinterpret_cast<unsigned short*>(unit(stage, r, lane >> 3))[lane & 7] = reinterpret_cast<const unsigned short*>(p)[(int64_t)(r0 + r) * ld + c0 + lane];
  }
  __syncwarp();
}
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
      for (int u = 0; u < NC / 8; ++u) add8(u, __ldg(reinterpret_cast<const uint4*>(A.bias + c0) + u));
    } else {
#pragma unroll
      for (int i = 0; i < NC; ++i)
        if (c0 + i < A.rowsB) v[i] += bf_value(__ldg(reinterpret_cast<const unsigned short*>(A.bias) + c0 + i));
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

// ---------------------------------------------------------------------------------------------- the product

// PAIR: two CTAs on neighbouring SMs (a cluster) work on one tile of 256 rows: each loads half of A and half of B, the
// first one's MMA thread multiplies on both SMs at once, and each holds its 128 rows of D in its own TMEM.
// That halves what an SM has to fetch per product: 128 x 256 tiles by single CTAs are bound by the traffic out of L2
// (8192^3: 820 TFLOP/s).
// SPLIT: that many CTAs (a cluster) share a tile's k; each then completes 1/SPLIT of every 32 columns.
template <int BN, bool SWAP, bool PAIR, int SPLIT>
__global__ void __launch_bounds__(kGemmThreads, 1) gemm_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB,
                                                               const __grid_constant__ GemmArgs A) {
  extern __shared__ __align__(1024) unsigned char raw[];
  __shared__ uint64_t full[kMaxStages], empty[kMaxStages], done[2], freed[2];
  __shared__ unsigned tmem_base;
  constexpr int kHalf = PAIR ? BN / 2 : BN;                         // rows of B that this CTA loads
  constexpr int kRows = PAIR ? 2 * kBM : kBM;                       // rows of a tile
  constexpr unsigned kStageA = kBM * 128, kStage = kStageA + kHalf * 128;
  constexpr int kChunks = BN / 32;
  constexpr unsigned kCols = 2 * BN < 32 ? 32 : 2 * BN;
  unsigned char* sm = raw + ((1024 - (smem_addr(raw) & 1023)) & 1023);
  uint4* staging = reinterpret_cast<uint4*>(sm + (size_t)A.stages * kStage);                     // 2 KB per epilogue warp
  float* sums = reinterpret_cast<float*>(sm + (size_t)A.stages * kStage + kEpiWarps * 2048);     // the cluster's partial sums
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  static_assert(!PAIR || SPLIT == 1, "a pair does not split k");
  constexpr int per = PAIR ? 2 : SPLIT, kOwn = 32 / SPLIT;
  const int side = PAIR ? blockIdx.x & 1 : 0, rank = SPLIT > 1 ? blockIdx.x % SPLIT : 0;
  const int tiles = A.tilesA * A.tilesB, first = blockIdx.x / per, step = gridDim.x / per;
  const int kb0 = (int)((int64_t)A.kblocks * rank / SPLIT), kb1 = (int)((int64_t)A.kblocks * (rank + 1) / SPLIT);

  start_dependents();
  if (threadIdx.x == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mapA) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mapB) : "memory");
    for (int s = 0; s < A.stages; ++s) { bar_init(smem_addr(&full[s]), 1); bar_init(smem_addr(&empty[s]), 1); }
    for (int i = 0; i < 2; ++i) { bar_init(smem_addr(&done[i]), 1); bar_init(smem_addr(&freed[i]), PAIR ? 2 * kEpiWarps : kEpiWarps); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    if constexpr (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_base)), "r"(kCols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_base)), "r"(kCols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
  }
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  if (PAIR || SPLIT > 1) cluster_sync();
  wait_for_previous();
  const unsigned tmem = tmem_base;
  bool ok = true;

  // tile t: A tiles in bands of 16, B tiles across a band, so that what runs at once shares its operands in L2
  auto tile_at = [&](int t, int& ta, int& tb) {
    const int band = 16 * A.tilesB, b = t / band, in = t - b * band, h = min(16, A.tilesA - 16 * b);
    tb = in / h;
    ta = 16 * b + in - tb * h;
  };

  if (warp == 0) {
    const bool issuer = elect();     // the warp stays together; one lane issues
    {
      int s = 0, issued = 0;
      unsigned ph = 0;
      for (int t = first; t < tiles && ok; t += step) {
        int ta, tb;
        tile_at(t, ta, tb);
        for (int kb = kb0; kb < kb1; ++kb) {
          ok = warp_wait(smem_addr(&empty[s]), ph ^ 1);
          if (!ok) break;
          const unsigned dst = smem_addr(sm) + s * kStage;
          unsigned bar = smem_addr(&full[s]);
          if (issuer && side == 0) bar_expect(bar, PAIR ? 2 * kStage : kStage);
          if (PAIR) bar = in_cta(bar, 0);
          auto load = [&](unsigned to, const CUtensorMap* map, int c0, int c1) {
            if (!issuer) return;
            if constexpr (PAIR) tma_load_pair(to, map, c0, c1, bar);
            else tma_load(to, map, c0, c1, bar);
          };
          const int ra = ta * kRows + side * kBM, rb = tb * BN + side * kHalf;
          if (A.mnA) {
            for (int i = 0; i < kBM / 64; ++i) load(dst + i * kBK * 128, &mapA, ra + i * 64, kb * kBK);
          } else {
            load(dst, &mapA, kb * kBK, ra);
          }
          if (A.mnB) {
            for (int i = 0; i < kHalf / 64; ++i) load(dst + kStageA + i * kBK * 128, &mapB, rb + i * 64, kb * kBK);
          } else {
            load(dst + kStageA, &mapB, kb * kBK, rb);
          }
          __syncwarp();
          ++issued;
          if (++s == A.stages) { s = 0; ph ^= 1; }
        }
      }
      // the last copies land before the CTA ends, whoever waits for them (a pair's second CTA stays until the first has seen them)
      for (int i = 0; i < A.stages && i < issued && side == 0; ++i) {
        if (--s < 0) { s = A.stages - 1; ph ^= 1; }
        bar_wait(smem_addr(&full[s]), ph);
      }
    }
  } else if (warp == 1) {
    if (side == 0) {
      const bool issuer = elect();
      const unsigned idesc = 1u << 4 | 1u << 7 | 1u << 10 | (unsigned)A.mnA << 15 | (unsigned)A.mnB << 16 | (unsigned)(BN >> 3) << 17 | (unsigned)(kRows >> 4) << 24;
      const unsigned stepA = A.mnA ? 2048 >> 4 : 32 >> 4, stepB = A.mnB ? 2048 >> 4 : 32 >> 4;
      int s = 0;
      unsigned ph = 0, buf = 0, aph = 0;
      for (int t = first; t < tiles && ok; t += step) {
        ok = warp_wait(smem_addr(&freed[buf]), aph ^ 1);
        if (!ok) break;
        tmem_fence_after();
        for (int kb = kb0; kb < kb1; ++kb) {
          ok = warp_wait(smem_addr(&full[s]), ph);
          if (!ok) break;
          tmem_fence_after();
          const unsigned base = smem_addr(sm) + s * kStage;
          const uint64_t da = descriptor(base, A.mnA), db = descriptor(base + kStageA, A.mnB);
          if (issuer) {
#pragma unroll
            for (int k = 0; k < kBK / 16; ++k) {
              if constexpr (PAIR) mma_pair(tmem + buf * BN, da + k * stepA, db + k * stepB, idesc, kb > kb0 || k > 0);
              else mma(tmem + buf * BN, da + k * stepA, db + k * stepB, idesc, kb > kb0 || k > 0);
            }
            if constexpr (PAIR) mma_commit_pair(smem_addr(&empty[s]));
            else mma_commit(smem_addr(&empty[s]));
          }
          __syncwarp();
          if (++s == A.stages) { s = 0; ph ^= 1; }
        }
        if (issuer) {
          if constexpr (PAIR) mma_commit_pair(smem_addr(&done[buf]));
          else mma_commit(smem_addr(&done[buf]));
        }
        __syncwarp();
        if (buf) aph ^= 1;
        buf ^= 1;
      }
    }
  } else {
    const int e = warp - 2, quarter = warp & 3, group = e >> 2;     // TMEM lanes 32 quarter.. belong to warps of that number mod 4
    uint4* stage = staging + e * 128;
    unsigned buf = 0, aph = 0;
    for (int t = first; t < tiles && ok; t += step) {
      int ta, tb;
      tile_at(t, ta, tb);
      const int r0 = ta * kRows + side * kBM + quarter * 32;
      float bias = 0.f;                                             // fetched before the wait
      if (SWAP && A.bias && r0 + lane < A.rowsA) bias = bf_value(__ldg(reinterpret_cast<const unsigned short*>(A.bias) + r0 + lane));
      if (!SWAP && A.bias && tb * BN + group * 32 < A.rowsB) asm volatile("prefetch.global.L1 [%0];" ::"l"(A.bias + tb * BN + group * 32));
      ok = warp_wait(smem_addr(&done[buf]), aph);
      if (!ok) break;
      tmem_fence_after();
      if constexpr (SPLIT == 1) {
        for (int c = group; c < kChunks; c += kEpiWarps / 4) {
          const int c0 = tb * BN + c * 32;
          if (c0 >= A.rowsB) break;
          float v[32];
          tmem_load32(tmem + buf * BN + c * 32 + ((unsigned)(quarter * 32) << 16), v);
          if constexpr (SWAP) finish_swapped<32>(A, v, stage, r0, c0, bias, lane);
          else finish<32>(A, v, stage, r0, c0, lane);
        }
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (PAIR) bar_arrive_cluster(in_cta(smem_addr(&freed[buf]), 0));
          else bar_arrive(smem_addr(&freed[buf]));
        }
        if (buf) aph ^= 1;
        buf ^= 1;
      } else {
        // one tile per cluster, at most one chunk per warp: what others complete goes to them, the rest stays
        static_assert(SPLIT == 1 || kChunks <= kEpiWarps / 4, "a warp keeps its chunk in registers");
        const int c0 = tb * BN + group * 32;
        const bool mine = group < kChunks && c0 < A.rowsB;
        float v[32], own[kOwn];
        float* slots = sums + (size_t)group * SPLIT * kOwn * kBM + quarter * 32 + lane;       // [SPLIT sources][kOwn][128]
        if (mine) {
          tmem_load32(tmem + group * 32 + ((unsigned)(quarter * 32) << 16), v);
#pragma unroll
          for (int o = 0; o < SPLIT; ++o) {
            if (o == rank) {
#pragma unroll
              for (int i = 0; i < kOwn; ++i) own[i] = v[o * kOwn + i];
            } else if (c0 + o * kOwn < A.rowsB) {
              const unsigned to = in_cta(smem_addr(slots + rank * kOwn * kBM), o);
#pragma unroll
              for (int i = 0; i < kOwn; ++i) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + i * kBM * 4), "f"(v[o * kOwn + i]) : "memory");
            }
          }
        }
        __syncwarp();
        cluster_sync();
        if (mine && c0 + rank * kOwn < A.rowsB) {
#pragma unroll
          for (int q = 0; q < SPLIT; ++q)
            if (q != rank) {
#pragma unroll
              for (int i = 0; i < kOwn; ++i) own[i] += slots[(q * kOwn + i) * kBM];
            }
          if constexpr (SWAP) finish_swapped<kOwn>(A, own, stage, r0, c0 + rank * kOwn, bias, lane);
          else finish<kOwn>(A, own, stage, r0, c0 + rank * kOwn, lane);
        }
        break;
      }
    }
    // a CTA that gave up before the exchange still takes its part in the barrier
    if (SPLIT > 1 && !ok) cluster_sync();
  }
  __syncwarp();
  if (SPLIT > 1 && warp < 2) cluster_sync();
  if (!ok && lane == 0) atomicAdd(&g_gave_up, 1u);
  tmem_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync();        // neither leaves while the other's MMA, copies or arrivals may reach it
  tmem_fence_after();
  if (warp == 1) {
    if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols));
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols));
  }
}

// ---------------------------------------------------------------------------------------------- elementwise parts

// Row-wise jobs, up to three to a launch (blockIdx.z): dz = dy act'(z) as bf16 rows of `ldo` elements with, per chunk of
// rows, the column sums of the unrounded dz; and the laying out of an operand whose rows TMA cannot take. Bound: HBM (dz
// reads two matrices and writes one: 8192 x 4096, 201 MB).
constexpr int kChunkRows = 64;
struct Job {
  const bf16 *in, *z;       // dy (or the operand), and z if the slope is taken
  bf16* out;                // or NULL
  float* sums;              // or NULL
  int64_t ldi, ldz, ldo, rows;
  int cols, vec;            // vec: 16-byte accesses everywhere
};
struct Jobs {
  Job job[3];
};

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
__global__ void __launch_bounds__(256) columns_kernel(const float* __restrict__ sums, int64_t chunks, int cols, bf16* __restrict__ out) {
  __shared__ float sh[8][33];
  start_dependents();
  wait_for_previous();
  const int lane = threadIdx.x & 31, r = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  float s = 0.f;
  if (c < cols) {
#pragma unroll 8
    for (int64_t i = r; i < chunks; i += 8) s += __ldg(sums + i * cols + c);
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

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
  static EncodeTiled f = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult r;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) != cudaSuccess || r != cudaDriverEntryPointSuccess) {
      (void)cudaGetLastError();
      p = nullptr;
    }
    return reinterpret_cast<EncodeTiled>(p);
  }();
  return f;
}

bool aligned(const void* p, unsigned a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
int64_t pad8(int64_t n) { return (n + 7) & ~(int64_t)7; }
int64_t pad256(int64_t n) { return (n + 255) & ~(int64_t)255; }

// A matrix; TMA takes it if it is 16-byte aligned, its rows a multiple of 16 bytes apart and none repeated
struct Matrix {
  const bf16* p;
  int64_t rows, cols, ld;
};
bool tma_ready(const Matrix& m) { return aligned(m.p, 16) && (m.rows <= 1 || (m.ld % 8 == 0 && m.ld >= m.cols)); }
int64_t laid_out_bytes(const Matrix& m) { return tma_ready(m) ? 0 : pad256(m.rows * pad8(m.cols) * 2); }

// rows of m are D's rows (or columns) if !mn, its columns if mn
bool make_map(CUtensorMap* map, const Matrix& m, int mn, int box_rows) {
  const EncodeTiled f = encode_tiled();
  if (!f) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)m.cols, (cuuint64_t)m.rows};
  const cuuint64_t strides[1] = {(cuuint64_t)(m.rows > 1 ? m.ld : pad8(m.cols)) * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)(mn ? kBK : box_rows)}, one[2] = {1, 1};
  return f(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<bf16*>(m.p), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
           CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename... P, typename... V>
int start(cudaLaunchConfig_t cfg, int cluster, void (*kernel)(P...), V... args) {
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return dmxh::cuda_ok(cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...)) ? DMX_OK : DMX_ERR_CUDA;
}
template <typename... P, typename... V>
int start(dim3 grid, cudaStream_t st, void (*kernel)(P...), V... args) {      // 256 threads
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(256);
  cfg.stream = st;
  return start(cfg, 1, kernel, args...);
}

struct Choice {
  int bn, split;
  bool pair;
};

// Tile width, split and pairing, by the time they take: what a stage of 64 k took measured on 8192^3 (ns; the narrow tiles are bound
// by what the SMs fetch from L2), the last tile's epilogue, a split's cluster barrier and exchange.
Choice choose(int64_t rowsA, int64_t rowsB, int kblocks, bool swap) {
  Choice best = {0, 1, false};
  float least = 0.f;
  const struct { int bn; bool pair; float stage; } forms[6] = {{256, true, 405.f}, {256, false, 435.f}, {128, true, 290.f},
                                                                {128, false, 290.f}, {64, false, 245.f}, {32, false, 200.f}};
  for (const auto& f : forms) {
    if (swap ? f.pair || f.bn != (rowsB <= 32 ? 32 : 64) : f.bn == 32) continue;
    const int rows = f.pair ? 2 * kBM : kBM, at_once = f.pair ? 74 : 148;
    const int64_t tiles = ((rowsA + rows - 1) / rows) * ((rowsB + f.bn - 1) / f.bn);
    const int most = swap ? 4 : f.pair || f.bn == 256 ? 1 : 2;
    for (int split = 1; split <= most; split *= 2) {
      if (split > 1 && (tiles * split > 148 || kblocks / split < 2)) break;
      const int64_t waves = (tiles * split + at_once - 1) / at_once;
      const float t = waves * ((kblocks + split - 1) / split) * f.stage + 8.f * f.bn + (split > 1 ? 1300.f : 0.f);
      if (best.bn == 0 || t < least) { best.bn = f.bn; best.split = split; best.pair = f.pair; least = t; }
    }
  }
  return best;
}

// 64 rows or fewer: b's rows take the 128 lanes (b keeps whichever way it lies; a, the narrow side, has to be K-major)
struct Form {
  bool exchanged;
  Choice choice;
};
Form form_of(int64_t rowsA, int64_t rowsB, int kblocks, int mnA) {
  const bool exchanged = rowsA <= 64 && !mnA;
  return {exchanged, exchanged ? choose(rowsB, rowsA, kblocks, true) : choose(rowsA, rowsB, kblocks, false)};
}

template <int BN, bool SWAP, bool PAIR, int SPLIT>
int launch_gemm(const Matrix& a, const Matrix& b, GemmArgs& A, cudaStream_t st) {
  constexpr int kHalf = PAIR ? BN / 2 : BN, kRows = PAIR ? 2 * kBM : kBM;
  CUtensorMap ma, mb;
  if (!make_map(&ma, a, A.mnA, kBM) || !make_map(&mb, b, A.mnB, kHalf)) return DMX_ERR_CUDA;
  A.tilesA = (A.rowsA + kRows - 1) / kRows;
  A.tilesB = (A.rowsB + BN - 1) / BN;
  const int stage = (kBM + kHalf) * 128, chunks = BN / 32;
  const int extra = 1024 + kEpiWarps * 2048 + (SPLIT > 1 ? chunks * 32 * kBM * 4 : 0);
  A.stages = (kSmemMost - extra) / stage;
  if (A.stages > kMaxStages) A.stages = kMaxStages;
  const int smem = A.stages * stage + extra;
  const auto kernel = gemm_kernel<BN, SWAP, PAIR, SPLIT>;
  static std::atomic<uint64_t> set{0};         // devices on which this kernel may use that much shared memory
  int device = 0;
  if (!dmxh::cuda_ok(cudaGetDevice(&device))) return DMX_ERR_CUDA;
  const uint64_t bit = (uint64_t)1 << (device & 63);
  if (!(set.load(std::memory_order_relaxed) & bit) || device > 63) {
    if (!dmxh::cuda_ok(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMost))) return DMX_ERR_CUDA;
    set.fetch_or(bit, std::memory_order_relaxed);
  }
  const int64_t tiles = (int64_t)A.tilesA * A.tilesB;
  constexpr int per = PAIR ? 2 : SPLIT;
  if (tiles * per > 0x7fffffff) return DMX_ERR_ARG;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(SPLIT > 1 || tiles * per < 148 ? tiles * per : 148));
  cfg.blockDim = dim3(kGemmThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  return start(cfg, per, kernel, ma, mb, A);
}

// D = A B^T with the epilogue in E (bias, residual, outputs, act). mn: the operand's rows run along D's extent.
int product(const Matrix& a, int mnA, const Matrix& b, int mnB, int64_t k, const GemmArgs& E, cudaStream_t st) {
  GemmArgs A = E;
  const int64_t rowsA = mnA ? a.cols : a.rows, rowsB = mnB ? b.cols : b.rows;
  A.kblocks = (int)((k + kBK - 1) / kBK);
  A.vecy = aligned(A.y, 16) && (rowsA <= 1 || A.ldy % 8 == 0);
  A.vecz = A.z && aligned(A.z, 16) && (rowsA <= 1 || A.ldz % 8 == 0);
  A.vecr = A.residual && aligned(A.residual, 16) && (rowsA <= 1 || A.ldr % 8 == 0);
  const Form f = form_of(rowsA, rowsB, A.kblocks, mnA);
  const Choice& c = f.choice;
  if (f.exchanged) {
    A.rowsA = (int)rowsB; A.rowsB = (int)rowsA;
    A.mnA = mnB; A.mnB = mnA;
    if (c.bn == 32) {
      if (c.split == 4) return launch_gemm<32, true, false, 4>(b, a, A, st);
      return c.split == 2 ? launch_gemm<32, true, false, 2>(b, a, A, st) : launch_gemm<32, true, false, 1>(b, a, A, st);
    }
    if (c.split == 4) return launch_gemm<64, true, false, 4>(b, a, A, st);
    return c.split == 2 ? launch_gemm<64, true, false, 2>(b, a, A, st) : launch_gemm<64, true, false, 1>(b, a, A, st);
  }
  A.rowsA = (int)rowsA; A.rowsB = (int)rowsB;
  A.mnA = mnA; A.mnB = mnB;
  if (c.pair) return c.bn == 256 ? launch_gemm<256, false, true, 1>(a, b, A, st) : launch_gemm<128, false, true, 1>(a, b, A, st);
  if (c.bn == 256) return launch_gemm<256, false, false, 1>(a, b, A, st);
  if (c.bn == 128) return c.split == 2 ? launch_gemm<128, false, false, 2>(a, b, A, st) : launch_gemm<128, false, false, 1>(a, b, A, st);
  return c.split == 2 ? launch_gemm<64, false, false, 2>(a, b, A, st) : launch_gemm<64, false, false, 1>(a, b, A, st);
}

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
  return rc != DMX_OK ? rc : product(a, 0, b, 0, K, E, st);
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
  GemmArgs E = {};
  E.act = DMX_ACT_NONE;
  if (products && dx && rc == DMX_OK) {        // dx[m, k] = sum_n dz[m, n] w[n, k]
    E.y = static_cast<bf16*>(dx); E.ldy = M > 1 ? lddx : K;
    rc = product(g, 0, b, 1, N, E, st);
  }
  if (products && dw && rc == DMX_OK) {        // dw[n, k] = sum_m dz[m, n] x[m, k]
    E.y = static_cast<bf16*>(dw); E.ldy = N > 1 ? lddw : K;
    rc = product(g, 1, a, 1, M, E, st);
  }
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
  unsigned n = 0;
  if (!dmxh::cuda_ok(cudaMemcpyFromSymbol(&n, g_gave_up, sizeof n))) return DMX_ERR_CUDA;
  unsigned& before = reported[device & 255];
  *errors = (int)(n >= before ? n - before : n);       // (below it: the device was reset)
  before = n;
  return DMX_OK;
}

}  // extern "C"
