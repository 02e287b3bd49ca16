// dmx_gemm.cuh — D[i, j] = sum_k A[i, k] B[j, k] on the 5th-generation tensor cores (bf16 operands, fp32 accumulation) with an
// epilogue of the including file's choice: the kernel behind the linear layer and the cross entropy of one.
//
// A producer warp moves tiles of A (128 rows) and B (32 to 256) of 64 k with TMA into a ring of shared memory
// stages, one thread issues tcgen05.mma on them into accumulators in TMEM, and sixteen warps take finished accumulators out
// (tcgen05.ld), apply the epilogue and store, while the next tile accumulates in the other half of TMEM. An
// operand whose rows run along k is K-major, one whose rows run across it MN-major; both are
// multiplied as they lie: only the descriptors differ, nothing is transposed in memory.
// Few tiles: k is split over the CTAs of a cluster, whose partial sums meet in distributed shared memory and
// are added in a fixed order.
// Every wait is bounded; a warp that gives up counts itself in a device word (dmx_linear_status), and its CTA lets its
// copies land, frees its TMEM and returns.
#pragma once
#include "dmx.h"

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <atomic>

#include "dmx_f32x2.cuh"
#include "dmx_host.h"

namespace dmx_gemm {

using namespace dmx_f32x2;
typedef __nv_bfloat16 bf16;

constexpr int kBM = 128, kBK = 64;            // tile rows of A; k per stage (128 bytes: one swizzle row)
constexpr int kEpiWarps = 16;                 // four per scheduler: with two a GELU epilogue took longer than 1024 k
constexpr int kGemmThreads = 64 + 32 * kEpiWarps;
constexpr int kMaxStages = 8;
constexpr int kSmemMost = 226 * 1024;
constexpr unsigned kPolls = 1u << 18;         // about a second

static __device__ unsigned g_gave_up;         // warps whose waits ran out, in kernels of the including file

struct GemmShape {
  int rowsA, rowsB, kblocks;                  // rows of D, columns of D, ceil(k / 64)
  int tilesA, tilesB, stages;
  int mnA, mnB;                               // operand is MN-major
  int ranges;                                 // of k, if E takes a range's part of D at a time
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
// Inputs are read behind the wait and with ordinary loads: a read-only one promises that its data do not change while the kernel is resident, which is
// while the one before still writes them.
__device__ __forceinline__ void start_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ __forceinline__ float bf_value(unsigned short u) { return __uint_as_float((unsigned)u << 16); }
__device__ __forceinline__ unsigned pack2(float a, float b) {
  __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<unsigned*>(&t);
}
// ---------------------------------------------------------------------------------------------- staging

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
// ---------------------------------------------------------------------------------------------- the product

// PAIR: two CTAs on neighbouring SMs (a cluster) work on one tile of 256 rows: each loads half of A and half of B, the
// first one's MMA thread multiplies on both SMs at once, and each holds its 128 rows of D in its own TMEM.
// That halves what an SM has to fetch per product: 128 x 256 tiles by single CTAs are bound by the traffic out of L2
// (8192^3: 820 TFLOP/s).
// SPLIT: that many CTAs (a cluster) share a tile's k; each then completes 1/SPLIT of every 32 columns.
// E: what becomes of D. A warp calls fetch for a tile's rows a tile ahead, begin for a tile before it waits for it, chunk for every 32 columns (or its share of them) of its 32 rows,
// a row per lane, and end (false: a wait in it ran out) before it hands the accumulators back; setup initializes what barriers end has.
// With kRanged k is cut into A.ranges parts, each a D of its own (E's member `range` says which). kStaging: bytes of a warp's staging buffer (2048, or 0 if it uses none), kOwnShared: shared memory that E declares itself.
template <int BN, bool PAIR, int SPLIT, class E>
__global__ void __launch_bounds__(kGemmThreads, 1) gemm_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB,
                                                               const __grid_constant__ typename E::Args A) {
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
  float* sums = reinterpret_cast<float*>(sm + (size_t)A.stages * kStage + kEpiWarps * E::kStaging);     // the cluster's partial sums
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  static_assert(!PAIR || SPLIT == 1, "a pair does not split k");
  constexpr int per = PAIR ? 2 : SPLIT, kOwn = 32 / SPLIT;
  const int side = PAIR ? blockIdx.x & 1 : 0, rank = SPLIT > 1 ? blockIdx.x % SPLIT : 0;
  const int every = A.tilesA * A.tilesB, tiles = E::kRanged ? every * A.ranges : every, first = blockIdx.x / per, step = gridDim.x / per;
  int kb0 = (int)((int64_t)A.kblocks * rank / SPLIT), kb1 = (int)((int64_t)A.kblocks * (rank + 1) / SPLIT);

  start_dependents();
  if (threadIdx.x == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mapA) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mapB) : "memory");
    for (int s = 0; s < A.stages; ++s) { bar_init(smem_addr(&full[s]), 1); bar_init(smem_addr(&empty[s]), 1); }
    for (int i = 0; i < 2; ++i) { bar_init(smem_addr(&done[i]), 1); bar_init(smem_addr(&freed[i]), PAIR ? 2 * kEpiWarps : kEpiWarps); }
    E::setup();
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

  // Tiles in turn, from the CTA's first by steps: A tiles in bands of 16, B tiles across a band, so that what runs at once shares its
  // operands in L2. (A band and a place in it are kept: divisions by the problem's extents cost an epilogue over a short k a tenth of its time.)
  const int band = 16 * A.tilesB;
  struct Walk {
    int t, b, in;
  };
  auto from = [&](int t) { return Walk{t, E::kRanged ? 0 : t / band, E::kRanged ? 0 : t % band}; };
  auto next = [&](Walk& w) {
    w.t += step;
    w.in += step;
    while (w.in >= band) { w.in -= band; ++w.b; }
  };
  auto place = [&](const Walk& w, int& ta, int& tb) {
    int b = w.b, in = w.in;
    if constexpr (E::kRanged) {
      const int range = w.t / every, t = w.t - range * every;
      kb0 = (int)((int64_t)A.kblocks * range / A.ranges);
      kb1 = (int)((int64_t)A.kblocks * (range + 1) / A.ranges);
      b = t / band;
      in = t - b * band;
    }
    const int h = min(16, A.tilesA - 16 * b);
    tb = h == 16 ? in >> 4 : in / h;
    ta = 16 * b + in - tb * h;
  };

  if (warp == 0) {
    const bool issuer = elect();     // the warp stays together; one lane issues
    {
      int s = 0, issued = 0;
      unsigned ph = 0;
      for (Walk w = from(first); w.t < tiles && ok; next(w)) {
        int ta, tb;
        place(w, ta, tb);
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
      for (Walk w = from(first); w.t < tiles && ok; next(w)) {
        if constexpr (E::kRanged) {
          int ta, tb;
          place(w, ta, tb);                    // (for its range of k)
        }
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
    E epilogue;
    int ta = 0, tb = 0;
    Walk w = from(first);
    if (w.t < tiles) {
      place(w, ta, tb);
      epilogue.fetch(A, ta * kRows + side * kBM + quarter * 32, lane);
    }
    while (w.t < tiles && ok) {
      const int r0 = ta * kRows + side * kBM + quarter * 32;
      if constexpr (E::kRanged) epilogue.range = w.t / every;
      epilogue.begin(A, r0, tb * BN + group * 32, lane);            // fetches before the wait
      const int tb_now = tb;
      next(w);
      if (w.t < tiles) {                                            // what the next tile's rows need is on its way meanwhile
        place(w, ta, tb);
        epilogue.fetch(A, ta * kRows + side * kBM + quarter * 32, lane);
      }
      ok = warp_wait(smem_addr(&done[buf]), aph);
      if (!ok) break;
      tmem_fence_after();
      if constexpr (SPLIT == 1) {
        for (int c = group; c < kChunks; c += kEpiWarps / 4) {
          const int c0 = tb_now * BN + c * 32;
          if (c0 >= A.rowsB) break;
          float v[32];
          tmem_load32(tmem + buf * BN + c * 32 + ((unsigned)(quarter * 32) << 16), v);
          epilogue.template chunk<32>(A, v, stage, r0, c0, lane);
        }
        ok = epilogue.end(A, r0, tb_now, group, lane, buf, aph);
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
        const int c0 = tb_now * BN + group * 32;
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
          epilogue.template chunk<kOwn>(A, own, stage, r0, c0 + rank * kOwn, lane);
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

// ---------------------------------------------------------------------------------------------- host

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiled encode_tiled() {
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

inline bool aligned(const void* p, unsigned a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline int64_t pad8(int64_t n) { return (n + 7) & ~(int64_t)7; }
inline int64_t pad256(int64_t n) { return (n + 255) & ~(int64_t)255; }

// A matrix; TMA takes it if it is 16-byte aligned, its rows a multiple of 16 bytes apart and none repeated
struct Matrix {
  const bf16* p;
  int64_t rows, cols, ld;
};
inline bool tma_ready(const Matrix& m) { return aligned(m.p, 16) && (m.rows <= 1 || (m.ld % 8 == 0 && m.ld >= m.cols)); }
inline int64_t laid_out_bytes(const Matrix& m) { return tma_ready(m) ? 0 : pad256(m.rows * pad8(m.cols) * 2); }

// rows of m are D's rows (or columns) if !mn, its columns if mn
inline bool make_map(CUtensorMap* map, const Matrix& m, int mn, int box_rows) {
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
int start(dim3 grid, int threads, cudaStream_t st, void (*kernel)(P...), V... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.stream = st;
  return start(cfg, 1, kernel, args...);
}
template <typename... P, typename... V>
int start(dim3 grid, cudaStream_t st, void (*kernel)(P...), V... args) { return start(grid, 256, st, kernel, args...); }

struct Choice {
  int bn, split;
  bool pair;
  float ns;
};

// Tile width, split and pairing, by the time they take: what a stage of 64 k took measured on 8192^3 (ns; the narrow tiles are bound
// by what the SMs fetch from L2), the last tile's epilogue, a split's cluster barrier and exchange.
inline Choice choose(int64_t rowsA, int64_t rowsB, int kblocks, bool swap) {
  Choice best = {0, 1, false, 0.f};
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
      if (best.bn == 0 || t < least) { best.bn = f.bn; best.split = split; best.pair = f.pair; best.ns = least = t; }
    }
  }
  return best;
}

// The same for products whose tiles may have little k: a tile takes the longer of its stages and its epilogue and a quarter of the other. What
// an epilogue takes per tile (ns) was measured on the cross entropy's sums at k = 64; slopes and plain stores take `weight` times it. A single CTA's tile of
// 256 columns then beats a pair's: 8192 x 30522 x 256 forward without bias 114 us against 141, at k = 1024 338 against 317.
// A pair's of 128 columns is for one wave over a long k: dx of 2048 x 30522 x 1024 takes 3 us less than single CTAs' of 128 columns.
inline Choice choose_by_tiles(int64_t rowsA, int64_t rowsB, int kblocks, bool swap, bool splits, float weight) {
  Choice best = {0, 1, false, 0.f};
  const struct { int bn; bool pair; float stage, epilogue; } forms[6] = {{256, true, 405.f, 2450.f}, {256, false, 435.f, 2000.f}, {128, true, 282.f, 1850.f},
                                                                          {128, false, 290.f, 1400.f}, {64, false, 245.f, 1050.f}, {32, false, 200.f, 800.f}};
  for (const auto& f : forms) {
    if (swap ? f.pair || f.bn != (rowsB <= 32 ? 32 : 64) : f.bn == 32) continue;
    const int rows = f.pair ? 2 * kBM : kBM, at_once = f.pair ? 74 : 148;
    const int64_t tiles = ((rowsA + rows - 1) / rows) * ((rowsB + f.bn - 1) / f.bn);
    const int most = !splits ? 1 : swap ? 4 : f.pair || f.bn == 256 ? 1 : 2;
    for (int split = 1; split <= most; split *= 2) {
      if (split > 1 && (tiles * split > 148 || kblocks / split < 2)) break;
      const int64_t waves = (tiles * split + at_once - 1) / at_once;
      const float k = (float)((kblocks + split - 1) / split) * f.stage, e = f.epilogue * weight;
      const float t = waves * (k > e ? k + 0.25f * e : e + 0.25f * k) + (split > 1 ? 1300.f : 0.f);
      if (best.bn == 0 || t < best.ns) best = {f.bn, split, f.pair, t};
    }
  }
  return best;
}

template <int BN, bool PAIR, int SPLIT, class E>
int launch_gemm(const Matrix& a, const Matrix& b, typename E::Args& A, cudaStream_t st) {
  constexpr int kHalf = PAIR ? BN / 2 : BN, kRows = PAIR ? 2 * kBM : kBM;
  CUtensorMap ma, mb;
  if (!make_map(&ma, a, A.mnA, kBM) || !make_map(&mb, b, A.mnB, kHalf)) return DMX_ERR_CUDA;
  A.tilesA = (A.rowsA + kRows - 1) / kRows;
  A.tilesB = (A.rowsB + BN - 1) / BN;
  const int stage = (kBM + kHalf) * 128, chunks = BN / 32;
  const int extra = 1024 + E::kOwnShared + kEpiWarps * E::kStaging + (SPLIT > 1 ? chunks * 32 * kBM * 4 : 0);
  A.stages = (kSmemMost - extra) / stage;
  if (A.stages > kMaxStages) A.stages = kMaxStages;
  const int smem = A.stages * stage + extra - E::kOwnShared;
  const auto kernel = gemm_kernel<BN, PAIR, SPLIT, E>;
  static std::atomic<uint64_t> set{0};         // devices on which this kernel may use that much shared memory
  int device = 0;
  if (!dmxh::cuda_ok(cudaGetDevice(&device))) return DMX_ERR_CUDA;
  const uint64_t bit = (uint64_t)1 << (device & 63);
  if (!(set.load(std::memory_order_relaxed) & bit) || device > 63) {
    if (!dmxh::cuda_ok(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMost - E::kOwnShared))) return DMX_ERR_CUDA;
    set.fetch_or(bit, std::memory_order_relaxed);
  }
  const int64_t tiles = (int64_t)A.tilesA * A.tilesB * (E::kRanged ? A.ranges : 1);
  constexpr int per = PAIR ? 2 : SPLIT;
  if (tiles * per > 0x7fffffff) return DMX_ERR_ARG;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(SPLIT > 1 || tiles * per < 148 ? tiles * per : 148));
  cfg.blockDim = dim3(kGemmThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  return start(cfg, per, kernel, ma, mb, A);
}

// ---------------------------------------------------------------------------------------------- dmx_linear.cu's, for others

// Row-wise jobs, up to three to a launch: dz = dy act'(z), or the laying out of an operand whose rows TMA cannot take.
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

int run_jobs(const Jobs& jobs, int n, int act, cudaStream_t st);
// m's copy at *ws (which moves on), if it needs one
void lay_out(Matrix& m, unsigned char*& ws, Jobs& jobs, int& n);
// y = A B^T, times *unit (device memory) if there is one, rounded to bf16. mn: the operand's rows run along D's extent.
int plain_product(const Matrix& a, int mnA, const Matrix& b, int mnB, int64_t k, const float* unit, bf16* y, int64_t ldy, cudaStream_t st);

// what it takes with a unit, by choose_by_tiles
float plain_product_ns(int64_t rowsA, int64_t rowsB, int64_t k, int mnA);
// the cross entropy's count of warps that gave up
bool loss_gave_up(unsigned* n);

}  // namespace dmx_gemm
