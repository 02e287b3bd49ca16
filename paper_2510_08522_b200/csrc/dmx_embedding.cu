// dmx_embedding.cu — rows of a table by token, scaled, and the table's gradient by sorted tokens.
//
// forward    y[n] = scale T[ids[n]]
// backward   dT[v] = scale (sum over n with ids[n] = v of dy[n]), added to what dT holds or not
//
// Both are bound by HBM. Backward first sorts the tokens by row (stably: by row, then by place): one cluster of eight CTAs sorts,
// eight bits a pass, counting digits per warp, joining the counts through distributed shared memory; the other CTAs of that
// launch write the table's zeros meanwhile, which takes longer than the sort of an ordinary batch. Then every warp sums a chunk of the sorted
// tokens over its columns, row after row in registers: each gradient row is read once, each row of the table written once. A row whose
// tokens reach over chunks leaves fp32 sums, one per chunk, which a third launch joins. Work is cut by tokens, not by rows: how
// often a token comes does not matter. Nothing is added atomically; the order of all sums is fixed by the shape and the ids.
#include "dmx_rows.cuh"

namespace {

using namespace dmx_rows;

constexpr int kSortCtas = 8, kSortThreads = 1024, kSortWarps = kSortThreads / 32, kDigits = 256;

// ---------------------------------------------------------------------------------------------- forward

struct GatherArgs {
  const void *ids, *table;
  void* y;
  int64_t N, V, ldt, ldy;
  int D, wide_ids;
  float scale;
};

__device__ __forceinline__ int64_t id_at(const void* ids, int wide, int64_t n) {
  return wide ? __ldg(static_cast<const long long*>(ids) + n) : (int64_t)__ldg(static_cast<const int*>(ids) + n);
}

// a warp takes 32 accesses of a row, four rows at a time
template <typename T, int W>
__global__ void __launch_bounds__(256) gather_kernel(const __grid_constant__ GatherArgs A) {
  typedef typename Vec<T, W>::type Raw;
  constexpr int kRows = 4;
  start_dependents();
  wait_for_previous();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = (blockIdx.y * 32 + lane) * W;
  const int64_t n0 = ((int64_t)blockIdx.x * 8 + warp) * kRows;
  if (c >= A.D) return;
  Raw r[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    r[k] = Raw{};
    if (n0 + k >= A.N) continue;
    const int64_t id = id_at(A.ids, A.wide_ids, n0 + k);
    if (id >= 0 && id < A.V) r[k] = *reinterpret_cast<const Raw*>(static_cast<const T*>(A.table) + id * A.ldt + c);
  }
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    if (n0 + k >= A.N) continue;
    if (A.scale != 1.f) {
      float x[W];
      widen<T>(r[k], x);
#pragma unroll
      for (int i = 0; i < W; ++i) x[i] *= A.scale;
      r[k] = narrow<T, W>(x);
    }
    *reinterpret_cast<Raw*>(static_cast<T*>(A.y) + (n0 + k) * A.ldy + c) = r[k];
  }
}

// ---------------------------------------------------------------------------------------------- the sort

struct SortArgs {
  const void* ids;
  int wide_ids, passes;
  int64_t N, V;
  unsigned *key[2], *place[2];     // passes go from one to the other; the last one ends in 0
  void* zero;                      // rows to clear, or NULL
  int64_t zero_ld;                 // in bytes
  int64_t zero_bytes;              // of a row
};

__device__ __forceinline__ void cluster_sync() { asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory"); }

__device__ void clear_rows(const SortArgs& A, int64_t cta, int64_t ctas) {
  unsigned char* p = static_cast<unsigned char*>(A.zero);
  if (A.zero_ld == A.zero_bytes || A.V == 1) {             // one piece
    const int64_t bytes = A.V * A.zero_bytes;
    int64_t head = (-(int64_t)reinterpret_cast<uintptr_t>(p)) & 15;
    if (head > bytes) head = bytes;
    const int64_t units = (bytes - head) / 16, tail = head + units * 16;
    for (int64_t i = cta * kSortThreads + threadIdx.x; i < units; i += ctas * kSortThreads) reinterpret_cast<uint4*>(p + head)[i] = make_uint4(0, 0, 0, 0);
    if (cta == 0) {                                        // (elements are 2 or 4 bytes)
      for (int64_t i = threadIdx.x * 2; i < head; i += 2 * kSortThreads) *reinterpret_cast<unsigned short*>(p + i) = 0;
      for (int64_t i = tail + threadIdx.x * 2; i < bytes; i += 2 * kSortThreads) *reinterpret_cast<unsigned short*>(p + i) = 0;
    }
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int64_t v = cta * kSortWarps + warp; v < A.V; v += ctas * kSortWarps)
    for (int64_t i = lane * 2; i < A.zero_bytes; i += 64) *reinterpret_cast<unsigned short*>(p + v * A.zero_ld + i) = 0;
}

__global__ void __cluster_dims__(kSortCtas, 1, 1) __launch_bounds__(kSortThreads) sort_kernel(const __grid_constant__ SortArgs A) {
  extern __shared__ unsigned counts[];                    // [warps][digits]: a warp's digits, then where its next one goes
  __shared__ unsigned totals[kSortCtas][kDigits];         // every CTA's digits
  __shared__ unsigned scan[8];
  start_dependents();
  wait_for_previous();
  if (blockIdx.x >= kSortCtas) {
    clear_rows(A, blockIdx.x - kSortCtas, gridDim.x - kSortCtas);
    return;
  }
  cluster_sync();                                         // all of it is there
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = blockIdx.x;
  const unsigned below = (1u << lane) - 1;
  // a warp's share: whole rounds of 32
  const int64_t rounds = (A.N + 32 * kSortWarps * kSortCtas - 1) / (32 * kSortWarps * kSortCtas);
  const int64_t first = ((int64_t)rank * kSortWarps + warp) * rounds * 32;
  unsigned* mine = counts + warp * kDigits;
  for (int pass = 0; pass < A.passes; ++pass) {
    const int from = (A.passes - pass) & 1, shift = 8 * pass;
    auto key_at = [&](int64_t n) -> unsigned {
      if (pass > 0) return __ldcg(A.key[from] + n);
      const int64_t id = id_at(A.ids, A.wide_ids, n);
      return id >= 0 && id < A.V ? (unsigned)id : (unsigned)A.V;     // what is in no row comes last
    };
    for (int i = lane; i < kDigits; i += 32) mine[i] = 0;
    __syncwarp();
    for (int64_t r = 0; r < rounds; ++r) {
      const int64_t n = first + r * 32 + lane;
      const bool live = n < A.N;
      if (!__any_sync(0xffffffffu, live)) break;
      const unsigned d = live ? key_at(n) >> shift & 255 : 256;
      const unsigned same = __match_any_sync(0xffffffffu, d);
      if (live && (same & below) == 0) mine[d] += __popc(same);
      __syncwarp();
    }
    __syncthreads();
    if (threadIdx.x < kDigits) {                          // prefix over the warps; the CTA's total goes to every CTA
      unsigned sum = 0;
      for (int w = 0; w < kSortWarps; ++w) {
        const unsigned c = counts[w * kDigits + threadIdx.x];
        counts[w * kDigits + threadIdx.x] = sum;
        sum += c;
      }
      for (int to = 0; to < kSortCtas; ++to) {
        unsigned at;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((unsigned)__cvta_generic_to_shared(&totals[rank][threadIdx.x])), "r"(to));
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(sum) : "memory");
      }
    }
    cluster_sync();
    if (threadIdx.x < kDigits) {                          // where this CTA's first key of a digit goes
      unsigned all = 0, before = 0;
      for (int r = 0; r < kSortCtas; ++r) {
        const unsigned c = totals[r][threadIdx.x];
        before += r < rank ? c : 0;
        all += c;
      }
      unsigned up = all;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned t = __shfl_up_sync(0xffffffffu, up, o);
        if (lane >= o) up += t;
      }
      if (lane == 31) scan[warp] = up;
      asm volatile("bar.sync 1, 256;" ::: "memory");
      unsigned start = up - all + before;
      for (int w = 0; w < warp; ++w) start += scan[w];
      for (int w = 0; w < kSortWarps; ++w) counts[w * kDigits + threadIdx.x] += start;
    }
    __syncthreads();
    for (int64_t r = 0; r < rounds; ++r) {
      const int64_t n = first + r * 32 + lane;
      const bool live = n < A.N;
      if (!__any_sync(0xffffffffu, live)) break;
      const unsigned k = live ? key_at(n) : 0, d = live ? k >> shift & 255 : 256;
      const unsigned same = __match_any_sync(0xffffffffu, d);
      unsigned at = 0;
      if (live) at = mine[d] + __popc(same & below);
      __syncwarp();
      if (live && (same & below) == 0) mine[d] += __popc(same);
      __syncwarp();
      if (live) {
        const unsigned p = pass > 0 ? __ldcg(A.place[from] + n) : (unsigned)n;
        A.key[from ^ 1][at] = k;
        A.place[from ^ 1][at] = p;
      }
    }
    __threadfence();
    cluster_sync();
  }
}

// ---------------------------------------------------------------------------------------------- the sums

struct SumArgs {
  const unsigned *key, *place;
  const void* dy;
  void* out;
  float* part;                     // [chunks][2][D]: what a chunk's first and last row got, where they go on
  int64_t N, V, lddy, ldout;
  int D, chunk, accumulate;        // chunk: tokens, a multiple of 32
  float scale;
};

template <typename O, int W>
__device__ __forceinline__ void finish_row(const SumArgs& A, unsigned v, int c, const float* acc) {
  O* q = static_cast<O*>(A.out) + (int64_t)v * A.ldout + c;
  float x[W];
#pragma unroll
  for (int i = 0; i < W; ++i) x[i] = acc[i] * A.scale;
  constexpr int kOut = W == 1 ? 1 : kWide<O>;
  static_assert(W % kOut == 0, "whole accesses");
#pragma unroll
  for (int k = 0; k < W; k += kOut) {
    typedef typename Vec<O, kOut>::type Raw;
    if (A.accumulate) {
      float old[kOut];
      widen<O>(*reinterpret_cast<const Raw*>(q + k), old);
#pragma unroll
      for (int i = 0; i < kOut; ++i) x[k + i] += old[i];
    }
    *reinterpret_cast<Raw*>(q + k) = narrow<O, kOut>(x + k);
  }
}

// T: type of dy, O: of the table's gradient; W elements a lane (8 or 1, so that either type's accesses are whole)
template <typename T, typename O, int W>
__global__ void __launch_bounds__(256) sum_kernel(const __grid_constant__ SumArgs A) {
  constexpr int kIn = W == 1 ? 1 : kWide<T>;
  typedef typename Vec<T, kIn>::type Raw;
  start_dependents();
  wait_for_previous();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int slices = (A.D + 32 * W - 1) / (32 * W);
  const int64_t unit = (int64_t)blockIdx.x * 8 + warp, chunk = unit / slices;
  const int c = ((int)(unit - chunk * slices) * 32 + lane) * W;
  const int64_t n0 = chunk * A.chunk, n1 = min(n0 + A.chunk, A.N);
  if (n0 >= A.N) return;
  const bool mine = c < A.D;
  const unsigned none = (unsigned)A.V;
  unsigned current = __ldg(A.key + n0);
  bool joined = n0 > 0 && __ldg(A.key + n0 - 1) == current;            // the row began in an earlier chunk
  if (current == none) return;
  float acc[W];
#pragma unroll
  for (int i = 0; i < W; ++i) acc[i] = 0.f;
  auto leave = [&](int which) {
    if (!mine) return;
    float* p = A.part + (chunk * 2 + which) * A.D + c;
#pragma unroll
    for (int i = 0; i < W; ++i) p[i] = acc[i];
  };
  auto flush = [&]() {
    if (joined) leave(0);
    else if (mine) finish_row<O, W>(A, current, c, acc);
  };
  bool over = false;
  for (int64_t n = n0; n < n1 && !over; n += 32) {
    const unsigned key = n + lane < n1 ? __ldg(A.key + n + lane) : none, place = n + lane < n1 ? __ldg(A.place + n + lane) : 0;
    const int count = (int)min((int64_t)32, n1 - n);
    for (int i = 0; i < count && !over; i += 8) {
      Raw r[8][W / kIn];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const unsigned k = __shfl_sync(0xffffffffu, key, i + j), p = __shfl_sync(0xffffffffu, place, i + j);
#pragma unroll
        for (int q = 0; q < W / kIn; ++q) {
          r[j][q] = Raw{};
          if (mine && k != none) r[j][q] = *reinterpret_cast<const Raw*>(static_cast<const T*>(A.dy) + (int64_t)p * A.lddy + c + q * kIn);
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const unsigned k = __shfl_sync(0xffffffffu, key, i + j);
        if (i + j >= count) break;
        if (k != current) {
          flush();
          current = k;
          joined = false;
#pragma unroll
          for (int q = 0; q < W; ++q) acc[q] = 0.f;
          if (k == none) { over = true; break; }
        }
        float x[W];
#pragma unroll
        for (int q = 0; q < W / kIn; ++q) widen<T>(r[j][q], x + q * kIn);
#pragma unroll
        for (int q = 0; q < W; ++q) acc[q] += x[q];
      }
    }
  }
  if (over) return;
  if (n1 < A.N && __ldg(A.key + n1) == current) leave(joined ? 0 : 1);     // it goes on in the next chunk
  else flush();
}

// The rows that reach over chunks: a CTA for each chunk in which one begins that goes on, and 32 columns of it. Its eight warps take the
// chunks behind it in turn.
template <typename O>
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ SumArgs A) {
  __shared__ float sh[8][32];
  start_dependents();
  wait_for_previous();
  const int64_t chunk = blockIdx.x, n0 = chunk * A.chunk, n1 = n0 + A.chunk;
  if (n1 >= A.N) return;
  const unsigned k = __ldg(A.key + n1);
  if (k == (unsigned)A.V || __ldg(A.key + n1 - 1) != k) return;
  if (__ldg(A.key + n0) == k && n0 > 0 && __ldg(A.key + n0 - 1) == k) return;            // it began earlier
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int c0 = blockIdx.y * 32; c0 < A.D; c0 += gridDim.y * 32) {
    const int c = c0 + lane;
    float s = 0.f;
    for (int64_t j = chunk + 1 + warp; j * A.chunk < A.N && __ldg(A.key + j * A.chunk) == k; j += 8)
      if (c < A.D) s += A.part[j * 2 * A.D + c];
    sh[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && c < A.D) {
      s = A.part[(chunk * 2 + 1) * A.D + c];
      for (int w = 0; w < 8; ++w) s += sh[w][lane];
      finish_row<O, 1>(A, k, c, &s);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------------------------- host

// Tokens a chunk: enough chunks for 16 warps on every SM, and 32 tokens at least (a chunk's ends cost it two rows of fp32).
int chunk_of(int64_t N, int64_t D, int W) {
  const int64_t slices = (D + 32 * W - 1) / (32 * W), chunks = (148 * 16 + slices - 1) / slices;
  const int64_t per = (N + chunks - 1) / chunks;
  return (int)((per + 31) / 32 * 32);
}

struct BackPlan {
  int64_t keys, part, total;
};
BackPlan back_plan(int64_t N, int64_t D) {
  BackPlan p;
  p.keys = pad256(N * 4);
  const int64_t chunk = chunk_of(N, D, 8), chunk1 = chunk_of(N, D, 1), least = chunk < chunk1 ? chunk : chunk1;
  p.part = pad256((N + least - 1) / least * 2 * D * (int64_t)sizeof(float));
  p.total = 4 * p.keys + p.part;
  return p;
}

bool type_ok(int t) { return t == DMX_F32 || t == DMX_BF16; }
bool sizes_ok(int64_t N, int64_t V, int64_t D) { return N >= 0 && V >= 0 && D >= 0 && N <= DMX_EMBEDDING_MAX && V <= DMX_EMBEDDING_MAX && D <= DMX_EMBEDDING_MAX_WIDTH; }

template <typename T, typename O>
int sums(const SumArgs& A, bool wide, cudaStream_t st) {
  const int W = wide ? 8 : 1;
  const int64_t chunks = (A.N + A.chunk - 1) / A.chunk, slices = (A.D + 32 * W - 1) / (32 * W), ctas = (chunks * slices + 7) / 8;
  const int rc = wide ? start(dim3((unsigned)ctas), 256, 1, 0, st, sum_kernel<T, O, 8>, A) : start(dim3((unsigned)ctas), 256, 1, 0, st, sum_kernel<T, O, 1>, A);
  if (rc != DMX_OK || chunks == 1) return rc;
  return start(dim3((unsigned)(chunks - 1), (unsigned)((A.D + 31) / 32 < 64 ? (A.D + 31) / 32 : 64)), 256, 1, 0, st, join_kernel<O>, A);
}

}  // namespace

extern "C" {

int dmx_embedding_forward(int64_t N, int64_t V, int64_t D, int dtype, int id_bytes, const void* ids, const void* table, int64_t ldt, float scale, void* y,
                          int64_t ldy, void* cuda_stream) {
  if (!sizes_ok(N, V, D) || !type_ok(dtype) || (id_bytes != 4 && id_bytes != 8) || (V > 1 && ldt < 0) || (N > 1 && ldy < D)) return DMX_ERR_ARG;
  if (N == 0 || D == 0) return DMX_OK;
  if (!ids || !y || (V > 0 && !table)) return DMX_ERR_ARG;
  const unsigned e = element_size(dtype);
  if (!aligned(ids, id_bytes) || !aligned(table, e) || !aligned(y, e)) return DMX_ERR_ALIGN;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  GatherArgs A = {ids, table, y, N, V, V > 1 ? ldt : D, N > 1 ? ldy : D, (int)D, id_bytes == 8, scale};
  const bool wide = wide_rows(table, V, ldt, D, dtype) && wide_rows(y, N, ldy, D, dtype);
  const int W = wide ? 16 / e : 1;
  const dim3 grid((unsigned)((N + 31) / 32), (unsigned)((D + 32 * W - 1) / (32 * W)));
  if (dtype == DMX_F32) return wide ? start(grid, 256, 1, 0, st, gather_kernel<float, 4>, A) : start(grid, 256, 1, 0, st, gather_kernel<float, 1>, A);
  return wide ? start(grid, 256, 1, 0, st, gather_kernel<bf16, 8>, A) : start(grid, 256, 1, 0, st, gather_kernel<bf16, 1>, A);
}

int64_t dmx_embedding_backward_workspace(int64_t N, int64_t V, int64_t D) {
  if (!sizes_ok(N, V, D)) return DMX_ERR_ARG;
  return N == 0 || D == 0 || V == 0 ? 0 : back_plan(N, D).total;
}

int dmx_embedding_backward(int64_t N, int64_t V, int64_t D, int id_bytes, const void* ids, int dtype, const void* dy, int64_t lddy, float scale,
                           int out_dtype, void* dtable, int64_t ldt, int accumulate, void* workspace, int64_t workspace_bytes, void* cuda_stream) {
  if (!sizes_ok(N, V, D) || !type_ok(dtype) || !type_ok(out_dtype) || (id_bytes != 4 && id_bytes != 8) || (N > 1 && lddy < 0) || (V > 1 && ldt < D)) return DMX_ERR_ARG;
  if (V == 0 || D == 0 || (N == 0 && accumulate)) return DMX_OK;
  const unsigned e = element_size(dtype), eo = element_size(out_dtype);
  if (!dtable || (N > 0 && (!ids || !dy))) return DMX_ERR_ARG;
  if (!aligned(ids, id_bytes) || !aligned(dy, e) || !aligned(dtable, eo) || !aligned(workspace, 256)) return DMX_ERR_ALIGN;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (N == 0) return dmxh::cuda_ok(cudaMemset2DAsync(dtable, (V > 1 ? ldt : D) * eo, 0, D * eo, V, st)) ? DMX_OK : DMX_ERR_CUDA;
  const BackPlan p = back_plan(N, D);
  if (workspace_bytes < p.total || !workspace) return DMX_ERR_ARG;
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  SortArgs S = {};
  S.ids = ids; S.wide_ids = id_bytes == 8; S.N = N; S.V = V;
  for (S.passes = 1; (uint64_t)V >> (8 * S.passes); ++S.passes) {}
  for (int i = 0; i < 2; ++i) {
    S.key[i] = reinterpret_cast<unsigned*>(ws + 2 * i * p.keys);
    S.place[i] = reinterpret_cast<unsigned*>(ws + (2 * i + 1) * p.keys);
  }
  if (!accumulate) { S.zero = dtable; S.zero_ld = (V > 1 ? ldt : D) * eo; S.zero_bytes = D * eo; }
  constexpr int kShared = kSortWarps * kDigits * 4;       // 32 KB
  const int rc = start(dim3(accumulate ? kSortCtas : 144), kSortThreads, 1, kShared, st, sort_kernel, S);
  if (rc != DMX_OK) return rc;
  const bool wide = wide_rows(dy, N, lddy, D, dtype) && wide_rows(dtable, V, ldt, D, out_dtype) && D % 8 == 0;
  SumArgs A = {S.key[0], S.place[0], dy, dtable, reinterpret_cast<float*>(ws + 4 * p.keys), N, V, N > 1 ? lddy : D, V > 1 ? ldt : D, (int)D,
               chunk_of(N, D, wide ? 8 : 1), accumulate != 0, scale};
  if (dtype == DMX_F32) return out_dtype == DMX_F32 ? sums<float, float>(A, wide, st) : sums<float, bf16>(A, wide, st);
  return out_dtype == DMX_F32 ? sums<bf16, float>(A, wide, st) : sums<bf16, bf16>(A, wide, st);
}

}  // extern "C"
