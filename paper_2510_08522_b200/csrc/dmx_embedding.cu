// dmx_embedding.cu — rows of a table by token, scaled, and the table's gradient by sorted tokens.
//
// forward    y[n] = scale T[ids[n]]
// backward   dT[v] = scale (sum over n with ids[n] = v of dy[n]), added to what dT holds or not
//
// Both are bound by HBM. Backward first sorts the tokens by row (stably: by row, then by place), eight bits a pass in two launches: every
// CTA counts its keys' digits, then moves its keys. Other CTAs of the second write the table's zeros meanwhile. Then every warp sums a chunk of the sorted
// tokens over its columns, row after row in registers: each gradient row is read once, each row of the table written once. A row whose
// tokens reach over chunks leaves fp32 sums, one per chunk, which a last launch joins. Work is cut by tokens, not by rows: how
// often a token comes does not matter. Nothing is added atomically but whole numbers; the order of all sums is fixed by the ids, the sizes and types, and by
// whether rows are 16-byte aligned (which says how many columns a lane takes, and so where chunks begin).
// Measured on B200 (replayed in graphs, data mostly in L2): forward of 32768 tokens (8400 distinct) x 1024 bf16 13 us, a call among others 17
// (13.1 at the measured copy rate), fp32 29 (26.4), unaligned 23, scaled 25. Gradient of 16384 tokens in 30522 x 1024 bf16 36 us (14.9), fp32 53 (29.9): six launches in a row, sort 14 us
// and 5 more for zeros meanwhile, sums 11, joins 6; 64 tokens 17 us (9.7), added 10; 65536 tokens (12400 distinct) added to 50257 x 771 fp32 74 us (34).
#include <atomic>
#include <type_traits>

#include "dmx_rows.cuh"

namespace {

using namespace dmx_rows;

constexpr int kSortCtas = 128, kSortThreads = 1024, kSortWarps = kSortThreads / 32, kDigits = 256;      // (CTAs: at most)
constexpr int kKept = 8;                                   // keys a lane that scatter_kernel keeps
constexpr int kFew = 4, kFewTokens = kFew * kSortThreads;  // keys a thread that sort_few_kernel keeps
constexpr int kJoinCtas = 148 * 12;                        // at most

// ---------------------------------------------------------------------------------------------- forward

struct GatherArgs {
  const void *ids, *table;
  void* y;
  int64_t N, V, ldt, ldy;
  int D, wide_ids;
  float scale;
};

__device__ __forceinline__ int64_t id_at(const void* ids, int wide, int64_t n) {
  return wide ? static_cast<const long long*>(ids)[n] : (int64_t)static_cast<const int*>(ids)[n];
}

// How a lane holds its share of 32 x W columns: W neighbours in one access (of dy's type; 16 bytes), or, where alignment allows no
// more, every 32nd element.
template <int W, bool WIDE>
struct Columns {
  int c, D;
  __device__ __forceinline__ Columns(int slice, int lane, int D_) : c(slice * 32 * W + (WIDE ? lane * W : lane)), D(D_) {}
  __device__ __forceinline__ int at(int i) const { return WIDE ? c + i : c + i * 32; }
  __device__ __forceinline__ bool has(int i) const { return WIDE ? c < D : c + i * 32 < D; }
};

template <typename T, int W, bool WIDE>
struct Share {
  typedef typename Vec<T, WIDE ? W : 1>::type Raw;
  Raw r[WIDE ? 1 : W];
  __device__ __forceinline__ void load(const T* row, const Columns<W, WIDE>& at, bool live) {
#pragma unroll
    for (int i = 0; i < (WIDE ? 1 : W); ++i) {
      load_if(r[i], row + at.at(i), live && at.has(i));
    }
  }
  __device__ __forceinline__ void add_to(float (&acc)[W]) const {
    float x[W];
#pragma unroll
    for (int i = 0; i < (WIDE ? 1 : W); ++i) widen<T>(r[i], x + i);
#pragma unroll
    for (int i = 0; i < W; ++i) acc[i] += x[i];
  }
};

// A warp takes 32 x W columns of four rows. Unaligned rows with four elements a lane: with one, 32768 x 1023 bf16 took 59 us, so 29 (any ids, scaled).
template <typename T, int W, bool WIDE>
__global__ void __launch_bounds__(256) gather_kernel(const __grid_constant__ GatherArgs A) {
  constexpr int kRows = 4;
  start_dependents();
  wait_for_previous();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const Columns<W, WIDE> at(blockIdx.y, lane, A.D);
  const int64_t n0 = ((int64_t)blockIdx.x * 8 + warp) * kRows;
  Share<T, W, WIDE> r[kRows];
  int64_t id[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) id[k] = n0 + k < A.N ? id_at(A.ids, A.wide_ids, n0 + k) : -1;
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const bool live = id[k] >= 0 && id[k] < A.V;
    r[k].load(static_cast<const T*>(A.table) + (live ? id[k] : 0) * A.ldt, at, live);
  }
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    if (n0 + k >= A.N) continue;
    T* to = static_cast<T*>(A.y) + (n0 + k) * A.ldy;
#pragma unroll
    for (int i = 0; i < (WIDE ? 1 : W); ++i) {
      if (A.scale != 1.f) {
        constexpr int n = WIDE ? W : 1;
        float x[n];
        widen<T>(r[k].r[i], x);
#pragma unroll
        for (int j = 0; j < n; ++j) x[j] *= A.scale;
        r[k].r[i] = narrow<T, n>(x);
      }
      if (at.has(i)) *reinterpret_cast<typename Share<T, W, WIDE>::Raw*>(to + at.at(i)) = r[k].r[i];
    }
  }
}

// ---------------------------------------------------------------------------------------------- the sort

struct SortArgs {
  const void* ids;
  int wide_ids, shift, passes, ctas;      // shift: of the pass's digit; ctas: that sort
  int64_t N, V, rounds;            // rounds: of 32 keys, a warp's share
  const uint2* from;               // key and place, or NULL: the first pass takes the ids
  uint2* to;
  unsigned* counts;                // [ctas][digits] of the pass
  unsigned* crossing;              // to be zeroed
  unsigned char* zero;             // rows to clear meanwhile, by the other CTAs, or NULL
  int64_t zero_rows, zero_ld, zero_bytes;      // the last two of a row, in bytes
};

__device__ void clear_rows(const SortArgs& A, int64_t cta, int64_t ctas) {
  unsigned char* p = A.zero;
  if (A.zero_ld == A.zero_bytes || A.zero_rows == 1) {     // one piece
    const int64_t bytes = A.zero_rows * A.zero_bytes;
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
  for (int64_t v = cta * kSortWarps + warp; v < A.zero_rows; v += ctas * kSortWarps)
    for (int64_t i = lane * 2; i < A.zero_bytes; i += 64) *reinterpret_cast<unsigned short*>(p + v * A.zero_ld + i) = 0;
}

__device__ __forceinline__ uint2 pair_at(const SortArgs& A, int64_t n) {
  if (n >= A.N) return make_uint2(0, 0);
  if (A.from) return A.from[n];
  const int64_t id = id_at(A.ids, A.wide_ids, n);
  return make_uint2(id >= 0 && id < A.V ? (unsigned)id : (unsigned)A.V, (unsigned)n);      // what is in no row comes last
}

// How often each digit comes among a CTA's keys
__global__ void __launch_bounds__(kSortThreads) count_kernel(const __grid_constant__ SortArgs A) {
  __shared__ unsigned sh[kDigits];
  start_dependents();
  wait_for_previous();
  if (blockIdx.x == 0 && threadIdx.x == 0 && A.crossing) *A.crossing = 0;
  if (threadIdx.x < kDigits) sh[threadIdx.x] = 0;
  __syncthreads();
  const int64_t n0 = (int64_t)blockIdx.x * A.rounds * kSortThreads, n1 = min(n0 + A.rounds * kSortThreads, A.N);
#pragma unroll 4
  for (int64_t n = n0 + threadIdx.x; n < n1; n += kSortThreads) atomicAdd(&sh[pair_at(A, n).x >> A.shift & 255], 1u);
  __syncthreads();
  if (threadIdx.x < kDigits) A.counts[blockIdx.x * kDigits + threadIdx.x] = sh[threadIdx.x];
}

// A CTA's keys to where they belong by the digit. Every warp ranks its keys in order (behind its earlier equal digits, and the equal ones in lanes
// below); the ranks become places by prefix sums over warps, CTAs (whose counts are there) and digits. A warp's keys stay in registers
// meanwhile if they are no more than eight a lane; else they are ranked a second time.
__global__ void __launch_bounds__(kSortThreads) scatter_kernel(const __grid_constant__ SortArgs A) {
  extern __shared__ unsigned counts[];                    // [warps][digits]: a warp's digits, then where its next one goes
  __shared__ unsigned quarter[4][kDigits], others[4][kDigits], earlier_ctas[4][kDigits], scan[4][8];
  start_dependents();
  wait_for_previous();
  if ((int)blockIdx.x >= A.ctas) {
    clear_rows(A, blockIdx.x - A.ctas, gridDim.x - A.ctas);
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = blockIdx.x;
  const int digit = threadIdx.x & 255, group = threadIdx.x >> 8;      // of the prefix sums: a digit of eight warps, of every fourth CTA
  const unsigned below = (1u << lane) - 1;
  const int64_t first = ((int64_t)rank * kSortWarps + warp) * A.rounds * 32, end = min(first + A.rounds * 32, A.N);
  const bool keep = A.rounds <= kKept;
  unsigned* mine = counts + warp * kDigits;
  // the key's rank behind what `mine` holds for its digit, which moves on
  auto ranked = [&](bool live, unsigned k) {
    const unsigned d = live ? k >> A.shift & 255 : 256;
    const unsigned same = __match_any_sync(0xffffffffu, d);
    const unsigned before = live ? mine[d] : 0;
    __syncwarp();
    if (live && (same & below) == 0) mine[d] = before + __popc(same);
    __syncwarp();
    return before + __popc(same & below);
  };
  uint2 pair[kKept];
  unsigned at[kKept];
  if (keep) {
#pragma unroll
    for (int r = 0; r < kKept; ++r)
      if (r < A.rounds) pair[r] = pair_at(A, first + r * 32 + lane);
  }
  unsigned before = 0, total = 0;                         // of the digit, in CTAs before this one, in all
#pragma unroll 8
  for (int c = group; c < A.ctas; c += 4) {
    const unsigned t = A.counts[c * kDigits + digit];
    before += c < rank ? t : 0;
    total += t;
  }
  earlier_ctas[group][digit] = before;
  others[group][digit] = total;
  for (int i = lane; i < kDigits; i += 32) mine[i] = 0;
  __syncwarp();
  if (keep) {
#pragma unroll
    for (int r = 0; r < kKept; ++r)
      if (r < A.rounds) at[r] = ranked(first + r * 32 + lane < A.N, pair[r].x);
  } else {
    for (int64_t n = first; n < end; n += 32) ranked(n + lane < A.N, pair_at(A, n + lane).x);
  }
  __syncthreads();
  unsigned c[8], sum = 0;                                 // prefix over the warps
#pragma unroll
  for (int w = 0; w < 8; ++w) c[w] = counts[(group * 8 + w) * kDigits + digit];
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    const unsigned t = c[w];
    c[w] = sum;
    sum += t;
  }
  quarter[group][digit] = sum;
  unsigned start = 0;
  total = 0;
#pragma unroll
  for (int q = 0; q < 4; ++q) { start += earlier_ctas[q][digit]; total += others[q][digit]; }
  unsigned up = total;                                    // prefix over the digits
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned t = __shfl_up_sync(0xffffffffu, up, o);
    if (lane >= o) up += t;
  }
  if (lane == 31) scan[group][warp & 7] = up;
  __syncthreads();
  start += up - total;
  for (int w = 0; w < (warp & 7); ++w) start += scan[group][w];
  for (int q = 0; q < group; ++q) start += quarter[q][digit];
#pragma unroll
  for (int w = 0; w < 8; ++w) counts[(group * 8 + w) * kDigits + digit] = c[w] + start;
  __syncthreads();
  if (keep) {
#pragma unroll
    for (int r = 0; r < kKept; ++r)
      if (r < A.rounds && first + r * 32 + lane < A.N) A.to[at[r] + mine[pair[r].x >> A.shift & 255]] = pair[r];
  } else {
    for (int64_t n = first; n < end; n += 32) {
      const uint2 p = pair_at(A, n + lane);
      const unsigned to = ranked(n + lane < A.N, p.x);
      if (n + lane < A.N) A.to[to] = p;
    }
  }
}

// All passes in one CTA, pairs on their way from pass to pass through shared memory: up to four keys a thread. Fewer launches, but one SM. The whole
// gradient of 30522 x 1024 bf16 this way and by the two launches a pass: 1024 tokens 19 and 27 us, 4096 24 and 30 us, 8192 35 and 32 us.
__global__ void __launch_bounds__(kSortThreads) sort_few_kernel(const __grid_constant__ SortArgs A) {
  extern __shared__ unsigned counts[];                    // [warps][digits], then the pairs
  __shared__ unsigned quarter[4][kDigits], scan[4][8];
  start_dependents();
  wait_for_previous();
  if (blockIdx.x > 0) {
    clear_rows(A, blockIdx.x - 1, gridDim.x - 1);
    return;
  }
  if (threadIdx.x == 0) *A.crossing = 0;
  uint2* pairs = reinterpret_cast<uint2*>(counts + kSortWarps * kDigits);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int digit = threadIdx.x & 255, group = threadIdx.x >> 8;
  const unsigned below = (1u << lane) - 1;
  const int rounds = (int)A.rounds, first = warp * rounds * 32 + lane, N = (int)A.N;
  unsigned* mine = counts + warp * kDigits;
  uint2 pair[kFew];
  unsigned at[kFew];
#pragma unroll
  for (int r = 0; r < kFew; ++r)
    if (r < rounds) pair[r] = pair_at(A, first + r * 32);
  for (int pass = 0; pass < A.passes; ++pass) {
    const int shift = 8 * pass;
    for (int i = lane; i < kDigits; i += 32) mine[i] = 0;
    __syncwarp();
#pragma unroll
    for (int r = 0; r < kFew; ++r) {
      if (r >= rounds) continue;
      const bool live = first + r * 32 < N;
      const unsigned d = live ? pair[r].x >> shift & 255 : 256;
      const unsigned same = __match_any_sync(0xffffffffu, d);
      const unsigned before = live ? mine[d] : 0;
      __syncwarp();
      if (live && (same & below) == 0) mine[d] = before + __popc(same);
      __syncwarp();
      at[r] = before + __popc(same & below);
    }
    __syncthreads();
    unsigned c[8], sum = 0;                               // prefix over the warps
#pragma unroll
    for (int w = 0; w < 8; ++w) c[w] = counts[(group * 8 + w) * kDigits + digit];
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      const unsigned t = c[w];
      c[w] = sum;
      sum += t;
    }
    quarter[group][digit] = sum;
    __syncthreads();
    unsigned start = 0, total = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const unsigned t = quarter[q][digit];
      start += q < group ? t : 0;
      total += t;
    }
    unsigned up = total;                                  // prefix over the digits
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned t = __shfl_up_sync(0xffffffffu, up, o);
      if (lane >= o) up += t;
    }
    if (lane == 31) scan[group][warp & 7] = up;
    __syncthreads();
    start += up - total;
    for (int w = 0; w < (warp & 7); ++w) start += scan[group][w];
#pragma unroll
    for (int w = 0; w < 8; ++w) counts[(group * 8 + w) * kDigits + digit] = c[w] + start;
    __syncthreads();
    const bool last = pass + 1 == A.passes;
#pragma unroll
    for (int r = 0; r < kFew; ++r)
      if (r < rounds && first + r * 32 < N) (last ? A.to : pairs)[at[r] + mine[pair[r].x >> shift & 255]] = pair[r];
    if (last) return;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kFew; ++r)
      if (r < rounds && first + r * 32 < N) pair[r] = pairs[first + r * 32];
  }
}

// ---------------------------------------------------------------------------------------------- the sums

struct SumArgs {
  const uint2* pair;               // sorted: key and place
  const void* dy;
  void* out;
  unsigned* crossing;              // how many chunks have a last row that begins there and goes on, then (from the 8th byte) which, and the row, in any order
  float* part;                     // [chunks][2][D]: what a chunk's first and last row got, where they go on
  int64_t N, V, lddy, ldout;
  int D, chunk, accumulate;        // chunk: tokens, a multiple of 8
  float scale;
};

// W neighbours of a row of the table's gradient: one or two accesses
template <typename O, int W> struct Whole;
template <> struct Whole<float, 8> { typedef uint4 type; static constexpr int n = 4; };
template <> struct Whole<float, 4> { typedef uint4 type; static constexpr int n = 4; };
template <> struct Whole<bf16, 8> { typedef uint4 type; static constexpr int n = 8; };
template <> struct Whole<bf16, 4> { typedef uint2 type; static constexpr int n = 4; };

// A lane's share of a row of the table's gradient
template <typename O, int W, bool WIDE>
struct Row {
  typedef Whole<O, WIDE ? W : 4> H;
  typedef typename std::conditional<WIDE, typename H::type, typename Vec<O, 1>::type>::type Unit;
  Unit r[WIDE ? W / H::n : W];
  __device__ __forceinline__ void load(const O* row, const Columns<W, WIDE>& at, bool live) {
    constexpr int n = WIDE ? W / H::n : W;
#pragma unroll
    for (int k = 0; k < n; ++k) {
      const int i = WIDE ? k * H::n : k;
      load_if(r[k], row + at.at(i), live && at.has(i));
    }
  }
};

// acc * scale (+ old) to the row
template <typename O, int W, bool WIDE>
__device__ __forceinline__ void finish_row(const SumArgs& A, unsigned v, const Columns<W, WIDE>& at, const float (&acc)[W], const Row<O, W, WIDE>& old) {
  O* row = static_cast<O*>(A.out) + (int64_t)v * A.ldout;
  float x[W];
#pragma unroll
  for (int i = 0; i < W; ++i) x[i] = acc[i] * A.scale;
  if constexpr (WIDE) {
    typedef Whole<O, W> H;
    if (!at.has(0)) return;
#pragma unroll
    for (int k = 0; k < W / H::n; ++k) {
      float* y = x + k * H::n;
      if (A.accumulate) {
        if constexpr (sizeof(O) == 4) {
          float o[4];
          widen<O>(old.r[k], o);
#pragma unroll
          for (int i = 0; i < 4; ++i) y[i] += o[i];
        } else {
          const unsigned* w = reinterpret_cast<const unsigned*>(&old.r[k]);
#pragma unroll
          for (int i = 0; i < H::n / 2; ++i) { y[2 * i] += __uint_as_float(w[i] << 16); y[2 * i + 1] += __uint_as_float(w[i] & 0xffff0000u); }
        }
      }
      typename H::type* q = reinterpret_cast<typename H::type*>(row + at.at(k * H::n));
      if constexpr (sizeof(O) == 4 || H::n == 8) *q = narrow<O, H::n>(y);
      else *q = make_uint2(pack2(y[0], y[1]), pack2(y[2], y[3]));
    }
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i) {
      if (!at.has(i)) continue;
      if (A.accumulate) {
        float o;
        widen<O>(old.r[i], &o);
        x[i] += o;
      }
      *reinterpret_cast<typename Vec<O, 1>::type*>(row + at.at(i)) = narrow<O, 1>(x + i);
    }
  }
}

// T: type of dy, O: of the table's gradient. A warp: a chunk of the sorted tokens, 32 x W columns, `kAhead` rows of dy on their way at a time,
// with ADD also what the table holds where a row ends.
template <typename T, typename O, int W, bool WIDE, bool ADD>
__global__ void __launch_bounds__(256, 2) sum_kernel(const __grid_constant__ SumArgs A) {
  constexpr int kAhead = ADD ? 8 : 16;
  start_dependents();
  wait_for_previous();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int slices = (A.D + 32 * W - 1) / (32 * W);
  const int64_t unit = (int64_t)blockIdx.x * 8 + warp, chunk = unit / slices;
  const int slice = (int)(unit - chunk * slices);
  const Columns<W, WIDE> at(slice, lane, A.D);
  const int64_t n0 = chunk * A.chunk, n1 = min(n0 + A.chunk, A.N);
  if (n0 >= A.N) return;
  const unsigned none = (unsigned)A.V;
  const unsigned front = A.pair[n0].x;
  bool joined = n0 > 0 && A.pair[n0 - 1].x == front;             // the row began in an earlier chunk
  if (front == none) return;
  float acc[W];
#pragma unroll
  for (int i = 0; i < W; ++i) acc[i] = 0.f;
  auto leave = [&](int which) {
    float* p = A.part + (chunk * 2 + which) * A.D;
#pragma unroll
    for (int i = 0; i < W; ++i)
      if (at.has(i)) p[at.at(i)] = acc[i];
  };
  bool open = false;                                                     // the last row goes on in the next chunk
  for (int64_t n = n0; n < n1; n += 32) {
    const uint2 pair = n + lane < n1 ? A.pair[n + lane] : make_uint2(none, 0);
    const unsigned key = pair.x, place = pair.y, after = n + lane + 1 < A.N ? A.pair[n + lane + 1].x : none;
    const unsigned some = __ballot_sync(0xffffffffu, key != none), ends = __ballot_sync(0xffffffffu, key != after) & some;
    const int count = __popc(some);                                      // (what is in no row comes last)
    for (int i = 0; i < count; i += kAhead) {
      // Shuffles before the loads: one among them waited for those on their way, it seems (few counters serve both): 65536 rows of 771 fp32
      // added to a table took 202 us that way and take 54 this way, whatever the number of rows at a time.
      unsigned p[kAhead], k[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        p[j] = __shfl_sync(0xffffffffu, place, i + j);
        k[j] = __shfl_sync(0xffffffffu, key, i + j);
      }
      Share<T, W, WIDE> r[kAhead];
      Row<O, W, WIDE> old[ADD ? kAhead : 1];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) r[j].load(static_cast<const T*>(A.dy) + (int64_t)p[j] * A.lddy, at, i + j < count);
      if constexpr (ADD) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) old[j].load(static_cast<const O*>(A.out) + (int64_t)k[j] * A.ldout, at, ends >> (i + j) & 1);
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        if (i + j >= count) continue;
        r[j].add_to(acc);
        open = true;
        if (ends >> (i + j) & 1) {
          if (joined) leave(0);
          else finish_row<O, W, WIDE>(A, k[j], at, acc, old[ADD ? j : 0]);
          joined = open = false;
#pragma unroll
          for (int q = 0; q < W; ++q) acc[q] = 0.f;
        }
      }
    }
    if (count < 32) break;
  }
  if (!open) return;
  leave(joined ? 0 : 1);
  if (!joined && slice == 0 && lane == 0) reinterpret_cast<uint2*>(A.crossing)[1 + atomicAdd(A.crossing, 1u)] = make_uint2((unsigned)chunk, A.pair[n1].x);
}

// The rows that reach over chunks, by the chunk in which they begin: a CTA takes 128 columns of one at a time, its four warps the chunks
// behind in turn. (Most such rows have one chunk behind: small CTAs, many of them.)
template <typename O>
__global__ void __launch_bounds__(128) join_kernel(const __grid_constant__ SumArgs A) {
  constexpr int kAtOnce = 6;
  __shared__ float sh[4][4][32];
  start_dependents();
  wait_for_previous();
  const int64_t chunks = (A.N + A.chunk - 1) / A.chunk;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, slices = (A.D + 127) / 128;
  const uint2* list = reinterpret_cast<const uint2*>(A.crossing) + 1;
  uint2 entry = list[blockIdx.x / slices];                 // (on its way with the count; there is room for every chunk, and no more CTAs than those take)
  const int64_t units = (int64_t)*A.crossing * slices;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    if (unit != blockIdx.x) entry = list[unit / slices];
    const int64_t chunk = entry.x;
    const unsigned k = entry.y;
    const Columns<4, false> at((int)(unit % slices), lane, A.D);
    Row<O, 4, false> old;
    if (warp == 0) old.load(static_cast<const O*>(A.out) + (int64_t)k * A.ldout, at, A.accumulate);
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    for (int64_t j = chunk + 1 + warp; j < chunks; j += 4 * kAtOnce) {
      unsigned x[kAtOnce][4], key[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {                  // (what is read of a chunk that is not in the row is left out)
        const int64_t q = j + 4 * u;
        load_if(key[u], A.pair + q * A.chunk, q < chunks);
#pragma unroll
        for (int i = 0; i < 4; ++i) load_if(x[u][i], A.part + q * 2 * A.D + at.at(i), q < chunks && at.has(i));
      }
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] += j + 4 * u < chunks && key[u] == k ? __uint_as_float(x[u][i]) : 0.f;
      if (j + 4 * (kAtOnce - 1) >= chunks || key[kAtOnce - 1] != k) break;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) sh[warp][i][lane] = s[i];
    __syncthreads();
    if (warp == 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[i] = at.has(i) ? A.part[(chunk * 2 + 1) * A.D + at.at(i)] : 0.f;
        for (int w = 0; w < 4; ++w) s[i] += sh[w][i][lane];
      }
      finish_row<O, 4, false>(A, k, at, s, old);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------------------------- host

// Tokens a chunk: enough chunks for 16 warps on every SM, as many as there is room for, and eight tokens at least. W: columns a lane. (Sixteen rows on
// their way in each of 16 warps beat eight in each of 24: 131072 tokens of 1024 bf16 92 and 94 us, added to a table 88 and 93.)
int chunk_of(int64_t N, int64_t D, int W) {
  const int64_t slices = (D + 32 * W - 1) / (32 * W), chunks = (148 * 16 + slices - 1) / slices;
  const int64_t per = (N + chunks - 1) / chunks;
  return (int)((per + 7) / 8 * 8);
}

struct BackPlan {
  int64_t keys, part, crossing, counts, total;
};
BackPlan back_plan(int64_t N, int64_t D) {
  BackPlan p;
  p.keys = pad256(N * 8);
  const int64_t chunk = chunk_of(N, D, 8), chunk4 = chunk_of(N, D, 4), least = chunk < chunk4 ? chunk : chunk4;
  p.part = pad256((N + least - 1) / least * 2 * D * (int64_t)sizeof(float));
  p.crossing = pad256((1 + (N + least - 1) / least) * 8);
  p.counts = kSortCtas * kDigits * 4;
  p.total = 2 * p.keys + p.part + p.crossing + p.counts;
  return p;
}

bool type_ok(int t) { return t == DMX_F32 || t == DMX_BF16; }
bool sizes_ok(int64_t N, int64_t V, int64_t D) { return N >= 0 && V >= 0 && D >= 0 && N <= DMX_EMBEDDING_MAX && V <= DMX_EMBEDDING_MAX && D <= DMX_EMBEDDING_MAX_WIDTH; }

template <typename T, typename O>
int sums(SumArgs A, bool wide, cudaStream_t st) {
  constexpr int kW = kWide<T>;
  const int W = wide ? kW : 4;
  A.chunk = chunk_of(A.N, A.D, W);
  const int64_t chunks = (A.N + A.chunk - 1) / A.chunk, slices = (A.D + 32 * W - 1) / (32 * W), ctas = (chunks * slices + 7) / 8;
  const dim3 grid((unsigned)ctas);
  int rc;
  if (A.accumulate) rc = wide ? start(grid, 256, 1, 0, st, sum_kernel<T, O, kW, true, true>, A) : start(grid, 256, 1, 0, st, sum_kernel<T, O, 4, false, true>, A);
  else rc = wide ? start(grid, 256, 1, 0, st, sum_kernel<T, O, kW, true, false>, A) : start(grid, 256, 1, 0, st, sum_kernel<T, O, 4, false, false>, A);
  if (rc != DMX_OK || chunks == 1) return rc;
  const int64_t most = (chunks - 1) * ((A.D + 127) / 128);
  return start(dim3((unsigned)(most < kJoinCtas ? most : kJoinCtas)), 128, 1, 0, st, join_kernel<O>, A);
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
  const int W = wide ? 16 / e : 4;
  const dim3 grid((unsigned)((N + 31) / 32), (unsigned)((D + 32 * W - 1) / (32 * W)));
  if (dtype == DMX_F32) return wide ? start(grid, 256, 1, 0, st, gather_kernel<float, 4, true>, A) : start(grid, 256, 1, 0, st, gather_kernel<float, 4, false>, A);
  return wide ? start(grid, 256, 1, 0, st, gather_kernel<bf16, 8, true>, A) : start(grid, 256, 1, 0, st, gather_kernel<bf16, 4, false>, A);
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
  uint2* pairs[2] = {reinterpret_cast<uint2*>(ws), reinterpret_cast<uint2*>(ws + p.keys)};      // the last pass ends in the first
  S.ids = ids; S.wide_ids = id_bytes == 8; S.N = N; S.V = V;
  S.rounds = (N + (int64_t)kSortThreads * kSortCtas - 1) / ((int64_t)kSortThreads * kSortCtas);
  S.ctas = (int)((N + S.rounds * kSortThreads - 1) / (S.rounds * kSortThreads));
  S.crossing = reinterpret_cast<unsigned*>(ws + 2 * p.keys + p.part);
  S.counts = reinterpret_cast<unsigned*>(ws + 2 * p.keys + p.part + p.crossing);
  S.zero_ld = (V > 1 ? ldt : D) * eo; S.zero_bytes = D * eo;
  int passes = 1;
  while ((uint64_t)V >> (8 * passes)) ++passes;
  constexpr int kShared = kSortWarps * kDigits * 4;       // 32 KB
  int rc = DMX_OK;
  if (N <= kFewTokens) {
    S.passes = passes;
    S.rounds = (N + kSortThreads - 1) / kSortThreads;
    S.to = pairs[0];
    S.zero = accumulate ? nullptr : static_cast<unsigned char*>(dtable);
    S.zero_rows = V;
    const int shared = kShared + (int)(passes > 1 ? N * 8 : 0);
    static std::atomic<uint64_t> set{0};                  // devices on which the kernel may use that much
    int device = 0;
    if (!dmxh::cuda_ok(cudaGetDevice(&device))) return DMX_ERR_CUDA;
    const uint64_t bit = (uint64_t)1 << (device & 63);
    if (!(set.load(std::memory_order_relaxed) & bit) || device > 63) {
      if (!dmxh::cuda_ok(cudaFuncSetAttribute(sort_few_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kShared + kFewTokens * 8))) return DMX_ERR_CUDA;
      set.fetch_or(bit, std::memory_order_relaxed);
    }
    rc = start(dim3(S.zero ? 296 : 1), kSortThreads, 1, shared, st, sort_few_kernel, S);
  }
  for (int i = 0; i < passes && N > kFewTokens && rc == DMX_OK; ++i) {
    S.shift = 8 * i;
    S.from = i == 0 ? nullptr : pairs[(passes - i) & 1];
    S.to = pairs[(passes - i - 1) & 1];
    S.zero = nullptr;
    rc = start(dim3((unsigned)S.ctas), kSortThreads, 1, 0, st, count_kernel, S);
    if (rc != DMX_OK) break;
    // the scattering launches, which take longer, clear their share of the rows meanwhile
    const int64_t v0 = V * i / passes, v1 = V * (i + 1) / passes;
    S.zero = accumulate || v1 == v0 ? nullptr : static_cast<unsigned char*>(dtable) + v0 * S.zero_ld;
    S.zero_rows = v1 - v0;
    rc = start(dim3((unsigned)(S.ctas + (S.zero ? 296 : 0))), kSortThreads, 1, kShared, st, scatter_kernel, S);
    S.crossing = nullptr;
  }
  if (rc != DMX_OK) return rc;
  // 16-byte accesses of dy, and as many elements of the table's rows: 8 to 32 bytes
  const int W = 16 / e;
  const bool wide = wide_rows(dy, N, lddy, D, dtype) && aligned(dtable, W * eo < 16 ? W * eo : 16) && (V <= 1 || ldt % (W * eo < 16 ? W : 16 / (int)eo) == 0);
  SumArgs A = {pairs[0], dy, dtable, reinterpret_cast<unsigned*>(ws + 2 * p.keys + p.part), reinterpret_cast<float*>(ws + 2 * p.keys), N, V, N > 1 ? lddy : D, V > 1 ? ldt : D, (int)D, 0, accumulate != 0, scale};
  if (dtype == DMX_F32) return out_dtype == DMX_F32 ? sums<float, float>(A, wide, st) : sums<float, bf16>(A, wide, st);
  return out_dtype == DMX_F32 ? sums<bf16, float>(A, wide, st) : sums<bf16, bf16>(A, wide, st);
}

}  // extern "C"
