/*
 * dmx.h — C ABI of the DYNAMIX data-parallel gradient step on one GPU.
 *
 * The operation (Algorithm 1, the body of the innermost loop over the workers: each worker
 * computes a gradient g_i at its own batch size x_i and the global model is updated under
 * BSP; Section "State representation", paragraph "Training Statistical Efficiency Metrics":
 * the controller reads gradient statistics, sigma_norm and sigma^2_norm):
 *
 *   K emulated workers hand in flat gradient vectors x_k[0..P) computed at batch sizes b_k.
 *   One call forms the batch-size-weighted aggregate g = sum_k b_k x_k / sum_k b_k, the
 *   statistics the batch-size policy reads, and the SGD-momentum update
 *   m <- beta*m + g, theta <- theta - lr*m, prev_agg <- g.
 *
 * The paper states no formula for the aggregate, the statistics or the optimizer; the
 * definitions below are this library's reading and are the contract.
 *
 * Conventions
 *   - Every function returns DMX_OK (0) or a negative DMX_ERR_* code. Nothing throws,
 *     aborts or traps, on the host or on the device.
 *   - "HOST" / "DEVICE" on a pointer says which memory it addresses.
 *   - dmx_step is asynchronous: it enqueues work on the given stream and returns. It does
 *     not allocate, does not synchronise and copies nothing host-to-device (worker pointers,
 *     weights and batch sizes travel as kernel arguments).
 *   - A handle may be used from one stream at a time (its scratch is shared by its calls).
 *   - A handle belongs to the CUDA device that was current in dmx_create: its tables and scratch
 *     live there. A step issued while another device is current returns DMX_ERR_HANDLE before
 *     anything is enqueued (make the handle's device current first).
 *   - Handles are looked up in a table of live handles, never read through the pointer first:
 *     a call on a destroyed (or never created) handle returns DMX_ERR_HANDLE and touches no
 *     freed memory. An address reused by a later create names that later handle.
 *   - dmx_step, dmx_step_adam and their _partial forms enqueue two kernel launches and nothing
 *     else, so (with per-kernel timing off) they can be captured in a CUDA graph and replayed:
 *     the kernels leave the handle's scratch ready for the next run.
 */
#ifndef DMX_H_
#define DMX_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct dmx_handle dmx_handle;

/* gradient element types */
enum { DMX_F32 = 0, DMX_BF16 = 1 };

/* return codes */
enum {
  DMX_OK = 0,
  DMX_ERR_ARG = -1,      /* null pointer, K/P/S out of range, aliasing buffers, bad dtype  */
  DMX_ERR_SEGMENTS = -2, /* segment table not o[0]=0 <= o[1] <= ... <= o[S]=P              */
  DMX_ERR_BATCH = -3,    /* some batch size < 1                                            */
  DMX_ERR_ALIGN = -4,    /* a device pointer is not 16-byte aligned                        */
  DMX_ERR_NOMEM = -5,    /* host or device allocation failed                               */
  DMX_ERR_CUDA = -6,     /* a CUDA runtime call failed (see dmx_last_cuda_error)           */
  DMX_ERR_HANDLE = -7,   /* handle is NULL, destroyed, or belongs to another CUDA device   */
  DMX_ERR_LIMIT = -8,    /* problem too large for the fixed scratch of dmx_step_static     */
  DMX_ERR_GUARD = -9     /* dmx_check_guards: a guard word beside the scratch was overwritten */
};

/* limits */
#define DMX_MAX_WORKERS 64
#define DMX_MAX_SEGMENTS 65536
#define DMX_MAX_PARAMS (((int64_t)1) << 40)

/*
 * Layout of out_state (fp32, length dmx_state_len = 16 + K + 2*S).
 * With B = sum_k b_k, q_k = sum_j x_kj^2, A = sum_j g_j^2,
 * D = sum_j sum_k b_k (x_kj - g_j)^2, a = prev_agg as passed in:
 */
enum {
  DMX_ST_B_TOTAL = 0,      /* B                                                            */
  DMX_ST_AGG_SQNORM = 1,   /* A                                                            */
  DMX_ST_TR_SIGMA = 2,     /* tr(Sigma)^ = D/(K-1); unbiased for the per-sample covariance */
                           /* trace when x_k is a mean of b_k i.i.d. samples; 0 if K == 1  */
  DMX_ST_G2 = 3,           /* |G|^2^ = A - tr(Sigma)^/B; unbiased, may be <= 0             */
  DMX_ST_GNS = 4,          /* gradient noise scale tr(Sigma)^ / |G|^2^ if |G|^2^ > 0 else 0
                              (the quantity behind the paper's large->medium->small
                              batch schedule, Section "RL Agent Inference Evaluation",
                              paragraph "Batch Size Adaptation Dynamics")                      */
  DMX_ST_COS_PREV = 5,     /* <g,a> / sqrt(A * |a|^2) if both norms > 0 else 0             */
  DMX_ST_DOT_PREV = 6,     /* <g,a>                                                        */
  DMX_ST_PREV_SQNORM = 7,  /* |a|^2                                                        */
  DMX_ST_SIGMA2_NORM = 8,  /* sigma^2_norm = tr(Sigma)^ / (B*A) if A > 0 else 0            */
  DMX_ST_SIGMA_NORM = 9,   /* sigma_norm = sqrt(max(sigma^2_norm, 0))                      */
  DMX_ST_WMEAN_SQNORM = 10,/* sum_k b_k q_k / B                                            */
  DMX_ST_FLAGS = 11,       /* bit mask stored as a float, DMX_FLAG_*                       */
  DMX_ST_HDR = 16          /* 12..15 reserved (0); then q_k [K], V_s [S], N_s [S]          */
};
/* V_s = (sum_{j in s} sum_k b_k (x_kj-g_j)^2)/(K-1): segment s's additive share of
 * tr(Sigma)^ (0 if K == 1).  N_s = sum_{j in s} g_j^2.  Empty segments give 0. */

enum {
  DMX_FLAG_NONFINITE = 1,  /* some q_k, |a|^2 or A is not finite as fp32                   */
  DMX_FLAG_G2_NONPOS = 2,  /* |G|^2^ <= 0 (or NaN): gns reported as 0                      */
  DMX_FLAG_COS_UNDEF = 4,  /* A == 0 or |a|^2 == 0 (first step): cosine reported as 0      */
  DMX_FLAG_SINGLE = 8,     /* K == 1: no across-worker variance                            */
  DMX_FLAG_INTERNAL = 16,  /* a bounded wait inside the kernel ran out; results invalid    */
  DMX_FLAG_BOUNDS = 32     /* checked build only: an index into the tables or the scratch was
                              out of range and the access was skipped; results invalid     */
};

/*
 * dmx_create — validate (K, P, segment table), choose the launch configuration for the
 * current CUDA device, build the device-side tables and allocate the reduction scratch.
 *   K            number of workers, 1..DMX_MAX_WORKERS
 *   P            number of parameters, 1..DMX_MAX_PARAMS-1
 *   seg_offsets  HOST, S+1 entries: o[0]=0 <= o[1] <= ... <= o[S]=P; segment s is
 *                [o[s], o[s+1]); zero-length segments allowed; the table is copied
 *   S            number of segments, 1..DMX_MAX_SEGMENTS
 *   grad_dtype   DMX_F32 or DMX_BF16 (params, momentum, prev_agg, out_state are fp32)
 *   out          HOST, receives the handle
 * Errors: DMX_ERR_ARG, DMX_ERR_SEGMENTS, DMX_ERR_NOMEM, DMX_ERR_CUDA. Synchronous. On any error
 * everything allocated so far is released and *out is NULL.
 * For tests of that clean-up: with the environment variable DMX_TEST_FAIL_ALLOC=n the n-th
 * allocation of a create call (counted from 1, the handle structure first, then the device
 * buffers) is refused on the host as if memory had run out; no device call is made for it.
 * dmx_agg_create honours the same variable.
 */
int dmx_create(int K, int64_t P, const int64_t* seg_offsets, int S, int grad_dtype,
               dmx_handle** out);

/* 16 + K + 2*S, or DMX_ERR_HANDLE. */
int dmx_state_len(const dmx_handle* h);

/*
 * dmx_step — one iteration: aggregate, statistics, SGD-momentum update, state vector.
 *   grad_ptrs    HOST array of K DEVICE pointers; each addresses P elements of grad_dtype,
 *                16-byte aligned, read only
 *   batch_sizes  HOST array of K ints, each >= 1
 *   params       DEVICE, P fp32, 16-byte aligned, updated in place: theta - lr*m'
 *   momentum     DEVICE, P fp32, 16-byte aligned, updated in place: m' = beta*m + g
 *   lr, beta     learning rate and momentum coefficient (used as fp32)
 *   prev_agg     DEVICE, P fp32, 16-byte aligned; in: the previous step's aggregate
 *                (zeros before the first step); out: this step's aggregate g
 *   out_state    DEVICE, dmx_state_len(h) fp32, 4-byte aligned, fully overwritten
 *   cuda_stream  a cudaStream_t passed as void*; NULL = the legacy default stream
 * Buffers stay owned by the caller and must stay alive and untouched until the stream has
 * passed the step. params, momentum, prev_agg, out_state and the gradient buffers must be
 * pairwise disjoint (checked by address range; gradient buffers may alias one another).
 * Argument errors return before anything is enqueued: DMX_ERR_HANDLE, DMX_ERR_ARG,
 * DMX_ERR_BATCH, DMX_ERR_ALIGN; a failed launch returns DMX_ERR_CUDA.
 * Data problems (non-finite inputs, zero norms, |G|^2^ <= 0) are not errors: they set
 * bits in out_state[DMX_ST_FLAGS].
 */
int dmx_step(dmx_handle* h, const void* const* grad_ptrs, const int32_t* batch_sizes,
             float* params, float* momentum, float lr, float beta, float* prev_agg,
             float* out_state, void* cuda_stream);

/*
 * dmx_step_adam — the same pass with the Adam update in place of SGD with momentum (the paper
 * evaluates both optimizers, Section "Workloads and Datasets", and its state vector carries
 * sigma_norm and sigma^2_norm when the optimizer is adaptive, Section "State representation"). With g the
 * aggregate (Kingma & Ba 2015, Algorithm 1, bias-corrected form):
 *   m' = beta1 m + (1-beta1) g          v' = beta2 v + (1-beta2) g^2
 *   mhat = m' / (1-beta1^t)             vhat = v' / (1-beta2^t)
 *   theta' = theta - lr * mhat / (sqrt(vhat) + eps)          prev_agg' = g
 *   first_moment, second_moment   DEVICE, P fp32 each, 16-byte aligned, updated in place
 *   t                             1-based step count of this call (bias correction), >= 1
 *   0 <= beta1, beta2 < 1, eps >= 0, else DMX_ERR_ARG
 * Everything else (arguments, errors, asynchrony, statistics) is as dmx_step. out_state has the
 * same layout; three of its reserved entries carry the optimizer-normalised gradient statistics,
 * with ghat_j = g_j / (sqrt(vhat_j) + eps), the aggregate in units of Adam's running scale:
 *   out_state[12] = mean_j ghat_j     out_state[13] = var_j ghat_j (population variance over
 *   the P parameters)                 out_state[14] = sqrt(max(out_state[13], 0))
 * (dmx_step leaves 12..15 at 0.) This reading of the gradient variance and standard deviation
 * normalized for an adaptive optimizer is this library's: the paper gives no formula.
 */
int dmx_step_adam(dmx_handle* h, const void* const* grad_ptrs, const int32_t* batch_sizes,
                  float* params, float* first_moment, float* second_moment, float lr, float beta1,
                  float beta2, float eps, int64_t t, float* prev_agg, float* out_state,
                  void* cuda_stream);
enum { DMX_ST_ADAM_GHAT_MEAN = 12, DMX_ST_ADAM_GHAT_VAR = 13, DMX_ST_ADAM_GHAT_STD = 14 };

/*
 * Sharding one problem by parameter range (several GPUs, or several passes on one).
 * Every output of the step is either per parameter or a sum over parameters, so a problem splits
 * by parameter range with one small exchange: shard r owns elements [lo, hi) of all K gradient
 * buffers and of params/momentum/prev_agg, runs the same fused pass on them, and emits its raw
 * fp64 sums; the shards' sums are added (an all-reduce of K + 5 + 2 S doubles: the one exchange
 * step, e.g. NCCL over NVLink), and the state vector is derived from the total. This mirrors
 * the paper's scaling of the worker loop over 8 to 32 nodes (Section "Scalability of DYNAMIX"); the
 * paper has no formula for it. In a cluster where worker k is GPU k, the gradient shards come from
 * a reduce-scatter-like exchange that leaves every GPU with all workers' values of its range.
 *
 *   dmx_shard_range     HOST only. [lo, hi) of shard `shard` of `nshards`: boundaries on multiples
 *                       of 1024 elements (pointer alignment survives), the last shard ends at P;
 *                       a shard may be empty (lo == hi) when P is small: skip it.
 *   dmx_shard_segments  HOST only. The shard's own segment table (S+1 entries, written to
 *                       shard_offsets): the problem's table clipped to [lo, hi) and shifted by lo;
 *                       segments outside the shard become empty. Create the shard's handle with
 *                       dmx_create(K, hi - lo, shard_offsets, S, dtype): S and the state layout
 *                       stay those of the whole problem.
 *   dmx_partials_len    K + 5 + 2 S.
 *   dmx_step_partial, dmx_step_adam_partial
 *                       as dmx_step / dmx_step_adam on the shard's buffers (pointers to element lo),
 *                       but instead of out_state they write `partials` (DEVICE, dmx_partials_len
 *                       doubles, 8-byte aligned): q_k [K] in the caller's worker order, <g,a>, |a|^2,
 *                       Adam's sum and sum of squares of ghat (0 for SGD), Vraw_s [S] (before the
 *                       division by K-1), N_s [S], and an error word (1 if a bounded wait inside
 *                       the kernel ran out, plus 65536 if the checked build found an index out
 *                       of range; added over the shards like the rest).
 *   dmx_finalize_partials
 *                       batch_sizes: HOST, K ints; partials: DEVICE, the entry-wise sum over all
 *                       shards; P_total: the whole problem's parameter count (Adam's mean); writes
 *                       out_state (DEVICE, 16 + K + 2 S fp32) exactly as dmx_step defines it.
 *                       Asynchronous, one small launch.
 * Errors as dmx_step; DMX_ERR_SEGMENTS for a bad table or a range outside it.
 */
int dmx_shard_range(int64_t P, int nshards, int shard, int64_t* lo, int64_t* hi);
int dmx_shard_segments(const int64_t* seg_offsets, int S, int64_t lo, int64_t hi, int64_t* shard_offsets);
int dmx_partials_len(const dmx_handle* h);
int dmx_step_partial(dmx_handle* h, const void* const* grad_ptrs, const int32_t* batch_sizes, float* params,
                     float* momentum, float lr, float beta, float* prev_agg, double* partials,
                     void* cuda_stream);
int dmx_step_adam_partial(dmx_handle* h, const void* const* grad_ptrs, const int32_t* batch_sizes,
                          float* params, float* first_moment, float* second_moment, float lr, float beta1,
                          float beta2, float eps, int64_t t, float* prev_agg, double* partials,
                          void* cuda_stream);
int dmx_finalize_partials(int K, int S, const int32_t* batch_sizes, const double* partials, int adam,
                          int64_t P_total, float* out_state, void* cuda_stream);

/*
 * dmx_step_host — the same step for a caller whose gradients sit in HOST memory (the end-to-end
 * form of Algorithm 1's worker loop on one machine: gradients arrive from the workers' side of
 * the bus, the model state stays resident on the GPU).
 *   host_grad_ptrs  HOST array of K HOST pointers (pinned memory for full copy speed), each P
 *                   elements of grad_dtype
 *   staging_ptrs    HOST array of K DEVICE pointers, caller-owned staging buffers of P elements
 *                   each, 16-byte aligned; they receive the copies and feed the step
 *   out_state_dev   DEVICE, as out_state of dmx_step
 *   out_state_host  HOST, dmx_state_len(h) fp32; filled before the call returns
 * Enqueues K host-to-device copies, the step, and the device-to-host copy of the state vector
 * on the stream, then waits for the stream (so this call, unlike dmx_step, is synchronous).
 * Other arguments and errors as dmx_step; a failed copy returns DMX_ERR_CUDA.
 */
int dmx_step_host(dmx_handle* h, const void* const* host_grad_ptrs, void* const* staging_ptrs,
                  const int32_t* batch_sizes, float* params, float* momentum, float lr, float beta,
                  float* prev_agg, float* out_state_dev, float* out_state_host, void* cuda_stream);

/*
 * Per-kernel device timing of the steps of a handle (for benchmarks; off by default).
 * With profiling on, each dmx_step records CUDA events on its stream before the fused pass,
 * between the two kernels and after finalize. dmx_get_profile waits for the last step's
 * events and returns the two durations in milliseconds. Errors: DMX_ERR_HANDLE,
 * DMX_ERR_ARG (no step recorded, or profiling off), DMX_ERR_CUDA.
 * For timeline tools every step is also bracketed by NVTX ranges on the host ("dmx_step" or
 * "dmx_step_adam", with "dmx fused pass" and "dmx finalize" inside); they cost a pointer test
 * when no tool is attached.
 */
int dmx_set_profiling(dmx_handle* h, int on);
int dmx_get_profile(dmx_handle* h, float* fused_ms, float* finalize_ms);

/* Number of kernels one dmx_step launches (2: fused pass, finalize). */
int dmx_launches_per_step(const dmx_handle* h);

/* Sizes of a handle's launch plan, for inspection and tests: CTAs of the fused pass, chunks of
 * its work list, (V, N) partial-sum slots. Any pointer may be NULL. DMX_ERR_HANDLE or DMX_OK. */
int dmx_scratch_info(const dmx_handle* h, int* grid, int* nchunks, int* nslots);

/*
 * Checks of the library's own machinery (the paper has no counterpart; robustness is one of its
 * stated requirements, and these are how this library shows it without ever faulting a GPU).
 *
 * dmx_check_guards — every scratch array a handle's kernels write lies between two guard regions
 *   filled with a fixed word by dmx_create. This reads them back (synchronous copies; call it when
 *   no step of the handle is running) and returns DMX_OK, or DMX_ERR_GUARD if a word has changed,
 *   i.e. some kernel wrote just outside its array.
 *
 * dmx_selftest_wait — every wait inside the fused pass is bounded: after a fixed number of polls
 *   it gives up, raises the handle's error word and the CTA drains; the step's state vector then
 *   carries DMX_FLAG_INTERNAL and the word is cleared for the next step. This launches one warp
 *   that waits, with a budget of `polls` (1..2^24; the fused pass itself uses 2^18, about one
 *   second on B200 at 4 us per unsuccessful poll) polls, on a barrier that nothing will ever
 *   complete (no copy in flight, nobody to arrive): the wait must run out. *timed_out (HOST)
 *   receives 1 if it did; *waited_ms (HOST) the time the warp spent waiting, by the GPU's timer.
 *   The handle's error word is raised exactly as by a failed wait in a step: the next step of the
 *   handle reports DMX_FLAG_INTERNAL (its other outputs are valid) and clears it. Synchronous.
 *   Errors: DMX_ERR_HANDLE, DMX_ERR_ARG, DMX_ERR_NOMEM, DMX_ERR_CUDA.
 */
int dmx_check_guards(dmx_handle* h);
int dmx_selftest_wait(dmx_handle* h, uint32_t polls, int* timed_out, double* waited_ms, void* cuda_stream);

/*
 * dmx_plan_chunks — the work list dmx_create builds for the fused pass (host only: no CUDA call,
 * no device needed). For inspection and for tests of the planning logic.
 * The P parameters are cut into tiles of tile_elems elements (the last may be ragged); tiles are
 * taken in groups of *group_tiles consecutive tiles; chunk c consists of num_tiles[c] tiles:
 * tile i of the chunk is first_tile[c] + (i / G) * group_stride[c] + i % G with G = *group_tiles.
 * Every tile belongs to exactly one chunk. The fused kernel's CTAs draw chunks in list order
 * (CTA b starts with chunk b), so the list's order is the schedule: full waves first, shrinking
 * waves towards the end, and the chunk holding a ragged last tile moved to the front.
 *   resident_ctas   CTAs the device runs at once (SM count x CTAs per SM); *grid receives the
 *                   number of CTAs the kernel is launched with
 *   first_tile, num_tiles, group_stride   HOST, capacity entries each (may be NULL with capacity 0)
 * Returns the number of chunks (the arrays are filled only if capacity is at least that), or
 * DMX_ERR_ARG. The tuning variables dmx_create reads (DMX_TILE_GROUP, DMX_CHUNK_TILES,
 * DMX_MIN_CHUNK_KB) apply here too.
 */
int dmx_plan_chunks(int64_t P, int K, int grad_dtype, int tile_elems, int resident_ctas,
                    int32_t* first_tile, int32_t* num_tiles, int32_t* group_stride, int capacity,
                    int* group_tiles, int* grid);

/*
 * Window statistics of the state vector over k consecutive steps, kept on the device.
 * The controller acts on metrics aggregated over k iterations (Section "System architecture";
 * Section "State representation": state vectors are built from metrics collected every k
 * iterations, as means and standard deviations); with this the host reads one vector per
 * window instead of one per step.
 *   dmx_agg_create   state_len = dmx_state_len(h) (> DMX_ST_FLAGS), k >= 1; allocates two fp64
 *                    vectors on the current device
 *   dmx_agg_push     out_state: DEVICE, state_len fp32, as written by a step (enqueue the push on
 *                    the step's stream, after it); window_out: DEVICE, 2*state_len fp32. On every
 *                    k-th push window_out receives, per entry i over the window's k vectors,
 *                    mean (at i) and population standard deviation sqrt(sum (x-mean)^2 / k) (at
 *                    state_len + i), and the window restarts; entry DMX_ST_FLAGS gets the OR of
 *                    the k flag words and spread 0. Other pushes leave window_out untouched.
 *                    *emitted (HOST, may be NULL) is set to 1 on the pushes that write, else 0.
 *                    Asynchronous, no allocation. The position inside the window is counted on the
 *                    host, by call (which is why *emitted is known when the call returns, without
 *                    waiting for the device): a handle's pushes must be issued one after the other
 *                    (not concurrently from several threads), in the order of the steps, and on
 *                    one stream, so that the device executes them in that same order.
 * Errors: DMX_ERR_ARG, DMX_ERR_NOMEM, DMX_ERR_HANDLE, DMX_ERR_CUDA.
 */
typedef struct dmx_agg dmx_agg;
int dmx_agg_create(int state_len, int k, dmx_agg** out);
int dmx_agg_push(dmx_agg* a, const float* out_state, float* window_out, int* emitted, void* cuda_stream);
int dmx_agg_destroy(dmx_agg* a);

/*
 * dmx_ctl_decide — the controller's decision at the end of an adjustment cycle, on the device
 * (Algorithm 1, the loops after the k training iterations: build each worker's state vector,
 * evaluate the policy, apply the action within the batch-size limits, compute the reward).
 * What the paper fixes: the action set {-100, -25, 0, +25, +100} and the update
 * x_i <- max(min(x_i + a_i, x_max), x_min) (Section "Action space and batch size adjustment"),
 * and the reward (Section "Reward function design")
 *   r_i = Abar_i + alpha*max(0, dA_i) - beta_t*T_iter,i - delta*(log2 x_i - 5) - eta*(sigma2_norm + sigma_norm)
 * with x_i the batch size used during the cycle; eta = 0 gives the SGD form. What it leaves open,
 * and this library defines: the layout of the state vector and the policy network.
 *
 *   K, M, H        workers (1..DMX_MAX_WORKERS); caller-supplied metrics per worker
 *                  (0..DMX_CTL_MAX_AUX: accuracy, accuracy gain, iteration time, network and system
 *                  figures); hidden width of the policy network (1..DMX_CTL_MAX_HIDDEN)
 *   state_len      length of the step's state vector (>= DMX_ST_HDR + K)
 *   window         DEVICE, 2*state_len fp32: window means then deviations, as dmx_agg_push emits
 *   aux            DEVICE, K x M fp32 row-major (may be NULL when M == 0)
 *   batch          DEVICE, K int32: batch sizes used during the cycle (each >= 1)
 *   weights        DEVICE, dmx_ctl_num_weights(M, H) fp32, row-major, in this order:
 *                  W1 (H x F), c1 (H), W2 (H x H), c2 (H), W3 (5 x H), c3 (5), F = dmx_ctl_num_features(M)
 *   col_acc, col_gain, col_titer   columns of aux holding Abar, dA, T_iter; -1 leaves the term out
 *   alpha, beta_t, delta, eta      reward coefficients
 *   b_min, b_max   batch-size limits (the paper uses 32 and 1024), 1 <= b_min <= b_max
 *   uniforms       DEVICE, K fp32 in [0,1), or NULL. NULL: the action with the largest logit (lowest
 *                  index on ties). Otherwise the action is drawn from softmax(logits): the smallest a
 *                  whose cumulative probability exceeds uniforms[i] (the caller owns the generator)
 *   next_batch     DEVICE out, K int32     action   DEVICE out, K int32 (index 0..4 into the action set)
 *   reward         DEVICE out, K fp32      logits   DEVICE out, K x 5 fp32
 *   features       DEVICE out, K x F fp32, or NULL
 *
 * State vector of worker i (F = M + 9 entries), with mean/dev the two halves of `window`:
 *   aux[i][0..M), log2 x_i - 5, x_i*K / mean[B_TOTAL], mean[worker_sqnorm i] / mean[WMEAN_SQNORM],
 *   mean[SIGMA_NORM], mean[SIGMA2_NORM], dev[SIGMA_NORM], mean[COS_PREV], dev[COS_PREV],
 *   log2(1 + max(mean[GNS], 0) / mean[B_TOTAL])          (ratios with a zero denominator give 0)
 * Policy: logits = W3 tanh(W2 tanh(W1 s + c1) + c2) + c3. Arithmetic is fp64, stored as fp32; the
 * action is chosen from the fp32 logits as emitted.
 * Asynchronous, one launch, no allocation, no host-device copy. Errors: DMX_ERR_ARG, DMX_ERR_CUDA.
 */
#define DMX_CTL_ACTIONS 5
#define DMX_CTL_MAX_AUX 32
#define DMX_CTL_MAX_HIDDEN 256
#define DMX_CTL_LOCAL_EXTRA 3
#define DMX_CTL_GLOBAL_FEATURES 6
int dmx_ctl_num_features(int M);          /* M + 9, or DMX_ERR_ARG */
int64_t dmx_ctl_num_weights(int M, int H);  /* H*F + H + H*H + H + 5*H + 5, or DMX_ERR_ARG */
int dmx_ctl_decide(int K, int M, int H, int state_len, const float* window, const float* aux,
                   const int32_t* batch, const float* weights, int col_acc, int col_gain, int col_titer,
                   float alpha, float beta_t, float delta, float eta, int b_min, int b_max,
                   const float* uniforms, int32_t* next_batch, int32_t* action, float* reward,
                   float* logits, float* features, void* cuda_stream);

/*
 * dmx_step_static — the same step without a handle and without any allocation.
 * (The paper has no counterpart: this entry point exists for the library's callers only.)
 *
 * For callers that cannot allocate device memory at the point where they need the step:
 * code running under an allocator or memory pool that must account for every byte, a
 * latency-critical loop that cannot afford the device-wide synchronisation a cudaMalloc may
 * bring, or a process whose memory budget is spoken for. dmx_create allocates tables and
 * reduction scratch; this call uses neither. Its reduction scratch is a fixed array of
 * DMX_STATIC_SCRATCH_BYTES inside the library's device image: every GPU on which the library
 * is loaded holds that array until the process exits.
 *
 *   K, P, seg_offsets, S, grad_dtype   as dmx_create, but S <= DMX_STATIC_MAX_SEGMENTS.
 *                                      seg_offsets is HOST memory. It is validated during the call
 *                                      and copied to the device by an asynchronous copy on the
 *                                      stream: from pageable memory the runtime has taken its copy
 *                                      when the call returns; from pinned memory the table must
 *                                      stay unchanged until the stream has passed the call (and
 *                                      for as long as a captured copy of the call may be replayed)
 *   grad_ptrs ... cuda_stream          as dmx_step
 *
 * It calls no cudaMalloc, cudaFree or other allocating routine; the caller still provides
 * every input and output buffer. It runs the plain-load kernel with one contiguous range of
 * tiles per CTA, so it is slower than dmx_step, and its sums are taken in a different order:
 * results agree with dmx_step to rounding, not bit for bit.
 *
 * The first call on each device looks up the array's device address (with that device
 * current). Make that first call outside any stream capture.
 * All calls on a GPU share the one array, and it keeps what the previous call left: the
 * kernels clear what they need at the start of each call, and two calls that overlap on
 * the same GPU (different streams, different threads) race on it. Keep calls on one GPU in
 * stream order.
 * Errors: as dmx_create and dmx_step, and DMX_ERR_LIMIT when S exceeds
 * DMX_STATIC_MAX_SEGMENTS or the partial sums of this device's grid would not fit in the array.
 */
#define DMX_STATIC_MAX_SEGMENTS 512
#define DMX_STATIC_SCRATCH_BYTES (1 << 20)
int dmx_step_static(int K, int64_t P, const int64_t* seg_offsets, int S, int grad_dtype,
                    const void* const* grad_ptrs, const int32_t* batch_sizes, float* params,
                    float* momentum, float lr, float beta, float* prev_agg, float* out_state,
                    void* cuda_stream);

/*
 * The operators on both sides of the gradient step: the layers whose backward pass makes a worker's gradient
 * (dmx_linear_*, dmx_group_norm_*) and an optimizer over a model's separate tensors (dmx_adamw_*). The paper
 * names the models and optimizers it trains with and no formula for any of them; the formulas below are the
 * contract. All pointers are DEVICE memory unless marked HOST, all calls are asynchronous on the given stream
 * and copy nothing to the host, none allocates except the create call, and empty problems (a zero extent) are
 * valid. Buffers must not overlap unless a call says so; this is the caller's to keep.
 */

/* activations of dmx_group_norm_* and dmx_linear_*: u, max(u, 0), u / (1 + exp(-u)), u * Phi(u) (Phi: the normal
 * distribution function, the erf form). The slope of DMX_ACT_RELU at 0 is 0. All are computed in fp32: Phi to 3e-7 absolutely (so
 * that u * Phi(u) is good to 4e-6 of itself at u = -2 and to 5e-4 at u = -4), exponentials and reciprocals to 2 ulp. */
enum { DMX_ACT_NONE = 0, DMX_ACT_RELU = 1, DMX_ACT_SILU = 2, DMX_ACT_GELU = 3 };

/*
 * dmx_adamw_* — AdamW over n tensors in one launch, moments in fp32 or in 8-bit block codes.
 * Per element, with s the optional gradient factor:
 *   g = s*grad       m' = b1 m + (1-b1) g       v' = b2 v + (1-b2) g^2
 *   p' = p (1 - lr*wd) - lr/(1-b1^t) * m' / (sqrt(v') / sqrt(1-b2^t) + eps)       (wd = 0 where decay[i] is 0)
 * Arithmetic is fp32; parameters of type DMX_BF16 are rounded once when written. Where g^2 overflows (|g| > 1.8e19) v' is
 * infinite and the update zero.
 *
 * State. Tensor i owns ceil(sizes[i]/256) consecutive blocks of DMX_ADAMW_BLOCK elements, the first one at
 * dmx_adamw_first_block(h, i), dmx_adamw_blocks(h) in all; element j of the tensor is element first*256 + j of
 * the state arrays, which hold blocks*256 entries each (zero them before the first step; entries past a
 * tensor's end stay zero):
 *   state_bits 32   m, v fp32; m_scale, v_scale NULL
 *   state_bits 8    m int8 codes c with first moment m_scale[block] * sgn(c) * (c/127)^2, v uint8 codes with
 *                   second moment (v_scale[block] * (c/255)^2)^2; m_scale, v_scale: one fp32 per block.
 *                   Each step writes the block's largest |m'| and sqrt(v') as its scales and the codes nearest to
 *                   (|x|/scale)^(1/2), or, with dither != 0, floor(that + u) with u in [0,1) in steps of 2^-16
 *                   from a hash of the element's state index (low 32 bits) and `seed`: give every step another
 *                   seed. A nonzero second moment keeps a nonzero code; an infinite one is held as 3.4e38. Dithering is what lets a second moment
 *                   decay: a change of 0.1 % is far below half a code. It is unbiased in the code x, not in the value, whose mean
 *                   comes out larger by 6 f (1-f) / x^2 of itself for x^4 (f: x's fraction): a second moment at code c without
 *                   gradient loses 1 - 1.5/c of what beta2 takes away, until it rests at code 1.
 *
 *   dmx_adamw_create     sizes: HOST, n entries >= 0 (n in 1..DMX_ADAMW_MAX_TENSORS); decay: HOST, n bytes, or
 *                        NULL for all 1; param_dtype, grad_dtype: DMX_F32 or DMX_BF16. Synchronous.
 *   dmx_adamw_bind       params, grads, copies: HOST arrays of n DEVICE pointers, copied to the handle's table on the
 *                        stream (the arrays may be reused when the call returns). A NULL gradient leaves its
 *                        tensor and its state alone. copies (NULL, or with NULL entries): bf16 copies of the
 *                        parameters, written by every step. Pointers need their element's alignment only;
 *                        16-byte aligned fp32 and 8-byte aligned bf16 tensors are faster. Bind again when a
 *                        buffer moves; not inside a stream capture.
 *   dmx_adamw_grad_norm  out[0] = sqrt(sum of squares of all bound gradients) (summed in fp64 from fp32 sums of
 *                        eight; bitwise reproducible), out[1] = min(1, max_norm / (out[0] + 1e-6)), or NaN if
 *                        out[0] is not finite
 *   dmx_adamw_step       grad_scale: one fp32 or NULL (1), e.g. out + 1 of the norm. If it is NaN the step leaves
 *                        everything as it is. t >= 1: this step's number; 0 <= beta1, beta2 < 1; eps, weight_decay >= 0
 *   dmx_adamw_moments    the values of 8-bit moments, blocks*256 of them each, as fp32 or bf16 (out_dtype)
 * m, v and the moments' outputs are 16-byte aligned. A handle's calls are issued on one stream at a time.
 * Errors: DMX_ERR_ARG (also a call before bind), DMX_ERR_ALIGN, DMX_ERR_NOMEM, DMX_ERR_HANDLE, DMX_ERR_CUDA.
 */
#define DMX_ADAMW_BLOCK 256
#define DMX_ADAMW_MAX_TENSORS 65536
typedef struct dmx_adamw dmx_adamw;
int dmx_adamw_create(int n, const int64_t* sizes, const uint8_t* decay, int param_dtype, int grad_dtype, int state_bits,
                     dmx_adamw** out);
int64_t dmx_adamw_blocks(const dmx_adamw* h);
int64_t dmx_adamw_first_block(const dmx_adamw* h, int i);
int dmx_adamw_bind(dmx_adamw* h, void* const* params, const void* const* grads, void* const* copies, void* cuda_stream);
int dmx_adamw_grad_norm(dmx_adamw* h, float max_norm, float* out, void* cuda_stream);
int dmx_adamw_step(dmx_adamw* h, void* m, void* v, float* m_scale, float* v_scale, const float* grad_scale, double lr,
                   double beta1, double beta2, double eps, double weight_decay, int64_t t, int dither, uint32_t seed,
                   void* cuda_stream);
int dmx_adamw_moments(dmx_adamw* h, const void* m, const void* v, const float* m_scale, const float* v_scale, int out_dtype,
                      void* out_m, void* out_v, void* cuda_stream);
int dmx_adamw_destroy(dmx_adamw* h);   /* as dmx_destroy */

/*
 * dmx_group_norm_* — group norm with an activation on channels-last data, and its gradient.
 * x is N images of L positions of C channels (DMX_F32 or DMX_BF16), G groups of C/G neighbouring channels:
 *   mean, var over a group's L*C/G values (var without Bessel's correction), rstd = 1/sqrt(var + eps),
 *   u = (x - mean) * rstd * weight + bias, y = act(u)
 * backward, with xh = (x - mean)*rstd, du = dy * act'(u), n = L*C/G and sums over the group:
 *   dweight = sum over images and positions of du*xh, dbias = the same of du,
 *   dx = rstd * (weight*du - (sum(weight*du) + xh * sum(weight*du*xh)) / n)
 * All arithmetic and all sums are fp32; y and dx are rounded once. A variance is summed from deviations: a thread's (at
 * most 128 values) from its first value, corrected by their mean, the threads', CTAs' and chunks' from one another's means, so
 * a mean far from zero costs no accuracy. Group norm's statistics do not depend on the batch size, which is why
 * it is the norm to use where a controller changes that.
 *   x, y, dy, dx       element (n, l, c) at n*image + l*row + c, strides in elements >= 0; x and dy may repeat rows or
 *                      images with strides 0 (a broadcast gradient); y and dx have each element in a place of its
 *                      own: images one after the other, or their rows in turn (DMX_ERR_ARG otherwise);
 *                      any alignment of the element type (16-byte aligned starts and strides are faster)
 *   weight, bias       fp32, C entries, or NULL for ones and zeros
 *   mean, rstd         fp32, N*G (written by forward, read by backward); NaN where L = 0: there is nothing to average
 *   dweight, dbias     fp32, C entries, or NULL
 *   workspace          at least dmx_group_norm_workspace(...) bytes, 16-byte aligned, contents undefined
 *   dmx_group_norm_plan   for inspection and tests (no device needed): plan (HOST) receives elements per access, whether an
 *                      image's slab stays on the chip (0/1), CTAs that share it (or chunks of an image), items that the CTAs
 *                      (clusters) take in turn, threads and shared memory of a CTA. wide: 16-byte accesses are possible.
 * Results are bitwise reproducible. y may be x itself, and dx may be dy or x, with the same strides.
 * Errors: DMX_ERR_ARG (C < 1, G not a divisor of C, C > DMX_GN_MAX_CHANNELS,
 * C/G > DMX_GN_MAX_GROUP, extents, strides, eps < 0, null pointers, workspace
 * too small), DMX_ERR_ALIGN, DMX_ERR_CUDA.
 */
#define DMX_GN_MAX_CHANNELS 65536
#define DMX_GN_MAX_GROUP 1024
int64_t dmx_group_norm_workspace(int64_t N, int64_t L, int C, int G, int dtype, int backward);
int dmx_group_norm_plan(int64_t N, int64_t L, int C, int G, int dtype, int wide, int backward, int64_t* plan);
int dmx_group_norm_forward(int64_t N, int64_t L, int C, int G, int dtype, const void* x, int64_t x_image, int64_t x_row,
                           const float* weight, const float* bias, float eps, int act, void* y, int64_t y_image,
                           int64_t y_row, float* mean, float* rstd, void* workspace, int64_t workspace_bytes,
                           void* cuda_stream);
int dmx_group_norm_backward(int64_t N, int64_t L, int C, int G, int dtype, const void* dy, int64_t dy_image,
                            int64_t dy_row, const void* x, int64_t x_image, int64_t x_row, const float* mean,
                            const float* rstd, const float* weight, const float* bias, int act, void* dx,
                            int64_t dx_image, int64_t dx_row, float* dweight, float* dbias, void* workspace,
                            int64_t workspace_bytes, void* cuda_stream);

/*
 * dmx_linear_* — matrix product with bias, activation and residual in its epilogue, and its gradient (bf16
 * operands, fp32 accumulation on the tensor cores).
 *   forward    z = x W^T + bias,  y = act(z) + residual        x: M x K, W: N x K, y, z, residual: M x N
 *   backward   dz = dy * act'(z),  dx = dz W,  dW = dz^T x,  dbias = column sums of dz   (the residual's gradient is dy)
 * Everything up to a store is fp32, with one exception: with an activation, dz is rounded to bf16 before the two
 * products of backward (the tensor cores take 16-bit operands); dbias is summed from the unrounded dz.
 *   x, w, bias, residual, z, y, dy, dx, dw, dbias   bf16, row-major, ld* = elements from row to row (>= 0; of outputs
 *              >= the row's length unless there is one row; inputs may repeat rows with 0); element alignment suffices. Operands whose start or rows are not
 *              16-byte aligned, or repeat, are first laid out in the workspace.
 *   bias, residual, z (forward: an output, written only if given)   may be NULL
 *   z          backward: forward's z, needed unless act is DMX_ACT_NONE
 *   dx, dw, dbias   each may be NULL and is then not computed
 *   workspace  at least dmx_linear_workspace(...) / dmx_linear_backward_workspace(...) bytes for the same
 *              arguments (0 is possible), 256-byte aligned, contents undefined
 * y may be the residual itself. K = 0 gives z = bias; M = 0 gives dW = 0 and dbias = 0. Results are bitwise reproducible.
 *   dmx_linear_status   every wait inside the kernels is bounded; *errors (HOST) receives how many warps gave up
 *                       on the current device since the last call (0 unless the device misbehaves; results
 *                       are invalid otherwise). Waits for everything issued to the device so far, on whatever stream, and
 *                       counts it; not inside a stream capture.
 *   dmx_linear_plan     for inspection and tests (no device needed): how a product of rows x cols over k is cut. plan (HOST)
 *                       receives tile width, pairing of CTAs (0/1), ranges of k, exchanged operands (0/1), most tiles a CTA takes.
 *                       rows_across: the operand that D's rows come from lies across k (dw); 0 for y and dx.
 * Errors: DMX_ERR_ARG (extents > DMX_LINEAR_MAX_EXTENT, strides, null pointers, workspace too small), DMX_ERR_ALIGN, DMX_ERR_CUDA.
 */
#define DMX_LINEAR_MAX_EXTENT 4194240
int64_t dmx_linear_workspace(int64_t M, int64_t N, int64_t K, const void* x, int64_t ldx, const void* w, int64_t ldw);
int dmx_linear_forward(int64_t M, int64_t N, int64_t K, const void* x, int64_t ldx, const void* w, int64_t ldw,
                       const void* bias, int act, const void* residual, int64_t ldr, void* y, int64_t ldy, void* z,
                       int64_t ldz, void* workspace, int64_t workspace_bytes, void* cuda_stream);
int64_t dmx_linear_backward_workspace(int64_t M, int64_t N, int64_t K, const void* dy, int64_t lddy, const void* x,
                                      int64_t ldx, const void* w, int64_t ldw, int act);
int dmx_linear_backward(int64_t M, int64_t N, int64_t K, const void* dy, int64_t lddy, const void* x, int64_t ldx,
                        const void* w, int64_t ldw, const void* z, int64_t ldz, int act, void* dx, int64_t lddx,
                        void* dw, int64_t lddw, void* dbias, void* workspace, int64_t workspace_bytes,
                        void* cuda_stream);
int dmx_linear_plan(int64_t rows, int64_t cols, int64_t k, int rows_across, int64_t* plan);
int dmx_linear_status(int* errors);

/*
 * dmx_layer_norm_* — layer norm over the rows of a matrix, and its gradient.
 * x is M rows of D values (DMX_F32 or DMX_BF16):
 *   mean, var over a row's D values (var without Bessel's correction), rstd = 1/sqrt(var + eps), y = (x - mean) * rstd * weight + bias
 * backward, with xh = (x - mean)*rstd and g = weight*dy, sums over the row:
 *   dx = rstd * (g - (sum(g) + xh * sum(g*xh)) / D) + add,  dweight = sum over rows of dy*xh,  dbias = the same of dy
 * All arithmetic and all sums are fp32; y and dx are rounded once. var is the sum of squared deviations from the rounded mean,
 * corrected by that mean's own deviation: a mean far from zero costs it no accuracy (the mean itself is one float).
 *   x, y, dy, add, dx  element (m, d) at m*ld + d, strides in elements; inputs may repeat rows (ld 0) or overlap them, y's and dx's
 *                      ld is >= D unless there is one row. Element alignment suffices (16-byte aligned rows are faster).
 *   weight, bias       fp32, D entries, or NULL for ones and zeros
 *   mean, rstd         fp32, M entries (written by forward, read by backward)
 *   add                what is added to dx before it is rounded (e.g. the gradient that reaches x past the norm), or NULL
 *   dweight, dbias     fp32, D entries, or NULL
 *   workspace          backward, if dweight or dbias is wanted: at least dmx_layer_norm_workspace(...) bytes, 16-byte aligned,
 *                      contents undefined
 * Results are bitwise reproducible (for rows that are 16-byte aligned and for others: sums have another order there). y may be x, and dx may be dy, x or add, with the same strides (unless rows repeat). M = 0 gives dweight = 0 and
 * dbias = 0.
 * Errors: DMX_ERR_ARG (D < 1, D > DMX_LN_MAX_WIDTH, M >= 2^40, strides, eps < 0, null pointers, workspace too small), DMX_ERR_ALIGN,
 * DMX_ERR_CUDA.
 */
#define DMX_LN_MAX_WIDTH 65536
int64_t dmx_layer_norm_workspace(int64_t M, int D, int dtype);
int dmx_layer_norm_forward(int64_t M, int D, int dtype, const void* x, int64_t ldx, const float* weight, const float* bias,
                           float eps, void* y, int64_t ldy, float* mean, float* rstd, void* cuda_stream);
int dmx_layer_norm_backward(int64_t M, int D, int dtype, const void* dy, int64_t lddy, const void* x, int64_t ldx,
                            const float* mean, const float* rstd, const float* weight, const void* add, int64_t ldadd,
                            void* dx, int64_t lddx, float* dweight, float* dbias, void* workspace,
                            int64_t workspace_bytes, void* cuda_stream);

/*
 * dmx_embedding_* — rows of a table by token, scaled, and the table's gradient.
 *   forward    y[n] = scale * table[ids[n]]                       table: V x D, y: N x D (DMX_F32 or DMX_BF16, both of dtype)
 *   backward   dtable[v] = scale * (sum over n with ids[n] = v of dy[n])   (+ dtable[v] if accumulate)
 * An id outside 0..V-1 (padding, an ignored place) gives a row of zeros and takes no gradient. Sums are fp32, in the order of n within
 * chunks of neighbouring places in the sorted order (where they begin goes by the sizes, the types and whether rows are 16-byte aligned); results are
 * rounded once and are bitwise reproducible.
 *   ids          N integers of id_bytes (4 or 8) bytes, aligned to their size
 *   dtable       V x D of out_dtype. Without accumulate every row is written, zeros where no token is. With it rows without
 *                a token are neither read nor written (a table tied to a head whose gradient is there already).
 *   table, y, dy, dtable   rows ld* elements apart; inputs may repeat rows (0); outputs' ld >= D unless there is one row. Element alignment
 *                suffices (16-byte aligned rows are faster).
 *   workspace    at least dmx_embedding_backward_workspace(...) bytes, 256-byte aligned, contents undefined
 * Errors: DMX_ERR_ARG (N or V > DMX_EMBEDDING_MAX, D > DMX_EMBEDDING_MAX_WIDTH, types, strides, null pointers, workspace too small),
 * DMX_ERR_ALIGN, DMX_ERR_CUDA.
 */
#define DMX_EMBEDDING_MAX 0x7fffffff
#define DMX_EMBEDDING_MAX_WIDTH 65536
int dmx_embedding_forward(int64_t N, int64_t V, int64_t D, int dtype, int id_bytes, const void* ids, const void* table,
                          int64_t ldt, float scale, void* y, int64_t ldy, void* cuda_stream);
int64_t dmx_embedding_backward_workspace(int64_t N, int64_t V, int64_t D);
int dmx_embedding_backward(int64_t N, int64_t V, int64_t D, int id_bytes, const void* ids, int dtype, const void* dy,
                           int64_t lddy, float scale, int out_dtype, void* dtable, int64_t ldt, int accumulate,
                           void* workspace, int64_t workspace_bytes, void* cuda_stream);

/*
 * dmx_cross_entropy_* — softmax cross entropy of a linear layer over a vocabulary, its logits never kept, and its gradient (bf16 operands, fp32
 * accumulation on the tensor cores).
 *   forward    z = x W^T + bias,  lse[n] = log(sum over v of exp(z[n, v])),  loss[n] = lse[n] - z[n, target[n]]     x: N x D, W: V x D
 *   backward   G[n, v] = (exp(z[n, v] - lse[n]) - [v = target[n]]) * dloss[n],  dx = G W,  dW = G^T x,  dbias = column sums of G
 * A row whose target lies outside 0..V-1 (an ignored place) has loss 0 and no gradient; its lse is computed all the same. (dW
 * multiplies its x by zeros: that x has to be finite, or dW is NaN where it is not.) No loss is
 * negative: it is log(sum of exponentials of the distances from the largest logit), at least log 1, and the largest logit's lead over the target's. backward
 * computes the logits again and goes through the vocabulary in pieces. Everything up to a store is fp32, with one exception: G is rounded to bf16 before the two
 * products (the tensor cores take 16-bit operands), in units of the largest finite |dloss|'s significand; dbias is summed from the unrounded G. Exponentials are good to 2 ulp and 0 below 2^-126; the tensor cores'
 * sums of D products may truncate at every step (lse of D = 4000 is good to 5e-6 of the logits' size). Logits
 * of -inf (a bias of -inf) are words that do not occur; a logit of +inf or NaN makes its row's loss and gradient NaN, as does a row without
 * any finite logit.
 *   x, w, bias, dx, dw, dbias   bf16, row-major, ld* = elements from row to row (>= 0; of outputs >= D unless there is one row; inputs may
 *              repeat rows with 0); element alignment suffices. Operands whose start or rows are not 16-byte aligned, or repeat, are first
 *              laid out in the workspace.
 *   bias       V entries, or NULL
 *   target     N integers of target_bytes (4 or 8) bytes, aligned to their size
 *   loss, lse, dloss   fp32, N entries; dloss with a stride in elements (0: one value for all rows)
 *   dx, dw, dbias   each may be NULL and is then not computed
 *   workspace  at least dmx_cross_entropy_workspace(...) / dmx_cross_entropy_backward_workspace(...) bytes for the same arguments, 256-byte aligned,
 *              contents undefined. Forward: 8 bytes for each row and 64 to 256 words, 4 for each row. Backward: for dx or dw a piece of G (bf16, 512 MB at
 *              most, or 256 words), for dbias fp32 sums over 32 rows each of that piece, for dx fp32 sums (N x D, both rounded up to 256) where there are several pieces, and
 *              with one the parts of products that are cut into ranges. Both: the operands that are laid out. dmx_cross_entropy_backward_workspace counts
 *              all outputs, ..._for those of `outputs` (1 for dx, 2 for dw, 4 for dbias, added): enough for a call that gives the others as NULL.
 *   dmx_cross_entropy_plan   for inspection and tests (no device needed): how a problem is cut. plan (HOST, 11 entries) receives forward's tile width, pairing
 *              of CTAs (0/1) and tiles across the vocabulary; the pieces and a piece's words; the gradient's first product's tile width and pairing; of
 *              dx and of dW the tile width and ranges of k that are added afterwards (0: none)
 * N = 0 gives dW = 0 and dbias = 0. Results are bitwise reproducible. Waits inside the kernels are bounded; dmx_linear_status counts these too.
 * Errors: DMX_ERR_ARG (extents < 1 of V or D, or > DMX_LINEAR_MAX_EXTENT, strides, null pointers, workspace too small), DMX_ERR_ALIGN,
 * DMX_ERR_CUDA.
 */
int64_t dmx_cross_entropy_workspace(int64_t N, int64_t V, int64_t D, const void* x, int64_t ldx, const void* w, int64_t ldw);
int dmx_cross_entropy_forward(int64_t N, int64_t V, int64_t D, const void* x, int64_t ldx, const void* w, int64_t ldw,
                              const void* bias, int target_bytes, const void* target, float* loss, float* lse, void* workspace,
                              int64_t workspace_bytes, void* cuda_stream);
int64_t dmx_cross_entropy_backward_workspace(int64_t N, int64_t V, int64_t D, const void* x, int64_t ldx, const void* w, int64_t ldw);
int64_t dmx_cross_entropy_backward_workspace_for(int64_t N, int64_t V, int64_t D, const void* x, int64_t ldx, const void* w, int64_t ldw, int outputs);
int dmx_cross_entropy_backward(int64_t N, int64_t V, int64_t D, const float* dloss, int64_t dloss_stride, const void* x, int64_t ldx,
                               const void* w, int64_t ldw, const void* bias, int target_bytes, const void* target,
                               const float* lse, void* dx, int64_t lddx, void* dw, int64_t lddw, void* dbias, void* workspace,
                               int64_t workspace_bytes, void* cuda_stream);
int dmx_cross_entropy_plan(int64_t N, int64_t V, int64_t D, int64_t* plan);

/* Frees the tables and the scratch. NULL is accepted; a handle that is not live (destroyed
 * already) gives DMX_ERR_HANDLE. The caller makes sure no step of this handle is still running. */
int dmx_destroy(dmx_handle* h);

/* Static, NUL-terminated description of a return code. */
const char* dmx_strerror(int code);

/* The cudaError_t (as int) of the last failed CUDA call made by this library on the
 * calling thread, 0 if none. */
int dmx_last_cuda_error(void);

#ifdef __cplusplus
}
#endif
#endif /* DMX_H_ */
