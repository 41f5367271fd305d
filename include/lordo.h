/*
 * lordo.h -- C ABI of the LoRDO optimizer hot path on one NVIDIA B200 (sm_100a).
 *
 * The library runs, for a list of weight matrices W_i (m_i x n_i) and K simulated workers held as
 * a replica axis on one GPU, the three recurring pieces of the paper's Algorithm 1 (Global
 * variant) and Algorithm 2 (Local variant):
 *
 *   lordo_inner_step       the per-step block: clip, project with error feedback, low-rank Adam
 *                          moments, (quasi-hyperbolic) update, back-projection onto W
 *   lordo_outer_step       the synchronisation block: state averaging, pseudo-gradient mean,
 *                          outer optimizer (averaging or Nesterov), broadcast
 *   lordo_refresh_subspace ComputeProjection (randomized range finder + QR) and the rotation of
 *                          the moments into the new basis
 *   lordo_init             the algorithms' "Require" block (initial P, zero states, anchor copy)
 *
 * Conventions
 *   - Every matrix is row-major with no padding. The replica axis is outermost and contiguous:
 *     W_i is [K][m][n]; u_i, v_i are [K][r][n]; P_i is [m][r] (Global) or [K][m][r] (Local).
 *   - All "device" pointers are CUDA device memory of the current device, owned by the caller,
 *     16-byte aligned, and must stay valid for the lifetime of the context. The library never
 *     allocates device memory; `workspace` (size from lordo_query_workspace) is caller-owned too.
 *   - Pointer *tables* (`void* const*`) are host arrays with one device pointer per matrix.
 *   - `stream` is a cudaStream_t passed as void* (NULL = the default stream). Calls enqueue work
 *     and return without synchronising, except lordo_init, lordo_poll_status,
 *     lordo_inner_step_host, lordo_profile_read and lordo_destroy. (A call that is handed new
 *     gradient pointers stages their table in one of two pinned slots and may wait for the copy
 *     that left that slot two changes ago, which has normally long finished.)
 *   - Shapes: n and r multiples of 8 (m too for a matrix projected from the right), 8 <= r <= min(m, n),
 *     K >= 1, H >= 1.
 *   - Errors are return codes (lordo_status); nothing throws or aborts. After a non-zero return
 *     from an argument check no device state was modified. Numerical trouble found on the device
 *     (non-finite gradient norm, breakdown of the QR) sets a sticky flag word that
 *     lordo_poll_status returns.
 *   - A context is not thread-safe. Call order is checked (LORDO_ERR_STATE): lordo_outer_step
 *     only after a multiple of H inner steps; Global lordo_refresh_subspace only directly after
 *     lordo_outer_step; Local lordo_refresh_subspace only before the first inner step of a round.
 */
#ifndef LORDO_H_
#define LORDO_H_

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define LORDO_API __attribute__((visibility("default")))
#else
#define LORDO_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef struct lordo_ctx lordo_ctx; /* opaque, host memory, library-owned */

typedef enum {
  LORDO_OK = 0,
  LORDO_ERR_INVALID_ARG = 1,
  LORDO_ERR_SHAPE = 2,
  LORDO_ERR_ALIGN = 3,
  LORDO_ERR_STATE = 4,
  LORDO_ERR_NOMEM = 5,
  LORDO_ERR_CUDA = 6,
  LORDO_ERR_NUMERIC = 7,
  LORDO_ERR_UNSUPPORTED = 8
} lordo_status;

typedef enum { LORDO_F32 = 0, LORDO_BF16 = 1 } lordo_dtype;
typedef enum { LORDO_GLOBAL = 0, LORDO_LOCAL = 1 } lordo_variant;                 /* Alg. 1 / Alg. 2 */
typedef enum { LORDO_QHM_NONE = 0, LORDO_QHM_LOW = 1, LORDO_QHM_FULL = 2 } lordo_qhm; /* Alg. 1, update cases */
typedef enum { LORDO_OUTER_AVG = 0, LORDO_OUTER_NESTEROV = 1 } lordo_outer;       /* OuterOpt */

/* device status flags returned by lordo_poll_status */
#define LORDO_FLAG_NONFINITE_GRAD 1u /* a gradient norm was NaN or Inf */
#define LORDO_FLAG_QR_BREAKDOWN 2u   /* a column of a sketch was (numerically) dependent on the columns before it */
#define LORDO_FLAG_DEVICE_TIMEOUT 4u /* a bounded wait inside a kernel gave up; results of that call are invalid */

typedef struct {
  int64_t m, n; /* W is m x n */
  int32_t r;    /* P is m x r; moments are r x n (projection from the left, Sec. 2) */
  int32_t side; /* 0: as in the paper, from the left. 1: from the right (not in the paper, which always projects
                   from the left; the side selection of GaLore-type methods for matrices with m > n): P is n x r,
                   g = (G^ + E) P, the update is U~ P^T, mu(.) of the full-rank QHM term gives one value per row,
                   ComputeProjection returns the top-r right singular subspace. It is the left-side method applied
                   to W^T, and the library keeps that view: the moments u, v of such a matrix are [K][r][m]
                   (transposed low-rank arrays), P is [n][r] / [K][n][r]. Needs m a multiple of 8; not available
                   together with time_buffer or oversample. */
} lordo_mat;

typedef struct {
  int32_t n_mats;
  const lordo_mat* mats;   /* host array [n_mats] */
  int32_t K;               /* workers held as replicas (paper: M) */
  int32_t H;               /* inner steps per round (paper: K_x = K_u = K_v) */
  int32_t w_dtype;         /* lordo_dtype of W */
  int32_t g_dtype;         /* lordo_dtype of the gradients */
  int32_t e_dtype;         /* lordo_dtype of the error buffer E */
  int32_t variant;         /* lordo_variant */
  int32_t error_feedback;  /* 1: g = P^T(G^ + E), E <- G^ + E - P g ; 0: g = P^T G^, E unused */
  float beta2;             /* second-moment decay */
  float eps;               /* Adam epsilon */
  float clip_rho;          /* clipping radius rho; <= 0 disables clipping */
  int32_t clip_scope;      /* 0: one norm per worker over all matrices; 1: one per matrix */
  int32_t sync_u, sync_v;  /* average u / v over workers in lordo_outer_step */
  int32_t outer;           /* lordo_outer */
  float outer_lr;          /* eta_s (Nesterov only) */
  float outer_momentum;    /* mu_s  (Nesterov only) */
  int32_t power_iters;     /* subspace iterations of the range finder (0..8) */
  uint64_t seed;           /* seed of the counter-based generator for P_0 and the sketches */
  int32_t check_mode;      /* 1: every contraction in fp32 FMA arithmetic (parity mode);
                              0: bf16 tensor-core contractions where operands are bf16 */
  int32_t warm_start;      /* 0: every refresh starts from a fresh random sketch; 1: block power iteration
                              started from the current P (max(power_iters, 1) iterations, no sketch), the
                              cheaper estimator the paper names as an alternative ComputeProjection */
  int32_t time_buffer;     /* 1: the up-link time buffer of App. "Worker Communication": every worker accumulates
                              T += eta * alpha (alpha = the step's low-rank update, r x n, workspace memory) and
                              lordo_outer_step rebuilds the pseudo-gradient as (1/K) sum_k P_k T_k instead of
                              reading it off the K weight replicas. Only the update forms without the full-rank
                              term factorise: lordo_inner_step with LORDO_QHM_FULL returns LORDO_ERR_UNSUPPORTED.
                              The basis does not move between two synchronisations (the call order that
                              lordo_refresh_subspace enforces), which the factorisation needs. 0: off */
  int32_t oversample;      /* p >= 0, a multiple of 8: the range finder of the refresh runs with r + p columns and its
                              basis is truncated to the top-r left singular subspace of its projection of the
                              signal (Rayleigh-Ritz; not in the paper, the randomized-SVD refinement of the range
                              finder). The refresh then runs in fp32 in both modes. Needs r + p <= min(m, n) and
                              <= 600 for every matrix and warm_start = 0. 0: off */
} lordo_config;

/* Host tables of device pointers, one entry per matrix. fp32 unless stated. */
typedef struct {
  void* const* W;      /* [K][m][n] in w_dtype; on entry to lordo_init replica 0 holds W_0 */
  void* const* E;      /* [K][m][n] in e_dtype; may be NULL when error_feedback == 0 */
  float* const* P;     /* [m][r] (Global) or [K][m][r] (Local); side 1: [n][r] / [K][n][r] */
  float* const* u;     /* [K][r][n] first moment; side 1: [K][r][m] */
  float* const* v;     /* [K][r][n] second moment; side 1: [K][r][m] */
  float* const* X0;    /* [m][n] model copy of the last synchronisation */
  float* const* B;     /* [m][n] outer momentum; may be NULL when outer == LORDO_OUTER_AVG */
  float* const* Delta; /* [m][n] aggregated pseudo-gradient of the last lordo_outer_step */
} lordo_buffers;

/* Bytes of device workspace lordo_init needs for this configuration. Host-only, no CUDA call. */
LORDO_API int lordo_query_workspace(const lordo_config* cfg, size_t* bytes);

/*
 * Needs an sm_100a device; with check_mode = 0 and one storage type throughout (bf16 with r <= 512, fp32 with
 * r <= 256 and side 0) also a driver that offers cuTensorMapEncodeTiled (CUDA 12.0 or later), else LORDO_ERR_CUDA.
 *
 * Algorithm 1 / 2 "Require": copies W[0] to every replica and to X0, zeroes E, u, v, B, Delta,
 * writes P_0 (Global: orthonormalised random matrix from `seed`; Local: first r columns of the
 * identity for every worker). Synchronises `stream` before returning. `*out` owns host memory
 * only and is released by lordo_destroy. `workspace` must be 256-byte aligned.
 */
LORDO_API int lordo_init(const lordo_config* cfg, const lordo_buffers* buf, void* workspace, size_t workspace_bytes,
               void* stream, lordo_ctx** out);

/*
 * Algorithm 1, the per-step lines (clip ... model update), for every matrix and worker.
 * G: host table of device pointers, G[i] is [K][m_i][n_i] in g_dtype, read only.
 * lr = eta_t; beta1, omega per call because the paper switches them after warm-up; form selects
 * the update case. Bias correction uses the count of inner steps done on this context.
 */
LORDO_API int lordo_inner_step(lordo_ctx* ctx, const void* const* G, float lr, float beta1, float omega, int form,
                     void* stream);

/*
 * Same step fed from HOST memory: copies G_host[i] (pinned or pageable host memory, [K][m][n] in
 * g_dtype) into the caller's device staging buffers G_stage[i], runs lordo_inner_step, copies the
 * K clip coefficients of matrix 0 back to clip_out_host (K floats, may be NULL) and synchronises.
 */
LORDO_API int lordo_inner_step_host(lordo_ctx* ctx, const void* const* G_host, void* const* G_stage, float lr, float beta1,
                          float omega, int form, float* clip_out_host, void* stream);

/*
 * Algorithm 1, synchronisation lines: u,v <- mean over workers (if sync_u / sync_v);
 * Delta = X0 - mean_k W_k; averaging: X0 <- X0 - Delta; Nesterov: B <- mu_s B + Delta,
 * X0 <- X0 - eta_s (Delta + mu_s B); every W_k <- X0.
 */
LORDO_API int lordo_outer_step(lordo_ctx* ctx, void* stream);

/*
 * Algorithm 1, lines "if t mod K_u = 0: u <- E_m[u]" and "if t mod K_v = 0: v <- E_m[v]" on their
 * own, for schedules whose state-synchronisation intervals K_u, K_v differ from the model interval
 * K_x = H (set sync_u = sync_v = 0 in the configuration and call this at the steps of your choice).
 * May be called between any two inner steps.
 */
LORDO_API int lordo_sync_states(lordo_ctx* ctx, int sync_u, int sync_v, void* stream);

/*
 * ComputeProjection and the moment-rotation lines of Algorithm 1 (Global: signal = Delta, G must
 * be NULL) or Algorithm 2 (Local: signal = c_k G_k + E_k per worker, G as for lordo_inner_step).
 * Range finder: Y = S Omega with an n x r integer sketch from `seed`, thin QR, `power_iters`
 * subspace iterations. If at least one inner step was done the moments are rotated with
 * Rot = P_new^T P_old: u <- Rot u, v <- (1-beta2^s)|(Rot o Rot)(v^ - u^ o u^) + (Rot u^) o (Rot u^)|.
 * beta1 is the first-moment decay used for the bias-corrected u^.
 */
LORDO_API int lordo_refresh_subspace(lordo_ctx* ctx, const void* const* G_or_null, float beta1, void* stream);

/* Synchronises `stream`, stores the sticky device flag word in *flags (may be NULL) and returns
 * LORDO_ERR_NUMERIC if it is non-zero, else LORDO_OK. */
LORDO_API int lordo_poll_status(lordo_ctx* ctx, void* stream, uint32_t* flags);

/*
 * Diagnostics (Sec. "Experimental Framework", Metrics). mssv_dev: one float per projection matrix
 * (n_mats for Global, n_mats * K for Local, matrix-major), the mean squared singular value
 * (1/r) sum_i sigma_i^2 of Rot = P_new^T P_old of the LAST lordo_refresh_subspace (1 = the subspace
 * did not move, 0 = it moved to an orthogonal one); valid until the next refresh overwrites the
 * rotation matrices; LORDO_ERR_STATE before the first refresh. e_norm_dev: [n_mats][K] floats,
 * ||E||_F of every error buffer. Either pointer may be NULL. Device pointers, caller-owned.
 */
LORDO_API int lordo_diagnostics(lordo_ctx* ctx, float* mssv_dev, float* e_norm_dev, void* stream);

/* Clears the sticky device flag word (after the caller has dealt with what lordo_poll_status reported). */
LORDO_API int lordo_clear_status(lordo_ctx* ctx, void* stream);

/*
 * Self-test of the failure path of the tensor-core kernels: every wait inside them (on a TMA
 * transfer, a tensor-core commit, another warp) is bounded; a wait that runs out sets
 * LORDO_FLAG_DEVICE_TIMEOUT and the kernel runs to its normal end, so the context stays usable.
 * This call enqueues a one-thread kernel that waits on a barrier nothing completes: about two
 * seconds later lordo_poll_status reports the flag. It touches no optimizer state.
 */
LORDO_API int lordo_selftest_wait_timeout(lordo_ctx* ctx, void* stream);

/* Counters for checkpoint / resume: {inner steps done, refreshes done, outer steps done, inner steps
 * done in the current round}. A checkpoint is the caller's tensors (W, E, P, u, v, X0, B, Delta) plus
 * these four numbers: restore the tensors into the buffers of a context made with the same
 * configuration, then call lordo_set_counters (which also makes the library rebuild its internal
 * copies of P before the next step). With time_buffer the low-rank accumulators of a round live in the
 * workspace and are not part of a checkpoint: lordo_set_counters then accepts round boundaries only
 * (in[3] == 0, where the accumulators are zero) and returns LORDO_ERR_UNSUPPORTED otherwise.
 * Global rule: a checkpoint taken between lordo_outer_step and lordo_refresh_subspace (a round boundary
 * with fewer refreshes than synchronisations) may run that refresh first thing after the restore. The
 * rotation matrices behind lordo_diagnostics' MSSV are workspace state too: after a restore MSSV returns
 * LORDO_ERR_STATE until a refresh has run on the new context. */
LORDO_API int lordo_get_counters(const lordo_ctx* ctx, int64_t out[4]);
LORDO_API int lordo_set_counters(lordo_ctx* ctx, const int64_t in[4]);

/* Device address of the clip coefficients of the last inner step, [n_mats][K] fp32 (library
 * workspace; valid until lordo_destroy). */
LORDO_API int lordo_clip_coefficients(const lordo_ctx* ctx, const float** device_ptr);

/* Number of kernels this context has launched so far. */
LORDO_API int64_t lordo_launch_count(const lordo_ctx* ctx);

/*
 * Per-kernel-class device timing with CUDA events on the call's stream. While enabled, every
 * call records an event pair around each class; lordo_profile_read synchronises `stream` and
 * returns the milliseconds accumulated since the previous read:
 * ms[0] clip norm, [1] projection g = P^T(cG+E), [2] moment update, [3] back-projection + weight
 * and error-buffer update, [4] state averaging, [5] outer update, [6] subspace refresh, [7] unused.
 */
LORDO_API int lordo_profile_enable(lordo_ctx* ctx, int on);
LORDO_API int lordo_profile_read(lordo_ctx* ctx, void* stream, float ms_out[8]);

/* Text of the last error of this context (library-owned, valid until the next call). */
LORDO_API const char* lordo_last_error(const lordo_ctx* ctx);
LORDO_API const char* lordo_status_string(int status);

LORDO_API int lordo_destroy(lordo_ctx* ctx);

/*
 * The counter-based generator behind P_0 and the sketches, exposed so that it can be compared
 * bit for bit with a host implementation: out[i*cols + j] = popcount(mix64(key + g*(i*cols+j+1))) - 32
 * with key chained from (seed, purpose, mat, index, replica); purpose 1 = P_0, 2 = sketch.
 * out_dev: device pointer, rows*cols floats.
 */
LORDO_API int lordo_fill_random(uint64_t seed, int32_t purpose, int32_t mat, int64_t index, int32_t replica, int64_t rows,
                      int64_t cols, float* out_dev, void* stream);

/*
 * (The paper has no counterpart for this entry point; it is a convenience of this library.)
 *
 * Clip coefficient c = min(1, rho / (||G||_2 + 1e-6)) of ONE gradient array, computed without any
 * device allocation: no context, no workspace. It is meant for callers that must not or cannot
 * allocate device memory at the point where they need the coefficient -- code running while a
 * memory pool is frozen or nearly exhausted, a plug-in that was handed fixed buffers by its host
 * framework, a monitoring hook that may not disturb the allocator of the job it watches.
 * The reduction's partial sums live in a fixed array inside the library image (128 KiB per GPU
 * that loads the library, held until the process exits), which bounds the input:
 * count <= lordo_clip_coefficient_static_max_count() (2^29 elements); larger inputs are rejected
 * with LORDO_ERR_UNSUPPORTED and nothing is launched.
 *
 *   G_dev         device pointer, `count` elements of g_dtype (lordo_dtype), 16-byte aligned,
 *                 count a multiple of 8; read only
 *   rho           clipping radius; <= 0 gives c = 1
 *   coef_out_dev  device pointer to one float, written by the call (caller-owned); NaN when the
 *                 sum of squares is NaN or infinite (this entry point has no status word)
 *
 * The call enqueues two kernels on `stream` and returns without synchronising. The first call on
 * each device looks up the device address of the static array (with that device current); make
 * that first call outside any stream capture (the address is cached for the life of the process
 * and does not survive a cudaDeviceReset). A CUDA error already pending on the thread makes the
 * call return LORDO_ERR_CUDA before it launches anything. All calls on a device share the array: it holds
 * whatever the previous call left (every slot a call reads it has written itself, so nothing needs
 * clearing), and two calls whose kernels overlap on the GPU -- different streams, no ordering
 * between them -- race on it. Calls on one stream are safe.
 */
LORDO_API int lordo_clip_coefficient_static(const void* G_dev, int g_dtype, int64_t count, float rho, float* coef_out_dev,
                                            void* stream);
LORDO_API int64_t lordo_clip_coefficient_static_max_count(void);

/* =============================================================================================
 * Parameters outside the low-rank path: embedding tables, norm gains, biases.
 *
 * A model trained with the calls above has parameters that are no matrices of a context. They are updated by AdamW in a group of
 * their own, for the same K workers held as replicas, and synchronised by the same outer step (the paper's comparison systems run
 * Adam on every parameter; the low-rank path is defined for matrices only). Conventions are those at the top of this file: arrays
 * are row-major, the replica axis is outermost, device memory belongs to the caller, calls enqueue on `stream` and return.
 * An array that a call writes overlaps no other of its arrays. Sizes need not be multiples of anything here. lordo_adamw_init and
 * lordo_adamw_poll_status synchronise; a group's calls on different streams have to be ordered by the caller.
 * ============================================================================================= */

typedef enum { LORDO_I32 = 0, LORDO_I64 = 1 } lordo_index;                     /* type of token arrays */
typedef enum { LORDO_STATES_F32 = 0, LORDO_STATES_8BIT = 1 } lordo_states;

/*
 * Embedding lookup: out[k][t][:] = scale * W[k][tokens[k][t]][:], rounded once to out_dtype.
 *   W       [K][V][d] in w_dtype (lordo_dtype)     tokens  [K][T] in `index` (lordo_index)     out  [K][T][d] in out_dtype
 * A token outside [0, V) -- padding -- gives a row of zeros. T may be 0. K <= 64, V and T <= 2^30, d <= 2^24. Any element-aligned
 * pointers; rows whose bytes are a multiple of 16, at 16-byte aligned addresses, are moved 16 bytes at a time. May be captured in a
 * graph.
 */
LORDO_API int lordo_embedding(const void* W, int w_dtype, int K, int64_t V, int64_t d, const void* tokens, int index, int64_t T,
                              float scale, void* out, int out_dtype, void* stream);

/*
 * Its gradient: dW[k][v][:] = scale * sum of dY[k][t][:] over the t with tokens[k][t] = v; accumulate = 1 adds that to dW, and rows
 * whose token does not occur are left as they are (accumulate = 0: they become zero). dY is [K][T][d] in y_dtype, dW [K][V][d] in
 * w_dtype. Tokens outside [0, V) take no part, whatever their rows of dY hold. Every sum is formed in fp32, in an order that depends
 * on the tokens alone, and rounded once: the same bits on every run. `workspace` (256-byte aligned, size from the query, which makes
 * no CUDA call) may be used by one call at a time. Limits as for lordo_embedding. May be captured in a graph.
 */
LORDO_API int lordo_embedding_grad_query_workspace(int K, int64_t V, int64_t d, int64_t T, size_t* bytes);
LORDO_API int lordo_embedding_grad(const void* dY, int y_dtype, const void* tokens, int index, int K, int64_t V, int64_t d, int64_t T,
                                   float scale, void* dW, int w_dtype, int accumulate, void* workspace, size_t workspace_bytes,
                                   void* stream);

/* One tensor of an AdamW group. */
typedef struct {
  int64_t n;           /* elements (of one worker) */
  int64_t row;         /* of a table whose gradient may be given by tokens: elements of a row, n a multiple; else 0 */
  int64_t max_tokens;  /* with row > 0: most tokens of a worker in one step */
  double weight_decay;
} lordo_tensor;

typedef struct {
  int32_t n_tensors;
  const lordo_tensor* tensors; /* host array [n_tensors] */
  int32_t K;                   /* workers held as replicas, 1 .. 64 */
  int32_t w_dtype, g_dtype;    /* lordo_dtype */
  int32_t states;              /* lordo_states: the moments in fp32, or in 8 bits (below) */
  double beta2, eps;           /* eps > 0; with 8-bit moments at least 2^-126. Rates are doubles here: 1 - 0.999f is 1.3e-5 off 0.001 */
  double clip_rho;             /* clipping radius; <= 0 disables clipping */
  int32_t clip_scope;          /* 0: one norm per worker over all tensors; 1: one per tensor */
  int32_t sync;                /* 1: the group takes part in synchronisations (X0, B); 0: lordo_adamw_outer_step is refused */
  int32_t sync_m, sync_v;      /* average the moments over workers in lordo_adamw_outer_step */
  int32_t outer;               /* lordo_outer */
  double outer_lr, outer_momentum;
  uint64_t seed;               /* of the rounding of 8-bit moments */
} lordo_adamw_config;

/*
 * Host tables of device pointers, one entry per tensor, 16-byte aligned.
 *
 * 8-bit moments: m and s = sqrt(v) are kept as OCP E4M3 codes, one scale per 256 consecutive elements of one worker's tensor (the last
 * block of a worker may be shorter): value = code * 2^(scale byte - 127) (OCP E8M0). A scale puts the largest magnitude of its block
 * into [128, 256), or is 2^-126 where that is smaller. A magnitude of t units of the scale's grid is rounded down after (u + 1/2) / 65536
 * was added, u being 16 bits of the generator behind lordo_fill_random for (seed, step, tensor, worker, element): the expected value
 * is the exact one, so averages with beta near 1, whose change in a step is a fraction of the distance between codes, keep moving.
 * sqrt(v) > 0 never becomes 0 (the smallest code instead); v itself is formed in fp32 and counts as 0 below 2^-126 (gradients of 1e-18 where beta2 is
 * 0.999). The step itself uses the moments before they are rounded. Infinities and NaN are kept as NaN; the scale of their block is that of its
 * finite magnitudes, so that the other elements keep theirs.
 */
typedef struct {
  void* const* W;   /* [K][n] in w_dtype; on entry to lordo_adamw_init replica 0 holds the initial weights */
  void* const* m;   /* [K][n] fp32, or E4M3 */
  void* const* v;   /* [K][n] fp32, or E4M3 of sqrt(v) */
  void* const* ms;  /* [K][ceil(n / 256)] E8M0, 8-bit moments only, else NULL */
  void* const* vs;
  float* const* X0; /* [n] model copy of the last synchronisation; NULL when sync == 0 */
  float* const* B;  /* [n] outer momentum; NULL when sync == 0 or outer == LORDO_OUTER_AVG */
} lordo_adamw_buffers;

/* The gradient of one tensor in one step. */
typedef struct {
  const void* G;       /* [K][n] in g_dtype, 16-byte aligned; with tokens: [K][T][row], the gradient of the lookup's output */
  const void* tokens;  /* NULL, or [K][T]: the gradient is scale * (sum of the rows of G that belong to each token), kept in fp32 */
  int64_t T;           /* 0 <= T <= max_tokens */
  int32_t index;       /* lordo_index */
  float scale;
} lordo_grad;

typedef struct lordo_adamw_ctx lordo_adamw_ctx; /* opaque, host memory, library-owned */

LORDO_API int lordo_adamw_query_workspace(const lordo_adamw_config* cfg, size_t* bytes); /* no CUDA call */

/* Copies W[0] to every replica and to X0, zeroes the moments and B, synchronises `stream`. `workspace` is 256-byte aligned. */
LORDO_API int lordo_adamw_init(const lordo_adamw_config* cfg, const lordo_adamw_buffers* buf, void* workspace, size_t workspace_bytes,
                               void* stream, lordo_adamw_ctx** out);

/*
 * One step on every tensor and worker, G: host array [n_tensors]:
 *   g = c_k G;  m <- beta1 m + (1-beta1) g;  v <- beta2 v + (1-beta2) g^2;  m^ = m / (1-beta1^s);  v^ = v / (1-beta2^s)
 *   W <- W - lr ((omega m^ + (1-omega) g) / (sqrt(v^) + eps) + weight_decay W)
 * omega = 1 is AdamW, omega < 1 the quasi-hyperbolic form of the low-rank path. c_k = min(1, rho / (norm + 1e-6)), or, with coef_dev
 * (K floats in device memory), coef_dev[k]: for instance the coefficients of a lordo_ctx. s counts the steps of this context. A gradient
 * norm that is NaN or infinite sets LORDO_FLAG_NONFINITE_GRAD (only where the norm is formed); its coefficient is then NaN or 0,
 * as the formula has it (lordo_inner_step takes 1 for NaN). The step count and the rates are host values, so a stream that is being
 * captured is refused (LORDO_ERR_UNSUPPORTED).
 */
LORDO_API int lordo_adamw_step(lordo_adamw_ctx* ctx, const lordo_grad* G, double lr, double beta1, double omega, const float* coef_dev,
                               void* stream);

/*
 * The synchronisation lines of Algorithm 1 for the group: m, v <- mean over the workers (sync_m, sync_v; 8-bit moments: the mean of v,
 * rounded once, the same codes for every worker); D = X0 - mean_k W_k; averaging: X0 <- X0 - D; Nesterov: B <- mu_s B + D,
 * X0 <- X0 - eta_s (D + mu_s B); every W_k <- X0. To be called wherever lordo_outer_step is; it keeps no schedule of its own. A stream that
 * is being captured is refused.
 */
LORDO_API int lordo_adamw_outer_step(lordo_adamw_ctx* ctx, void* stream);

LORDO_API int lordo_adamw_poll_status(lordo_adamw_ctx* ctx, void* stream, uint32_t* flags); /* as lordo_poll_status */
LORDO_API int lordo_adamw_clear_status(lordo_adamw_ctx* ctx, void* stream);
/* {steps done, synchronisations done}: with the caller's tensors, all that a checkpoint needs. */
LORDO_API int lordo_adamw_get_counters(const lordo_adamw_ctx* ctx, int64_t out[2]);
LORDO_API int lordo_adamw_set_counters(lordo_adamw_ctx* ctx, const int64_t in[2]);
/* Device address of the clip coefficients of the last step that formed them, [n_tensors][K] fp32 (1 before that). */
LORDO_API int lordo_adamw_clip_coefficients(const lordo_adamw_ctx* ctx, const float** device_ptr);
LORDO_API int64_t lordo_adamw_launch_count(const lordo_adamw_ctx* ctx);
LORDO_API const char* lordo_adamw_last_error(const lordo_adamw_ctx* ctx);
LORDO_API int lordo_adamw_destroy(lordo_adamw_ctx* ctx);

#ifdef __cplusplus
}
#endif
#endif /* LORDO_H_ */
