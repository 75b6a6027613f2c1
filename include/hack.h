/*
 * hack.h - C ABI of the B200 (sm_100a) library for the per-scale decoding step of head-aware
 * KV-cache compression in next-scale visual autoregressive transformers.
 *
 * One "step" serves one (layer, scale): the new scale's keys/values join the cache (Eq. 3), every
 * candidate key of a head whose cache would exceed its budget is scored with a small query subset
 * (Eq. 9), a budgeted subset is selected per head with the contextual rule (Eq. 10) or the
 * structural rule (Eq. 11) under asymmetric budgets (Eq. 7-8), the survivors are compacted into a
 * ragged per-head cache, and the scale's queries attend over it (Eq. 4 on the compressed cache,
 * compression preceding attention, section "Asymmetric Head Budget Allocation").
 *
 * Conventions for every entry point
 *  - Q, K, V, O are CALLER-OWNED DEVICE buffers, dense row-major [batch, n_heads, N_k, head_dim]
 *    in the cache's dtype, 16-byte aligned, N_k = side_k^2 of the scale being decoded.  Only the
 *    *_host entry point takes host pointers.
 *  - `stream` is a cudaStream_t passed as void* (NULL = the legacy default stream).  Calls only
 *    enqueue work and return; nothing synchronises unless stated.
 *  - Layers and scales are 0-based.  Each layer walks its scales in order 0,1,2,...; a call for
 *    any other scale returns HACK_ERR_STATE.  Within a scale a layer is served either by
 *    hack_scale_step, or by [hack_score, hack_select,] hack_compact, hack_attend in that order.
 *  - Stored lengths are a function of the schedule, the budgets and the head type only (the
 *    selection decides WHICH entries survive, never HOW MANY), so the library keeps them on the
 *    host and never reads anything back from the device to plan a launch.
 *  - Candidate index j of a head in a step: j < L addresses the L entries stored before the step
 *    (ascending original position), j >= L the new scale's token j - L.
 *  - Argument errors are detected on the host before anything is launched and leave the cache
 *    unchanged.  Nothing traps on the device.  There is no CPU fallback.
 *  - The cache (K/V planes, position plane, scratch) is owned by the library and released by
 *    hack_free_cache.  A cache is not thread safe; use one cache per stream of work.
 */
#ifndef HACK_H_
#define HACK_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#if defined(__GNUC__)
#define HACK_API __attribute__((visibility("default")))
#else
#define HACK_API
#endif

typedef struct hack_cache hack_cache_t; /* opaque, library-owned */

typedef enum {
  HACK_OK = 0,
  HACK_ERR_INVALID_ARG = 1, /* NULL pointer, size or index out of range, misaligned buffer */
  HACK_ERR_UNSUPPORTED = 2, /* head_dim / dtype / n_obs outside what the kernels implement */
  HACK_ERR_OOM = 3,         /* device or host allocation failed */
  HACK_ERR_CUDA = 4,        /* a CUDA call failed; hack_last_error() has the text */
  HACK_ERR_STATE = 5,       /* call out of order for this layer (wrong scale or phase) */
  HACK_ERR_TIMEOUT = 6      /* a bounded device-side wait expired (reported by hack_poll_status) */
} hack_status_t;

typedef enum { HACK_F32 = 0, HACK_BF16 = 1 } hack_dtype_t;

/* Overflow rule for structural heads when B_S < N_init + N_k (the paper is silent): */
enum { HACK_OVERFLOW_KEEP_PROTECTED = 0, /* keep every protected entry, exceed B_S */
       HACK_OVERFLOW_COMPETE = 1 };      /* protect only the initial scales; keep exactly B_S */

/* Which n = min(N_obs, N_k) queries of the current scale form the subset Q~ of Eq. 9.  The method
 * uses uniform spacing; the others are the alternatives of the paper's query-subset ablation. */
enum { HACK_OBS_UNIFORM = 0, /* floor(m * N_k / n), m = 0..n-1 */
       HACK_OBS_INIT = 1,    /* the first n tokens of the scale */
       HACK_OBS_RECENT = 2,  /* the last n tokens of the scale */
       HACK_OBS_CALLER = 3,  /* rows given per scale with hack_set_obs_rows (random sampling: the
                                caller draws them) */
       HACK_OBS_FULL = 4 };  /* every query of the scale, whatever n_obs: the ablation's full-attention
                                reference; costs ceil(N_k / 32) scoring rounds per step */

typedef struct {
  int32_t n_layers, n_heads, head_dim, batch; /* head_dim in {64, 128} */
  int32_t n_scales;
  const int32_t* scale_sides;        /* host, [n_scales], copied at init; N_k = side^2 */
  int32_t dtype;                     /* hack_dtype_t of Q/K/V/O and of the cache */
  const uint8_t* head_is_contextual; /* host, [n_layers*n_heads], 1 = contextual, 0 = structural
                                        (offline classification, Eq. 6); copied at init */
  int32_t budget_c, budget_s;        /* B_C, B_S: entries per head, >= 1 (Eq. 7-8) */
  int32_t n_obs;                     /* query subset size N_obs, 1..32 (Eq. 9; paper uses 32) */
  int32_t n_init_scales;             /* leading scales always kept in structural heads (paper: 2) */
  float sm_scale;                    /* softmax scale; 0 selects 1/sqrt(head_dim) */
  int32_t overflow_policy;           /* HACK_OVERFLOW_* */
  int32_t device;                    /* CUDA device ordinal */
  int32_t obs_sampler;               /* HACK_OBS_*; 0 = the method's uniform rule */
  int32_t merge_last;                /* 1: at the last scale, contextual heads fold the entries that step
                                        discards into their nearest retained counterparts (the merge
                                        described after Eq. 10; see hack_compact).  bf16 caches only. */
} hack_config_t;

/* Host-side plan of one step of one layer (all lengths in entries per head). */
typedef struct {
  int32_t n_new;                 /* N_k */
  int32_t stored_c, stored_s;    /* L before the step, contextual / structural heads */
  int32_t cand_c, cand_s;        /* T' = L + N_k */
  int32_t kept_c, kept_s;        /* length after the step */
  int32_t triggered_c, triggered_s; /* 1 if T' exceeds the type's budget (strictly) */
  int32_t n_obs_rows;            /* min(N_obs, N_k) */
} hack_step_info_t;

/* Buffer strides a caller of the separate stage calls must use. */
typedef struct {
  int32_t cand_stride; /* floats per (batch, head) row of `scores`: max T' over all steps */
  int32_t kept_stride; /* int32 per (batch, head) row of `idx`: max kept length over all steps */
  int32_t max_new;     /* largest N_k */
} hack_limits_t;

/* Eq. 7, B = alpha*B_C + (1-alpha)*B_S, solved under one of the paper's two allocation rules
 * (appendix, "Model-Specific Configurations").  Host only, no device work.
 *   rule 0 ("fraction"): B_C = floor(param*T_K); B_S = floor((B - alpha*B_C)/(1-alpha)).
 *   rule 1 ("ratio"):    B_C : B_S = 1 : param; B_C = floor(B/(alpha+param*(1-alpha))), B_S = param*B_C.
 * B_S is clamped to T_K and both results are at least 1.  INVALID_ARG unless 0 < alpha < 1. */
HACK_API hack_status_t hack_split_budget(int32_t budget, double alpha, int32_t rule, double param,
                                int32_t total_tokens, int32_t* budget_c, int32_t* budget_s);

/* Allocate the ragged per-head cache for the whole stack (Eq. 5, 8: per head at most its type's
 * budget, or the protected set if that is larger) and all scratch.  *out is set only on
 * success.  Capacity per head = the largest stored length its type reaches over the schedule. */
HACK_API hack_status_t hack_init_cache(const hack_config_t* cfg, hack_cache_t** out);
/* Release everything; synchronises the device first.  NULL is accepted. */
HACK_API hack_status_t hack_free_cache(hack_cache_t* cache);
/* HACK_OBS_CALLER only: the query rows that form Q~ (Eq. 9) at `scale`, for every layer, batch
 * element and head.  rows: host, n = min(N_obs, N_k) distinct indices in [0, N_k), used in the
 * order given (the scores do not depend on the order).  Copied to the device synchronously: a
 * set-up call, made before the steps of that scale are enqueued; the rows stay in force across
 * hack_reset.  A step that has to score while its scale has no rows fails with HACK_ERR_STATE.
 * INVALID_ARG for a wrong n, an index out of range or a repeated index; STATE if the cache was
 * not created with HACK_OBS_CALLER. */
HACK_API hack_status_t hack_set_obs_rows(hack_cache_t* cache, int32_t scale, const int32_t* rows, int32_t n);
/* New image: all layers back to scale 0 with empty caches.  Enqueues nothing. */
HACK_API hack_status_t hack_reset(hack_cache_t* cache);

HACK_API hack_status_t hack_get_limits(const hack_cache_t* cache, hack_limits_t* out);
/* Plan of step (layer, scale) given the layer's current state; scale must be the layer's next. */
HACK_API hack_status_t hack_step_info(const hack_cache_t* cache, int32_t layer, int32_t scale,
                             hack_step_info_t* out);

/* Subset-attention importance (Eq. 9 and the TOPK argument of Eq. 10-11).  For every (b,h) whose
 * type is triggered in this step: scores[(b*H+h)*cand_stride + j] = sum over the
 * min(N_obs, N_k) uniformly spaced query rows i = floor(m*N_k/n) of
 * Softmax_j(sm_scale * <Q[i], K_cand[j]>) over all T' candidates (stored ++ k_new).  Rows of
 * heads that are not triggered are left untouched.  Does not change the cache. */
HACK_API hack_status_t hack_score(hack_cache_t* cache, int32_t layer, int32_t scale, const void* q,
                         const void* k_new, float* scores, void* stream);

/* Budgeted selection per head from fp32 `scores` (layout as above).  Contextual heads keep the
 * B_C best candidates (Eq. 10).  Structural heads keep every entry of the first n_init_scales
 * scales and of the scale being decoded and fill the remaining M = B_S - |protected| slots with
 * the best of the rest (Eq. 11).  Order: score descending on the fp32 bit pattern, ties to the
 * lower candidate index.  Heads that are not triggered keep everything.  Output
 * idx[(b*H+h)*kept_stride + r], r < kept, ascending candidate indices; kept_out[b*H+h] their
 * count (may be NULL).  Does not change the cache. */
HACK_API hack_status_t hack_select(hack_cache_t* cache, int32_t layer, int32_t scale, const float* scores,
                          int32_t* idx, int32_t* kept_out, void* stream);

/* Gather the surviving K/V rows (Eq. 10-11) into the layer's ragged cache in ascending original
 * position; evicted entries are gone for good.  `idx` as written by hack_select for this step;
 * each head's row must hold exactly hack_step_info's kept_c / kept_s entries.  In place.
 * With merge_last, at the last scale, a contextual head that evicts then folds every discarded
 * entry e into the retained entry c whose key has the largest cosine similarity to k_e (lowest
 * index among equals) with weight w_e = max(similarity, 0):
 *   k_c <- (k_c + sum w_e k_e) / (1 + sum w_e), v_c likewise, rounded to bf16
 * (the paper states the operation in one sentence; measure, weights and the treatment of V are this
 * library's reading).  hack_scale_step does the same. */
HACK_API hack_status_t hack_compact(hack_cache_t* cache, int32_t layer, int32_t scale, const int32_t* idx,
                           const void* k_new, const void* v_new, void* stream);

/* O = Softmax(sm_scale * Q K^T) V over the head's compacted cache, all N_k queries, no mask
 * inside the scale (Eq. 4 on the compressed cache).  Requires hack_compact for this scale;
 * completes the step (the layer then expects scale + 1). */
HACK_API hack_status_t hack_attend(hack_cache_t* cache, int32_t layer, int32_t scale, const void* q,
                          void* out, void* stream);

/* hack_attend that also returns the attention variance of every head (Eq. 6, offline head
 * classification): sigma[b*H + h] = sum_j Var_i A[i, j], A = Softmax(sm_scale * Q K^T) the attention
 * matrix of this step's queries (rows) over the head's cache as it stands (columns), Var the
 * population variance over the queries.  For Eq. 6 proper, create the cache with budgets >= T_K, so
 * that nothing is evicted, and call this at the last scale: A is then the N_K x T_K matrix of the
 * final generation step.  sigma: device, [batch*n_heads] floats, written on `stream`.  State rules
 * of hack_attend.  UNSUPPORTED unless the cache is bf16 and the scale has at least 32 tokens (and
 * batch*n_heads*N_k >= 128): the statistics come from the tensor-core attention kernel. */
HACK_API hack_status_t hack_attend_variance(hack_cache_t* cache, int32_t layer, int32_t scale, const void* q,
                                   void* out, float* sigma, void* stream);

/* Head types from the variance matrix (Eq. 6 and the paragraph after it): all n_layers*n_heads heads
 * are ranked by sigma (host, row-major [n_layers][n_heads], already averaged over the samples) and
 * the round(alpha * n_layers * n_heads) lowest are marked contextual (1), the others structural (0);
 * equal values rank by (layer, head).  head_is_contextual: host, [n_layers*n_heads], the mask
 * hack_config_t takes.  Host only.  INVALID_ARG unless 0 <= alpha <= 1 and sigma is finite. */
HACK_API hack_status_t hack_classify_heads(const double* sigma, int32_t n_layers, int32_t n_heads, double alpha,
                                  uint8_t* head_is_contextual);

/* The whole step for one (layer, scale): score -> select -> compact -> attend; heads whose
 * candidate count does not exceed their budget skip scoring and selection and keep everything
 * (section "KV Cache Compression for VAR": compress whenever the length exceeds the budget).
 * bf16 caches: at most two launches (one cluster launch that scores, selects and compacts, one
 * attention launch that also appends the rows of heads which keep the whole new scale); a step that
 * merges takes seven, one whose candidate lists are beyond a cluster the launches of the stages.  The
 * attention of heads that do not depend on the compression runs beside it; steps whose heads fit into
 * shared memory are one launch (fp32 caches too).  `stream` orders everything (also inside a stream
 * capture). */
HACK_API hack_status_t hack_scale_step(hack_cache_t* cache, int32_t layer, int32_t scale, const void* q,
                              const void* k, const void* v, void* out, void* stream);

/* Scores without any allocation (the paper has no counterpart: this exists for deployment).
 * For callers that cannot allocate device memory when they need scores - a server whose pool
 * already owns all of HBM, so cudaMalloc would fail, or a decode loop that cannot afford the
 * device-wide synchronisation cudaMalloc/cudaFree imply - and therefore cannot create a cache.
 * Computes what hack_score computes, on dense caller-owned device tensors:
 *   q       [n_rows, n_queries, head_dim]   (n_rows = batch*heads, dtype as given)
 *   k_cand  [n_rows, n_cand, head_dim]      all candidate keys of each row, in candidate order
 *   scores  [n_rows, score_stride] fp32, score_stride >= n_cand; columns j < n_cand are written.
 * sm_scale 0 selects 1/sqrt(head_dim).  Runs on the calling thread's current device.
 * Intermediates live in a fixed array inside the library's device image (about 8.3 MiB, held
 * by every GPU that loads the library until the process exits), hence the limits
 * n_rows <= 512 and n_rows*n_cand <= 65536; larger sizes return HACK_ERR_UNSUPPORTED.
 * No cudaMalloc, cudaFree or other allocating call is made.  The first call on a device is a
 * set-up call: it resolves the array's address (cudaGetSymbolAddress) and, because CUDA loads a
 * module's device image lazily, it is also the moment the driver reserves those 8.3 MiB on that
 * device and loads the kernels, those of every size and dtype.  Make it at start-up, before the caller's own pool claims the rest of the memory and
 * before any stream capture; every later call on that device leaves the device's memory as it is.
 * All calls share the array: calls that overlap on the GPU race, so keep them on one stream or
 * order them yourself.  Only enqueues; does not synchronise. */
HACK_API hack_status_t hack_score_noalloc(const void* q, const void* k_cand, float* scores,
                                          int32_t n_rows, int32_t n_queries, int32_t n_cand,
                                          int32_t score_stride, int32_t head_dim, int32_t dtype,
                                          int32_t n_obs, float sm_scale, void* stream);

/* Same step with HOST buffers (pinned memory, or the copies are not asynchronous): Q/K/V go to
 * library-owned device staging, the step runs on `stream`, O comes back; the call returns without
 * synchronising, and once `stream` has been synchronised out_host is complete.  The uploads and
 * the download run on two private streams with three staging sets, so the upload of the next
 * call overlaps this call's kernels; the host buffers of a call must stay valid until `stream`
 * has passed that call.  The staging sets and streams are created by the first such call on a
 * cache (make it outside any stream capture). */
HACK_API hack_status_t hack_scale_step_host(hack_cache_t* cache, int32_t layer, int32_t scale,
                                   const void* q_host, const void* k_host, const void* v_host,
                                   void* out_host, void* stream);

/* Stored length of every (batch, head) of a layer, host_out[b*H+h].  Host bookkeeping only. */
HACK_API hack_status_t hack_get_lengths(const hack_cache_t* cache, int32_t layer, int32_t* host_out);
/* Test inspection (synchronises the device): copy one head's stored rows to host memory.
 * which = 0: K rows, 1: V rows (dtype of the cache, [len, head_dim]); 2: original global token
 * positions (int32 [len]).  `bytes` is the size of host_out and must cover the stored length. */
HACK_API hack_status_t hack_read_head(hack_cache_t* cache, int32_t layer, int32_t b, int32_t h,
                             int32_t which, void* host_out, size_t bytes);

/* KV bytes (K and V rows only): currently stored, the peak since init/reset, and reserved. */
HACK_API hack_status_t hack_kv_bytes(const hack_cache_t* cache, size_t* live, size_t* peak, size_t* reserved);
/* Number of the library's own kernel launches enqueued through this cache since init. */
HACK_API hack_status_t hack_launch_count(const hack_cache_t* cache, uint64_t* launches);
/* Per-stage device timing for benchmarks.  enable != 0: from now on every stage's launches are
 * bracketed by two CUDA events on the caller's stream (a few microseconds of overhead per
 * stage); accumulators are cleared.  Synchronises the device. */
HACK_API hack_status_t hack_stage_timing(hack_cache_t* cache, int32_t enable);
/* Synchronises the device and returns the accumulated device time in ms and the number of kernel
 * launches per stage since timing was enabled: [0] score, [1] select, [2] compact, [3] attend.  In
 * hack_scale_step on a bf16 cache scoring, selection and compaction are one launch, counted under
 * [0], and a step that is one launch altogether is counted under [3]. */
HACK_API hack_status_t hack_stage_times(hack_cache_t* cache, double* ms, uint64_t* launches);
/* Synchronises `stream`, then reports the device status word: HACK_OK, or HACK_ERR_TIMEOUT if a
 * bounded device-side wait gave up (the word is cleared by the call). */
HACK_API hack_status_t hack_poll_status(hack_cache_t* cache, void* stream);
/* Limit, in SM clock cycles, of every bounded device-side wait (mbarrier waits of the tensor-core
 * kernels) in launches made through this cache from now on; 0 restores the default of about one
 * second.  What counts is a launch's own time, not that in which it waits for the launch ahead of it
 * in the stream; waits for a whole unit of work of the attention get the limit once per wait in it.
 * A wait that outlasts the limit raises the status word (hack_poll_status then returns
 * HACK_ERR_TIMEOUT), the CTA drains what it has in flight, frees its tensor memory and returns; the
 * results of that launch are undefined and the cache should be reset.  Meant for tests of that path
 * (a limit of a few cycles makes the first wait that is not already satisfied give up) and for
 * callers that want a tighter bound than a second.  INVALID_ARG for a negative limit. */
HACK_API hack_status_t hack_set_wait_limit(hack_cache_t* cache, int64_t cycles);
/* 1 if this library is the checked build (compiled with HACK_DEBUG_CHECKS), else 0.  The checked
 * build stands in for a memory checker: its kernels compare every ragged index they form with its
 * bound, skip the access on a violation and put the site's code into the status word
 * (hack_poll_status then returns HACK_ERR_STATE), and its planes carry one guard row behind the
 * rows of every (layer, batch, head). */
HACK_API int32_t hack_debug_build(void);
/* Checked build only: synchronises the device and counts the guard rows (K, V and position planes)
 * that no longer hold their pattern; hack_last_error() names the first.  UNSUPPORTED in the normal
 * build. */
HACK_API hack_status_t hack_debug_check(hack_cache_t* cache, int32_t* violations);
/* ------------------------------------------------------------------------------------------------
 * From a layer's projections to its steps: rotary positions and norms of queries and keys.
 *
 * A tensor here is [batch, heads, tokens, head_dim] with any strides but the last, which is 1: a view
 * of the projection's output [batch, tokens, heads, head_dim] as well as the dense layout of the steps.
 * Every row starts on a 16-byte boundary (base address and strides).  head_dim is 64 or 128, dtype
 * HACK_F32 or HACK_BF16; sums and products are fp32, rounded once.  Nothing is allocated or kept.
 * An output may be its input (same address, same strides); other overlaps are not allowed.
 * A call with no tokens does nothing.  `device` is made current for the call.  Arrays of numbers (positions,
 * weights, gains, lengths) start on a multiple of their elements' size.
 * ---------------------------------------------------------------------------------------------- */
typedef struct { int64_t batch, head, token; } hack_strides_t;   /* in elements */

enum { HACK_ROPE_HALF = 0,    /* element i of the rotated part pairs with element i + rotary_dim / 2 */
       HACK_ROPE_PAIRS = 1 }; /* element 2i pairs with element 2i + 1 */
/* Frequencies of contexts longer than the trained one (D: dimensions an axis rotates, factor: the stretch) */
enum { HACK_ROPE_PLAIN = 0,   /* f_i = base^(-2i / D) */
       HACK_ROPE_LINEAR = 1,  /* f_i / factor */
       HACK_ROPE_BASE = 2,    /* base grows to base * factor^(D / (D - 2)) */
       HACK_ROPE_BANDS = 3 }; /* pairs that turn more than turns_fast times within trained_length stay as they are, those
                                 that turn less than turns_slow times are divided by factor, a linear ramp over the pair
                                 numbers between; cosine and sine are multiplied by 1 + 0.1 ln(factor) */
#define HACK_ROPE_MAX_PAIRS 64

/* A rotation.  Plain data, filled by hack_rope_plan (or by the caller); nothing on a device belongs to it.
 * Pair i of a token at position p turns by the angle p * freq[i], formed in 64 bits:
 *   y0 = gain * (x0 cos - x1 sin),  y1 = gain * (x0 sin + x1 cos).
 * With two axes a token has two positions (a grid's row and column): the first half of the pairs turns by the
 * first, the second half by the second.  Elements from rotary_dim on pass unchanged. */
typedef struct {
  int32_t head_dim, rotary_dim, layout, axes;
  float gain;
  int32_t reserved;
  double freq[HACK_ROPE_MAX_PAIRS];
} hack_rope_plan_t;

/* Host only.  rotary_dim: a multiple of 2 * axes in 2..head_dim.  turns_fast, turns_slow: 0 selects 32 and 1. */
HACK_API hack_status_t hack_rope_plan(int32_t head_dim, int32_t rotary_dim, int32_t layout, int32_t axes, double base,
                                      int32_t scaling, double factor, int64_t trained_length, double turns_fast,
                                      double turns_slow, hack_rope_plan_t* out);

typedef struct {
  int32_t device, dtype, batch, n_heads, n_tokens;
  int32_t transpose;          /* 1: by the opposite angles, which is the gradient of the rotation */
  int32_t positions_f32;      /* positions: 0 int32, 1 fp32; [batch, n_tokens, axes] */
  int32_t reserved;
  int64_t positions_stride;   /* elements from one batch element's positions to the next's; 0: shared */
  hack_strides_t x, y;
} hack_rope_args_t;
/* y = x with the rotation of its token's position. */
HACK_API hack_status_t hack_rope(const hack_rope_plan_t* plan, const hack_rope_args_t* args, const void* x, void* y,
                                 const void* positions, void* stream);

enum { HACK_NORM_NONE = 0,
       HACK_NORM_RMS = 1,     /* x / sqrt(mean x^2 + eps) */
       HACK_NORM_L2 = 2 };    /* x / max(|x|, eps); eps is one whose fp32 reciprocal is finite */
typedef struct {
  int32_t device, dtype, batch, n_heads, n_kv_heads, n_tokens, head_dim;
  int32_t norm;               /* HACK_NORM_*, of every row of q and k on its own */
  float eps;
  int32_t positions_f32;
  int64_t positions_stride;
  hack_strides_t q, k, v, q_out, k_out, v_out;
} hack_qkv_args_t;
/* Queries and keys normalised per head, multiplied by a weight per channel (fp32 [head_dim], may be NULL) and a gain
 * per head (fp32 [n_heads] or [n_kv_heads], may be NULL), and rotated (plan and positions NULL: not); values
 * copied: one pass from the projection's output to what hack_scale_step takes.  v and v_out may both be NULL, and so
 * may k and k_out. */
HACK_API hack_status_t hack_qk_norm_rope(const hack_rope_plan_t* plan, const hack_qkv_args_t* args, const void* q, const void* k,
                                         const void* v, void* q_out, void* k_out, void* v_out, const void* positions,
                                         const float* q_weight, const float* k_weight, const float* q_gain,
                                         const float* k_gain, void* stream);

/* hack_scale_step from the projections of a layer: hack_qk_norm_rope into buffers of the cache's own (created by the first
 * call on a cache, which must be outside any stream capture), then the step.  args describe the inputs, with as many
 * key as query heads, n_tokens = N_k of the scale and the cache's batch, heads, head_dim, dtype and device; its output strides are
 * not looked at.  out: dense [batch, n_heads, N_k, head_dim]. */
HACK_API hack_status_t hack_scale_step_qkv(hack_cache_t* cache, int32_t layer, int32_t scale, const hack_rope_plan_t* plan,
                                           const hack_qkv_args_t* args, const void* q, const void* k, const void* v,
                                           const void* positions, const float* q_weight, const float* k_weight,
                                           const float* q_gain, const float* k_gain, void* out, void* stream);

/* ------------------------------------------------------------------------------------------------
 * Caches of 4 bits: rows of keys and values in a little over a quarter of their bf16 bytes, and the
 * attention that reads them.
 *
 * A row of head_dim elements is blocks of 16 that share a scale s, one of the 256 values
 * (1 + m/8) 2^(e-20), byte 8 e + m: the smallest with 7 s >= the block's largest |x|, or the largest
 * of all.  An element is c * s, c = x / s rounded to the nearest whole number (ties to even) and
 * limited to -7..7; byte j of a row holds c + 8 of element 2j in its low and of element 2j + 1 in its
 * high half.  c * s has no more than seven significant bits: bf16 holds it exactly.  NaN is stored as
 * 0, what is beyond 26 880 as that.
 * The planes are the caller's device buffers, 16-byte aligned: codes [rows, head_dim / 2] and scales
 * [rows, head_dim / 16] bytes of K and of V.  Head i = b * n_kv_heads + h owns rows
 * [first, first + cap), first = row_off[i] (device) or, row_off NULL, i * cap.  A head whose rows are
 * not all among the planes' `rows` counts as one without any; heads may share rows that are only read,
 * those appended to must be a head's own.  How many of them are in use is the caller's to keep, on the
 * device, so that a captured graph can be replayed with other lengths: lens, int32
 * [batch * n_kv_heads].  The library only reads it; a length below 0 counts as 0, one beyond cap as cap.
 * new_lens (device, int32 [batch], may be NULL): of a padded batch, how many of the call's tokens each
 * batch element really has; the others are not read, and their outputs are left as they were.
 * ---------------------------------------------------------------------------------------------- */
typedef struct {
  int32_t device, batch, n_kv_heads, head_dim;   /* head_dim 64 or 128 */
  int32_t cap, reserved;                         /* cap: at most 2^31 - 512 */
  int64_t rows;                                  /* of each plane */
  const int64_t* row_off;
  void *k_codes, *v_codes, *k_scales, *v_scales;
} hack_kv4_t;

typedef struct {
  int32_t dtype, n_tokens;
  hack_strides_t k, v;
} hack_kv4_rows_t;
/* Rows k, v [batch, n_kv_heads, n_tokens, head_dim] join behind the lens rows of every head; rows that would
 * not fit are dropped.  The step after it is hack_kv4_attend with `appended`, and then lens += n_tokens, by
 * the caller. */
HACK_API hack_status_t hack_kv4_append(const hack_kv4_t* kv, const hack_kv4_rows_t* rows, const void* k, const void* v,
                                       const int32_t* lens, const int32_t* new_lens, void* stream);
/* The values of rows first[i] .. first[i] + n_tokens - 1 of every head, in dense or strided tensors (k, v of
 * `rows` are the outputs' strides); rows outside [0, cap) give zeros. */
HACK_API hack_status_t hack_kv4_read(const hack_kv4_t* kv, const hack_kv4_rows_t* rows, void* k_out, void* v_out,
                                     const int32_t* first, void* stream);
/* The rows that a layer of a cache holds (every head its own number of them, hack_get_lengths) join a 4-bit
 * cache of the same batch, heads and head_dim behind its lens rows. */
HACK_API hack_status_t hack_store_kv4(hack_cache_t* cache, int32_t layer, const hack_kv4_t* kv, const int32_t* lens,
                                      void* stream);

typedef struct {
  int32_t dtype;                 /* of q and out */
  int32_t n_heads, n_queries;    /* n_heads a multiple of n_kv_heads: query head h reads stored head h / (n_heads / n_kv_heads) */
  int32_t max_len;               /* no head attends over more rows (launches are planned for it): a longer one's length, which
                                    the queries' positions go by as well, counts as this */
  int32_t appended;              /* 1: the n_queries (or new_lens[b]) rows behind lens count too: those just appended */
  int32_t causal;                /* 1: query i of n, at position length - n + i, sees no later rows */
  int32_t window, n_sink;        /* window > 0: of the rows up to its position a query sees the last `window` (itself
                                    counted) and the first n_sink */
  float sm_scale;                /* 0 selects 1 / sqrt(head_dim) */
  int32_t wait_polls;            /* limit of the device-side waits, in polls of a barrier; 0: most of a second.  For tests: a
                                    limit of 1 makes the first wait that is not already satisfied give up */
  int64_t workspace_bytes;       /* size of the workspace given */
  hack_strides_t q, out;
  int32_t form;                  /* 0: the library chooses its kernel by the sizes; HACK_KV4_FEW or HACK_KV4_MANY: that one, for
                                    measurements and tests */
  int32_t reserved;
} hack_kv4_attend_t;
enum { HACK_KV4_FEW = 1,         /* 8 or 16 query rows a CTA, any type */
       HACK_KV4_MANY = 2 };      /* tiles of 128 query rows, bf16 */
/* Device memory that a call of these sizes needs (it may be 0); it depends on the struct's sizes alone. */
HACK_API hack_status_t hack_kv4_workspace(const hack_kv4_t* kv, const hack_kv4_attend_t* args, size_t* bytes);
/* O = Softmax(sm_scale Q K^T) V over the stored rows that a query sees; a query that sees none gets zeros, one with a NaN
 * that sees any NaN.  Logits, softmax and sums are fp32 numbers; in bf16 calls a probability p is rounded to bf16 once, for the
 * product with the values and for the sum it is divided by alike, which moves a result by at most 2^-8 sum p |v - out| besides
 * its own rounding (2^-8 |out|).  workspace: 16-byte aligned, its contents need no preparation and mean nothing after the call;
 * calls that may overlap on the GPU need workspaces of their own. */
HACK_API hack_status_t hack_kv4_attend(const hack_kv4_t* kv, const hack_kv4_attend_t* args, const void* q, void* out,
                                       const int32_t* lens, const int32_t* new_lens, void* workspace, void* stream);

/* Synchronises `stream`, then reports whether a bounded device-side wait of hack_kv4_attend on this device gave up since the
 * last call: HACK_OK or HACK_ERR_TIMEOUT (what that call wrote is undefined).  Nothing else reports it: hack_poll_status is about
 * a cache's own steps.  A loop of calls asks once where it reads its results. */
HACK_API hack_status_t hack_kv4_poll_status(int32_t device, void* stream);

/* Text of the calling thread's last error; never NULL. */
HACK_API const char* hack_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* HACK_H_ */
