/*
 * mcce -- cache-conditional MoE decode step for many independent token streams (NVIDIA B200, sm_100a).
 *
 * C ABI of libmcce.so.  Plain pointers and sizes only; every pointer is marked HOST or DEVICE.
 * The method is "Mixture of Cache-Conditional Experts" (arXiv 2412.00099); the citations below name
 * the equation, section or algorithm of that paper which defines each operation.
 *
 * Notation (paper, Sec. 2.1 / 2.2 / 3.3): N = E routed experts per layer, top-K selection, top-J
 * guaranteed experts, cache set C of `cache_capacity` experts per (stream, layer), promotion strength
 * lambda, logit range Delta_avg.  S independent token streams, L MoE layers, hidden size d, expert
 * intermediate size I.  Streams and layers are independent of one another; tokens of one stream are
 * sequential because the cache state carries over.
 *
 * Ownership: the caller owns every buffer, including the workspace, and keeps them alive until
 * mcce_destroy.  The library allocates no device memory and creates no streams (except the three internal
 * streams of the pipelined entry points).  Weights are borrowed.
 * Errors: every call returns 0 on success or a negative MCCE_E* code; nothing throws, aborts or prints.
 * Kernel launches are asynchronous on the given stream unless a function says that it synchronises.
 * A context is not thread-safe; distinct contexts are independent.
 */
#ifndef MCCE_H_
#define MCCE_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
  MCCE_OK = 0,
  MCCE_EINVAL = -1,   /* bad argument or unsupported configuration                      */
  MCCE_ENOSPC = -2,   /* workspace too small                                            */
  MCCE_ESTATE = -3,   /* weights not set, or a counter would overflow (reset needed)    */
  MCCE_ECUDA = -4,    /* a CUDA call failed; see mcce_last_cuda_error                   */
  MCCE_ETIMEOUT = -5, /* a bounded wait inside a kernel gave up: the launch it happened in is incomplete (results,
                         cache state and internal buffers), the CUDA context stays usable; mcce_reset brings the
                         mcce context back to a defined state                                             */
  MCCE_ELIMIT = -6,   /* problem larger than the fixed array of mcce_route_trace_static   */
  MCCE_EINDEX = -7,   /* an expert id outside [0, E) reached the grouping pass (the pair was skipped), or a
                         check of the checked mode failed: a grouping position outside [0, S*K), more than C
                         resident experts, or two resident experts with the same recency key               */
  MCCE_ENONFINITE = -8 /* checked mode: a router logit was NaN or infinite                               */
};

enum { MCCE_F32 = 0, MCCE_BF16 = 1, MCCE_E4M3 = 2 /* rows of mcce_dispatch only */ };
enum { MCCE_DELTA_RUNNING = 0, MCCE_DELTA_FIXED = 1 };
enum { MCCE_FFN_AUTO = 0, MCCE_FFN_SIMT = 1, MCCE_FFN_TENSOR = 2 };
/* How the router's ranking r is changed in favour of cached experts (Sec. 3):
 * CACHE_PRIOR  Eq. 7, the paper's main method: rank by z' = z + lambda*Delta_avg*m~_t;
 * MAX_RANK     Algorithm 1: promote(r[:J]; promote(r[:M] ∩ C; r)) with M = max_rank;
 * CUMSUM       Algorithm 2: the same with M = the smallest number of top-ranked experts whose router
 *              probabilities sum to at least cum_threshold. */
enum { MCCE_RERANK_CACHE_PRIOR = 0, MCCE_RERANK_MAX_RANK = 1, MCCE_RERANK_CUMSUM = 2 };

typedef struct mcce_ctx mcce_ctx; /* opaque; host memory owned by the library */

typedef struct {
  int32_t n_layers;       /* L >= 1                                                              */
  int32_t n_experts;      /* E = N routed experts per layer, 1..256                              */
  int32_t top_k;          /* K, 1..min(E,16)                                                     */
  int32_t top_j;          /* J, 0..K: router's top-J experts are always selected (Sec. 3.3)      */
  int32_t n_shared;       /* always-on experts per layer, weight 1, never cached, >= 0           */
  int32_t d_model;        /* d, multiple of 8                                                    */
  int32_t d_ff;           /* I, multiple of 8                                                    */
  int32_t cache_capacity; /* C >= 1 experts per (stream, layer); C >= E means nothing is evicted */
  int32_t n_streams;      /* S >= 1                                                              */
  float lambda;           /* promotion strength of Eq. 7, finite, >= 0 (paper: [0,1])            */
  int32_t delta_mode;     /* MCCE_DELTA_RUNNING: Delta_avg is the cumulative mean, per (stream,
                             layer), of max(z)-min(z) including the current token (Eq. 8);
                             MCCE_DELTA_FIXED: per-layer constants given to mcce_set_router
                             (appendix "Logit Range Estimation")                                 */
  int32_t renorm;         /* 1: weights renormalised over the K selected experts (Sec. 2.1)      */
  int32_t hidden_dtype;   /* MCCE_F32 or MCCE_BF16                                               */
  int32_t weight_dtype;   /* expert weights; must equal hidden_dtype                             */
  int32_t ffn_impl;       /* MCCE_FFN_AUTO picks the tensor-core path when it applies            */
  int32_t device;         /* CUDA device ordinal                                                 */
  int32_t rerank_mode;    /* MCCE_RERANK_*; lambda / delta_mode only matter for CACHE_PRIOR      */
  int32_t max_rank;       /* M of Algorithm 1, 0..E (MAX_RANK only)                              */
  float cum_threshold;    /* p of Algorithm 2, >= 0 (CUMSUM only)                                */
  int32_t track_lifetime; /* 1: record how long experts stay cached (mcce_lifetime_stats)         */
  int32_t route_impl;     /* MCCE_ROUTE_AUTO (0) picks per launch what was measured faster;
                             MCCE_ROUTE_TWO_KERNELS: logits kernel, then routing tail;
                             MCCE_ROUTE_FUSED: the single cooperative kernel wherever it can run.  That kernel
                             adds the parts of its split reduction of Eq. 3 in the order in which they arrive,
                             so the last bit of a logit (and with it a selection between two experts whose
                             logits are equal to within rounding) can differ between runs; the two-kernel path
                             adds them in a fixed order.  The deterministic and the checked mode never use it */
  int32_t deterministic;  /* 1: repeated runs give identical bits (the paper's runs are deterministic, Sec. 4.1):
                             y = sum_k w_k E_k(x) + shared experts is added in slot order on every path (the
                             tensor-core path then writes one fp32 row per (stream, slot) and sums them in a
                             second pass instead of adding into y with atomics), and the router logits come
                             from the two-kernel path                                                       */
  int32_t checked;        /* 1: checked mode.  Every routing launch is followed by kernels that verify the
                             logits (finite), the cache state (at most C resident experts per (stream,
                             layer), distinct recency keys) and every grouping pass (positions inside
                             [0, S*K)); a violation is recorded and reported by mcce_cache_stats as
                             MCCE_ENONFINITE / MCCE_EINDEX.  Costs a few small launches per call          */
} mcce_config;

typedef struct {
  int64_t steps;       /* (stream, token, layer) routing steps                                   */
  int64_t selections;  /* K * steps, denominator of Eq. 4                                        */
  int64_t misses;      /* selected experts absent from the cache as it was before the token      */
  int64_t cold_misses; /* misses on experts that had never been resident (compulsory misses)     */
} mcce_stats;

/* Bytes of DEVICE workspace mcce_create needs for this configuration (0 if the config is invalid). */
size_t mcce_workspace_bytes(const mcce_config* cfg /*HOST*/);

/* Validates cfg, carves `workspace` (DEVICE, 256-byte aligned, >= mcce_workspace_bytes) into the
 * state arrays, zeroes them (cache empty) and returns a context.  Synchronises the device. */
int mcce_create(const mcce_config* cfg /*HOST*/, void* workspace /*DEVICE*/, size_t workspace_bytes,
                mcce_ctx** out /*HOST*/);
int mcce_destroy(mcce_ctx* ctx);

/* Router G of Eq. 3: z = W_r[l] x.  Wr: DEVICE fp32 [L,E,d], row-major.  fixed_delta: DEVICE fp32 [L],
 * required iff delta_mode == MCCE_DELTA_FIXED, else may be NULL.  Borrowed. */
int mcce_set_router(mcce_ctx* ctx, const float* Wr, const float* fixed_delta);

/* Experts E_i of Eq. 1 as SwiGLU: E_i(x) = W_d (silu(W_g x) * (W_u x)).  DEVICE, weight_dtype,
 * row-major: Wg, Wu [L,E,I,d]; Wd [L,E,d,I]; shared experts shWg, shWu [L,n_shared,I,d],
 * shWd [L,n_shared,d,I] (NULL when n_shared == 0).  Borrowed. */
int mcce_set_experts(mcce_ctx* ctx, const void* Wg, const void* Wu, const void* Wd, const void* shWg,
                     const void* shWu, const void* shWd);

/* Root-mean-square norm in front of every layer's router and experts in mcce_decode_step_chained (mcce_rmsnorm's
 * formulas).  weight: DEVICE fp32 [L,d], 16-byte aligned, borrowed; eps finite, >= 0; d at most
 * MCCE_NORM_MAX_D.  NULL: no norm (the state after mcce_create). */
int mcce_set_norm(mcce_ctx* ctx, const float* weight, float eps);

/* Empties every cache, or loads an initial cache content (Sec. 4.8 "Impact of Initial Cache State"):
 * init_order HOST int32 [L,S,C], resident experts most-recently-used first, -1 padding; NULL = empty.
 * These entries count as older than anything touched later.  Counters are zeroed.  The running
 * Delta statistics are kept iff keep_delta_stats != 0, or replaced when delta_sum (HOST fp32 [L,S])
 * is given together with delta_count (tokens it was summed over).  Synchronises. */
int mcce_reset(mcce_ctx* ctx, const int32_t* init_order, int keep_delta_stats, const float* delta_sum,
               int64_t delta_count);

/* n_steps tokens of routing for every (stream, layer): Eq. 3 logits (or given logits), Eq. 8 range
 * statistic, mask m~_t = cache OR top-J, Eq. 7 promotion z' = z + lambda*Delta_avg*m~_t, top-K of z'
 * (ties to the lower expert index), weights = softmax of the UNMODIFIED z over the selected experts
 * (Sec. 3.3), Eq. 4 miss counting against the cache as it was before the token, LRU update in which
 * the selected expert with the higher router weight counts as older (Sec. 4.2).
 *   hidden     DEVICE hidden_dtype [n_steps,L,S,d], or NULL
 *   logits_in  DEVICE fp32 [n_steps,L,S,E], or NULL; exactly one of the two is non-NULL
 *   sel_idx    DEVICE int32 [n_steps,L,S,K] out, rank order of z'
 *   sel_w      DEVICE fp32  [n_steps,L,S,K] out
 *   logits_out DEVICE fp32  [n_steps,L,S,E] out, optional: the logits the decision was taken on
 * When E is a multiple of 4, rows of logits are read and written four floats at a time: logits_in and
 * logits_out must then be 16-byte aligned (MCCE_EINVAL otherwise; 4-byte alignment suffices for other E).
 */
int mcce_route_step(mcce_ctx* ctx, int32_t n_steps, const void* hidden, const float* logits_in,
                    int32_t* sel_idx, float* sel_w, float* logits_out, void* cuda_stream);

/* Eq. 1 for one token of every (stream, layer): groups the (stream, slot) pairs by expert, runs the
 * SwiGLU experts group by group and combines y = sum_k w_k E_sel_k(x) (slot order) + shared experts.
 *   hidden DEVICE hidden_dtype [L,S,d]; sel_idx DEVICE int32 [L,S,K]; sel_w DEVICE fp32 [L,S,K];
 *   y DEVICE fp32 [L,S,d] out.
 * With bf16 weights the intermediate silu(g)*u is rounded to bf16 before the down projection.  On the
 * tensor-core path the K + n_shared terms of a stream are added into y with fp32 atomic adds in no fixed
 * order, so the last bits of y may differ between runs, unless the configuration sets `deterministic`
 * (the fp32-pipe path always sums in slot order).
 * An entry of sel_idx outside [0, E) (padding, an uninitialised buffer) is skipped: the pair contributes
 * nothing to y, and the next mcce_cache_stats reports MCCE_EINDEX. */
int mcce_moe_forward(mcce_ctx* ctx, const void* hidden, const int32_t* sel_idx, const float* sel_w,
                     float* y, void* cuda_stream);

/* One token in sequential-layer mode: the layers are chained through a residual stream instead of being
 * independent, as in a real decoder (the paper changes nothing in the forward pass but the ranking, Sec. 2.2).
 * For l = 0..L-1: route layer l on its input x_l, run its experts, x_{l+1} = x_l + y_l rounded to the hidden
 * dtype.  Without mcce_set_norm there is no normalisation layer: the logit scale may drift with depth, which the
 * per-layer Delta_avg absorbs.  With it, layer l routes and runs its experts on mcce_rmsnorm(x_l, weight[l]), as
 * pre-norm decoders do, and the residual stream x_l itself stays as it is.
 *   x0     DEVICE hidden_dtype [S,d]: input of layer 0        x_out DEVICE hidden_dtype [S,d]: output of layer L-1
 *   sel_idx DEVICE int32 [L,S,K], optional: the selections of every layer
 * Cache state, counters, Delta statistics and the miss trace advance exactly as with mcce_route_step.  Launches
 * L rounds of the single-layer kernels on the stream (asynchronous).  On the tensor-core path the expert
 * outputs are summed with fp32 atomics, so x_{l+1} can differ in its last bit between runs, and with it,
 * rarely, a near-tie routing decision of a later layer. */
int mcce_decode_step_chained(mcce_ctx* ctx, const void* x0, void* x_out, int32_t* sel_idx, void* cuda_stream);

/* One whole decode step from HOST buffers: copies hidden [L,S,d] to the device, routes, runs the
 * experts and copies y [L,S,d] (and, if non-NULL, sel_idx [L,S,K]) back.  Staging lives in the
 * workspace.  hidden_host / y_host should be pinned.  Synchronises the stream before returning. */
int mcce_decode_step_host(mcce_ctx* ctx, const void* hidden_host, float* y_host, int32_t* sel_idx_host,
                          void* cuda_stream);

/* The same decode step, pipelined over successive tokens.  Routing needs only the hidden states of its token and
 * the cache state that the previous token's routing left (Sec. 3.3: the mask m_t is the cache after token t-1),
 * not the previous token's experts; so routing, grouping and the row copy of step t+1 run on an internal stream
 * while the expert kernels of step t, which stream all the weights, still run on cuda_stream.  Two sets of
 * buffers ("slots") alternate.
 *
 * mcce_pipeline_submit_host enqueues, without waiting, the upload of hidden_host [L,S,d] on an internal copy-in
 * stream, the step, and the download of y [L,S,d] (and sel_idx [L,S,K] if non-NULL) on an internal copy-out
 * stream once the step has finished.  A call blocks only if the step submitted two calls earlier has not yet
 * left the device, so the upload of token t+1 and the download of token t-1 also run while token t computes.
 * The host buffers of a submitted step must stay valid, and y_host must not be read, until mcce_pipeline_wait
 * (or the second following submit) returns.  hidden_host / y_host must be pinned for the copies to be
 * asynchronous.
 *
 * mcce_pipeline_submit is its twin for DEVICE buffers: hidden [L,S,d] (hidden_dtype), y [L,S,d] fp32 out, sel_idx
 * [L,S,K] int32 out or NULL.  Nothing is copied.  The library reads `hidden` on its internal stream, which does
 * not wait for cuda_stream: hidden must be complete when the call is made, or hidden_ready (a cudaEvent_t, may be
 * NULL) must mark its completion.  y and sel_idx are complete in cuda_stream order.  y is cleared on the internal
 * stream while the previous step may still compute: consecutive calls must use different y buffers, and neither
 * hidden nor y of a step may be touched by the caller until that step has finished on cuda_stream.
 *
 * The three internal streams and their events are the only CUDA objects the library creates (on the first
 * submit); it still allocates no device memory.  Always use the same cuda_stream per context, and call
 * mcce_pipeline_wait before using any other entry point of the context that routes or runs experts. */
int mcce_pipeline_submit_host(mcce_ctx* ctx, const void* hidden_host, float* y_host, int32_t* sel_idx_host,
                              void* cuda_stream);
int mcce_pipeline_submit(mcce_ctx* ctx, const void* hidden /*DEVICE*/, float* y /*DEVICE*/, int32_t* sel_idx /*DEVICE*/,
                         void* hidden_ready /*cudaEvent_t or NULL*/, void* cuda_stream);
/* Waits until every submitted step has finished (and, for host buffers, has been copied back). */
int mcce_pipeline_wait(mcce_ctx* ctx);

/* Eq. 4 counters, summed over streams: total and per layer (HOST [L], may be NULL).  Synchronises.
 * The counters are always written; the return value also carries what the kernels of this context recorded
 * since the last mcce_reset, in this order of precedence: MCCE_ETIMEOUT (a bounded wait gave up),
 * MCCE_EINDEX (an expert id out of range was skipped, or a check of the checked mode failed),
 * MCCE_ENONFINITE (checked mode: a non-finite logit). */
int mcce_cache_stats(mcce_ctx* ctx, mcce_stats* total /*HOST*/, mcce_stats* per_layer /*HOST*/);

/* Cache lifetimes (the statistic of the paper's Table 2): a lifetime is the number of tokens from the
 * token that loaded an expert into a (stream, layer) cache to the token that evicted it; experts still
 * resident are not counted.  total / per_layer (HOST, [L], may be NULL) receive {evictions, sum of
 * lifetimes, sum of squared lifetimes}; mean = sum/evictions, variance = sumsq/evictions - mean^2.
 * Needs track_lifetime = 1 in the configuration (MCCE_ESTATE otherwise).  Not part of the state that
 * mcce_get_cache_state exports.  Synchronises. */
typedef struct { int64_t evictions, sum, sum_sq; } mcce_lifetime;
int mcce_lifetime_stats(mcce_ctx* ctx, mcce_lifetime* total /*HOST*/, mcce_lifetime* per_layer /*HOST*/);

/* Per-token miss trace (the data behind the paper's hit / miss timelines of Sec. 4.6): while a buffer is set,
 * every routed token writes one word per (layer, stream) whose bit k says that the k-th selected expert was
 * not in the cache.  trace: DEVICE uint32 [capacity_tokens, L, S], caller-owned; tokens beyond the capacity
 * are not recorded; recording restarts at entry 0 when the buffer is set and after mcce_reset.  NULL with
 * capacity 0 turns it off. */
int mcce_set_miss_trace(mcce_ctx* ctx, uint32_t* trace, int64_t capacity_tokens);

/* Logit range from a calibration set (appendix "Logit Range Estimation": Delta_avg estimated once over a
 * calibration set instead of during inference).  After some tokens have been routed in MCCE_DELTA_RUNNING
 * mode, writes for every layer the mean over its streams of the running estimate of Eq. 8,
 *   delta[l] = (1/S) sum_s sum_range[l][s] / tokens,
 * accumulated in double precision and rounded once to fp32: the constants to hand to mcce_set_router of a
 * context in MCCE_DELTA_FIXED mode.  delta HOST fp32 [L].  MCCE_ESTATE if no token has been routed yet.
 * Synchronises. */
int mcce_calibrate_delta(mcce_ctx* ctx, float* delta /*HOST*/);

/* Canonical cache state: order HOST int32 [L,S,C] most-recently-used first, -1 padded; optional
 * ever HOST uint8 [L,S,E]; delta_sum HOST fp32 [L,S] and *delta_count (optional).  Synchronises. */
int mcce_get_cache_state(mcce_ctx* ctx, int32_t* order, uint8_t* ever, float* delta_sum,
                         int64_t* delta_count);

/* Result of the expert-grouping pass of the last mcce_moe_forward (histogram, scan, stable scatter):
 * offsets HOST int32 [L,E+1]; perm HOST int32 [L,S*K], perm[l][pos] = s*K+slot of the pair placed at
 * pos, pairs of one expert contiguous and in increasing (s,slot) order.  Synchronises. */
int mcce_get_grouping(mcce_ctx* ctx, int32_t* offsets, int32_t* perm);

/* Belady's optimal eviction (Sec. 4.8 "Optimal Cache Eviction") replayed on a recorded selection trace: the
 * lossless bound that LRU cannot beat and that the paper's lossy rerouting can.  For every (stream, layer)
 * and every capacity the trace is replayed from an empty cache; on a miss the expert is inserted, and while
 * the cache is over capacity the resident expert whose next use lies farthest ahead is evicted, never one
 * the current token itself selects.  Context-free.
 *   sel_trace  DEVICE int32 [n_tokens, L, S, K]: the sel_idx output of mcce_route_step (K distinct experts)
 *   capacities DEVICE int32 [n_capacities], each >= K
 *   next_use_scratch DEVICE int32 [n_tokens, L, S, K], overwritten
 *   misses     DEVICE int64 [n_capacities, L, S] out
 * Asynchronous on the stream.  Capacities below K are the caller's error (the result is then undefined). */
int mcce_belady_replay(const int32_t* sel_trace, int32_t n_tokens, int32_t n_layers, int32_t n_streams,
                       int32_t n_experts, int32_t top_k, const int32_t* capacities, int32_t n_capacities,
                       int32_t* next_use_scratch, int64_t* misses, void* cuda_stream);

/* ---- operators around the experts ----------------------------------------------------------------------------
 * What a decoder layer needs on either side of its experts, and the gradients for training it.  Context-free: the
 * device that is current when the call is made is used, every buffer is the caller's, launches are asynchronous on
 * the stream, nothing is allocated and nothing is kept between calls; a call may be captured into a graph.  A
 * workspace is used only while the call's kernels run: calls that can overlap need one each.  Sums, statistics and
 * weights are held in fp32; every result is rounded once, to nearest even, to the type of its buffer.  Results do
 * not depend on the order in which threads run (no atomics on data): repeated calls give identical bits.  Where a call
 * does not say that an output may be one of its inputs, no output and no workspace may share memory with another tensor of the
 * call: refused, from the addresses, sizes and strides.  (Columns of one buffer, side by side, share none.)
 */

/* Rows for mcce_rmsnorm and its gradient.  Row strides (ld_*) are in elements, 0 means d; the columns of a row are
 * contiguous and rows of a tensor do not overlap. */
enum { MCCE_NORM_MAX_D = 16384 };
typedef struct {
  int64_t rows;          /* 0..2^31-1                                                                         */
  int32_t d;             /* columns, 1..MCCE_NORM_MAX_D                                                                 */
  int32_t dtype;         /* x, sum, out, and the gradients: MCCE_F32 or MCCE_BF16                             */
  int32_t add_dtype;     /* MCCE_F32 (what mcce_moe_forward returns) or dtype                                 */
  int32_t weight_dtype;  /* MCCE_F32 or dtype                                                                 */
  int32_t quant_group;   /* columns that share a scale: 32, 64, 128, or 0 for one scale per row               */
  float eps;             /* finite, >= 0                                                                      */
  int64_t ld_x, ld_add, ld_sum, ld_out, ld_q;
} mcce_norm;

/* Root-mean-square norm of the residual stream, with the residual's addition:
 *   h = x + add, rounded to dtype (h = x without add);    r = 1 / sqrt(mean_j h_j^2 + eps);    n_j = h_j r weight_j
 *   sum = h;    out = n rounded to dtype;    for every group G of columns
 *   scales_G = max(max_{j in G} |n_j|, 2^-100) / 448;    q_j = e4m3(n_j / scales_G)
 *   x   DEVICE dtype [rows,d]; add DEVICE add_dtype [rows,d] or NULL; weight DEVICE weight_dtype [d]
 *   sum DEVICE dtype [rows,d] out or NULL; may be x itself (same stride)
 *   out DEVICE dtype [rows,d] out or NULL
 *   q   DEVICE e4m3 (one byte: 4 exponent bits, 3 mantissa bits, largest value 448) [rows,d] out or NULL
 *   scales DEVICE fp32 [rows, ceil(d / quant_group)] out, contiguous; given exactly when q is.  The last group of a
 *       row may be shorter.  q_j * scales_G is within 2^-4 |n_j| (or half a subnormal step) of n_j.  The quotient is formed in fp32
 *       as n_j * (448 / max), both operations rounded to nearest, from n_j in fp32.
 * One of sum, out and q at least.  Apart from sum == x no output may overlap another tensor of the call.  A row that holds a NaN is
 * NaN throughout; the sum of squares is formed in fp32, so one beyond 3.4e38 counts as infinite (r = 0) and squares
 * below 1e-45 as zero. */
int mcce_rmsnorm(const mcce_norm* n /*HOST*/, const void* x, const void* add, const void* weight, void* sum,
                 void* out, void* q, float* scales, void* cuda_stream);

/* Its gradient.  With g_j = dout_j weight_j and r as above, formed again from h:
 *   dx_j = r g_j - h_j r^3 mean_i(h_i g_i) + dsum_j;    dweight_j = sum over the rows of dout_j h_j r
 * dx is the gradient of x and of add alike (they enter as a sum).  The gradient of the 8-bit output is not part of
 * it: hand in the gradient with respect to n as dout.
 *   dout DEVICE dtype [rows,d], stride ld_out;    h DEVICE dtype [rows,d], stride ld_x: the `sum` of the forward call (x without add)
 *   dsum DEVICE dtype [rows,d], stride ld_add, or NULL: the gradient that reaches h past the norm
 *   dx   DEVICE dtype [rows,d] out, stride ld_sum; may be dout or dsum itself (same stride)
 *   dweight DEVICE fp32 [d] out, or NULL: not wanted (no workspace needed then).  Rounded parts are added in a fixed order.
 *   workspace DEVICE, 16-byte aligned, mcce_rmsnorm_backward_workspace_bytes(n) bytes (0 for an invalid n).
 * add_dtype, quant_group and ld_q are ignored. */
size_t mcce_rmsnorm_backward_workspace_bytes(const mcce_norm* n /*HOST*/);
int mcce_rmsnorm_backward(const mcce_norm* n /*HOST*/, const void* dout, const void* h, const void* dsum,
                          const void* weight, void* dx, float* dweight, void* workspace, size_t workspace_bytes,
                          void* cuda_stream);

/* Token rows for mcce_dispatch, mcce_combine and mcce_combine_backward: n_layers independent problems of n_tokens
 * tokens with top_k (token, slot) pairs each, P = n_tokens * top_k <= 2^30 pairs per layer. */
typedef struct {
  int32_t n_layers;    /* 1..65535                                                                        */
  int32_t n_tokens;    /* >= 0                                                                            */
  int32_t top_k;       /* 1..16                                                                           */
  int32_t n_experts;   /* 1..256 (mcce_dispatch)                                                          */
  int32_t d;           /* columns of a row, 1..2^24                                                       */
  int32_t dtype;       /* sorted rows: MCCE_F32 or MCCE_BF16; MCCE_E4M3 too in mcce_dispatch              */
  int32_t token_dtype; /* y, add and dy: MCCE_F32, or dtype (mcce_combine and its gradient)               */
  int32_t scale_cols;  /* fp32 scales that travel with a row, 0: none (mcce_dispatch)                     */
  int64_t ld_token;    /* stride in elements of the token rows (x; y and dy), 0 means d; tokens of layer l start at row l * n_tokens */
  int64_t ld_rows;     /* stride in elements of the sorted rows, 0 means d; layer l starts at row l * P   */
} mcce_rows;

/* Sorts token rows by expert: the pairs (t, k) of a layer, in the order t * top_k + k, go into their expert's bucket
 * (a stable counting sort, the grouping of mcce_get_grouping).  A pair whose expert id is outside [0, n_experts) --
 * padding, a dropped token -- goes nowhere.
 *   sel_idx DEVICE int32 [L,T,K]
 *   offsets DEVICE int32 [L,E+1] out: bucket e of layer l is positions offsets[l][e] .. offsets[l][e+1]
 *   perm    DEVICE int32 [L,P] out: pair at every position, or NULL;    inv DEVICE int32 [L,T,K] out: position of every pair, -1 if it has none
 *   x       DEVICE dtype [L,T,d] or NULL (only sort);    rows DEVICE dtype [L,P,d] out: rows[l][inv[l][t][k]] = x[l][t]
 *   scales  DEVICE fp32 [L,T,scale_cols];    row_scales DEVICE fp32 [L,P,scale_cols] out: likewise; contiguous, NULL without scale_cols
 * perm, rows and row_scales are left as they were behind position offsets[l][E].  A token's row is read once.
 * The gradient with respect to x is mcce_combine without weights.
 *   workspace DEVICE, 16-byte aligned, mcce_dispatch_workspace_bytes(r) bytes (0 is possible: it may be NULL then). */
size_t mcce_dispatch_workspace_bytes(const mcce_rows* r /*HOST*/);
int mcce_dispatch(const mcce_rows* r /*HOST*/, const int32_t* sel_idx, const void* x, const float* scales,
                  int32_t* offsets, int32_t* perm, int32_t* inv, void* rows, float* row_scales, void* workspace,
                  size_t workspace_bytes, void* cuda_stream);

/* Brings rows back to their tokens (the weighted sum of Eq. 1):  y[l][t] = add[l][t] + sum_k sel_w[l][t][k] rows[l][inv[l][t][k]],
 * added in slot order, then add.  A pair whose position is outside [0, P) contributes nothing, whatever its weight or
 * any row holds; a token without pairs gets add, or 0.
 *   rows DEVICE dtype [L,P,d];  inv DEVICE int32 [L,T,K];  sel_w DEVICE fp32 [L,T,K], or NULL: every weight is 1
 *   add  DEVICE token_dtype [L,T,d], stride ld_token, or NULL;    y DEVICE token_dtype [L,T,d] out; may be add itself */
int mcce_combine(const mcce_rows* r /*HOST*/, const void* rows, const int32_t* inv, const float* sel_w,
                 const void* add, void* y, void* cuda_stream);

/* Its gradient:  drows[l][inv[l][t][k]] = sel_w[l][t][k] dy[l][t];    dw[l][t][k] = sum_j dy[l][t][j] rows[l][inv[l][t][k]][j],
 * 0 for a pair without a position.  (The gradient of add is dy.)  The positions of a layer must be distinct, as
 * mcce_dispatch makes them; rows of drows at other positions are left as they were.
 *   dy DEVICE token_dtype [L,T,d];  rows DEVICE dtype [L,P,d], NULL if dw is
 *   drows DEVICE dtype [L,P,d] out, stride ld_rows; may be rows itself;    dw DEVICE fp32 [L,T,K] out, or NULL */
int mcce_combine_backward(const mcce_rows* r /*HOST*/, const void* dy, const void* rows, const int32_t* inv,
                          const float* sel_w, void* drows, float* dw, void* cuda_stream);

/* Seeded synthetic inputs (counter-based: Philox4x32-10 keyed by (seed, 0), counter = (element
 * block, t, tensor_id), Box-Muller with fixed-order fp32 series); no counterpart in the paper, whose
 * inputs are text corpora.  out DEVICE, dtype MCCE_F32/MCCE_BF16; elements [start, start+count) of the
 * tensor, value = std * n.  start must be a multiple of 4. */
int mcce_gen_normal(void* out, int32_t dtype, uint64_t start, uint64_t count, uint32_t seed,
                    uint32_t tensor_id, uint32_t t, float std, void* cuda_stream);
/* AR(1) hidden states: h <- (t==0 ? n_t : rho*h + c*n_t) on state DEVICE fp32 [count]; emits
 * x = h + offset_scale * n_offset (offset omitted when offset_scale == 0) as dtype.  count % 4 == 0. */
int mcce_gen_hidden_step(float* state, void* x_out, int32_t dtype, uint64_t count, uint32_t seed,
                         uint32_t t, float rho, float c, float offset_scale, void* cuda_stream);
/* Raw Philox words, DEVICE uint32 [n_blocks,4], for checking the generator bit by bit. */
int mcce_gen_philox_words(uint32_t* out, uint64_t start_block, uint64_t n_blocks, uint32_t seed,
                          uint32_t tensor_id, uint32_t t, void* cuda_stream);

/* Per-kernel device time, for measurement (no counterpart in the paper).  When enabled, every launch
 * of this context is bracketed by a pair of CUDA events on its stream; mcce_profile_read waits for the
 * recorded events and returns, per kernel kind, the summed milliseconds and the number of launches
 * (HOST arrays of MCCE_N_KERNELS entries), clearing the sums if reset != 0. */
enum {
  MCCE_K_ROUTE = 0,    /* fused route kernel (with bf16 hidden states: its tail, on the logits of MCCE_K_ROUTE_GEMM) */
  MCCE_K_GROUP = 1,    /* grouping, first pass: histograms of the selected experts per chunk of pairs */
  MCCE_K_GATHER = 2,   /* grouping, second pass: scan, stable scatter, and the activation rows copied into expert
                          order on the way (clears y on the tensor-core path) */
  MCCE_K_FFN_UP = 3,   /* H = silu(X Wg^T) * (X Wu^T), all groups    */
  MCCE_K_FFN_DOWN = 4, /* O = H Wd^T, all groups                     */
  MCCE_K_COMBINE = 5,  /* weighted sum over slots + shared experts (fp32-pipe path; fused into FFN_DOWN otherwise) */
  MCCE_K_ROUTE_GEMM = 6, /* router logits on the tensor cores (bf16 hidden states) */
  MCCE_N_KERNELS = 7
};
int mcce_profile(mcce_ctx* ctx, int enable);
int mcce_profile_read(mcce_ctx* ctx, double* ms /*HOST*/, int64_t* launches /*HOST*/, int reset);

/* Routing with no context, no workspace and no allocation of any kind.  The paper has no counterpart
 * to this call; it exists for callers that cannot allocate device memory where they need routing
 * decisions: a server whose memory pool already owns the whole GPU, a plug-in that only receives input
 * and output buffers, or a latency-critical callback that must not enter the allocator.
 *
 * Routes n_steps tokens of every (stream, layer) with the routing kernels of mcce_route_step, starting from
 * EMPTY caches, zero counters and (running mode) an empty Delta statistic.  From hidden states the logits
 * are formed on the fp32 pipe for both hidden dtypes (a context given bf16 hidden states uses the tensor
 * cores instead, so its logits can differ in the last bits and, at a near tie, so can a selection).  The cache
 * state it needs while it runs lives in a fixed array inside the library image
 * (mcce_route_trace_static_limit() bytes = 4 MiB, resident on every GPU that loads the library until
 * the process exits) instead of in a workspace.  The state needs about L*S*(4*E + 4*ceil(E/32) + 12)
 * bytes; a configuration that does not fit is refused with MCCE_ELIMIT and nothing is launched.
 *   cfg         HOST; n_layers, n_streams, n_experts, top_k, top_j, cache_capacity, lambda, delta_mode,
 *               renorm, hidden_dtype, d_model, rerank_mode, max_rank and cum_threshold are used and checked
 *               as in mcce_create; the rest is ignored
 *               (hidden must be 16-byte aligned, and so must logits_in when E is a multiple of 4)
 *   hidden, Wr  DEVICE [n_steps,L,S,d] (hidden_dtype) and fp32 [L,E,d], or both NULL
 *   logits_in   DEVICE fp32 [n_steps,L,S,E], or NULL; exactly one of hidden / logits_in is given
 *   fixed_delta DEVICE fp32 [L], only for MCCE_DELTA_FIXED
 *   sel_idx, sel_w  DEVICE outputs [n_steps,L,S,K], as in mcce_route_step
 *   totals_host HOST, optional: Eq. 4 counters summed over everything; asking for them makes the call
 *               wait for the stream, otherwise it only enqueues work
 * The device that is current when the call is made is used.  The first call on each device looks up
 * the array's device address and keeps it for the life of the process; make that first call outside any
 * stream capture, and do not call again on a device after cudaDeviceReset (the address is then stale).  The call uses no
 * cudaMalloc / cudaFree and no allocating library routine.  Every call on a device shares the one
 * array and first clears the part it uses, so nothing carries over between calls -- and two calls
 * whose GPU work overlaps (different streams, or different host threads) race on it: serialise them. */
size_t mcce_route_trace_static_limit(void);
int mcce_route_trace_static(const mcce_config* cfg /*HOST*/, int32_t n_steps, const void* hidden, const float* Wr,
                            const float* logits_in, const float* fixed_delta, int32_t* sel_idx, float* sel_w,
                            mcce_stats* totals_host, void* cuda_stream);

/* Self-test of the bounded waits that the tensor-core kernels use (no counterpart in the paper).  Launches
 * a one-CTA kernel that waits on a barrier nothing ever arrives at, with a limit of limit_ns (1..1e9).  The
 * wait must give up and the kernel must return: MCCE_OK then, and the context's error word is set, so that
 * the next mcce_cache_stats reports MCCE_ETIMEOUT until mcce_reset clears it.  The GPU context stays usable.
 * Synchronises. */
int mcce_selftest_wait_timeout(mcce_ctx* ctx, uint64_t limit_ns);

/* 1 if mcce_moe_forward of this context runs the tcgen05/TMA expert kernels, 0 if the fp32-pipe ones. */
int mcce_uses_tensor_path(const mcce_ctx* ctx);

/* Which kernels mcce_route_step runs for a launch of n_tokens tokens from hidden states, once the router is
 * set (Eq. 3 and the routing rule of Sec. 3.3 either way; this is introspection for tests and benchmarks):
 * MCCE_ROUTER_FP32_PIPE      the fused route kernel forms the logits itself on the fp32 pipe (fp32 hidden states);
 * MCCE_ROUTER_GEMM_TAIL      tcgen05 GEMM with the experts as MMA rows, then the routing tail;
 * MCCE_ROUTER_RESIDENT_TAIL  tcgen05 GEMM with the router resident in shared memory, then the routing tail;
 * MCCE_ROUTER_FUSED          the router-resident GEMM and the tail in one cooperative kernel.
 * Negative: an error code. */
enum { MCCE_ROUTE_AUTO = 0, MCCE_ROUTE_TWO_KERNELS = 1, MCCE_ROUTE_FUSED = 2 };
enum { MCCE_ROUTER_FP32_PIPE = 0, MCCE_ROUTER_GEMM_TAIL = 1, MCCE_ROUTER_RESIDENT_TAIL = 2, MCCE_ROUTER_FUSED = 3 };
int mcce_router_kernel_kind(const mcce_ctx* ctx, int32_t n_tokens);

const char* mcce_strerror(int code);
int mcce_last_cuda_error(const mcce_ctx* ctx); /* cudaError_t of the last failed CUDA call */

#ifdef __cplusplus
}
#endif
#endif /* MCCE_H_ */
