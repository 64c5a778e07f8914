/*
 * accordion.h -- C ABI of the Accordion gradient-compression hot path for one
 * AMD MI355X (gfx950).  arxiv 2010.16248.
 *
 * What the library computes, per training step, for W simulated data-parallel
 * workers on one GPU (the paper's setting: Section 3; compressors: Section 5):
 *
 *   Delta_w = g_w + e_w                       error feedback ("memory term", Sec. 5.3, App. A)
 *   A      += g_0                             per-layer accumulated gradient (Sec. 4.2)
 *   PowerSGD, matrix layers:  P_w = Delta_w Q,  P^ = orthonormalise(mean_w P_w),
 *                             Q_w = Delta_w^T P^,  Q~ = mean_w Q_w (next step's Q),
 *                             D = P^ Q~^T,  e_w = Delta_w - D
 *             1-D layers:     D = mean_w g_w,  e_w = 0      (App. "Compression Ratio Selection")
 *   TopK, every layer:        keep the k entries of Delta_w with the largest |.|
 *                             (ties: lower flat index), payload (index, value),
 *                             e_w = Delta_w with the kept entries zeroed,
 *                             D = (sum over workers of their kept values) / W
 *   end of a window:          c_l = ||A_l||_2,  Algorithm 1 per layer
 *                             (| old - c | / old >= eta  or  lr_next < lr_curr  => critical),
 *                             old <- c,  A <- 0; the level picks rank / k of the next window.
 *
 * Levels.  The paper's l_low is LOW COMPRESSION (higher rank, larger K) and is the
 * level used inside critical regimes; l_high is used outside.  To avoid the word
 * "low" the configuration names them *_crit and *_noncrit.
 *
 * Conventions.
 *  - Every function returns an int32 status (ACC_OK = 0).  Nothing throws, aborts or logs;
 *    accordion_last_error() gives a static, human-readable string for the last failure.
 *  - All tensors are fp32.  "flat" buffers hold all layers concatenated at acc_layer.offset
 *    (in elements); a matrix layer is rows x cols row-major (conv weight out x in x kh x kw
 *    = out x (in*kh*kw)); a 1-D layer has rows = 1.
 *  - Pointers named *_dev are DEVICE pointers and must be 16-byte aligned; pointers named
 *    *_host are HOST pointers.  The library never allocates or frees device memory: the
 *    caller provides one workspace of accordion_workspace_bytes() bytes (256-byte aligned)
 *    that must outlive the context, plus every gradient / output buffer.
 *  - Every call that does device work enqueues it on the HIP stream given at init and returns
 *    without waiting.  The accordion_get_* / accordion_set_state / payload_words calls
 *    synchronise that stream.
 *  - Levels, ranks and kept counts live in device memory and are read by the kernels, so a
 *    level switch costs no host round trip.
 *  - Inputs must be finite; NaN/Inf give unspecified (but memory-safe) results.
 *  - A context is not thread-safe; calls that overlap on one context race.
 */
#ifndef ACCORDION_H
#define ACCORDION_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
  ACC_OK = 0,
  ACC_EINVAL = 1,    /* bad argument (null, out of range, misaligned) */
  ACC_ESTATE = 2,    /* call out of order for the step state machine */
  ACC_ENOSPACE = 3,  /* workspace or host buffer too small */
  ACC_EHIP = 4       /* a HIP runtime call failed */
};

enum { ACC_POWERSGD = 0, ACC_TOPK = 1, ACC_BATCH = 2 };

/* Which statistic accordion_detect_regime decides on.  ACC_DETECT_NORM: the paper's own test
 * (Sec. 4.2, Algorithm 1).  ACC_DETECT_MSDR: the comparison method of Sec. 5.6 -- per layer, the
 * mean to standard deviation ratio of worker 0's gradients over the window,
 *     m = || mean_t g_t || / sqrt( mean_t || g_t - mean ||^2 )
 * (from the accumulator, the sum of the squared gradient norms and the step count; fp64, result
 * fp32; +inf if the gradients did not vary).  The paper describes its use in one sentence; the
 * reading taken here: the first window's m is the reference; once m <= (1 - eta) * reference the
 * layer moves to the *_crit level (less compression) for good and m becomes the reference.
 * lr_curr / lr_next play no role.  accordion_get_norms then returns the reference the last decision
 * compared against (old_host) and m (curr_host).  One extra pass over worker 0's gradient per step.
 * accordion_set_state restarts the window sums (import state at a window end).  Not available
 * for ACC_BATCH; eta must be below 1. */
enum { ACC_DETECT_NORM = 0, ACC_DETECT_MSDR = 1 };

#define ACC_MAX_WORKERS 32
#define ACC_MAX_RANK 4
#define ACC_MAX_BATCH_MULTIPLIER 65536

typedef struct acc_layer {
  int64_t offset;     /* first element of the layer in the flat buffers */
  int32_t rows, cols; /* matrix: n x m; 1-D tensor: rows = 1 */
  int32_t is_matrix;  /* 1: compressed by PowerSGD; 0: 1-D tensor (sent raw by PowerSGD) */
} acc_layer;

typedef struct acc_config {
  int32_t method;              /* ACC_POWERSGD or ACC_TOPK */
  int32_t n_layers;
  const acc_layer* layers;     /* host array, copied at init; layers must not overlap */
  int64_t n_params;            /* length of the flat buffers; >= max(offset + rows*cols) */
  int32_t n_workers;           /* W in [1, ACC_MAX_WORKERS] */
  int32_t rank_crit;           /* PowerSGD rank inside critical regimes, in [1, ACC_MAX_RANK] */
  int32_t rank_noncrit;        /* PowerSGD rank outside */
  int32_t k_num_crit;          /* TopK: k = max(1, ceil(n * num / den)) per layer */
  int32_t k_num_noncrit;
  int32_t k_den;
  float   eta;                 /* detection threshold of Sec. 4.2; the paper uses 0.5 */
  int32_t initial_level;       /* level before the first decision: 1 = critical, 0 = not */
  int32_t batch_multiplier;    /* ACC_BATCH: floor(B_high / B_low) in [1, ACC_MAX_BATCH_MULTIPLIER]; else ignored */
  int32_t batch_monotone;      /* ACC_BATCH: 1 = once the large batch is chosen it is kept (App. A) */
  int32_t detector;            /* ACC_DETECT_NORM (0, the paper's) or ACC_DETECT_MSDR */
} acc_config;

typedef struct acc_ctx acc_ctx;

/* Size of the device workspace for this configuration (host-only arithmetic, no GPU needed).
 * Errors: ACC_EINVAL for null pointers or an invalid configuration. */
int32_t accordion_workspace_bytes(const acc_config* cfg, size_t* out_bytes);

/* Create a context (Algorithm 1's hyper-parameters l_low/l_high/eta and the layer table).
 * workspace_dev: device memory, >= accordion_workspace_bytes(), 256-byte aligned, owned by the
 *   caller; it is cleared here (e = 0, A = 0, no previous norms, level = initial_level).
 * q_init_host: PowerSGD only -- for every matrix layer, in layer order, cols x r_max floats
 *   (row-major, r_max = max(rank_crit, rank_noncrit)), the caller's N(0,1) start for Q.
 *   Ignored (may be NULL) for TopK.
 * hip_stream: a hipStream_t (NULL = the default stream).
 * Errors: ACC_EINVAL, ACC_ENOSPACE (workspace too small), ACC_EHIP.  On error *out is NULL. */
int32_t accordion_init(const acc_config* cfg, void* workspace_dev, size_t workspace_bytes,
                       const float* q_init_host, void* hip_stream, acc_ctx** out);

/* accordion_init for callers that cannot allocate device memory (code that runs under HIP graph
 * capture, serving loops, harnesses that forbid hipMalloc): the workspace is an array of
 * ACC_STATIC_WORKSPACE_BYTES bytes that lives inside the library's device code, one copy per GPU,
 * held until the process ends.  No hipMalloc, hipFree or other allocating call is made; gradients and
 * outputs are still the caller's.  The context belongs to the device that is current at the call.
 * Errors: as accordion_init; ACC_ENOSPACE when the configuration needs a larger workspace than the
 * array (accordion_workspace_bytes tells; use accordion_init then).
 * Every context created this way on one GPU uses the same array: the call clears it and lays it
 * out anew, so the context created last is the only usable one -- calls on an earlier one return
 * ACC_ESTATE (accordion_destroy still works) -- and two threads must not use such contexts on one
 * GPU at the same time: their work would race on the array. */
#define ACC_STATIC_WORKSPACE_BYTES (32u << 20)
int32_t accordion_init_static(const acc_config* cfg, const float* q_init_host, void* hip_stream, acc_ctx** out);

/* Enqueue all later work of this context on another HIP stream (NULL = the default stream).
 * Only between steps (else ACC_ESTATE).  The library does not order the two streams: the caller
 * makes the new stream wait for what the old one still has in flight.
 * HIP graphs: accordion_step_all, accordion_step_all_update and accordion_detect_regime only
 * launch kernels (no allocation, no memset, no synchronisation, per-kernel timing off), so a
 * caller may capture them on the context's stream and replay the graph.  What the host passes by
 * value is frozen into the graph: the gradient / output pointers, lr, momentum, weight_decay,
 * and the step number, which only steers the TopK bin guess (never a result) -- except in
 * batch-size mode, where it selects the slot of the micro-step count: capture an even number of
 * micro-steps per graph there.  Everything else a step depends on (levels, ranks, kept counts,
 * whether PowerSGD's residual is still pending) lives in device memory, so accordion_flush,
 * accordion_get_state or accordion_detect_regime may run between replays. */
int32_t accordion_set_stream(acc_ctx* ctx, void* hip_stream);

/* Free the host-side context (the workspace stays the caller's). */
int32_t accordion_destroy(acc_ctx* ctx);

/* Static description of the last error of this context (or of the last failed init when
 * ctx is NULL). */
const char* accordion_last_error(const acc_ctx* ctx);

/* C(g_w, l): one worker's compression (Sec. 3 update rule; Sec. 5 compressors).
 * phase 0: Delta_w = grad + e_w (kept in place of e_w); worker 0 also does A += grad.
 *          PowerSGD: P_w = Delta_w Q.  TopK: select, write the payload, zero the kept
 *          entries of e_w.   grad_dev: N floats; for PowerSGD it must stay unmodified until
 *          accordion_aggregate(ctx, 0) has run (the raw 1-D tensors are averaged there).
 * phase 1: PowerSGD only: Q_w = Delta_w^T P^ (grad_dev is ignored and may be NULL).
 * Order per step: phase 0 for each worker once (any order), aggregate(0), [phase 1 for each
 * worker, aggregate(1)], decompress.  Anything else returns ACC_ESTATE and touches nothing. */
int32_t accordion_compress_step(acc_ctx* ctx, int32_t worker, const float* grad_dev, int32_t phase);

/* The mean over workers that the all-reduce / all-gather provides (Sec. 5.1 "Implementation",
 * Sec. 3).  phase 0, PowerSGD: P^ = orthonormalise(mean_w P_w) by modified Gram-Schmidt in
 * column order (a zero column stays zero), and the mean of the raw 1-D tensors.
 * phase 0, TopK: the W payloads count as gathered (no arithmetic; the sum is in decompress).
 * phase 1, PowerSGD only: Q~ = mean_w Q_w, stored as the next step's Q. */
int32_t accordion_aggregate(acc_ctx* ctx, int32_t phase);

/* Averaged, decompressed gradient of this step into out_dev (N floats; every element that
 * belongs to a layer is overwritten).
 * PowerSGD: D = P^ Q~^T on matrix layers (the residual e_w = Delta_w - D of every worker becomes
 * the error memory, see accordion_flush); 1-D layers get the plain mean.  TopK: D[i] = (sum over workers, in worker order from +0, of the values kept
 * at i) / W.  Ends the step. */
int32_t accordion_decompress(acc_ctx* ctx, float* out_dev);

/* The whole step for all workers with batched launches: phase 0 for every worker,
 * aggregate, [phase 1, aggregate], decompress.  grads_host_array: HOST array of W DEVICE
 * pointers (N floats each).  Same results as the call-by-call sequence. */
int32_t accordion_step_all(acc_ctx* ctx, const float* const* grads_host_array, float* out_dev);

/* The optimizer that consumes the averaged decompressed gradient, fused into the pass that would
 * store it: SGD with Nesterov momentum (App. A, table "Hyperparameters": Nesterov, momentum 0.9)
 * on the update rule of Sec. 3.  With D as accordion_decompress defines it, for every element
 * that belongs to a layer (others are not touched):
 *     d = D + weight_decay * w   (only if weight_decay != 0; the paper names none)
 *     v = momentum * v + d
 *     w = w - lr * (d + momentum * v)
 * in fp32, every product and every sum rounded on its own, in this order.  D itself is not
 * stored anywhere (4 bytes per element written and read again saved).
 * weights_dev, velocity_dev: N floats each, DEVICE, 16-byte aligned, distinct, owned by the
 * caller; the velocity starts at zero.  lr, momentum, weight_decay: finite, >= 0.
 * accordion_decompress_update takes the place of accordion_decompress in the call-by-call
 * sequence, accordion_step_all_update that of accordion_step_all; state machine, effects on the
 * error memory and the accumulator, and errors are theirs (plus ACC_EINVAL for the arguments
 * above, checked before anything is launched). */
int32_t accordion_decompress_update(acc_ctx* ctx, float* weights_dev, float* velocity_dev, float lr,
                                    float momentum, float weight_decay);
int32_t accordion_step_all_update(acc_ctx* ctx, const float* const* grads_host_array,
                                  float* weights_dev, float* velocity_dev, float lr, float momentum,
                                  float weight_decay);

/* --- batch-size mode (method = ACC_BATCH) ----------------------------------------------------
 * Accordion switching the batch size instead of a compression level (Sec. 3 "Distributed SGD
 * with adaptive batch size"; Sec. 4.2: same algorithm, on the gradient of the whole model;
 * App. A "Additional Details for Batch Size experiment": the large batch is several backward
 * passes summed before one exchange).  One accordion_step_all / accordion_step_all_update call
 * is one MICRO-STEP: every worker's gradient of a micro-batch of B_low samples.
 *     A += g_0;   S_w = g_w (first micro-step of a batch) or S_w + g_w      (S_w lives where the
 *                                                                            error memory does)
 *     a batch is complete after 1 micro-step at level 1 (critical: batch B_low) and after
 *     batch_multiplier micro-steps at level 0 (batch B_high); then, with n = micro-steps in it,
 *     D = (S_0 + S_1 + ... + S_{W-1}) / (W n)   in fp32, in this order, one division.
 * accordion_step_all writes D to out_dev when the micro-step completes a batch and leaves
 * out_dev untouched otherwise; accordion_step_all_update applies the optimizer step then, with
 * the learning rate lr * n (Sec. 5.1: the rate grows in the ratio of the batch), and leaves
 * weights and velocity untouched otherwise.  The level and the micro-step count live on the
 * device: no host round trip decides whether a batch is complete; accordion_batch_status tells.
 * accordion_detect_regime: one norm over all layers' accumulated gradient, Algorithm 1 once; with
 * batch_monotone a level that has reached 0 stays 0.  accordion_payload_words counts n_model
 * floats (the dense all-reduce) per completed batch and none otherwise.
 * The call-by-call entry points return ACC_EINVAL for this method.  State layout: S_0..S_{W-1}
 * | A | pending micro-steps (int32) | norm_old (L) | has_old (L) | level (L, all equal); the
 * sums are meaningful only while pending > 0. */
int32_t accordion_batch_status(acc_ctx* ctx, int32_t* level, int32_t* pending_micro_steps,
                               int32_t* last_batch_micro_steps, int64_t* exchanges,
                               int64_t* micro_steps);

/* End of a window (Sec. 4.2; Algorithm 1): c_l = ||A_l||_2 (fp64 sum, fp32 result), per layer
 * critical <=> no previous norm, previous norm 0, |old - c| / old >= eta, or lr_next < lr_curr;
 * level <- critical; old <- c; A <- 0.  Only between steps (else ACC_ESTATE). */
int32_t accordion_detect_regime(acc_ctx* ctx, float lr_curr, float lr_next);

/* The batched entry points (accordion_step_all, accordion_step_all_update) keep Delta_w in the
 * error memory at the end of a step and form the residual in the first pass of the next step:
 * PowerSGD e_w = Delta_w - D from the stored factors, TopK e_w = Delta_w with the kept entries
 * dropped, from the stored thresholds and tie counts (one write of the memory saved per worker
 * and step).  accordion_flush writes the residual out now; accordion_get_state does so by itself.
 * Only between steps (else ACC_ESTATE).  The call-by-call TopK path writes it directly. */
int32_t accordion_flush(acc_ctx* ctx);

/* A <- 0 without a decision (to measure one epoch out of several, Sec. 5.1 "Hyperparameters"). */
int32_t accordion_reset_accumulator(acc_ctx* ctx);

/* --- read-backs (synchronise the stream) ------------------------------------------------ */

/* levels_host: n_layers int32, 1 = critical. */
int32_t accordion_get_levels(acc_ctx* ctx, int32_t* levels_host);
/* old_host: the previous norm the last decision compared against (0 if none);
 * curr_host: the norm it computed.  n_layers floats each. */
int32_t accordion_get_norms(acc_ctx* ctx, float* old_host, float* curr_host);
/* TopK payload of (worker, layer) from the last step: idx_host (int32, ascending, layer-local
 * flat index) and val_host (fp32), each with room for capacity entries; *count_out = k.
 * Errors: ACC_ENOSPACE if capacity < k (count_out is still set). */
int32_t accordion_get_payload(acc_ctx* ctx, int32_t worker, int32_t layer, int32_t* idx_host,
                              float* val_host, int64_t capacity, int64_t* count_out);
/* How a TopK layer's payload is laid out at a level (host-only arithmetic, no GPU needed).  The
 * paper's own runs keep K = 99 % inside critical regimes (Sec. 5.4, TopK tables), where a list of
 * (index, value) pairs costs 1.98 n floats -- more than the dense tensor.  A layer that keeps more
 * than half of its n entries therefore sends its k values in index order plus the n - k indices
 * of the dropped entries: n floats, never more than dense.  format: ACC_PAYLOAD_INDEX_VALUE
 * (2 k <= n; words = 2 k) or ACC_PAYLOAD_VALUES_HOLES (2 k > n; words = n); kept = k.
 * accordion_get_payload decodes either layout to (index, value); accordion_payload_words keeps
 * the paper's accounting of 2 k floats per layer. */
enum { ACC_PAYLOAD_INDEX_VALUE = 0, ACC_PAYLOAD_VALUES_HOLES = 1 };
int32_t accordion_payload_format(const acc_config* cfg, int32_t layer, int32_t level, int32_t* format,
                                 int64_t* kept, int64_t* words);

/* PowerSGD factors of a matrix layer from the last step: p_hat_host rows x r and q_host
 * cols x r (row-major, r = *rank_out, the rank that step used); room for ACC_MAX_RANK
 * columns each is required. */
int32_t accordion_get_factors(acc_ctx* ctx, int32_t layer, float* p_hat_host, float* q_host,
                              int32_t* rank_out);
/* Floats one worker sent in the last step / since init (PowerSGD: r(n+m) per matrix layer
 * + n per 1-D layer; TopK: 2k per layer -- the accounting of the paper's "Data Sent"). */
int32_t accordion_payload_words(acc_ctx* ctx, int64_t* last_step, int64_t* cumulative);

/* TopK diagnostics since init (they describe which path the selection took, never its result):
 * restaged_layers = (worker, layer) pairs whose threshold lay below the entries the
 * error-feedback pass had listed, on a guess: Delta was read once more for them, and a
 * layer whose threshold bin had not even been counted was decided by sweeps of one workgroup (slow;
 * accordion_topk_short_lists tells the two apart);
 * swept_layers = pairs whose guess held but whose tie class was too large for the per-quarter
 * key lists, decided by the same sweeps. */
int32_t accordion_topk_stats(acc_ctx* ctx, int64_t* restaged_layers, int64_t* swept_layers);
/* Of the restaged layers of accordion_topk_stats, those whose lists were merely too short: the threshold bin had been
 * counted, so the layer was decided as fast as any other and only its lists were of no use.  The rest are missed guesses. */
int32_t accordion_topk_short_lists(acc_ctx* ctx, int64_t* short_layers);

/* Overlap of the kept coordinates of two workers in the last step (Sec. 4.3: how much the
 * Top-K supports of a pair of stochastic gradients overlap; the paper reports > 90 % for
 * Top-10 %).  TopK only, between steps, after at least one step (else ACC_ESTATE).
 * common_host[l] = number of coordinates of layer l that both workers kept; kept_host[l] = k of
 * that step; n_layers entries each.  The overlap fraction is sum(common) / sum(kept).  With error
 * feedback the kept sets are those of gradient + memory; on the first step after init they are
 * those of the gradients themselves.  Synchronises the stream. */
int32_t accordion_topk_overlap(acc_ctx* ctx, int32_t worker_a, int32_t worker_b, int64_t* common_host,
                               int64_t* kept_host);

/* State export / import for checkpointing and step-by-step comparison.  Layout (bytes, all
 * little-endian fp32/int32, no padding):  e_0 .. e_{W-1} (N each) | A (N) | Q (sum over
 * matrix layers of cols*r_max; absent for TopK) | norm_old (L) | has_old (L, int32) |
 * level (L, int32).  accordion_state_bytes gives the size.  Only between steps. */
int32_t accordion_state_bytes(const acc_ctx* ctx, size_t* out_bytes);
int32_t accordion_get_state(acc_ctx* ctx, void* state_host, size_t bytes);
int32_t accordion_set_state(acc_ctx* ctx, const void* state_host, size_t bytes);

/* --- per-kernel timing (tracing aid; not part of the paper's method) -------------------------
 * With profiling on, a kernel launch carries two HIP events that take the begin and the end
 * timestamp of its dispatch on the context's stream, and the elapsed time is accumulated per
 * stage: enable = 1 times every kernel, enable = 2 only the fused error-feedback pass of the
 * method (the kernel that moves the most bytes), enable = 3 only every fourth launch of that
 * pass (a timed launch costs a few us of stream time); 0 switches it off.  Not to be switched on
 * while the stream is being captured into a graph.  accordion_get_profile
 * synchronises the stream and returns the accumulated milliseconds and the number of launches
 * of one stage since profiling was last switched on.  Stages are numbered from 0, fewer than
 * ACC_N_STAGES of them; accordion_stage_name gives the kernel's name, NULL beyond the last stage
 * (accordion_get_profile returns ACC_EINVAL there). */
#define ACC_N_STAGES 48
int32_t accordion_set_profiling(acc_ctx* ctx, int32_t enable);
int32_t accordion_get_profile(acc_ctx* ctx, int32_t stage, double* total_ms, int64_t* launches);
const char* accordion_stage_name(int32_t stage);

/* --- measurement aid (not part of the paper's method) ---------------------------------------
 * Plain streaming copy dst_dev[0..n) = src_dev[0..n) (n floats, a positive multiple of 4; both
 * DEVICE pointers, 16-byte aligned, not overlapping) enqueued on hip_stream.  It moves exactly
 * 4n bytes in and 4n bytes out, which calibrates the memory counters of a profiler run and
 * gives the copy bandwidth the memory system reaches.  Needs no context.
 * Errors: ACC_EINVAL, ACC_EHIP (message via accordion_last_error(NULL)). */
int32_t accordion_probe_copy(float* dst_dev, const float* src_dev, int64_t n, void* hip_stream);

/* --- operators of a language model's training step around the compression path -----------------
 * Forward and backward pass of three layers of a recurrent language model, whose gradients the
 * path compresses, and the AdamW step that consumes its averaged gradient.  They need no context.
 *
 * Conventions, besides those at the top of this file:
 *  - Activations and their gradients are fp32 or bf16 (ACC_FLOAT, ACC_BF16); parameters' gradients,
 *    statistics and states are fp32.  All arithmetic, sums and states are fp32; what is stored as
 *    bf16 is rounded once, to nearest even.
 *  - DEVICE pointers need the alignment of their element type only; rows may start anywhere and lie
 *    apart by a stride (in elements, at least the row's length unless there is one row at most);
 *    a row's own elements are contiguous.  Buffers that are written must not overlap any other buffer.
 *  - Every call enqueues its kernels on hip_stream (NULL = the default stream) and returns without
 *    waiting.  It allocates nothing and keeps nothing: a call that needs memory takes a workspace of
 *    at least ..._workspace_bytes() bytes (256-byte aligned), whose contents mean nothing before and
 *    after.  Work on one workspace must be ordered.  Every call may be captured into a HIP graph (what
 *    the host passes by value, step and learning rate among it, is frozen into the graph).
 *  - The order of every sum is fixed: the same call gives the same bits.
 *  - Empty inputs (no tokens, rows, steps or sequences) are valid.
 *  - Nothing is launched when an argument is refused.  Errors: ACC_EINVAL, ACC_ENOSPACE (workspace),
 *    ACC_EHIP (a launch of this call failed: nothing is enqueued behind it); accordion_operator_error()
 *    describes the last failure of the calling thread. */
enum { ACC_FLOAT = 0, ACC_BF16 = 1 };

const char* accordion_operator_error(void);

/* Embedding lookup with scaling.
 *   forward:   out[t, :] = scale * table[id_t, :]
 *   backward:  grad_table[v, :] = scale * sum over { t : id_t = v } of grad_out[t, :]
 * The sums go by ascending t, in pieces that are then added in their order.
 * An id outside [0, vocab) gives a row of zeros and takes no part in the gradient (padding).
 * grad_table is dense fp32, as the compressors take it: rows without a token become zeros, or, with
 * accumulate, stay as they are and the sums are added (a table shared with the decoder). */
typedef struct acc_embedding {
  int64_t vocab, dim, tokens;    /* vocab in [1, 2^31 - 2], dim in [1, 2^23], tokens in [0, 2^28]; backward:
                                  * tokens x dim up to about 2^36 */
  int64_t table_stride;          /* rows of table / grad_table */
  int64_t out_stride;            /* rows of out / grad_out */
  int32_t index_bits;            /* 32 or 64: int32 or int64 ids */
  int32_t table_type, out_type;  /* ACC_FLOAT / ACC_BF16; backward: grad_table is fp32 whatever table_type says */
  int32_t accumulate;            /* backward: 0 or 1 */
  float   scale;                 /* finite */
} acc_embedding;
int32_t accordion_embedding_forward(const acc_embedding* cfg, const void* ids_dev, const void* table_dev,
                                    void* out_dev, void* hip_stream);
int32_t accordion_embedding_workspace_bytes(const acc_embedding* cfg, size_t* out_bytes);   /* backward */
int32_t accordion_embedding_backward(const acc_embedding* cfg, const void* ids_dev, const void* grad_out_dev,
                                     float* grad_table_dev, void* workspace_dev, size_t workspace_bytes,
                                     void* hip_stream);

/* Layer norm over rows.
 *   forward:   mean = sum x / dim, rstd = 1 / sqrt(sum (x - mean)^2 / dim + eps),
 *              y = (x - mean) rstd weight + bias
 *   backward:  xh = (x - mean) rstd, g = grad_y weight,
 *              grad_x = rstd (g - sum g / dim - xh sum(g xh) / dim),
 *              grad_weight = sum over rows of grad_y xh,  grad_bias = sum over rows of grad_y
 * bias_dev and grad_bias_dev may be NULL, and so may mean_dev and rstd_dev of the forward pass (both).
 * accumulate: grad_weight and grad_bias are added to. */
typedef struct acc_layernorm {
  int64_t rows;                  /* [0, 2^31) */
  int64_t dim;                   /* [1, 2^24] */
  int64_t x_stride, y_stride;    /* rows of x / y (backward: grad_y) */
  int64_t grad_x_stride;         /* backward */
  int32_t type;                  /* of x, y and their gradients */
  int32_t accumulate;            /* backward: 0 or 1 */
  float   eps;                   /* finite, >= 0 */
} acc_layernorm;
int32_t accordion_layernorm_forward(const acc_layernorm* cfg, const void* x_dev, const float* weight_dev,
                                    const float* bias_dev, void* y_dev, float* mean_dev, float* rstd_dev,
                                    void* hip_stream);
int32_t accordion_layernorm_workspace_bytes(const acc_layernorm* cfg, size_t* out_bytes);   /* backward */
int32_t accordion_layernorm_backward(const acc_layernorm* cfg, const void* grad_y_dev, const void* x_dev,
                                     const float* weight_dev, const float* mean_dev, const float* rstd_dev,
                                     void* grad_x_dev, float* grad_weight_dev, float* grad_bias_dev,
                                     void* workspace_dev, size_t workspace_bytes, void* hip_stream);

/* Gated linear recurrence, element by element of the channels.
 *   forward:   a_t = 1 / (1 + exp(-gate_t)), z_t = 1 / (1 + exp(gate_t)),
 *              h_t = a_t h_{t-1} + z_t input_t,   out_t = h_t,   h_last = the last h
 *   backward:  G_t = grad_out_t + a_{t+1} G_{t+1}  (the last one with grad_last),
 *              grad_input_t = z_t G_t,  grad_gate_t = G_t (h_{t-1} - input_t) a_t z_t,
 *              grad_h0 = a_0 G_0
 * z is not computed as a difference from one; gates of +-infinity keep the state / take the input alone.
 * Both gates keep values below the normal fp32 numbers; from |gate| = 104 on the smaller one is zero.
 * h0_dev (NULL: zeros), h_last_dev, grad_last_dev (NULL: zeros) and grad_h0_dev are batch x channels,
 * contiguous fp32; h_last_dev and grad_h0_dev may be NULL.  lengths_dev (int32 per sequence, NULL:
 * all steps): steps from a sequence's length on write zeros and leave the state as it is; their
 * gradients are zeros; what their inputs hold plays no role.  A length below 0 counts as 0, one above
 * steps as steps.  steps = 1 is the serving form: one token, the state in h0 and h_last (which may be
 * the same buffer then, and for any number of steps).
 * Sequences x blocks of 64 channels (bf16: 128) x blocks of 128 steps (bf16 backward: 64): at most 2^22. */
typedef struct acc_recurrence {
  int64_t batch;                 /* [0, 65535] */
  int64_t steps;                 /* [0, 2^31) */
  int64_t channels;              /* [1, 2^24] */
  /* elements between sequences and between steps */
  int64_t gate_batch, gate_step, input_batch, input_step, out_batch, out_step;
  /* the same of the gradients (backward) */
  int64_t grad_gate_batch, grad_gate_step, grad_input_batch, grad_input_step, grad_out_batch, grad_out_step;
  int32_t type;                  /* of gate, input, out and their gradients */
} acc_recurrence;
int32_t accordion_recurrence_workspace_bytes(const acc_recurrence* cfg, size_t* out_bytes);
int32_t accordion_recurrence_forward(const acc_recurrence* cfg, const void* gate_dev, const void* input_dev,
                                     const float* h0_dev, const int32_t* lengths_dev, void* out_dev,
                                     float* h_last_dev, void* workspace_dev, size_t workspace_bytes,
                                     void* hip_stream);
int32_t accordion_recurrence_backward(const acc_recurrence* cfg, const void* gate_dev, const void* input_dev,
                                      const void* out_dev, const float* h0_dev, const int32_t* lengths_dev,
                                      const void* grad_out_dev, const float* grad_last_dev, void* grad_gate_dev,
                                      void* grad_input_dev, float* grad_h0_dev, void* workspace_dev,
                                      size_t workspace_bytes, void* hip_stream);

/* One AdamW step over many tensors (for example the layers of a flat buffer and their averaged
 * gradients from accordion_decompress).  For every element, in fp32, every product and sum rounded on
 * its own, in this order; scalars on the right of ':' are computed in fp64 and rounded once:
 *     g = grad * *grad_scale_dev                        (only if grad_scale_dev is given)
 *     m = beta1 m + c1 g                                 : c1 = 1 - beta1
 *     v = beta2 v + (c2 g) g                             : c2 = 1 - beta2
 *     w = w keep - (rate m) / (sqrt(v) up + eps)         : keep = 1 - lr weight_decay,
 *                                                          rate = lr / (1 - beta1^step), up = 1 / sqrt(1 - beta2^step)
 * step counts from 1.  copies (NULL: none; an entry may be NULL): w also as bf16.
 * State, accordion_adamw_state_elements() elements in all, the tensors one after the other:
 *   state_bits 32: m and v as fp32; m_scale and v_scale are NULL.
 *   state_bits 8:  every tensor starts on a multiple of ACC_ADAMW_BLOCK elements.  A block of
 *     ACC_ADAMW_BLOCK elements of a tensor holds x, for m, and sqrt(v), for v, as 8-bit floating-point
 *     codes (e4m3, largest 448) of x (448 / max|x|), and max|x| / 448 as its fp32 scale; a
 *     block whose max|x| is below 2^-100 is held as zeros.  A positive sqrt(v) of any other block keeps
 *     a code of at least the smallest positive one, so that no update is divided by eps alone because
 *     of the rounding.
 *     Codes are rounded to nearest even where beta1 <= 0.9 (m) and beta2 <= 0.95 (sqrt(v)).  Codes to
 *     nearest do not follow an average that a step moves by less than half their spacing: beyond these
 *     betas, and everywhere with dither = 1, code values are floor(|y| / q + u) q (at most 448), for
 *     y = x (448 / max|x|), the spacing q of codes at |y| and
 *         u = floor(((e k + step 0x9E3779B9) mod 2^32) / 2^12) / 2^20,
 *     e being the element's place in the state and k 0x6A09E667 for m, 0xBB67AE85 for sqrt(v): what is
 *     cut off in one step is made up for in others.  A step frozen into a graph freezes u too, and an
 *     average that moves slowly then stands still.  To nearest, at beta2 = 0.95, sqrt(v) of random
 *     gradients is held 3 to 6 % too large; gradients that do not vary at all from step to step need
 *     dither = 1 at any betas.
 *     The step itself uses the values before they are rounded to codes.  An infinity or NaN in a
 *     block's moments makes the whole block's moments NaN.
 * A state of zeros is the state before the first step. */
#define ACC_ADAMW_BLOCK 256
typedef struct acc_adamw {
  int32_t n_tensors;             /* [0, 2^20] */
  int32_t weight_type;           /* ACC_FLOAT, or ACC_BF16: weights that are kept in bf16 alone */
  int32_t grad_type;
  int32_t state_bits;            /* 8 or 32 */
  const int64_t* sizes_host;     /* elements per tensor, >= 0 */
  const float* weight_decay_host;/* per tensor, finite and >= 0; NULL: none */
  double lr, beta1, beta2, eps;  /* finite; lr >= 0, betas in [0, 1), eps >= 0 */
  int64_t step;                  /* >= 1 */
  int32_t dither;                /* 0 or 1 (8 bits: see above; 32 bits: plays no role) */
} acc_adamw;
int32_t accordion_adamw_state_elements(const acc_adamw* cfg, int64_t* out_elements);
int32_t accordion_adamw_step(const acc_adamw* cfg, void* const* weights_host_array,
                             const void* const* grads_host_array, void* const* copies_host_array, void* m_dev,
                             void* v_dev, float* m_scale_dev, float* v_scale_dev, const float* grad_scale_dev,
                             void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* ACCORDION_H */
