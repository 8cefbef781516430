/*
 * sats.h -- C ABI of the routed, threshold-sparsified gated-MLP library for
 * AMD Instinct MI355X (gfx950).
 *
 * The operation (per token, independently):
 *
 *   route:  r = route_lut[token_id]      1 = base path, 0 = sparse path
 *           (the decision of the token-routing rule, Section 3.2, Eq. 13,
 *            precomputed per vocabulary id; a score below tau selects the
 *            sparse path, any other the base path)
 *   for each layer l = 0 .. n_layers-1, with h the layer input:
 *     a_j  = W_gate_T[l][j] . h  (a = h W_gate)        gated MLP, Eq. 1
 *     g    = SiLU(a) = a / (1 + exp(-a))                 Eq. 2
 *     keep = all columns                   if r == 1     (base MLP, Eq. 1)
 *            { j : |g_j| >= thresholds[l] } if r == 0    (CATS mask, Eq. 4-5)
 *     u_j  = W_up_T[l][j] . h              for j in keep  (x W_up, Eq. 1)
 *     y    = sum_{j in keep} g_j u_j W_down[l][j]         (Eq. 1)
 *     next h = rho(y / sqrt(mean(y^2) + 1e-6))    between layers
 *   out = rho(y of the last layer)
 *
 * rho rounds to the activation type (bf16: round to nearest even).  All
 * products and sums are float32.  The normalisation between layers is this
 * library's convention for chaining bare MLP layers (the paper places each
 * MLP inside a transformer block); a one-layer call is exactly Eq. 1 with the
 * Eq. 5 mask.
 *
 * Layouts (row-major, dense, no padding):
 *   x, out        [n_tokens][d]
 *   token_ids     [n_tokens]
 *   W_gate_T      [n_layers][d_ff][d]      W_gate transposed: row j = column j of W_gate
 *   W_up_T        [n_layers][d_ff][d]      W_up transposed: row j = column j of W_up
 *   W_down        [n_layers][d_ff][d]      row j = the output weights of neuron j
 * (every weight matrix holds one row of d weights per neuron: a linear
 * layer's weight as it is stored for W_gate and W_up, and its transpose for
 * W_down)
 *   thresholds    [n_layers]               float32, >= 0 or +inf
 *   route_lut     [vocab]                  uint8
 *
 * Ownership: every pointer is a DEVICE pointer owned by the caller and must
 * stay valid until the enqueued work has completed.  The library keeps no
 * pointer past that.  It owns a device workspace per (device, stream),
 * allocated on first use and grown when a larger shape arrives (a hipMalloc
 * on that call: call sats_reserve() first where allocation is not allowed).
 *
 * Errors: every call returns SATS_OK or a negative code synchronously, for
 * conditions the host can check (null pointers, shapes, overlap of out with
 * x other than exact equality, HIP launch failures).  The text of the last
 * error of the calling thread is returned by sats_last_error().  Execution
 * is asynchronous on `stream`; device-side faults surface at the caller's
 * next synchronisation.  n_tokens == 0 returns SATS_OK and enqueues nothing.
 *
 * Unchecked preconditions (device contents): 0 <= token_ids[i] < vocab;
 * thresholds not NaN and not negative; x and weights finite.
 *
 * Determinism: results do not depend on the run, on the batch a token is in
 * (for batches of one size class: 1 token, 2 to 64, and above 64 the batches
 * whose passes of up to 2048 rows split d_ff into as many chunks) or on the
 * stream; every reduction has a fixed order and no floating-point atomics
 * are used.  Only a batch whose workspace cannot be had runs on other kernels
 * (see sats_reserve), with results that agree within rounding.
 *
 * Concurrency: calls on different streams use different workspaces and may
 * overlap.  Calls on one stream are ordered by the stream; they may come from
 * several threads, each call's work is enqueued as a whole.  A graph that
 * recorded a call uses the workspace of the stream it was recorded on: a
 * replay must not overlap that stream's calls, nor replays of other graphs
 * recorded there.
 */
#ifndef SATS_H
#define SATS_H

#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef uint16_t sats_bf16; /* raw bfloat16 bits */

enum {
  SATS_OK = 0,
  SATS_ERR_NULL = -1,      /* a required pointer is NULL                        */
  SATS_ERR_SHAPE = -2,     /* d < 1, d_ff < 1, n_layers < 1, n_tokens < 0, or too large */
  SATS_ERR_HIP = -3,       /* a HIP runtime call or kernel launch failed        */
  SATS_ERR_WORKSPACE = -4, /* workspace allocation failed                       */
  SATS_ERR_ARG = -5,       /* other invalid argument (partial overlap of out and x)        */
  SATS_ERR_DEVICE = -6     /* reported by sats_device_status: a device-side wait gave up  */
};

/*
 * Routed sparse forward (Section 3.2 routing over the Section 2 CATS-masked
 * gated MLP).  route_lut == NULL sends every token to the sparse path (the
 * static sparse model) and token_ids may then be NULL.  out may equal x
 * exactly (in-place); any other overlap is rejected.
 */
int sats_mlp_forward(const sats_bf16 *x, const int32_t *token_ids,
                     const sats_bf16 *W_gate_T, const sats_bf16 *W_up_T,
                     const sats_bf16 *W_down, const float *thresholds,
                     const uint8_t *route_lut, sats_bf16 *out,
                     int64_t n_tokens, int64_t d, int64_t d_ff, int64_t n_layers,
                     hipStream_t stream);

/*
 * Allocation-free variant of sats_mlp_forward, for callers that cannot
 * allocate device memory: code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc.  Same arguments, computation and results
 * as sats_mlp_forward (the same kernels), but the workspace is a fixed device
 * array of the library, SATS_NOALLOC_SCRATCH_BYTES (16 MiB) on each device
 * that runs it, held until the process ends, instead of a per-stream
 * allocation; the call allocates and frees nothing.  That covers single-token
 * calls at d <= 4096 and d_ff <= 16384 (any number of layers up to 64, bf16)
 * and batches whose kernels' workspace fits: a batch that sats_mlp_forward
 * takes on the matrix-core products of prompts (more than 64 tokens, or d no
 * multiple of 128 or d_ff none of 64) runs on those where their workspace
 * fits, else, as any other batch, in passes of up to 64 tokens where that
 * one fits (the outputs then agree with sats_mlp_forward's within rounding).
 * The two differ in size, so a call may fit where one of fewer tokens does
 * not: 4096 x 14336 takes 65 tokens and not 64.  A call whose workspace does
 * not fit returns SATS_ERR_WORKSPACE before any device work.  Every call on a
 * device shares that device's array and leaves its last contents there: a
 * call that is not on the prompt products first clears the array's arrival
 * counters with a small kernel (no memset), and calls that overlap on one
 * device (other streams or threads) race and must not be issued.
 * sats_device_status also reports a bounded wait that gave up in such a call.
 */
#define SATS_NOALLOC_SCRATCH_BYTES (16u << 20)
int sats_mlp_forward_noalloc(const sats_bf16 *x, const int32_t *token_ids,
                             const sats_bf16 *W_gate_T, const sats_bf16 *W_up_T,
                             const sats_bf16 *W_down, const float *thresholds,
                             const uint8_t *route_lut, sats_bf16 *out,
                             int64_t n_tokens, int64_t d, int64_t d_ff, int64_t n_layers,
                             hipStream_t stream);

/* Base path for every token: the unmasked gated MLP of Eq. 1, same layout. */
int sats_mlp_dense(const sats_bf16 *x, const sats_bf16 *W_gate_T,
                   const sats_bf16 *W_up_T, const sats_bf16 *W_down,
                   sats_bf16 *out, int64_t n_tokens, int64_t d, int64_t d_ff,
                   int64_t n_layers, hipStream_t stream);

/* float32 twins: x, weights and out are float32; rho rounds to float32. */
int sats_mlp_forward_f32(const float *x, const int32_t *token_ids,
                         const float *W_gate_T, const float *W_up_T,
                         const float *W_down, const float *thresholds,
                         const uint8_t *route_lut, float *out,
                         int64_t n_tokens, int64_t d, int64_t d_ff, int64_t n_layers,
                         hipStream_t stream);
int sats_mlp_dense_f32(const float *x, const float *W_gate_T, const float *W_up_T,
                       const float *W_down, float *out, int64_t n_tokens, int64_t d,
                       int64_t d_ff, int64_t n_layers, hipStream_t stream);

/*
 * Introspection for tests and measurement: the same computation as
 * sats_mlp_forward, plus extra stores.  Any of the extra outputs may be NULL.
 *   route_out     [n_tokens]                 decision used (1 base, 0 sparse)
 *   active_count  [n_layers][n_tokens]       |keep| of each token at each layer
 *   active_idx    [n_layers][n_tokens][d_ff] keep set, ascending, first
 *                                            active_count entries valid
 *   layer_in      [n_layers][n_tokens][d]    input h of each layer
 */
int sats_mlp_forward_inspect(const sats_bf16 *x, const int32_t *token_ids,
                             const sats_bf16 *W_gate_T, const sats_bf16 *W_up_T,
                             const sats_bf16 *W_down, const float *thresholds,
                             const uint8_t *route_lut, sats_bf16 *out,
                             int64_t n_tokens, int64_t d, int64_t d_ff, int64_t n_layers,
                             hipStream_t stream, uint8_t *route_out,
                             int32_t *active_count, int32_t *active_idx,
                             sats_bf16 *layer_in);
int sats_mlp_forward_inspect_f32(const float *x, const int32_t *token_ids,
                                 const float *W_gate_T, const float *W_up_T,
                                 const float *W_down, const float *thresholds,
                                 const uint8_t *route_lut, float *out,
                                 int64_t n_tokens, int64_t d, int64_t d_ff, int64_t n_layers,
                                 hipStream_t stream, uint8_t *route_out,
                                 int32_t *active_count, int32_t *active_idx,
                                 float *layer_in);

/*
 * LoRA-aware routed sparse forward (Section 5, the fine-tuned routed
 * models): sparse-path tokens run the base weights plus rank-r adapters on
 * the three projections,
 *   W_gate + scale A_gate B_gate,  W_up + scale A_up B_up,  W_down + scale A_down B_down,
 * and base-path tokens run the base weights alone (both paths share them, so
 * the adapters are not merged in).  The CATS threshold applies to
 * |SiLU(h (W_gate + scale A_gate B_gate))|.  Device arrays in the activation
 * type, stacked over n_layers like the weights, row-major:
 *   A_gate [d][rank], B_gate [rank][d_ff], A_up [d][rank],
 *   B_up_T [d_ff][rank] (B_up transposed, like W_up_T),
 *   A_down [d_ff][rank], B_down [rank][d].
 * The adapters run inside the same launches as the base computation: the up
 * adapter only for kept columns, the down adapter's first factor only over
 * kept rows.  rank is 8, 16, 32 or 64; the adapter arrays must be 16-byte
 * aligned.  Batches of two or more bf16 tokens whose shapes fit the matrix-core
 * path (d a multiple of 128 and at most 4096, d_ff a multiple of 64) run in
 * passes of up to 64 tokens (above 128 tokens 2048) with every row on the matrix cores: each row
 * applies its own route and keep rule, the gate and up adapter terms are
 * added in float32 before SiLU and the keep rule, z = p A_down is summed per
 * column tile of at most 64 (above 128 tokens per chunk of d_ff, 16 of them)
 * and scale z B_down is added with the output.  Otherwise the
 * shapes must fit the single-token path (d <= 4096, d and d_ff multiples of
 * 16 bytes' worth of elements) and tokens are processed one after another,
 * each on its own route.  Other arguments and the optional
 * inspection outputs as in sats_mlp_forward_inspect.  Errors: SATS_ERR_NULL
 * (a required array), SATS_ERR_SHAPE (rank or shape), SATS_ERR_ARG
 * (alignment, non-finite scale), and those of sats_mlp_forward.
 */
int sats_mlp_forward_lora(const sats_bf16 *x, const int32_t *token_ids, const sats_bf16 *W_gate_T,
                          const sats_bf16 *W_up_T, const sats_bf16 *W_down, const sats_bf16 *A_gate,
                          const sats_bf16 *B_gate, const sats_bf16 *A_up, const sats_bf16 *B_up_T,
                          const sats_bf16 *A_down, const sats_bf16 *B_down, int64_t rank, float scale,
                          const float *thresholds, const uint8_t *route_lut, sats_bf16 *out, int64_t n_tokens,
                          int64_t d, int64_t d_ff, int64_t n_layers, hipStream_t stream, uint8_t *route_out,
                          int32_t *active_count, int32_t *active_idx, sats_bf16 *layer_in);
int sats_mlp_forward_lora_f32(const float *x, const int32_t *token_ids, const float *W_gate_T, const float *W_up_T,
                              const float *W_down, const float *A_gate, const float *B_gate, const float *A_up,
                              const float *B_up_T, const float *A_down, const float *B_down, int64_t rank,
                              float scale, const float *thresholds, const uint8_t *route_lut, float *out,
                              int64_t n_tokens, int64_t d, int64_t d_ff, int64_t n_layers, hipStream_t stream,
                              uint8_t *route_out, int32_t *active_count, int32_t *active_idx, float *layer_in);

/*
 * Allocate the workspace of (current device, stream) for calls of up to
 * max_tokens tokens at this d, d_ff, n_layers and element size (2 = bf16,
 * 4 = f32), so that later calls of that size or smaller allocate nothing.
 * Without it a call allocates what it needs, once; a buffer that a captured
 * call has used is kept until sats_release, also where a later call grows it.
 * A batch whose matrix-core workspace is not there and cannot be allocated
 * (under stream capture, or for want of memory) runs on other kernels in
 * passes of 64 tokens, and its results agree with the usual ones within
 * rounding: bf16 prompts of more than 64 tokens (LoRA: 128), float32 batches,
 * and bf16 batches with d no multiple of 128 or d_ff none of 64.  A size that
 * could not be allocated is not tried again until the next sats_reserve or
 * sats_release.
 */
int sats_reserve(int64_t max_tokens, int64_t d, int64_t d_ff, int64_t n_layers,
                 int elem_bytes, hipStream_t stream);

/*
 * Synchronise `stream` and report whether a kernel of this library on it
 * raised the device error flag since the last check (SATS_ERR_DEVICE; the
 * flag is cleared).  The single-token path's second reduction stage waits
 * for the other workgroups of its launch with a bounded wait that raises
 * the flag instead of hanging; the call also surfaces asynchronous HIP
 * errors of the stream.
 */
int sats_device_status(hipStream_t stream);

/*
 * SATS calibration (Section 3.1, Eq. 6-10): the offline step that produces
 * the per-layer thresholds the forward calls take.  Unlike the forward
 * calls, these take and return their small arrays in HOST memory, use
 * device buffers of their own (kept per device from call to call and grown
 * when a call needs more; calls are serialised; sats_release frees them),
 * and synchronise `stream` before returning, also when they fail.
 *
 * sats_calibration_curves -- one layer.  h [n][d] holds the layer's inputs
 * for n calibration rows (device, bf16; the base-path inputs in a stack),
 * W_gate_T, W_up_T, W_down [d_ff][d] each (device, bf16).  For
 * each level q_k of levels[n_levels] (host, ascending in [0, 1]) the
 * candidate threshold t_k is the Eq. 3 order statistic v_(ceil(q_k N)) of the
 * N = n d_ff post-gate magnitudes |SiLU(h W_gate)| (q_k = 0 gives t_k = 0;
 * q_k is taken to 1e-6), and
 *   err_out[k] = Err(t_k) = mean over rows of ||y - y_t|| / (||y|| + 1e-6)   (Eq. 6)
 *   sp_out[k]  = #{|g| < t_k} / N                      (the layer sparsity at t_k)
 * with y the dense MLP output of the row and y_t the output with the neurons
 * of |g| < t_k removed.  t_out, err_out, sp_out: host arrays [n_levels];
 * err_rows (device float [n][n_levels], or NULL) receives the per-row terms.
 * g and u accumulate in float32; p = g u enters the error product as two
 * bf16 terms (about 16 bits of p); the sums have a fixed order.
 * Shapes: d a multiple of 128 up to 4096, d_ff a multiple of 64.
 *
 * sats_calibrate_sats -- a stack.  The n_cal rows of x_cal (device bf16
 * [n_cal][d]) run through the base path of the n_layers-layer stack (the
 * forward calls' own inter-layer normalisation); every layer's curves are
 * measured on its inputs at the candidate levels 0, coarse_step,
 * 2 coarse_step, ... (Eq. 3 percentiles); for a budget b each layer takes
 * its largest candidate with Err <= b (Eq. 7), S(b) is the mean layer
 * sparsity (Eq. 9), and b* minimises |S(b) - s_tar| over every distinct
 * error value (Eq. 10; the smallest b on ties).  Then, per layer, levels
 * fine_step apart strictly between the two coarse levels adjacent to the
 * level of its choice (both sides of it) are added and b* is chosen again.  With guardrail != 0 (and n_layers > 1) the last
 * layer keeps its CATS threshold at level s_tar (its sparsity counts in S).
 * thresholds_out: host float [n_layers]; budget_out, realized_out: host
 * doubles (may be NULL) receiving b* and S(b*).
 */
int sats_calibration_curves(const sats_bf16 *h, const sats_bf16 *W_gate_T, const sats_bf16 *W_up_T,
                            const sats_bf16 *W_down, int64_t n, int64_t d, int64_t d_ff,
                            const double *levels, int64_t n_levels, float *t_out, double *err_out,
                            double *sp_out, float *err_rows, hipStream_t stream);
int sats_calibrate_sats(const sats_bf16 *x_cal, int64_t n_cal, const sats_bf16 *W_gate_T,
                        const sats_bf16 *W_up_T, const sats_bf16 *W_down, int64_t d, int64_t d_ff,
                        int64_t n_layers, double s_tar, double coarse_step, double fine_step,
                        int guardrail, float *thresholds_out, double *budget_out,
                        double *realized_out, hipStream_t stream);

/*
 * Routing-table construction (Section 3.2, Eq. 11-14), the offline step that
 * produces route_lut.  token_ids [n_tokens] with loss_base and loss_sparse
 * [n_tokens] (device, float32: the next-token cross-entropy of each
 * occurrence of the routing corpus on the base and the sparse path) give
 * each id x the score s(x) = mean over its occurrences of
 * d = max(0, loss_sparse - loss_base) (Eq. 11-12; d taken in float32 and
 * rounded to a multiple of 2^-32, so that the per-id sums are exact;
 * s = +inf for an id without occurrences).  heldout_ids [n_heldout] (device)
 * calibrate the threshold: tau* minimises |R(tau) - r_tar| over the distinct
 * finite scores of the held-out ids and +inf (Eq. 14; the smallest on ties),
 * R(tau) being the fraction of held-out occurrences whose id scores below
 * tau.  route_lut [vocab] (device) receives 0 (sparse path) where
 * s(x) < tau*, else 1 (base path) -- the table the forward calls take.
 * scores [vocab] (device double, or NULL) receives s; tau_out and
 * realized_out (host, or NULL) receive tau* and R(tau*); the selection of
 * tau* runs on the device.  Synchronises the stream; its device buffers are
 * kept per device from call to call (calls are serialised; sats_release
 * frees them).  On an error route_lut is left as it was.  Errors:
 * SATS_ERR_NULL, SATS_ERR_SHAPE,
 * SATS_ERR_ARG (r_tar outside [0, 1], an id outside [0, vocab), a loss
 * difference NaN or >= 2^31).  The per-id sums of d must stay below 2^32.
 */
int sats_route_table(const float *loss_base, const float *loss_sparse, const int32_t *token_ids, int64_t n_tokens,
                     const int32_t *heldout_ids, int64_t n_heldout, int64_t vocab, double r_tar,
                     uint8_t *route_lut, double *scores, double *tau_out, double *realized_out, hipStream_t stream);

/*
 * Execution options: which kernels the forward calls made afterwards on the
 * calling thread run.  Every field's default, 0, is the library's own
 * choice; sats_set_options(NULL) restores the defaults.  Meant for tests
 * and measurement (results of every choice agree with the definition above
 * within the stated tolerances); nothing else changes the kernels a call
 * takes.  Errors: SATS_ERR_ARG for a value outside its range.
 *   batch_path      SATS_BATCH_AUTO, or for batches of 2 or more tokens (float32
 *                   and shapes without a matrix-core kernel for the base-path
 *                   group: SPLIT takes the compacted kernels):
 *                   SATS_BATCH_MFMA     every token on the matrix cores, each
 *                                       with its own route and keep rule;
 *                   SATS_BATCH_SPLIT    the base-path group on the matrix
 *                                       cores, the sparse group on the
 *                                       compacted kernels;
 *                   SATS_BATCH_COMPACT  every token on the compacted kernels
 *                                       (gate, then up and down over the
 *                                       union of kept rows of each 4-token
 *                                       tile, with a per-row token mask).
 *   single_token    SATS_SINGLE_AUTO: one-token calls on the single-token
 *                   kernels where the shape fits them; SATS_SINGLE_OFF: on
 *                   the batch kernels.
 *   dec_block_cols  single-token layer launch: gate columns per workgroup,
 *                   one partial of y each (1 .. 64; 0 = d_ff over the
 *                   compute units, at least 8).
 *   lora_per_token  1: LoRA batches token after token on the single-token
 *                   kernels instead of the matrix-core passes.
 */
enum { SATS_BATCH_AUTO = 0, SATS_BATCH_MFMA = 1, SATS_BATCH_SPLIT = 2, SATS_BATCH_COMPACT = 3 };
enum { SATS_SINGLE_AUTO = 0, SATS_SINGLE_OFF = 1 };
typedef struct {
  int batch_path;
  int single_token;
  int dec_block_cols;
  int lora_per_token;
} sats_options;
int sats_set_options(const sats_options *opt);

/*
 * The kernels a forward call (without adapters) of this shape would run
 * under the calling thread's options, answered on the host without device
 * work: *path receives SATS_PATH_SINGLE_TOKEN, SATS_PATH_BATCH_MFMA,
 * SATS_PATH_BATCH_SPLIT or SATS_PATH_BATCH_COMPACT (for the first pass of
 * up to 64 tokens; 0 for n_tokens == 0).  For float32 batches it is
 * SATS_PATH_BATCH_COMPACT on every path: it does not tell their matrix-core
 * kernels (batch_path AUTO or MFMA, rows in 16-byte pieces, d <= 4096) from the
 * compacted ones.  elem_bytes: 2 (bf16) or 4 (float32); aligned16: whether x,
 * out and the weights are 16-byte aligned; n_cus: compute units of the device
 * (0: the current device's).  Errors: SATS_ERR_NULL, SATS_ERR_SHAPE and
 * SATS_ERR_ARG as for the forward calls.
 */
enum { SATS_PATH_SINGLE_TOKEN = 1, SATS_PATH_BATCH_MFMA = 2, SATS_PATH_BATCH_SPLIT = 3,
       SATS_PATH_BATCH_COMPACT = 4 };
int sats_query_path(int64_t n_tokens, int64_t d, int64_t d_ff, int elem_bytes, int aligned16, int n_cus,
                    int *path);

/*
 * Serving: what a token passes between two MLPs, and from the last one to the
 * next id.  bf16 or float32 throughout (elem_bytes 2 or 4; a cache also 8 bits), sums and softmax
 * statistics in float32 or wider, each result rounded once.
 *
 * Keys and values are kept in pages of page_size tokens.  A cache holds them
 * for every layer, in device arrays of the caller, each head's part of a page
 * contiguous:
 *   k, v   [n_layers][n_pages][n_kv_heads][page_size][head_dim]
 * page_size is a power of two up to 4096, head_dim a multiple of 8 up to 256,
 * both arrays 16-byte aligned.
 *
 * A batch names the new tokens of n_seqs sequences, whose rows follow each
 * other: sequence s has rows q_start[s] .. q_start[s + 1] - 1 of n_tokens, and
 * with them kv_len[s] tokens in all, so that new token i is at place
 * kv_len[s] - (q_start[s + 1] - q_start[s]) + i.  table[s] is its page table
 * row: token j is in page table[s][j / page_size] at j % page_size, -1 where
 * there is no page.  max_q_len and max_kv_len are upper bounds, on the host,
 * of the new tokens and the length of any sequence; they decide the launches
 * (a batch replayed from a graph may change within them).
 *
 * The state of the pages is the table [n_seqs][max_pages], the lengths
 * len[n_seqs] and refs[n_pages], the number of table entries that name each
 * page.  A page of 0 refs is free.
 *
 * Device contents are not trusted as far as memory goes: a length, sequence or
 * page number out of its range is cut off or passed over (the key of a page
 * that is not there is not seen, the token of one is not stored), and reads or
 * writes nothing outside the arrays.
 */
typedef struct {
  void *k, *v;
  int64_t n_layers, n_pages, n_kv_heads, page_size, head_dim;
  int32_t elem_bytes;
} sats_kv_cache;

typedef struct {
  const int32_t *table, *q_start, *kv_len; /* device */
  int64_t n_seqs, max_pages, n_tokens, max_q_len, max_kv_len;
} sats_kv_batch;

/*
 * A cache of 8 bits: every call that takes a cache takes &c8.kv, whose elem_bytes says
 * the format.  k and v hold codes, a byte each, and the scale arrays (4-byte aligned) a byte b for
 * each row of head_dim codes (a token's head):
 *   k_scale, v_scale   [n_layers][n_pages][n_kv_heads][page_size]
 * Code c stands for c 2^(b - 127), and for NaN where b is 255.  Codes are E4M3 numbers (4 bits
 * of exponent, 3 of mantissa, 448 at most, 0x7f and 0xff NaN) or whole numbers from -127 to 127.
 * A row is written with the smallest b from 1 to 254 for which its largest magnitude is
 * within the codes, each value to the nearest code, ties to even (at most, one that does not
 * read as an infinity); a row that holds an infinity or NaN as zeros under 255.  Values are
 * attended to, and read, as bf16 holds them, which is exactly (below 2^-126: cut off or rounded to its
 * step; codes of other origin must not stand for more than the largest bf16 number); what a value
 * adds to a result may be left out where it is below 2^-117.
 * page_size is at least 16 and head_dim a multiple of 16.  q_elem_bytes (2 or 4) is the
 * type of what is appended and of the queries and results of an attention over the cache.
 */
enum { SATS_KV_E4M3 = 17, SATS_KV_INT8 = 18 }; /* elem_bytes of a sats_kv_cache8's kv */
typedef struct {
  sats_kv_cache kv;
  uint8_t *k_scale, *v_scale;
  int32_t q_elem_bytes;
} sats_kv_cache8;

/*
 * Groups of a batch's sequences that share a prefix (sats_prefix_attention): the sequences seq_start[g] ..
 * seq_start[g + 1] - 1 (which follow each other in the batch) have their first len[g] tokens
 * in common (as far as each has them), as after sats_cache_fork.  seq_start [n_groups + 1] and len [n_groups]
 * are device data (n_groups <= 65535); sequences outside of every group, and groups of one or
 * with no prefix, are fine.  max_tokens (new tokens of a group), max_len (of a prefix) and max_own (of
 * any sequence's tokens behind its prefix, the new ones included) are upper bounds on the host:
 * what is beyond them is cut off.
 */
typedef struct {
  const int32_t *seq_start, *len; /* device */
  int64_t n_groups, max_tokens, max_len, max_own;
} sats_kv_prefix;

typedef struct {
  int32_t *table, *len, *refs; /* device */
  int64_t n_seqs, max_pages;
} sats_kv_pages;

/*
 * Norm of each head of q and k, and the position rotation, in one pass:
 *   x <- x / sqrt(mean(x^2) + eps) * weight       (q_norm, k_norm [head_dim]; NULL: no norm)
 *   (a, b) <- (a cos - b sin, b cos + a sin)      for the rot_dim / 2 pairs
 * A pair is (i, i + rot_dim / 2), with interleaved (2 i, 2 i + 1); dims from
 * rot_dim on are not rotated.  rope [n_pos][rot_dim] (float32, device) holds the
 * rot_dim / 2 cosines of a position, then the sines.  Rows of heads are dense;
 * the strides are elements from one token to the next, so q, k and v may be
 * parts of one projection's output.  An output may be its own input (same
 * pointer and stride); other overlap is rejected (rows of one stride may lie
 * between each other), and so are inputs or q_out in the cache.  Arrays and
 * strides on 16 bytes, with head_dim and rot_dim multiples of 32 bytes' worth of elements,
 * move in 16-byte pieces, others element by element.
 *
 * sats_qk_norm_rope: positions [n_tokens] (device; cut off to 0 .. n_pos - 1).
 * sats_qkv_append: the batch's tokens; keys and values (these as they are) go
 * to their places in `layer` of the cache.  positions NULL: the tokens' places.
 */
int sats_qk_norm_rope(const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *q_norm,
                      const void *k_norm, float eps, const float *rope, int64_t n_pos, const int32_t *positions,
                      void *q_out, int64_t q_out_stride, void *k_out, int64_t k_out_stride, int64_t n_tokens,
                      int64_t n_q_heads, int64_t n_kv_heads, int64_t head_dim, int64_t rot_dim, int interleaved,
                      int elem_bytes, hipStream_t stream);
int sats_qkv_append(const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                    const void *q_norm, const void *k_norm, float eps, const float *rope, int64_t n_pos,
                    const int32_t *positions, void *q_out, int64_t q_out_stride, const sats_kv_cache *cache,
                    int64_t layer, const sats_kv_batch *batch, int64_t n_q_heads, int64_t rot_dim, int interleaved,
                    hipStream_t stream);

/*
 * Attention of the batch's new tokens over one layer of the cache:
 *   out = sum_j p_j v_j,   p = softmax over the visible j of scale (q . k_j)
 * A token at place i sees the keys j <= i; with window > 0 only those with
 * i - j < window or j < n_sinks.  Query head h reads cache head
 * h / (n_q_heads / n_kv_heads).  q [n_tokens][n_q_heads][head_dim] at q_stride
 * elements a token; out the same, dense; lse [n_tokens][n_q_heads] (float32, or
 * NULL) the logarithm of the sum of exp(scale q . k_j).  A token that sees
 * nothing gives zeros and -inf.  What a key that is not seen holds (NaN,
 * infinities) does not matter.  q, out and rows of q on 16 bytes; q, out, lse and
 * the cache must not overlap.
 */
int sats_paged_attention(const void *q, int64_t q_stride, const sats_kv_cache *cache, int64_t layer,
                         const sats_kv_batch *batch, int64_t n_q_heads, float scale, int64_t window, int64_t n_sinks,
                         void *out, float *lse, hipStream_t stream);

/*
 * The same attention for a batch whose sequences share prefixes: the keys of a
 * prefix are read once for each tile of its group's rows (of a cache head 128 rows, 16 of float32, whose
 * sequence does not matter), from the pages of the first of its
 * sequences that is as long, or as long as any (shorter ones see of it what they have), the others
 * from each sequence's own.  With window > 0 a sequence may have given back the pages that its new
 * tokens do not see: each page of the prefix is then the longest sequence's that has one in its place.  A
 * sequence has to have the pages of the prefix that its new tokens see.  Results agree with
 * sats_paged_attention's within rounding.  Scratch memory as said at sats_reserve_prefix.
 */
int sats_prefix_attention(const void *q, int64_t q_stride, const sats_kv_cache *cache, int64_t layer,
                          const sats_kv_batch *batch, const sats_kv_prefix *prefix, int64_t n_q_heads, float scale,
                          int64_t window, int64_t n_sinks, void *out, float *lse, hipStream_t stream);

/*
 * Keys and values of the batch's tokens as they are in `layer` of the cache (of any format):
 * token t's go to row t of k_out and v_out, [n_tokens][n_kv_heads][head_dim] of elem_bytes (2 or
 * 4) at strides in elements; either may be NULL.  With q_start the running sums of kv_len that
 * reads whole sequences.  A token whose page is not there reads zeros; rows that are of
 * no sequence stay as they were.  The outputs may not overlap each other or the cache.
 */
int sats_cache_read(const sats_kv_cache *cache, int64_t layer, const sats_kv_batch *batch, void *k_out, int64_t k_stride,
                    void *v_out, int64_t v_stride, int elem_bytes, hipStream_t stream);

/*
 * Bookkeeping of the pages, on the device.  A call takes n items (up to 65535;
 * seqs NULL: sequences 0 .. n - 1); a sequence may be in it once.
 *
 * sats_cache_extend: item i's sequence grows by add[i] tokens: its table gets
 * the pages that these need (also the one that the sequence ends inside of, where
 * it was given back).  A last page that is not full and that other sequences
 * share is replaced by a copy of its own.
 * sats_cache_fork: sequence dst[i], which has to be empty, becomes a copy of
 * src[i] (no dst is a src): full pages are shared, a last page that is not full
 * is copied (its tokens, in every layer).
 * New pages are the free pages of lowest number, in ascending order over the
 * items (a copy first).  Without enough free pages nothing changes.  status
 * (device int32 [2], or NULL): pages that were missing, and items that were left
 * out (no such sequence, no room in the table, dst in use, add < 0).
 *
 * sats_cache_free: gives back the pages that lie wholly in the tokens
 * begin[i] .. end[i] - 1 of item i's sequence (NULL: from 0, to its length); their
 * table entries become -1.  An end at or past the length cuts the sequence to
 * begin[i] tokens.
 * sats_cache_compact: moves pages (contents, table entries, refs) so that those in
 * use are 0 .. n_used - 1: the ones beyond go to the free ones below, both in
 * ascending order.  n_used: device int32, or NULL.
 * sats_cache_copy: contents of pages src_pages[i] to dst_pages[i], every layer
 * (no page twice in dst_pages, none in both; no bookkeeping).
 */
int sats_cache_extend(const sats_kv_cache *cache, const sats_kv_pages *pages, const int32_t *seqs, const int32_t *add,
                      int64_t n, int32_t *status, hipStream_t stream);
int sats_cache_fork(const sats_kv_cache *cache, const sats_kv_pages *pages, const int32_t *src, const int32_t *dst,
                    int64_t n, int32_t *status, hipStream_t stream);
int sats_cache_free(const sats_kv_cache *cache, const sats_kv_pages *pages, const int32_t *seqs, const int32_t *begin,
                    const int32_t *end, int64_t n, hipStream_t stream);
int sats_cache_compact(const sats_kv_cache *cache, const sats_kv_pages *pages, int32_t *n_used, hipStream_t stream);
int sats_cache_copy(const sats_kv_cache *cache, const int32_t *src_pages, const int32_t *dst_pages, int64_t n,
                    hipStream_t stream);

/*
 * The next id of n rows of logits [vocab], `stride` elements apart, from one
 * number u[i] of [0, 1) a row.  Per row (device arrays, or NULL for the value in
 * brackets): temperature [1; not above 0: the largest logit], top_k [0: all],
 * top_p [1], min_p [0].  Id i weighs w_i = round(2^40 exp((l_i - max) / T)), a whole
 * number (the exponential in float32; NaN logits count as -inf).  In the order of
 * falling logit, the lower id first where two are equal, an id is kept while its
 * rank is below top_k, the weights before it are below top_p times those of the
 * top k, and exp(..) >= min_p; the first id always, one of weight 0 never.
 * tokens[i] is the first id, in the order of ids, at which the running sum of kept
 * weights exceeds u[i] times their total, so that it does not depend on any order
 * of summation; -1 for a row without a logit above -inf.  prob [n] (or NULL): its
 * share of the kept weights; n_kept [n] (or NULL): how many ids were kept.
 * vocab <= 2^22.
 */
int sats_sample(const void *logits, int elem_bytes, int64_t stride, int64_t n, int64_t vocab, const float *temperature,
                const int32_t *top_k, const float *top_p, const float *min_p, const float *u, int32_t *tokens,
                float *prob, int32_t *n_kept, hipStream_t stream);

/*
 * Rules on logits, ahead of sats_sample: out = logits [n][vocab] after, in this order and in float32,
 *   l <- l / repetition (l > 0) or l repetition (else)   ids among the row's ids so far
 *   l <- l - frequency count - presence [count > 0]      count: of the id in the answer
 *   l <- l + the sum of the id's biases, in their order
 *   l <- -infinity                                       ids without a bit in the row's mask
 * each rounded once to the type of out (elem_bytes and out_elem_bytes: 2 or 4; strides in elements).
 * out may be logits itself (same stride and type): eight neighbours that no rule changes are then not
 * touched; other overlap is rejected.  All arrays are on the device; max_history, n_bias or n_masks 0: no such rule:
 *   history        [n_seqs][history_stride] ids so far, the prompt first: of row i the first history_len[s] of row
 *                  s = seqs[i] (seqs NULL: i), at most max_history; from prompt_len[s] on (NULL: 0) they are
 *                  the answer
 *   repetition, frequency, presence   [n], a number a row (NULL: 1, 0, 0)
 *   bias_ids, bias [n_bias] ids and what is added to them, of row i from bias_start[i] to bias_start[i + 1] - 1
 *   masks          [n_masks][mask_stride] bits, id x in bit x % 32 of word x / 32; row i has mask
 *                  mask_of[i] (NULL: i), none where that is no mask
 * Ids outside the vocabulary are passed over, lengths cut off to their arrays.  vocab <= 2^22, n < 65536.
 */
typedef struct {
  const int32_t *seqs, *history, *history_len, *prompt_len;
  int64_t n_seqs, history_stride, max_history;
  const float *repetition, *frequency, *presence;
  const int32_t *bias_start, *bias_ids;
  const float *bias;
  int64_t n_bias;
  const uint32_t *masks;
  const int32_t *mask_of;
  int64_t n_masks, mask_stride;
} sats_logit_rules;
int sats_adjust_logits(const void *logits, int elem_bytes, int64_t stride, const sats_logit_rules *rules, void *out,
                       int out_elem_bytes, int64_t out_stride, int64_t n, int64_t vocab, hipStream_t stream);

/*
 * Allocate the scratch memory of (current device, stream) for sats_prefix_attention calls over such a cache, of
 * batches and prefixes up to these sizes (their pointers may be NULL) and any window: the batch's rows, n_q_heads a
 * token, in each of the parts that a launch splits their keys into, head_dim + 2 floats each (where
 * rows have many keys 196608 of them and more), and a page table row a group.  Else as
 * sats_reserve_serving, which covers the other calls; a stream's scratch memory is one for all.
 */
int sats_reserve_prefix(const sats_kv_cache *cache, const sats_kv_batch *batch, const sats_kv_prefix *prefix, int64_t n_q_heads,
                        hipStream_t stream);

/*
 * Allocate the scratch memory of (current device, stream) for serving calls: page calls
 * of up to max_items items over n_pages pages, sampling of max_rows rows of vocab
 * logits, attention of any batch with heads of head_dim (zeros: none).
 * Without it a call allocates what it needs, once; a call under stream capture that
 * would have to allocate returns SATS_ERR_WORKSPACE.  A stream's scratch memory is as
 * large as the largest of these needs (grown, at least twice as large where there is
 * that much) and kept until sats_release: sampling 8 bytes a logit and 24 KB a row, of
 * 512 rows at most (525 MB for 512 x 128256); attention 256 KB x (head_dim + 2); pages
 * 16 bytes a page and 20 an item.
 */
int sats_reserve_serving(int64_t max_items, int64_t n_pages, int64_t max_rows, int64_t vocab, int64_t head_dim,
                         hipStream_t stream);

/* Free every workspace of the calling process, and the kept buffers of the
 * routing-table construction and of the calibration (waits for calls that
 * other threads are issuing, and synchronises each device).  Graphs that
 * recorded a call of the library must not be replayed afterwards. */
int sats_release(void);

/* Thread-local text of the last error returned on this thread ("" if none). */
const char *sats_last_error(void);

/*
 * Kernel timing for measurement.  sats_timing_begin(kind, capacity) arms
 * HIP-event pairs around the next `capacity` launches of one kernel kind
 * (SATS_K_*), recorded on the stream the kernel is launched on.
 * sats_timing_end(kind, &total_ms, &count) waits for the recorded events,
 * returns the summed duration and the number of launches timed, and disarms.
 * SATS_K_ROUTE_ACCUM times the per-chunk pass over the routing split
 * (route_part_kernel; for vocabularies past 2^22 ids the atomic form,
 * route_accum_kernel), SATS_K_ROUTE_MERGE the merge of its entries.
 */
enum { SATS_K_GATE = 0, SATS_K_UP = 1, SATS_K_DOWN = 2, SATS_K_INSPECT = 3, SATS_K_DENSE = 4,
       SATS_K_DEC_LAYER = 5, SATS_K_DEC_LORA_V = 6, SATS_K_CAL_ERR = 7, SATS_K_CAL_GATEUP = 8,
       SATS_K_ROUTE_ACCUM = 9, SATS_K_LORA_V = 10, SATS_K_DEC_REDUCE = 11, SATS_K_DENSE_DOWN = 12,
       SATS_K_DEC_REDUCE_LORA = 13, SATS_K_ROUTE_MERGE = 14, SATS_K_COUNT = 15 };
int sats_timing_begin(int kind, int capacity);
int sats_timing_end(int kind, double *total_ms, int64_t *count);
const char *sats_kernel_name(int kind);

#ifdef __cplusplus
}
#endif

#endif /* SATS_H */
