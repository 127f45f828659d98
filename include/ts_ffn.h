/*
 * ts_ffn.h -- C ABI of libtsffn: the decode-time activation-sparse dReLU FFN
 * of Turbo Sparse (arXiv 2406.05955) on one GB300 (sm_103a).
 *
 * The operation (Eq. 1 in Sec. 2 with the dReLU of Eq. 2 in Sec. 3.2):
 *     g = x W_gate,  u = x W_up,  c = max(0, g) * max(0, u),  y = c W_down
 * Only neurons with g_j > 0 cost W_up bytes and only neurons with g_j > 0 and
 * u_j > 0 ("active", the non-zero activations counted in Sec. 6.2) cost
 * W_down bytes; the result equals the dense formula.
 *
 * Layout. All three weight matrices are neuron-major, [m][d] row-major:
 * row j of w_gate / w_up is neuron j's input weights (column j of the paper's
 * d x m matrices), row j of w_down is neuron j's output row (row j of the
 * paper's m x d W_down). Activations x are [batch][d] in the weight dtype;
 * outputs y and the residual stream h are [batch][d] fp32. Rows of every
 * weight matrix must start on 16-byte boundaries (pointer 16-byte aligned
 * and d * sizeof(element) a multiple of 16).
 *
 * Ownership. Weights, x, y, h and index lists are caller-owned device
 * memory; a handle borrows the weight pointers (they must outlive it) and
 * owns only its scratch, allocated once by *_create.
 *
 * Weights are taken to be constant. A call may read weight rows while the
 * kernel before it on the stream ends: if that very kernel writes weights, put
 * an event wait or another operation between. (MoE calls, stacks of more than
 * two tokens and bf16 forwards of more than 8 with a 16-byte aligned x read
 * them after it.)
 *
 * Execution. Every *_forward call is asynchronous on `stream`, performs no
 * host synchronisation and no allocation, and may be captured in a CUDA
 * graph. One forward may be in flight per handle at a time.
 *
 * Errors. Argument errors are returned synchronously and nothing is
 * launched. Errors the GPU detects (an out-of-range or unsorted index list)
 * never trap: the offending entries are skipped, a status word in the
 * handle's scratch records it, and ts_*_get_error reports it.
 */
#ifndef TS_FFN_H
#define TS_FFN_H

#include <stdint.h>
#include <cuda_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    TS_OK = 0,
    TS_ERR_INVALID_ARG = 1,  /* bad pointer, size, alignment or batch       */
    TS_ERR_CUDA = 2,         /* a CUDA runtime call failed                   */
    TS_ERR_OOM = 3,          /* scratch allocation failed                    */
    TS_ERR_BAD_INDEX = 4,    /* the GPU saw an out-of-range/unsorted list    */
    TS_ERR_TIMEOUT = 5,      /* a bounded device-side wait gave up           */
    TS_ERR_UNSUPPORTED = 6,  /* valid request this build does not handle     */
    TS_ERR_SCRATCH = 7       /* a scratch guard zone was overwritten         */
} ts_status;

/*
 * Weight storage. TS_F32 and TS_BF16 rows hold d elements. TS_INT4 rows (the
 * weight-only 4-bit storage of the paper's INT4 models, Tables 7-9) hold d/2
 * bytes of 4-bit codes followed by d/32 little-endian IEEE binary16 scales,
 * one per group of 32 consecutive elements: weight i = scale[i/32] *
 * (code[i] - 8). Group G's codes are the 16 bytes at offset 16G, read as four
 * little-endian 32-bit words w0..w3; element 8s + 2t + h of the group
 * (s, t in 0..3, h in 0..1) is nibble s + 4h of word t, i.e. bits
 * [4(s + 4h), 4(s + 4h) + 4) of w_t (the order in which one tensor-core lane
 * consumes them). An INT4 row is 9d/16 bytes and needs d to be a multiple of
 * 256; its activations x are bf16.
 */
typedef enum {
    TS_F32 = 0,
    TS_BF16 = 1,
    TS_INT4 = 2,
    TS_E4M3 = 3  /* only where named below: 8-bit floating point (4 exponent and 3 fraction bits, largest value
                    448, no infinity) with fp32 scales for blocks of 128: the products over many tokens */
} ts_dtype;

typedef struct ts_ffn ts_ffn;     /* one dReLU FFN (one layer or one expert) */
typedef struct ts_moe ts_moe;     /* one top-k MoE layer over ts_ffn experts */
typedef struct ts_graph ts_graph; /* a captured multi-layer forward          */
typedef struct ts_predictor ts_predictor; /* one layer's activation predictor */

/* Human-readable name of a status code (static string, never NULL). */
const char* ts_status_str(ts_status s);

/* ABI version of this library (major * 100 + minor). */
int ts_version(void);

/*
 * Create a handle for one dReLU FFN (Eq. 1 + Eq. 2).
 *   d, m       model width and number of neurons (d >= 1, m >= 1)
 *   wdtype     storage type of the weights (and of x, except INT4: bf16 x)
 *   w_gate, w_up, w_down  device pointers, [m][d] each, or [m][9d/16] bytes
 *              for TS_INT4 (borrowed)
 *   max_batch  largest batch a forward may pass (1..64)
 * Allocates the handle's scratch on the current device.
 * Returns TS_ERR_INVALID_ARG for bad sizes/pointers/alignment, TS_ERR_OOM if
 * scratch cannot be allocated, TS_ERR_CUDA for other CUDA failures.
 */
ts_status ts_ffn_create(ts_ffn** out, int d, int m, ts_dtype wdtype, const void* w_gate,
                        const void* w_up, const void* w_down, int max_batch);
void ts_ffn_destroy(ts_ffn* h);

/*
 * y = dReLU-FFN(x) for `batch` tokens (Eq. 1 + Eq. 2), on `stream`.
 *   x          device [batch][d], wdtype
 *   y          device [batch][d] fp32, overwritten
 *   active_idx NULL: the active sets are detected from the signs of g and u.
 *              Otherwise a device list of n_active neuron ids (0 <= n_active
 *              <= m), strictly ascending, shared by every token of the
 *              batch: the predictor-driven mode of Sec. 7. Gate, up and
 *              down then touch only listed rows, and listed neurons that
 *              are not dReLU-active contribute 0; unlisted neurons are
 *              skipped even if they would be active.
 * batch == 0 is a no-op. Equivalent to ts_ffn_gate_up then ts_ffn_down.
 */
ts_status ts_ffn_forward(ts_ffn* h, const void* x, int batch, float* y, cudaStream_t stream,
                         const int32_t* active_idx, int n_active);

/*
 * y = (Combined(x) * Mask(x)) W_down with the top-k magnitude mask of Eq. 3
 * and Eq. 4 (Sec. 3.2): per token, Mask keeps the `keep` neurons with the
 * largest |Combined| = max(0, g) max(0, u) (Eq. 2), a lower neuron index
 * winning a tie; the others contribute 0.
 *   x, batch, y, stream   as ts_ffn_forward (no predictor list)
 *   keep                  0 <= keep <= m; keep >= the number of dReLU-active
 *                         neurons gives ts_ffn_forward's result up to the
 *                         fp32 summation order of the down projection (the
 *                         masked path gathers W_down by column slices)
 * The per-token both-active sets that ts_ffn_get_active reports afterwards
 * are the kept active neurons. The selection compares the fp32 c values.
 * Errors: TS_ERR_INVALID_ARG for a bad keep or batch, TS_ERR_UNSUPPORTED for
 * INT4 rows.
 */
ts_status ts_ffn_forward_topk(ts_ffn* h, const void* x, int batch, float* y, cudaStream_t stream, int keep);

/*
 * First step alone: gate GEMV + ReLU + compaction, then the gathered up
 * projection over gate-active rows + dReLU product + second compaction
 * (into the handle's scratch). Arguments as ts_ffn_forward. Batches of more
 * than 8 tokens (INT4: 2) take several steps: ts_ffn_forward must be used.
 */
ts_status ts_ffn_gate_up(ts_ffn* h, const void* x, int batch, cudaStream_t stream,
                         const int32_t* active_idx, int n_active);

/* Second step alone: gathered down projection of the rows the preceding
   ts_ffn_gate_up on this handle marked active; writes y [batch][d] fp32.
   After another call of the same batch (forward, top-k, stack), the rows and
   c that it left. */
ts_status ts_ffn_down(ts_ffn* h, int batch, float* y, cudaStream_t stream);

/*
 * Pre-norm residual stack of n_layers FFNs on the fp32 residual h [batch][d]
 * (updated in place): for each layer l,
 *     x = round_wdtype(h / sqrt(mean(h^2) + 1e-5)),  x[d-1] = 1,
 *     h = h + FFN_l(x).
 * (The normalisation and bias channel are synthetic glue: the paper studies
 * the FFN alone.) active_idx / n_active: NULL, or per-layer lists as in
 * ts_ffn_forward (an entry may be NULL). All layers need the same d, wdtype.
 */
ts_status ts_stack_forward(ts_ffn* const* layers, int n_layers, float* h, int batch,
                           cudaStream_t stream, const int32_t* const* active_idx,
                           const int* n_active);

/*
 * Active sets of the last forward on this handle, copied to host memory
 * (synchronises `stream`). token >= 0 selects one token, -1 the union over
 * the batch. gate_idx / both_idx are host arrays of at least m entries
 * (either may be NULL); the lists come back ascending (neuron ids).
 */
ts_status ts_ffn_get_active(ts_ffn* h, cudaStream_t stream, int token, int32_t* gate_idx,
                            int* n_gate, int32_t* both_idx, int* n_both);

/* Synchronise `stream`, return and clear the device status word:
   TS_OK, TS_ERR_BAD_INDEX, or TS_ERR_TIMEOUT (a bounded device-side wait ran
   out; the kernels wound down instead of hanging and the results of that
   forward are undefined). */
ts_status ts_ffn_get_error(ts_ffn* h, cudaStream_t stream);

/*
 * Scratch guard check (a debugging aid, not part of the method). Every block
 * of a handle's device scratch (partial sums, bitmaps, c values, status
 * word, ...) is followed by a guard zone filled with one byte value when the
 * handle is created. This call synchronises `stream` and compares every zone
 * with its fill: TS_OK if all are intact, TS_ERR_SCRATCH if a kernel wrote
 * past the end of a block, TS_ERR_INVALID_ARG for a NULL handle.
 * ts_ffn_poke_guard overwrites one byte of guard zone i (0 <= i < the number
 * of blocks; TS_ERR_INVALID_ARG otherwise) from the host, so that a test can
 * check that the check fires; the handle stays usable.
 */
ts_status ts_ffn_check_scratch(ts_ffn* h, cudaStream_t stream);
ts_status ts_ffn_poke_guard(ts_ffn* h, int i);

/*
 * Test hook for the failure-detection path (not part of the method): while
 * `on` is nonzero, forwards on this handle make one consumer warp of every
 * gate+up CTA wait on a barrier that nothing arrives at. The wait, like every
 * device-side wait of the library, gives up after about one second, records
 * TS_ERR_TIMEOUT in the status word and lets the kernels wind down, so the
 * CUDA context stays usable. Such a forward takes a few seconds and its
 * output is undefined. Returns TS_ERR_INVALID_ARG for a NULL handle.
 */
ts_status ts_ffn_set_test_stall(ts_ffn* h, int on);

/*
 * One FFN forward with no handle and no device allocation. The paper has no
 * counterpart: this is a calling convention, not part of the method. It
 * computes exactly what ts_ffn_forward computes, up to the order of sums, for
 * callers that cannot allocate device memory when they run the FFN (a memory
 * pool that is full or must not grow, code that must not take the implicit
 * device synchronisation of cudaFree, a plain C caller with nowhere to keep
 * a handle).
 *   d, m, wdtype, w_gate, w_up, w_down   as ts_ffn_create (borrowed for the call)
 *   x, batch, y, stream, active_idx, n_active   as ts_ffn_forward
 * Scratch: a fixed array of the library's static device memory (~0.8 MB per
 * device), sized for m <= TS_NOALLOC_MAX_M and batch <= TS_NOALLOC_MAX_BATCH;
 * larger sizes return TS_ERR_UNSUPPORTED and launch nothing. Nothing is
 * allocated or freed by this call.
 * Set-up: the first call on a device (that device current) looks up the
 * scratch address and sets kernel attributes; make that first call before
 * any stream capture on the device. Each call compares the current context
 * with the one the set-up was made in and repeats the set-up when the
 * context was recreated (e.g. after cudaDeviceReset).
 * Concurrency: all calls on a device share the one scratch, so calls whose
 * executions overlap (other streams, unordered host threads) race; the
 * caller serialises them.
 * Errors: argument errors as ts_ffn_create / ts_ffn_forward. A device-side
 * list error (unsorted or out-of-range ids) skips the offending entries but
 * is not reported by this entry point.
 */
#define TS_NOALLOC_MAX_M 16384
#define TS_NOALLOC_MAX_BATCH 64
ts_status ts_ffn_forward_noalloc(int d, int m, ts_dtype wdtype, const void* w_gate,
                                 const void* w_up, const void* w_down, const void* x, int batch,
                                 float* y, cudaStream_t stream, const int32_t* active_idx,
                                 int n_active);

/*
 * Top-k MoE layer (Sec. 4; Mixtral: 2 of 8 experts, Sec. 6.2):
 *     r = x W_r^T, pick the top_k largest logits (lower expert index wins a
 *     tie), w = softmax over the picked logits,
 *     y_t = sum_k w_{t,k} * FFN_{e_{t,k}}(x_t),
 * each expert itself a neuron-sparse dReLU FFN.
 *   w_router   device [n_experts][d], wdtype (bf16 when the experts are
 *              TS_INT4; borrowed)
 *   experts    n_experts handles (same d and wdtype; borrowed)
 *   n_experts  1..16, top_k 1..min(4, n_experts), max_batch 1..8 (1..2 for
 *              INT4 experts)
 */
ts_status ts_moe_create(ts_moe** out, int d, int n_experts, int top_k, ts_dtype wdtype,
                        const void* w_router, ts_ffn* const* experts, int max_batch);
void ts_moe_destroy(ts_moe* h);

/* y [batch][d] fp32 = MoE(x [batch][d] wdtype), on `stream`. */
ts_status ts_moe_forward(ts_moe* h, const void* x, int batch, float* y, cudaStream_t stream);

/* Pre-norm residual stack of MoE layers on h [batch][d] fp32 (in place),
   with the same glue as ts_stack_forward. */
ts_status ts_moe_stack_forward(ts_moe* const* layers, int n_layers, float* h, int batch,
                               cudaStream_t stream);

/* Routing of the last forward, to host memory (synchronises `stream`):
   sel [batch][top_k] expert ids (largest logit first), w [batch][top_k]. */
ts_status ts_moe_get_routing(ts_moe* h, cudaStream_t stream, int32_t* sel, float* w);

/* Per-expert active sets of the last MoE forward (synchronises `stream`):
   as ts_ffn_get_active for expert `expert` and batch token `token` (-1: the
   union over the tokens routed to that expert). */
ts_status ts_moe_get_active(ts_moe* h, cudaStream_t stream, int expert, int token,
                            int32_t* gate_idx, int* n_gate, int32_t* both_idx, int* n_both);

/* As ts_ffn_get_error, for the MoE layer's router and grouped kernels. */
ts_status ts_moe_get_error(ts_moe* h, cudaStream_t stream);

/* As ts_ffn_check_scratch, for the MoE layer's scratch. */
ts_status ts_moe_check_scratch(ts_moe* h, cudaStream_t stream);

/*
 * Activation predictor of one FFN layer (Sec. 7: a predictor per FFN block,
 * per expert for MoE; the paper gives no architecture, so this is a reading):
 * a two-layer ReLU MLP over the layer's input x,
 *     hid = max(0, W1 x),   s = W2 hid      (s[j]: score of neuron j),
 * and a batch's list is the K neurons with the largest key
 * key[j] = max over the batch's tokens of s[t][j], a lower neuron id winning
 * a tie, emitted in ascending id order -- the input of the predictor-driven
 * mode of ts_ffn_forward / ts_stack_forward.
 *   d, r, m    input width, hidden width, neurons; d and r multiples of 256
 *              (bf16) or 128 (fp32), r / that multiple one of 1, 2, 4, 8
 *   dtype      TS_BF16 or TS_F32: the type of W1, W2 and x
 *   w1, w2     device [r][d] and [m][r], row-major (borrowed, 16-byte aligned)
 *   max_batch  largest batch of a prediction, 1..8
 * Scores accumulate in fp32. Returns TS_ERR_UNSUPPORTED for sizes without a
 * kernel, TS_ERR_OOM if scratch cannot be allocated. The handle owns its
 * scratch (hidden-layer partials, per-neuron keys and a histogram of the
 * keys), which serves one prediction at a time: predictions with the same
 * handle must not overlap on the GPU (use one stream, or one handle per
 * stream).
 */
ts_status ts_predictor_create(ts_predictor** out, int d, int r, int m, ts_dtype dtype, const void* w1,
                              const void* w2, int max_batch);
void ts_predictor_destroy(ts_predictor* p);

/* As ts_ffn_check_scratch, for the predictor's scratch. */
ts_status ts_predictor_check_scratch(ts_predictor* p, cudaStream_t stream);

/*
 * list[0..K) = the predicted neurons for the batch x [batch][d] (device,
 * predictor dtype), ascending; `list` is a caller-owned device buffer of at
 * least K int32. scores: NULL, or a device [batch][m] fp32 buffer that
 * receives s. batch == 0 or K == 0 is a no-op. 0 <= K <= m, else
 * TS_ERR_INVALID_ARG. Asynchronous on `stream`.
 */
ts_status ts_predict(ts_predictor* p, const void* x, int batch, int K, int32_t* list, float* scores,
                     cudaStream_t stream);

/*
 * ts_stack_forward with a predictor per layer: for each layer l,
 *     x = round_wdtype(h / sqrt(mean(h^2) + 1e-5)),  x[d-1] = 1,
 *     lists[l][0..K[l]) = ts_predict(preds[l], x, K[l]),
 *     h = h + FFN_l(x) over the listed neurons only (predictor-driven mode).
 * preds[l] must match layer l's d, m and activation dtype (bf16 for INT4
 * layers). lists[l]: caller-owned device buffers of K[l] int32 that keep the
 * lists for inspection. K[l] == 0 leaves h unchanged for that layer.
 */
ts_status ts_stack_forward_predicted(ts_ffn* const* layers, ts_predictor* const* preds, int n_layers,
                                     float* h, int batch, const int* K, int32_t* const* lists,
                                     cudaStream_t stream);

/*
 * Capture a whole multi-layer forward once as a CUDA graph and replay it.
 * The captured calls keep the pointers given here; replaying reads and
 * writes the same buffers. ts_graph_capture_stack captures
 * ts_stack_forward(layers, n_layers, h, batch, ., active_idx, n_active);
 * ts_graph_capture_moe_stack captures ts_moe_stack_forward.
 */
ts_status ts_graph_capture_stack(ts_graph** out, ts_ffn* const* layers, int n_layers, float* h,
                                 int batch, const int32_t* const* active_idx, const int* n_active);
ts_status ts_graph_capture_moe_stack(ts_graph** out, ts_moe* const* layers, int n_layers,
                                     float* h, int batch);
/* Captures ts_stack_forward_predicted(layers, preds, n_layers, h, batch, K, lists, .). */
ts_status ts_graph_capture_stack_predicted(ts_graph** out, ts_ffn* const* layers, ts_predictor* const* preds,
                                           int n_layers, float* h, int batch, const int* K,
                                           int32_t* const* lists);
/*
 * The same stack as ts_graph_capture_stack (Eq. 1 with the dReLU of Eq. 2 per
 * layer, the stack glue between layers), fused into one persistent launch:
 * every CTA (one per SM, all resident at once by a cooperative launch) runs
 * each layer's gate+up phases and its share of the down projection, then the
 * CTAs meet at a grid barrier, sum the partial down projections by column
 * slices into h, meet again and go on with the next layer. No launch gaps
 * between layers; one launch per replay, plus a memset that clears the
 * barrier words.
 *   layers, n_layers, h, batch, active_idx, n_active   as ts_graph_capture_stack
 * Supported: bf16 layers of one width d, batch 1 or 2, the same grid for
 * every layer; otherwise TS_ERR_UNSUPPORTED (capture the unfused stack then).
 * The graph owns a small device table of the layers' parameters (allocated
 * here, freed by ts_graph_destroy). Replays are bitwise identical to the
 * unfused graph's only up to the fp32 summation order of the reduction (the
 * partials are added in CTA order in both, in different groupings).
 * Device-side errors (bad list entries, a barrier that waited past its
 * bound: TS_ERR_TIMEOUT, after which the CTAs stop and h is undefined) are
 * reported by ts_ffn_get_error on layers[0] (barriers) and on each layer
 * (lists).
 */
ts_status ts_graph_capture_stack_fused(ts_graph** out, ts_ffn* const* layers, int n_layers, float* h,
                                       int batch, const int32_t* const* active_idx, const int* n_active);
ts_status ts_graph_launch(ts_graph* g, cudaStream_t stream);
void ts_graph_destroy(ts_graph* g);

/*
 * Layers of routed experts over many tokens at once (a prompt, a large batch).
 *
 * The forwards above read single weight rows, which pays while few tokens leave
 * most neurons inactive. Over a prompt every neuron is active for some token, so
 * the same layer (Sec. 4: top_k of n_experts, each expert Eq. 1 + Eq. 2) is a few
 * large matrix products. The steps are entry points of their own:
 *     ts_route         experts of every token, tokens of every expert
 *     ts_gather_rows   rows in the experts' order, copied
 *     ts_quant_rows    the same, rounded to TS_E4M3
 *     ts_grouped_*     each expert's rows times its weights
 *     ts_combine_rows  each token's rows summed by their routing weights
 * and ts_prompt_forward runs them in a row. All are asynchronous on `stream`, do
 * not allocate and may be captured in a CUDA graph. The paper has no counterpart to
 * how tokens are grouped or rounded to 8 bits: these are readings.
 */

/*
 * Routing of `tokens` tokens from the router's logits.
 *   logits     device [tokens][n_experts] fp32
 *   n_experts  1..256, top_k 1..min(8, n_experts); tokens * top_k below 2^30
 *   sel, w     device [tokens][top_k]: the picked experts, largest logit first (the
 *              lower index wins a tie), and the softmax over the picked logits
 *   offsets    device [n_experts + 1]: expert e has rows offsets[e] .. offsets[e + 1] - 1
 *   rows       device [tokens * top_k]: the token of each row, ascending within an
 *              expert; entries from offsets[n_experts] on are left as they were
 *   slots      device [tokens][top_k]: the row of each pick
 * An expert whose logit is -infinity or NaN is never picked. A token with fewer
 * experts left than top_k (padding: none) gets sel = -1, w = 0, slot = -1 for the
 * rest. Picks of logit +infinity share the weight equally. tokens == 0 writes
 * offsets only. No atomics: the same logits give the same rows.
 */
ts_status ts_route(const float* logits, int tokens, int n_experts, int top_k, int32_t* sel, float* w,
                   int32_t* offsets, int32_t* rows, int32_t* slots, cudaStream_t stream);

/*
 * out[r] = x[rows[r]] for r < min(*n, max_rows); the rows of `out` behind are left as they were.
 *   x         device, n_src rows of k elements (TS_BF16 or TS_F32), ldx elements apart
 *   rows      device [max_rows] int32, NULL: row r itself. An entry outside
 *             0..n_src-1 leaves its row of `out` as it was.
 *   n         device int32 (as &offsets[n_experts] of ts_route), NULL: max_rows
 *   out       device [max_rows][k], same type
 * Rows of x and out start on 16-byte boundaries. TS_ERR_UNSUPPORTED: k above 2^24 or max_rows above 2^30.
 */
ts_status ts_gather_rows(const void* x, int64_t ldx, ts_dtype dtype, int n_src, int k, const int32_t* rows,
                         const int32_t* n, int max_rows, void* out, cudaStream_t stream);

/*
 * Rows rounded to TS_E4M3 with an fp32 scale for each block of 128 elements:
 *     scale[b][r] = max |x[rows[r]][128 b .. 128 b + 127]| / 448
 * (at least 2^-100; 1 where the block is all zero) and q[r][i] = x / scale (as an fp32 quotient), rounded to the
 * nearest, ties to even. Arguments as ts_gather_rows (TS_BF16 or TS_F32; k a multiple of 16).
 *   q         device [max_rows][k] e4m3
 *   scale     device [ceil(k / 128)][max_rows] fp32: a block's scales lie together
 * NaN stays NaN in its place; a block that holds an infinity has an infinite scale and
 * stands for NaN throughout.
 */
ts_status ts_quant_rows(const void* x, int64_t ldx, ts_dtype dtype, int n_src, int k, const int32_t* rows,
                        const int32_t* n, int max_rows, void* q, float* scale, cudaStream_t stream);

/*
 * y[t][:] = sum over j < top_k of w[t][j] * src[slots[t][j]][:], in order of j, in fp32.
 *   src       device [n_rows][n] TS_F32 or TS_BF16, on a boundary of its elements
 *   slots, w  device [tokens][top_k]; a slot outside 0..n_rows-1 adds nothing
 *   top_k     1..8; n 1..2^30, at most 2^30 tokens
 *   y         device [tokens][n] fp32, overwritten
 */
ts_status ts_combine_rows(const void* src, ts_dtype dtype, int n_rows, int n, const int32_t* slots, const float* w,
                          int tokens, int top_k, float* y, cudaStream_t stream);

typedef struct ts_grouped ts_grouped; /* matrix products of groups of rows, each with its own weights */

typedef enum {
    TS_NK = 0,  /* a weight matrix is [n][k]: y = x W^T (as w_gate, w_up) */
    TS_KN = 1   /* [k][n]: y = x W (as w_down, stored by neuron)          */
} ts_layout;

/*
 * Products of ragged groups of rows: for each group e,
 *     y[r] = x[r] . W_e                                      (plain)
 *     y[r] = max(0, x[r] . W_e) * max(0, x[r] . U_e)         (gated: Eq. 1 with the dReLU of Eq. 2)
 * for offsets[e] <= r < offsets[e + 1]. One group is an ordinary matrix product.
 * A gated product is 0 unless both factors are positive (so where either is NaN).
 *   n_groups   1..256
 *   n, k       outputs (at most 2^30) and inputs of a weight matrix
 *   wdtype     TS_BF16 (x bf16) or TS_E4M3 (x e4m3)
 *   layout     TS_NK, or TS_KN for plain TS_BF16 products
 *   w          host array of n_groups device pointers (borrowed, 16-byte aligned), each
 *              [n][k] or [k][n]; rows of weights start on 16-byte boundaries
 *   w_up       NULL, or the same for U (gated)
 *   scale, scale_up  TS_E4M3: host arrays of device pointers, each [ceil(n / 128)][ceil(k / 128)]
 *              fp32: a scale for each 128 x 128 block of weights. NULL for TS_BF16.
 *   max_rows   largest number of rows of a forward, at most 2^30
 * k must be a multiple of 8 (TS_BF16) or 16 (TS_E4M3), at most 2^28, n a multiple of 8 for TS_KN.
 * Products are exact, sums are held in fp32; those of bf16 weights are truncated at every 16 of k within 256 of k, for
 * TS_BF16 outputs within 1024 (over Gaussian rows, relative in 2-norm, 2.4e-7 and, before the rounding, 1e-6). Returns TS_ERR_INVALID_ARG,
 * TS_ERR_UNSUPPORTED (wdtype or layout without a kernel), TS_ERR_OOM or TS_ERR_CUDA.
 */
ts_status ts_grouped_create(ts_grouped** out, int n_groups, int n, int k, ts_dtype wdtype, ts_layout layout,
                            const void* const* w, const void* const* w_up, const float* const* scale,
                            const float* const* scale_up, int max_rows);
void ts_grouped_destroy(ts_grouped* h);

/*
 * One forward over `rows` rows (0..max_rows; 0 is a no-op).
 *   x, ldx     device, rows of k elements ldx apart, each starting on a 16-byte boundary
 *   x_scale, ld_scale  TS_E4M3: device [ceil(k / 128)][ld_scale] fp32, ld_scale >= rows (as
 *              ts_quant_rows writes them). NULL for TS_BF16.
 *   offsets    device [n_groups + 1] int32, ascending, within 0..rows; NULL with one
 *              group: all rows. A group whose bounds are descending or out of range is
 *              skipped and recorded (ts_grouped_get_error: TS_ERR_BAD_INDEX).
 *   y, ldy     device, rows of n elements ldy apart (ydtype TS_BF16, rounded once, or TS_F32), on a boundary
 *              of its elements; rows that no group has are left as they were
 * One forward may be in flight per handle (a replay of a graph that holds one counts), and its device is the current
 * one (else TS_ERR_INVALID_ARG).
 */
ts_status ts_grouped_forward(ts_grouped* h, const void* x, int64_t ldx, const float* x_scale, int64_t ld_scale,
                             const int32_t* offsets, int rows, void* y, int64_t ldy, ts_dtype ydtype,
                             cudaStream_t stream);
/* As ts_ffn_get_error and ts_ffn_check_scratch. */
ts_status ts_grouped_get_error(ts_grouped* h, cudaStream_t stream);
ts_status ts_grouped_check_scratch(ts_grouped* h, cudaStream_t stream);
/* As ts_ffn_set_test_stall: one warp that keeps sums, after its last tile, of every CTA of the next forwards. */
ts_status ts_grouped_set_test_stall(ts_grouped* h, int on);

typedef struct ts_experts ts_experts; /* the weights of one layer of experts, for many tokens */
typedef struct ts_prompt ts_prompt;   /* scratch of layers over many tokens                    */

/*
 * One layer over many tokens: top_k of n_experts dReLU FFNs (Sec. 4), or a single one.
 *   d, m       model width and neurons of an expert; multiples of 8 (TS_BF16) or 16 (TS_E4M3), at most 2^24
 *   n_experts  1..256, top_k 1..min(8, n_experts)
 *   wdtype     TS_BF16 or TS_E4M3; activations x are bf16 either way
 *   w_router   device [n_experts][d] bf16; NULL with one expert, which then has weight 1
 *   w_gate, w_up   host arrays of n_experts device pointers, each [m][d]
 *   w_down     the same, each [m][d] (by neuron, as ts_ffn_create) for TS_BF16, [d][m] for TS_E4M3
 *   s_gate, s_up, s_down   TS_E4M3: host arrays of device pointers to scales as in ts_grouped_create,
 *              [ceil(m / 128)][ceil(d / 128)] twice and [ceil(d / 128)][ceil(m / 128)]. NULL for TS_BF16.
 * All weights are borrowed. The handle has no scratch: it may be used by forwards with different ts_prompt at once.
 */
ts_status ts_experts_create(ts_experts** out, int d, int m, int n_experts, int top_k, ts_dtype wdtype,
                            const void* w_router, const void* const* w_gate, const void* const* w_up,
                            const void* const* w_down, const float* const* s_gate, const float* const* s_up,
                            const float* const* s_down);
void ts_experts_destroy(ts_experts* e);

/* Scratch for forwards of up to max_tokens tokens through any layers of these sizes (arguments as
   ts_experts_create; n_experts and top_k may be smaller in a layer). One forward may be in flight per
   handle (a replay of a graph that holds one counts); scratch, layer and the current device are one
   device (else TS_ERR_INVALID_ARG). */
ts_status ts_prompt_create(ts_prompt** out, int d, int m, int n_experts, int top_k, ts_dtype wdtype, int max_tokens);
void ts_prompt_destroy(ts_prompt* p);

/*
 * y[t] = sum over the picked experts of w * FFN_e(x[t]) (one expert: FFN(x[t])), as ts_moe_forward and
 * ts_ffn_forward compute it for few tokens, with c = max(0, g) max(0, u) rounded to bf16 before the down product
 * (a GEMM operand), and for TS_E4M3 x and c rounded to e4m3 by ts_quant_rows.
 *   x       device [tokens][d] bf16, 0 <= tokens <= max_tokens
 *   y       device [tokens][d] fp32, overwritten (a token with no expert, all of its router logits NaN: 0)
 */
ts_status ts_prompt_forward(ts_prompt* p, ts_experts* e, const void* x, int tokens, float* y, cudaStream_t stream);

/* Routing of the last forward (of its top_k), to host memory (synchronises `stream`): sel and w [tokens][top_k],
   which is nothing after a forward of no tokens. TS_ERR_INVALID_ARG before any forward, after one that failed on
   its way, after a layer of one expert without a router, and where what ran last on the GPU had another number of
   tokens or another top_k than the last call: the call was captured and not replayed yet, or an earlier one replayed. */
ts_status ts_prompt_get_routing(ts_prompt* p, cudaStream_t stream, int32_t* sel, float* w);
/* As ts_ffn_get_error and ts_ffn_check_scratch. */
ts_status ts_prompt_get_error(ts_prompt* p, cudaStream_t stream);
ts_status ts_prompt_check_scratch(ts_prompt* p, cudaStream_t stream);

/* ---------------------------------------------------------------------------------------------
 * Adapted layers: what serving and tuning low-rank adapters of a layer needs beside its frozen weights.
 *     ts_list_rows              the rows of every adapter
 *     ts_adapt_rows             each row's share of its adapter, added to a product; its backward pass by rows
 *     ts_adapter_grads          gradients of the adapters
 *     ts_adapters_backward      these two as the backward pass of the first
 *     ts_drelu_rows             the gated activation of products computed apart, kept in 8 bits
 *     ts_drelu_rows_backward    its backward pass from what was kept
 *     ts_balance                loss on uneven routing, with the experts' counts
 *     ts_route_backward         gradient of the router's logits
 *     ts_combine_rows_backward  backward pass of ts_combine_rows
 * The backward pass of the frozen bf16 weights themselves is products that are there: by x, dg . W_gate is ts_grouped_*
 * with TS_KN, dy . W_down^T with TS_NK; that of ts_gather_rows is ts_combine_rows with weights of 1. All are
 * asynchronous on `stream`, keep nothing between calls, do not allocate and may be captured in a CUDA graph. No
 * result depends on timing: the same inputs give the same bits. The paper has no counterpart to any of them (its
 * training is of all weights): these are readings.
 */

/*
 * Rows by group: group i has list entries offsets[i] .. offsets[i + 1] - 1, ascending, and group n_groups the rows of none
 * (an id outside 0..n_groups-1).
 *   ids       device [n_rows] int32, n_rows below 2^30
 *   n_groups  1..255
 *   rows      device [n_rows] int32
 *   offsets   device [n_groups + 2] int32; offsets[n_groups + 1] = n_rows
 * The three share no memory.
 */
ts_status ts_list_rows(const int32_t* ids, int n_rows, int n_groups, int32_t* rows, int32_t* offsets, cudaStream_t stream);

/*
 * Low-rank adapters of many requests beside a shared product: with i = ids[t],
 *     h[t] = scale[i] * x[t] A_i^T,      out[t] = y[t] + h[t] B_i
 * and h[t] = 0, out[t] = y[t] for a row of no adapter (an id outside 0..n_adapters-1). Given dy, B, A and dx for x, A, B
 * and y it is the backward pass by rows: dh[t] = scale[i] * dy[t] B_i^T, dx[t] + dh[t] A_i.
 *   x, ldx     device, rows of k bf16 (a multiple of 8), ldx apart
 *   a, b       device [n_adapters][r][k] and [n_adapters][r][n] bf16, n a multiple of 8; row j of B_i is what
 *              component j adds, as row j of w_down is
 *   scale      device [n_adapters] fp32, NULL: 1
 *   ranks      device [n_adapters] int32, NULL: r. Components from ranks[i] on count as 0 and are not read.
 *   n_adapters 1..255, r 1..128
 *   ids        device [rows] int32; read where there is no list: up to 512 rows
 *   list, offsets   as ts_list_rows writes them from ids for n_adapters groups, or NULL
 *   y, ldy     device, rows of n of ydtype (TS_BF16 or TS_F32), ldy apart
 *   out, ldo   the same; may be y itself. NULL (y as well): h alone
 *   h          device [rows][r] fp32, or NULL
 * out and h share no memory with x, with y (but for an out that is y) and with each other: an adapter around the identity, where y is
 * x, has an out of its own. They may lie between each other's rows, as columns of one buffer (rows equally far apart).
 * Rows of x, y and out and the matrices start on 16-byte boundaries. Weights are finite. Products are exact, sums are in
 * fp32; h enters the second product in 16 (ydtype TS_BF16) or 24 significant bits; out is rounded once.
 * TS_ERR_UNSUPPORTED: k or n above 2^24, or rows above 2^30.
 */
ts_status ts_adapt_rows(const void* x, int64_t ldx, int rows, int k, const void* a, const void* b, const float* scale,
                        const int32_t* ranks, int n_adapters, int r, int n, const int32_t* ids, const int32_t* list,
                        const int32_t* offsets, const void* y, int64_t ldy, ts_dtype ydtype, void* out, int64_t ldo, float* h,
                        cudaStream_t stream);

/* Whether waits in calls of ts_adapt_rows and ts_adapter_grads on the current device have given up since this was last called
   (synchronises `stream`): TS_OK, or TS_ERR_TIMEOUT, after which their outputs are not to be used. The answer is about the calls
   of all streams and threads on the device that are done by then, and is given once: one caller asks for all of them. After
   TS_ERR_CUDA nothing that was recorded is lost. */
ts_status ts_adapt_get_error(cudaStream_t stream);
/* Failure-detection test hook: a bounded wait of the next calls over many rows runs out. */
void ts_adapt_set_test_stall(int on);

/*
 * Gradients of adapters: grad[i] = sum over the rows t of adapter i of h[t]^T x[t], so of B_i from h and dy, and of A_i from
 * dh and x, with h and dh as ts_adapt_rows gives them.
 *   h          device [rows][r] fp32
 *   x, ldx     device, rows of k, ldx apart, TS_BF16 (k a multiple of 8) or TS_E4M3 (of 16)
 *   x_scale, ld_scale  TS_E4M3: device [ceil(k / 128)][ld_scale] fp32, ld_scale >= rows (as ts_quant_rows writes
 *              them). NULL for TS_BF16.
 *   list, offsets   as ts_list_rows writes them
 *   grad       device [n_adapters][r][k] fp32, on a 16-byte boundary: overwritten (0 for an adapter without rows), or
 *              added to if accumulate is not 0; shares no memory with h, x and x_scale
 * Products and sums are in fp32, h in 24 significant bits: infinities and NaN of x and h come out as they do in fp32 (but for
 * an infinity times an h below 2^-133, which is NaN).
 */
ts_status ts_adapter_grads(const float* h, int r, const void* x, int64_t ldx, ts_dtype xdtype, const float* x_scale,
                           int64_t ld_scale, int rows, int k, int n_adapters, const int32_t* list, const int32_t* offsets,
                           float* grad, int accumulate, cudaStream_t stream);

/*
 * The backward pass of ts_adapt_rows (x, A, B, y to out, with h): in one call, which lets the two sums of rows overlap,
 *     ts_adapt_rows of dy, B, A, dx to out, with dh      dh[t] = scale[i] dy[t] B_i^T, out[t] = dx[t] + dh[t] A_i
 *     ts_adapter_grads of dh and x to da, of h and dy to db
 * with the arguments of those: dy rows of n bf16, h what the forward gave, x its rows (TS_BF16, or TS_E4M3 with x_scale), dx and
 * out rows of k of dxdtype (both NULL: not wanted), dh device [rows][r] fp32 (scratch, needed), list and offsets as
 * ts_list_rows writes them (needed). out may be dx itself; out, dh, da and db share no memory with dy, h, x and x_scale
 * (which are read after out is written: where dx is dy, out is another buffer) and with one another.
 */
ts_status ts_adapters_backward(const void* dy, int64_t ldy, int rows, int n, const void* a, const void* b, const float* scale,
                               const int32_t* ranks, int n_adapters, int r, int k, const int32_t* list, const int32_t* offsets,
                               const float* h, const void* x, int64_t ldx, ts_dtype xdtype, const float* x_scale,
                               int64_t ld_scale, const void* dx, int64_t lddx, ts_dtype dxdtype, void* out, int64_t ldo, float* dh,
                               float* da, float* db, int accumulate, cudaStream_t stream);

/*
 * The gated activation (Eq. 2) of rows whose two products were computed apart: c = max(0, g) max(0, u), 0 unless both are
 * positive (so where either is NaN), for rows r < min(*n, rows); the others, all of them where *n is negative, are left as
 * they were. What its backward pass needs is kept in TS_E4M3: each factor where both are positive and 0 elsewhere, with a
 * scale for each 128 of a row,
 *     scale = the smallest power of two, at least 2^-100, with max / scale <= 448 (1 where all are 0)
 *     q     = factor / scale rounded to the nearest, ties to even, but at least 2^-9 where the factor is positive
 * (a factor above 1.875 * 2^127 is kept as that).
 *   g, u       device, rows of m (a multiple of 16) of dtype (TS_BF16 or TS_F32), ldg and ldu apart
 *   n          device int32 (as &offsets[n_experts] of ts_route), NULL: rows
 *   c, ldc     device, rows of m bf16, ldc apart
 *   q_gate, q_up   device [rows][m] e4m3, s_gate, s_up device [ceil(m / 128)][rows] fp32; or NULL, all four
 * All rows start on 16-byte boundaries. c may be a bf16 g or u itself (its rows as far apart); otherwise what is written shares no
 * memory with what is read. TS_ERR_UNSUPPORTED: m above 2^24 or rows above 2^30.
 */
ts_status ts_drelu_rows(const void* g, int64_t ldg, const void* u, int64_t ldu, ts_dtype dtype, const int32_t* n, int rows,
                        int m, void* c, int64_t ldc, void* q_gate, void* q_up, float* s_gate, float* s_up,
                        cudaStream_t stream);

/*
 * The backward pass of ts_drelu_rows from what it kept, with factors g = s_gate q_gate and u = s_up q_up:
 *     dg = dc u,  du = dc g,  c = g u  where both are positive, 0 elsewhere (whatever dc is there)
 * rounded to bf16 (c, of 4 and 4 significant bits, is exact unless it leaves bf16's normal numbers). Rows from min(*n, rows)
 * on are left as they were.
 *   dc, ldd    device, rows of m of dtype (TS_BF16 or TS_F32), ldd apart
 *   dg, du     device, rows of m bf16, ldg and ldu apart
 *   c, ldc     the same, for the gradient of the down product's weights; or NULL
 * One of them may be a bf16 dc itself; otherwise they share no memory with what is read and with one another.
 */
ts_status ts_drelu_rows_backward(const void* dc, int64_t ldd, ts_dtype dtype, const void* q_gate, const void* q_up,
                                 const float* s_gate, const float* s_up, const int32_t* n, int rows, int m, void* dg,
                                 int64_t ldg, void* du, int64_t ldu, void* c, int64_t ldc, cudaStream_t stream);

/*
 * How evenly tokens are routed. A token is live if any of its logits is above -infinity; p[t] is the softmax over its
 * logits (-infinity and NaN count as none, equal +infinities share), and over the live tokens and the picks
 *     share[e] = mean of p[t][e],   loss = n_experts * sum_e (counts[e] / picks) share[e]
 * which is 1 where both are even, and 0 without picks. Sums over tokens are in fp32, of a thread's tokens, its CTA's and all CTAs' in turn.
 *   logits     device [tokens][n_experts] fp32; sel device [tokens][top_k], as ts_route takes and gives them (an
 *              entry outside 0..n_experts-1 is no pick)
 *   loss       device [1] fp32
 *   counts     device [n_experts] int32: picks of each expert
 *   share      device [n_experts] fp32
 *   totals     device [2] int32: live tokens, picks
 *   work       device, ts_balance_work(tokens, n_experts) fp32 (0: may be NULL), not shared by calls in flight at once
 * What is written shares no memory with what is read.
 */
long long ts_balance_work(int tokens, int n_experts); /* -1: sizes that ts_balance refuses */
ts_status ts_balance(const float* logits, int tokens, int n_experts, const int32_t* sel, int top_k, float* loss,
                     int32_t* counts, float* share, int32_t* totals, float* work, cudaStream_t stream);

/*
 * Gradient of the router's logits, overwritten, from the routing weights' (dw, or NULL) and the balance loss's (dloss with
 * the counts and totals of ts_balance for these logits, or all three NULL):
 *     dlogits[t][e] = sum over the picks j of e of w_j (dw_j - sum_i w_i dw_i)
 *                   + dloss n_experts / (picks * live tokens) p_e (counts[e] - sum_f counts[f] p_f)
 * The counts have no gradient. A token that is not live, and an expert of logit -infinity or NaN, gets 0; a live token without
 * a pick (dropped, where an expert takes a limited number of tokens) has the balance loss's term only.
 *   logits     device [tokens][n_experts] fp32 (with dloss); sel, w device [tokens][top_k] as ts_route gives them, dw
 *              the same (with dw)
 *   dloss      device [1] fp32
 *   dlogits    device [tokens][n_experts] fp32; may be logits itself, and shares no memory with what else is read
 */
ts_status ts_route_backward(const float* logits, int tokens, int n_experts, const int32_t* sel, const float* w, int top_k,
                            const float* dw, const int32_t* counts, const int32_t* totals, const float* dloss, float* dlogits,
                            cudaStream_t stream);

/*
 * The backward pass of ts_combine_rows for slots as ts_route gives them, where a row belongs to one token:
 *     dsrc[r] = (sum over the j with slots[t][j] = r of w[t][j]) dy[t]   for t = rows[r], if slots names r there
 *     dw[t][j] = sum over i of dy[t][i] src[slots[t][j]][i]              0 for a slot outside 0..n_rows-1
 * Other rows of dsrc are left as they were.
 *   dy         device [tokens][n] of dydtype (TS_F32 or TS_BF16)
 *   src, dsrc  device [n_rows][n] of dtype (TS_F32 or TS_BF16); dsrc shares no memory with src and dy
 *   rows       device [n_rows] int32: token of each row
 *   slots, w, dw   device [tokens][top_k], top_k 1..8; n 1..2^30, at most 2^30 tokens
 */
ts_status ts_combine_rows_backward(const void* dy, ts_dtype dydtype, const void* src, ts_dtype dtype, int n_rows, int n,
                                   const int32_t* slots, const float* w, const int32_t* rows, int tokens, int top_k,
                                   void* dsrc, float* dw, cudaStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* TS_FFN_H */
