/*
 * tabpack_ops.h -- operators of a student network, beside the packs of
 * tabpack.h: one residual network of gated blocks that a selected ensemble
 * (pack_select_greedy, pack_online_predict) is distilled into and that then
 * answers alone, its head's weights in 8 bits where that is wanted.  (The
 * paper has no counterpart.)
 *
 * Conventions, beside those of tabpack.h:
 *   - No handle: every call works on cuda_stream (NULL: the legacy default
 *     stream) of the current device and is asynchronous; it returns once the
 *     work is enqueued.  Nothing is kept from one call for the next, so calls
 *     on different streams or from different threads do not affect each other.
 *   - All data pointers are device pointers, owned by the caller; outputs and
 *     workspaces do not overlap inputs.  Workspaces are 256-byte aligned and
 *     hold as many bytes as the operator's _bytes entry says (which needs no
 *     GPU); their contents matter only within a call.
 *   - "T" is float32 for TP_FP32 and bf16 for TP_BF16.  Matrices are row-major;
 *     ld* is the distance of two rows in elements (at least the row's length;
 *     any value and any alignment of T is taken, multiples of 16 bytes are
 *     faster).  Matrices without an ld argument are contiguous.
 *   - rows = 0 is a valid call: nothing is written, but gradients that are
 *     sums over the rows become zero.
 *   - Sums, means and softmax statistics are fp32.  Infinities and NaN act on
 *     the rows (and the sums over rows) that hold them.
 *   - Results do not depend on the order in which blocks run: the same call
 *     gives the same bits.
 *   - On failure pack_last_error(NULL) on the same thread describes the cause.
 */
#ifndef TABPACK_OPS_H
#define TABPACK_OPS_H

#include "tabpack.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Waits for the stream; TP_ETIMEOUT if a bounded wait of a tensor-core
 * product has given up on this device since the calling thread's last check
 * of this stream (the first one: ever), whichever stream the product ran on.
 * That product's outputs are undefined.                                     */
tp_status pack_ops_check(void* cuda_stream);

/* Failure detection of the tensor-core products, for tests.  Every wait
 * inside a product gives up after 2 or 4 s: the CTA lets its own copies and MMAs
 * finish, frees its tensor memory and exits.  After this call the
 * process's next launch that shares out a tile's reduction between clusters
 * spoils one of its flags, so that the cluster that waits for it gives up
 * after 4 s (site 47).                                                      */
tp_status pack_debug_ops_withhold(void);

/* ------------------------------------------------------------------------
 * Gated feed-forward block, with weights [out, in] and no biases:
 *   g = x Wg^T,  u = x Wu^T,  h = act(g) u,  y = h Wd^T
 * x: T [rows, d]; w_gate_up: T [2 f, d], Wg above Wu; w_down: T [d_out, f];
 * y: T [rows, d_out].  act: relu(v), silu(v) = v / (1 + exp(-v)), or gelu(v)
 * = v Phi(v).  1 <= d, f, d_out <= 131072; rows < 2^31 - 256; no matrix above 2^40 elements.
 * TP_BF16: fp32 sums; h is rounded to bf16 once (act to 2^-16 of itself before
 * that; below 2^-119 it may be 0).  TP_FP32: operands as three bf16 parts
 * each, whose products above 2^-24 are summed in fp32.                      */
typedef enum { TP_ACT_RELU = 0, TP_ACT_SILU = 1, TP_ACT_GELU = 2 } tp_act;

/* Bytes of `saved` and of the workspaces of a forward and a backward call
 * (any output may be NULL).                                                 */
tp_status pack_gated_bytes(int64_t rows, int32_t d, int32_t f, int32_t d_out, int32_t precision, int64_t* saved,
                           int64_t* forward, int64_t* backward);

/* saved: NULL, or memory (256-byte aligned) that the backward pass of the
 * same rows reads: h, act(g) and u act'(g).                                 */
tp_status pack_gated_forward(const void* x, int64_t ldx, const void* w_gate_up, const void* w_down, int64_t rows,
                             int32_t d, int32_t f, int32_t d_out, int32_t act, int32_t precision, void* y, void* saved,
                             void* workspace, int64_t workspace_bytes, void* cuda_stream);

/* Gradients from dy: T [rows, d_out], with x and the weights of the forward
 * call and what it saved: dx T [rows, d], dw_gate_up T [2 f, d], dw_down
 * T [d_out, f], all overwritten.  relu'(0) = 0.  TP_BF16: the gradients at g
 * and u are rounded to bf16 once.                                           */
tp_status pack_gated_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, const void* w_gate_up,
                              const void* w_down, const void* saved, int64_t rows, int32_t d, int32_t f, int32_t d_out,
                              int32_t precision, void* dx, void* dw_gate_up, void* dw_down, void* workspace,
                              int64_t workspace_bytes, void* cuda_stream);

/* ------------------------------------------------------------------------
 * RMS norm of a residual stream:
 *   s = x + residual (x without one),  n = s / sqrt(mean(s^2) + eps) w
 * x, residual: T [rows, d] (residual may be NULL), w: float32 [d], d in
 * 1..16384, eps >= 0.  sum: T [rows, d], s rounded once (may be NULL); the
 * norm is taken of s before that rounding.  The sum of a row's squares is an
 * fp32 value: where it overflows (|s| from about 10^19 / sqrt(d) on) n is 0,
 * and where it and eps are 0 NaN.  Outputs, either or both:
 *   y: T [rows, d], n rounded once (may be NULL);
 *   q, scale: int8 [rows, d] and float32 [rows] (may both be NULL): scale =
 *   max |n| / 127 over the row, q = n / scale rounded to the nearest integer,
 *   ties to even, and at most 127 in magnitude (a scale below 2^-126 may be
 *   too small by its own rounding); a row with scale 0 has q = 0.  A row with an
 *   infinite or NaN n has q = 0 and scale NaN.                              */
tp_status pack_rms_norm(const void* x, int64_t ldx, const void* residual, int64_t ldr, const float* w, int64_t rows,
                        int32_t d, float eps, int32_t precision, void* sum, void* y, int8_t* q, float* scale,
                        void* cuda_stream);

/* Its gradients at s (the sum as it was stored): with t = dy w and r = 1 /
 * sqrt(mean(s^2) + eps), dx = r (t - s r^2 mean(t s)) + dsum, which is the
 * gradient of x and of residual alike; dw = sum over the rows of dy s r.
 *   dy, s: T [rows, d]; dsum: T [rows, d], the gradient that reaches the
 *   stored sum from elsewhere (may be NULL); dx: T [rows, d]; dw: float32
 *   [d] (may be NULL; then no workspace is needed).                        */
tp_status pack_rms_norm_bytes(int64_t rows, int32_t d, int64_t* backward);
tp_status pack_rms_norm_backward(const void* dy, int64_t lddy, const void* s, int64_t lds, const float* w,
                                 const void* dsum, int64_t lddsum, int64_t rows, int32_t d, float eps,
                                 int32_t precision, void* dx, float* dw, void* workspace, int64_t workspace_bytes,
                                 void* cuda_stream);

/* ------------------------------------------------------------------------
 * 8-bit product with a scale per row and per output channel:
 *   y[r, c] = (sum_k q[r, k] w[c, k]) scale[r] w_scale[c] + bias[c]
 * q: int8 [rows, k]; scale: float32 [rows]; w: int8 [n, k]; w_scale: float32
 * [n]; bias: float32 [n] or NULL; y: T [rows, n].  1 <= k, n <= 131072.  The
 * integer sums are exact while they and their partial sums stay below 2^24,
 * and fp32 sums beyond that.                                                */
tp_status pack_product_q8_bytes(int64_t rows, int32_t k, int32_t n, int32_t precision, int64_t* workspace);
tp_status pack_product_q8(const int8_t* q, int64_t ldq, const float* scale, const int8_t* w, const float* w_scale,
                          const float* bias, int64_t rows, int32_t k, int32_t n, int32_t precision, void* y,
                          void* workspace, int64_t workspace_bytes, void* cuda_stream);

/* ------------------------------------------------------------------------
 * Distillation of m students from one teacher's top logits, loss and
 * gradient in one call.
 *   z: T [m, rows, n], the students' logits; ids: int32 [rows, k] and top:
 *   float32 [rows, k], the classes and logits of the teacher's k entries of
 *   a row, 1 <= k <= 128, 2 <= n <= 2^31 - 1024.  An id outside 0..n-1 (such
 *   as -1) or a logit of -inf is no entry.  labels: int32 [rows] or NULL; a
 *   label outside 0..n-1 is none.
 * For a row of student i with p = softmax(top / tau) over the row's entries:
 *   kd = tau^2 sum_j p_j (log p_j - log softmax(z / tau)[id_j]),
 *   ce = -log softmax(z)[label],
 *   loss[i] = mean over all rows of alpha kd + (1 - alpha) ce,
 * kd = 0 for a row without entries, ce = 0 for a row without a label (also
 * when labels is NULL), both 0 where every logit of the student is -inf.
 * Entries with p_j = 0 add nothing; one with p_j > 0 on a class whose student logit
 * is -inf makes the loss +inf.  Entries of the same class add up.
 *   dz: T [m, rows, n] (may be NULL): the gradient of loss[i] at its logits,
 *   alpha tau (softmax(z / tau) - p) + (1 - alpha) (softmax(z) - onehot),
 *   over rows; loss: float32 [m].  2^-60 <= tau <= 2^60, 0 <= alpha <= 1.
 * kd is a difference of fp32 logarithms, whose rounding tau^2 multiplies: above
 * tau = 100 or so the loss loses its digits, while dz keeps them.           */
tp_status pack_distill_bytes(int64_t m, int64_t rows, int64_t* workspace);
tp_status pack_distill(const void* z, int64_t m, int64_t rows, int32_t n, const int32_t* ids, const float* top,
                       int32_t k, const int32_t* labels, float tau, float alpha, int32_t precision, float* loss,
                       void* dz, void* workspace, int64_t workspace_bytes, void* cuda_stream);

/* ------------------------------------------------------------------------
 * Embedding lookup with scaling, for category columns: y[i] = scale
 * table[ids[i]], 0 for an id outside 0..vocab-1 (such as -1).
 *   ids: n integers of id_bytes (4 or 8); table: [vocab, d], float32 or bf16
 *   by table_precision, rows ldt elements apart; y: T [n, d], T by precision.
 *   0 <= n < 2^31 - 4095, 1 <= vocab < 2^31 - 4095, 1 <= d <= 131072, no matrix
 *   above 2^40 elements.                                                    */
tp_status pack_embed(const void* ids, int32_t id_bytes, int64_t n, const void* table, int64_t ldt, int32_t vocab, int32_t d,
                     float scale, int32_t table_precision, int32_t precision, void* y, void* cuda_stream);

/* Its gradient: dtable[v] = scale times the sum of dy[i] over the i with
 * ids[i] = v, all of dtable written (0 where there is none).  dy: T [n, d] by
 * precision; dtable: [vocab, d], contiguous, by table_precision.  fp32 sums
 * of sorted tokens, joined in a fixed order; rounded once.                  */
tp_status pack_embed_bytes(int64_t n, int32_t vocab, int32_t d, int64_t* backward);
tp_status pack_embed_backward(const void* dy, int64_t lddy, const void* ids, int32_t id_bytes, int64_t n, int32_t vocab,
                              int32_t d, float scale, int32_t precision, int32_t table_precision, void* dtable,
                              void* workspace, int64_t workspace_bytes, void* cuda_stream);

/* ------------------------------------------------------------------------
 * Dropout whose mask is a function of its arguments and never stored:
 *   y(r, c) = x(r, c) / (1 - p) where kept, 0 where dropped, + residual(r, c)
 * Kept iff word c & 3 of Philox4x32-10 at counter (r, c >> 2, step, site) under
 * key (seed low, seed high) is >= floor(p 2^32): the rule of pack_train_step's
 * masks, whose site is (member << 4) | layer.  Its gradient at x is the same
 * call of dy without a residual; at residual it is dy.
 *   x, residual (may be NULL), y: T [rows, d]; 0 <= p < 1; 1 <= d <= 131072;
 *   rows < 2^31 - 255, no matrix above 2^40 elements.  What x holds where it is
 *   dropped does not matter (NaN and infinities included).  Rounded once;
 *   1 / (1 - p) is an fp32 value.                                           */
tp_status pack_dropout(const void* x, int64_t ldx, const void* residual, int64_t ldr, int64_t rows, int32_t d, float p,
                       uint64_t seed, uint32_t step, uint32_t site, int32_t precision, void* y, void* cuda_stream);

/* ------------------------------------------------------------------------
 * Layer norm of a residual stream:
 *   s = x + residual, rounded to T (x without one),
 *   y = (s - m) r w + b,  m = mean(s),  r = 1 / sqrt(mean((s - m)^2) + eps)
 * x, residual: T [rows, d] (residual may be NULL), w, b: float32 [d] (b may
 * be NULL), d in 1..16384, eps >= 0.  Outputs, any of them NULL: sum: T
 * [rows, d], s; y: T [rows, d], rounded once; stats: float32 [rows, 2], 8-byte
 * aligned, m and r of every row.  sum may be x or residual, if rows of it are d
 * apart.  A row's sums are fp32 values, of the differences from its first
 * element and of their squares: constant rows give b exactly, others errors of
 * the size of their spread, whatever their mean; where the squares overflow r is
 * 0, and where they and eps are 0 it is infinite and y NaN.                 */
tp_status pack_layer_norm(const void* x, int64_t ldx, const void* residual, int64_t ldr, const float* w, const float* b,
                          int64_t rows, int32_t d, float eps, int32_t precision, void* sum, void* y, float* stats,
                          void* cuda_stream);

/* Its gradients: with h = (s - m) r and t = dy w, dx = r (t - mean(t) - h
 * mean(t h)) + dsum, which is the gradient of x and of residual alike; dw and
 * db = the sums over the rows of dy h and of dy.
 * m is the mean as it was kept, a float32 value: h is off by up to 2^-24 |m| r.
 *   dy, s: T [rows, d], s as it was stored; stats: of the forward call; dsum:
 *   T [rows, d], the gradient that reaches the stored sum from elsewhere (may
 *   be NULL); dx: T [rows, d]; dw, db: float32 [d] (either may be NULL; with
 *   both, no workspace is needed).                                          */
tp_status pack_layer_norm_bytes(int64_t rows, int32_t d, int64_t* backward);
tp_status pack_layer_norm_backward(const void* dy, int64_t lddy, const void* s, int64_t lds, const float* w,
                                   const float* stats, const void* dsum, int64_t lddsum, int64_t rows, int32_t d,
                                   int32_t precision, void* dx, float* dw, float* db, void* workspace,
                                   int64_t workspace_bytes, void* cuda_stream);

/* ------------------------------------------------------------------------
 * 8-bit floating point (e4m3) with a scale for each block of 128.
 * Quantisation: a block is 128 columns of one row (block_rows 1: activations)
 * or of 128 rows (block_rows 128: weights); the last ones are shorter.
 *   scale = max |x| / 448 over the block, as a float32; q = the e4m3 number
 *   nearest to x / scale (ties to even, at most 448 in magnitude); q = 0 where
 *   scale is 0.  A block with an infinity or a NaN has q = 0 and scale NaN.
 *   x: T [rows, k]; q: [rows, k] bytes, ldq apart; scale: float32
 *   [ceil(rows / block_rows), ceil(k / 128)].  1 <= k <= 131072, rows <
 *   2^31 - 255 (2^23 - 128 in blocks of 128 rows).                          */
tp_status pack_quantise_f8(const void* x, int64_t ldx, int64_t rows, int32_t k, int32_t block_rows, int32_t precision,
                           void* q, int64_t ldq, float* scale, void* cuda_stream);

/* The product of such operands:
 *   y[r, c] = sum_b scale[r, b] w_scale[c / 128, b] sum_{k in block b}
 *             q[r, k] w[c, k] + bias[c]
 * q: e4m3 [rows, k], scale: float32 [rows, ceil(k / 128)]; w: e4m3 [n, k],
 * w_scale: float32 [ceil(n / 128), ceil(k / 128)]; bias: float32 [n] or NULL; y:
 * T [rows, n].  1 <= k, n <= 131072.  fp32 sums; rounded once.  The two scales
 * may be any numbers: where the product of a row's and a column block's is no
 * normal fp32 number they are applied one after the other, by a path that takes
 * that row some hundred times as long.
 * aligned: whether q and w start at multiples of 16 bytes, as their rows do
 * (ldq and ldw): others are copied into the workspace first.                */
tp_status pack_product_f8_bytes(int64_t rows, int32_t k, int32_t n, int32_t aligned, int64_t* workspace);
tp_status pack_product_f8(const void* q, int64_t ldq, const float* scale, const void* w, int64_t ldw, const float* w_scale,
                          const float* bias, int64_t rows, int32_t k, int32_t n, int32_t precision, void* y,
                          void* workspace, int64_t workspace_bytes, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif
