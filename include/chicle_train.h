/*
 * chicle_train.h - C ABI of the operators of a local training step on one MI355X.
 *
 * Beside CoCoA the uni-tasks of the paper run local SGD (Section 2.2, Section 5.1): every solver makes some steps on the
 * samples of its chunks and the trainer merges the models.  These are the operators of such a step for models over
 * categorical data with many classes: rows of a table looked up by token, layer norm, the softmax loss over all classes,
 * and the clipping of the step's gradients by their common norm, each with its gradients; and, where the rows come in sequences, of
 * layers between lookup and loss: a root-mean-square norm on a residual stream, a gated recurrence, and rows kept in 8 bits until
 * the backward pass.
 *
 * Conventions
 *   - every function returns CHICLE_OK (0) or a negative chicle_status (chicle_round.h); nothing throws or aborts;
 *     chicle_train_last_error() gives a message for the calling thread's last failure; a refused call enqueues nothing;
 *   - all pointers are device pointers unless said otherwise; work is enqueued on the given stream and nothing waits for it;
 *     the functions keep nothing from one call for the next and may be called from several threads and on several streams;
 *   - no device memory is allocated: what a call needs is the `workspace`, 16-byte aligned, of at least the bytes that the
 *     function's _bytes companion (host, pure) gives for the same sizes; it may be used again by work that is enqueued behind
 *     the call on the same stream, and holds nothing that a caller needs;
 *   - matrices are row-major with unit column stride; ld is the distance of rows in elements (at least the row's length); data
 *     begins at any multiple of its element's size; outputs overlap no inputs unless said otherwise;
 *   - type (chicle_type) is that of all matrices and parameter vectors of a call.  Sums, statistics and losses are held in
 *     32 bits or more (the loss's derivatives by the logits, in 16-bit types, to twice the type's bits), and results of a 16-bit
 *     type are rounded once, where they are stored;
 *   - label and token arrays hold 32-bit integers, or 64-bit ones where `wide` is not 0.  A negative one means "none": no loss, a row
 *     of zeros, no gradient.  One past the end is treated like that too, and sets a bit of *flags (1: label, 2: token), an
 *     int32 of the caller's, or NULL (4: offsets of sequences that are no rows of the call; 8: a scan whose workgroups gave up waiting for one another, after seconds, as
 *     where something else writes into its workspace: its results are not defined);
 *   - results do not depend on timing: the same call on the same inputs gives the same bits.
 */
#ifndef CHICLE_TRAIN_H
#define CHICLE_TRAIN_H

#include <stddef.h>
#include <stdint.h>
#include "chicle_round.h"

#ifdef __cplusplus
extern "C" {
#endif

enum chicle_type { CHICLE_F32 = 0, CHICLE_BF16 = 1, CHICLE_F16 = 2 };

/* Softmax cross entropy of rows x (n x d) against classes w (classes x d):
 *   lse_i = log sum_v exp(x_i . w_v),  loss_i = lse_i - x_i . w_label(i),  0 for a row without a label.
 * The logits are not kept (softmax_loss_grad keeps those of a piece of the rows in 32 bits, at most 1 GB or 256 rows of them, and in 16
 * bits those of up to 64 rows or of less than 192 tiles of 256 x 256; else in 16 bits its workspace is x laid out, dx in 32 bits and their
 * derivatives for a piece of the classes, 1 GB or 4 bytes for every row and min(8 d, 2^24 / d) classes, and w, if its rows are no whole
 * slices of 128 bytes).  n may be 0.  Limits: n, d and classes below 2^22, 2^21 and 2^23, and n * classes below 2^42.
 * Errors: EINVAL (arguments), ENOMEM (workspace), EDEVICE. */
size_t chicle_softmax_loss_bytes(const void *x, int64_t ldx, const void *w, int64_t ldw, int64_t n, int64_t d, int64_t classes, int32_t type,
                                 int32_t with_grad);
int chicle_softmax_loss(const void *x, int64_t ldx, const void *w, int64_t ldw, const void *labels, int32_t wide, int64_t n, int64_t d,
                        int64_t classes, int32_t type, float *loss, float *lse, void *workspace, size_t workspace_bytes, int32_t *flags,
                        void *hip_stream);

/* The same with the gradients of sum_i row_weight_i loss_i: dx (n x d) and dw (classes x d).  A row without a label counts nowhere,
 * whatever x and row_weight hold there, and its dx is 0.  row_weight: n floats.  In half precision the derivatives by the logits have one scale
 * for all rows: each is off by up to 2^-39 of the largest weight of a row with a label, which a row shows whose weight is less than some 2^-20 of it. */
int chicle_softmax_loss_grad(const void *x, int64_t ldx, const void *w, int64_t ldw, const void *labels, int32_t wide, const float *row_weight,
                             int64_t n, int64_t d, int64_t classes, int32_t type, float *loss, void *dx, int64_t lddx, void *dw, int64_t lddw,
                             void *workspace, size_t workspace_bytes, int32_t *flags, void *hip_stream);

/* out_i = scale * table[id_i]; table has n_rows rows of d values.  Limits: n and n_rows below 2^31, d below 2^23. */
int chicle_embed(const void *table, int64_t ld, int64_t n_rows, const void *ids, int32_t wide, int64_t n, int64_t d, int32_t type, float scale,
                 void *out, int64_t ldo, int32_t *flags, void *hip_stream);

/* Its gradient: dtable[v] = scale * sum over the i with id_i = v of dout_i, for all n_rows rows; or, where accumulate is not 0,
 * added to what dtable holds (rows that no token has are not touched; each touched row is rounded once).  Limits: n and n_rows
 * below 2^31 - 1, d below 2^23. */
size_t chicle_embed_grad_bytes(int64_t n, int64_t d, int64_t n_rows);
int chicle_embed_grad(const void *ids, int32_t wide, const void *dout, int64_t ldd, int64_t n, int64_t d, int64_t n_rows, int32_t type, float scale,
                      int32_t accumulate, void *dtable, int64_t ldo, void *workspace, size_t workspace_bytes, int32_t *flags, void *hip_stream);

/* Layer norm over rows of d values: y = (x - mean) rstd gamma + beta, rstd = 1 / sqrt(var + eps); mean and rstd (n floats each) are
 * what the gradient takes.  The sum of (x - mean)^2 is a 32-bit number: values below 2^63 / sqrt(d) have it.  Limits: n and d below 2^31. */
int chicle_layer_norm(const void *x, int64_t ldx, const void *gamma, const void *beta, int64_t n, int64_t d, int32_t type, float eps,
                      void *y, int64_t ldy, float *mean, float *rstd, void *hip_stream);

size_t chicle_layer_norm_grad_bytes(int64_t n, int64_t d, int32_t type);
int chicle_layer_norm_grad(const void *dy, int64_t lddy, const void *x, int64_t ldx, const void *gamma, const float *mean, const float *rstd,
                           int64_t n, int64_t d, int32_t type, void *dx, int64_t lddx, void *dgamma, void *dbeta, void *workspace,
                           size_t workspace_bytes, void *hip_stream);

/* Rows kept in 8 bits (packed rows): whole numbers q from -127 to 127, 32 neighbouring columns with one scale 2^e, the least power of two from
 * 2^-126 on with max |x| <= 127 2^e; q = x 2^-e, rounded to nearest even.  A value is off by at most half of 2^e; by less than 2^e where x
 * is near the largest number of its type (q stops at 63 there, so that what is finite stays finite).  A group with an infinity or NaN unpacks to NaN.
 * q: n rows of d bytes, ldq apart, a multiple of 32 that has room for d in whole groups, 16-byte aligned; the bytes behind the last column, up to a whole
 * group, are written as zeros.  scales: a byte e + 127 for a group (255: NaN, 0: zeros), rows ldq / 32 apart.  Limits: n and d below 2^31. */
int chicle_pack8(const void *x, int64_t ldx, int64_t n, int64_t d, int32_t type, void *q, void *scales, int64_t ldq, void *hip_stream);
int chicle_unpack8(const void *q, const void *scales, int64_t ldq, int64_t n, int64_t d, int32_t type, void *out, int64_t ldo, void *hip_stream);

/* Root-mean-square norm of rows on a residual stream: r = x + residual (residual may be NULL: r = x), rounded to the type;
 * rstd = 1 / sqrt(sum_c r_c^2 / d + eps), y = r rstd gamma.  sum (or NULL) gets r; sum8 (or NULL) gets r as packed rows, ldsum8 bytes apart.  y is of the
 * type where y_scales is NULL, else packed rows, ldy bytes apart, made from the 32-bit values.  rstd: n floats, which the gradient takes.
 * Values may be as large as the type's largest; where eps is 0, the root of a row's mean square is 2^-127 or more, since rstd is one over it (a row of zeros
 * has no norm then: rstd infinite, y NaN).
 * Limits: n and d below 2^31. */
int chicle_rms_norm(const void *x, int64_t ldx, const void *residual, int64_t ldres, const void *gamma, int64_t n, int64_t d, int32_t type, float eps,
                    void *sum, int64_t ldsum, void *y, int64_t ldy, void *y_scales, void *sum8, void *sum8_scales, int64_t ldsum8, float *rstd,
                    void *hip_stream);

/* Its gradients: dx, that of x as of the residual, with dsum added, which reaches r on the other way (or NULL), and dgamma, from r: of the type
 * where sum_scales is NULL, else packed rows, ldsum bytes apart. */
size_t chicle_rms_norm_grad_bytes(int64_t n, int64_t d, int32_t type);
int chicle_rms_norm_grad(const void *dy, int64_t lddy, const void *sum, int64_t ldsum, const void *sum_scales, const void *gamma, const float *rstd,
                         const void *dsum, int64_t lddsum, int64_t n, int64_t d, int32_t type, void *dx, int64_t lddx, void *dgamma, void *workspace,
                         size_t workspace_bytes, void *hip_stream);

/* Gated linear recurrence over the rows of sequences, column by column: a = 1 / (1 + exp(-f)), h_t = a_t h_{t-1} + (1 - a_t) u_t, y_t = h_t.
 * Sequence j has the rows offsets[j] to offsets[j + 1] - 1 (sequences + 1 integers, ascending, 32-bit ones, or 64-bit ones where wide is not 0); none where
 * they are equal.  offsets NULL: one sequence of all rows.  Rows of no sequence (before the first offset, from the last one on) get zeros, whatever
 * they hold.  Offsets that descend or are no rows of the call set a bit of *flags, and results are then not defined; nothing is read or
 * written outside of the tensors.  h0 (or NULL: zeros) and last (or NULL): sequences x d floats, the state before a sequence's first row and
 * after its last.  u is of the type where u_scales is NULL, else packed rows, ldu bytes apart.  states (or NULL): n / 32, rounded up, x d floats, the state
 * that enters every 32nd row, which the gradient takes.  Of a gate beyond +-103.97 (150 ln 2, where its smaller share, down to 2^-149 before, is rounded
 * to 0), +-infinity too, nothing comes through on the side that it closes, whatever is there: f = +infinity masks a row.  An infinity or NaN that
 * does come in stays in its column, as one or the other, until a gate closes or the sequence ends (the gradients', until it begins).
 * Limits: n, d and sequences below 2^31, and n / 128 times d / 64, each rounded up, below 2^23. */
size_t chicle_gated_scan_bytes(int64_t n, int64_t d, int32_t type);
int chicle_gated_scan(const void *f, int64_t ldf, const void *u, int64_t ldu, const void *u_scales, const void *offsets, int32_t wide, int64_t sequences,
                      const float *h0, int64_t n, int64_t d, int32_t type, void *y, int64_t ldy, float *last, float *states, void *workspace,
                      size_t workspace_bytes, int32_t *flags, void *hip_stream);

/* Its gradients by f, u and, where dh0 is not NULL, h0, from dy and, where it is not NULL, dlast, the gradient of `last`; the other arguments are
 * those of the forward call, and what it left in states.  Rows of no sequence get zeros.  h - u, and its product with h's gradient, are 32-bit numbers. */
int chicle_gated_scan_grad(const void *f, int64_t ldf, const void *u, int64_t ldu, const void *u_scales, const void *offsets, int32_t wide,
                           int64_t sequences, const float *h0, const float *states, const void *dy, int64_t lddy, const float *dlast, int64_t n, int64_t d,
                           int32_t type, void *df, int64_t lddf, void *du, int64_t lddu, float *dh0, void *workspace, size_t workspace_bytes,
                           int32_t *flags, void *hip_stream);

/* One row of each of n sequences: state = a state + (1 - a) u, in place, y = state.  state: n x d floats, rows ldstate apart (a state
 * that overlaps another tensor of the call is refused). */
int chicle_gated_step(const void *f, int64_t ldf, const void *u, int64_t ldu, float *state, int64_t ldstate, int64_t n, int64_t d, int32_t type, void *y,
                      int64_t ldy, void *hip_stream);

/* The 2-norm of `count` tensors together (norm: one float), and, where out is not NULL, out_k = in_k * min(1, max_norm / (norm + 1e-6)).
 * in, out, sizes and types are host arrays of count entries: device pointers of contiguous tensors, numbers of values and
 * chicle_types.  out_k may be in_k, and overlaps no other tensor of the call (outputs that overlap one another are refused).  A norm that is infinite
 * or no number scales as the formula says.  Limit: 100000 tensors. */
size_t chicle_clip_grads_bytes(int32_t count);
int chicle_clip_grads(const void *const *in, void *const *out, const int64_t *sizes, const int32_t *types, int32_t count, float max_norm,
                      float *norm, void *workspace, size_t workspace_bytes, void *hip_stream);

/* *out = *flags, and *flags = 0, in one step beside what other streams' work reports: no report is lost, none is taken twice. */
int chicle_train_take_flags(int32_t *flags, int32_t *out, void *hip_stream);

/* Message for the last failure on the calling thread (host). */
const char *chicle_train_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* CHICLE_TRAIN_H */
