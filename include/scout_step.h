/*
 * scout_step.h - operators of a replayed training step around its layers, on the device.
 *
 * A replay that starts from the step's tokens and ends at its loss (Sec. 6) leaves more
 * surfaces than a layer's: the embedding table's gradient, the activations and norms
 * between blocks, the loss of every token and the gradients of the output projection.
 * Exact consensus (Sec. 5.3) compares their bits, so these operators too give the same
 * bits wherever the hardware is healthy: no floating-point atomics, every sum in an order
 * that the sizes and the token ids fix, and random numbers from a counter.
 *
 *   scout_embed_forward / scout_embed_backward   rows of a table, and the table's gradient
 *   scout_dropout                                and its gradient, which is the same call
 *   scout_join_forward / scout_join_backward     a block's output joins the residual stream:
 *        norm, dropout, gate and scale, sum, the next block's norm
 *   scout_loss_forward / scout_loss_backward     softmax cross entropy over a vocabulary,
 *        from hidden states and output projection; the scores are never kept
 *
 * Conventions are those of scout_replay.h: plain C, error codes, caller-owned memory, work
 * enqueued on `stream`, scratch of the size the *_workspace calls return (256-byte aligned,
 * no initialisation, one for each of two calls that may run at the same time).  Matrices
 * have a row stride in elements, at least their columns, and adjacent columns; they are
 * aligned to their element size, and rows that lie on 16-byte boundaries are faster.
 * Types are SCOUT_DT_F32, SCOUT_DT_BF16 and SCOUT_DT_F16; sums, statistics and products of
 * elements are fp32, rounded to the result's type once.  Inputs and outputs of a call do
 * not overlap, save where it says so.  Waits of the join's and the loss's kernels on their
 * own copies and products are bounded; scout_replay_waits counts those that gave up.
 */
#ifndef SCOUT_STEP_H
#define SCOUT_STEP_H

#include "scout.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- token embedding ----------------------------------------------------------------
 * y[t] = scale * table[ids[t]], and zeros where ids[t] is outside 0..vocab-1 (padding, or
 * a token of another part of the vocabulary).
 *   id_dtype     SCOUT_DT_I32 or SCOUT_DT_I64
 *   dtype        of table;  out_dtype  of y: dtype or SCOUT_DT_F32
 *   ids          device [rows]
 *   table        device [vocab][dim], row stride table_stride
 *   y            device [rows][dim], row stride y_stride
 *   scale        finite */
SCOUT_API int scout_embed_forward(uint32_t id_dtype, uint32_t dtype, uint32_t out_dtype, uint64_t rows,
                                  uint64_t dim, uint64_t vocab, const void *ids, const void *table,
                                  uint64_t table_stride, float scale, void *y, uint64_t y_stride, void *stream);

/* d_table[v] = (accumulate ? d_table[v] : 0) + scale * sum over t with ids[t] = v of dy[t]
 * Tokens are sorted by id; the sum over a token's places runs in their order, in pieces
 * whose borders follow from the sizes and the ids.  With accumulate, rows without a token
 * are neither read nor written; without it every row is written.  What stands in dy where
 * the id is outside 0..vocab-1 is not read.
 *   dtype        of dy;  out_dtype  of d_table: dtype or SCOUT_DT_F32
 * rows up to 2^30, vocab up to 2^31 - 1; beyond that SCOUT_ERR_UNSUPPORTED. */
SCOUT_API int scout_embed_backward_workspace(uint64_t rows, uint64_t dim, uint64_t vocab, uint64_t *bytes);
SCOUT_API int scout_embed_backward(uint32_t id_dtype, uint32_t dtype, uint32_t out_dtype, uint64_t rows,
                                   uint64_t dim, uint64_t vocab, const void *ids, const void *dy,
                                   uint64_t dy_stride, float scale, void *d_table, uint64_t d_table_stride,
                                   uint32_t accumulate, void *workspace, uint64_t workspace_bytes, void *stream);

/* ---- dropout from a counter ------------------------------------------------------------
 * Place (r, c) of a matrix has the 16-bit number h_{c mod 8} of the eight that
 *     Philox4x32-10(counter = (c / 8, r, offset low, offset high), key = (seed low, seed high))
 * returns (low half of a word before its high half), with offset = `offset` + (d_offset ?
 * *d_offset : 0) modulo 2^64.  With cut = min(65535, floor(65536 p + 1/2)) it is kept where
 * h >= cut:
 *     y = x * (65536 / (65536 - cut))    where kept, else 0 (whatever x is)
 * The mask depends on the place, seed and offset alone: it is made again wherever it is
 * needed and never stored.  The gradient of x is the same call on the gradient of y.
 *   p            0 <= p < 1
 *   d_offset     device, one number, or NULL; read when the kernel runs, so that a captured
 *                call can drop other places each time it is replayed
 * rows up to 2^32, cols below 2^31.  y may be x, with x's row stride. */
SCOUT_API int scout_dropout(uint32_t dtype, uint64_t rows, uint64_t cols, const void *x, uint64_t x_stride, void *y,
                            uint64_t y_stride, double p, uint64_t seed, uint64_t offset, const uint64_t *d_offset,
                            void *stream);

/* ---- a block joins the residual stream ---------------------------------------------------
 * With x the residual stream, b the block's output, all per row of `dim` elements, and
 *     rms(z) = (mean of z^2 + eps)^(-1/2):
 *     u = post ? b * rms(b) * post : b            norm behind the block
 *     u = dropout(u)                              as scout_dropout, with p, seed, offset
 *     y = x + scale * gate * u                    (x NULL: 0; gate NULL: 1)
 *     n = y * rms(y) * norm                       norm before the next block (norm NULL: none)
 * y is rounded to the stream's type where it is stored; n is made from what it was before.
 * gate has one row for every rows / groups rows in turn: one of learned scales (groups = 1),
 * one per sequence, one per token (groups = rows).
 *   stats        device [2][rows] fp32: rms(b), rms(y); 0 where there is no such norm */
typedef struct {
    uint32_t dtype;            /* of b, n, dn, db                                       */
    uint32_t stream_dtype;     /* of x, y, dy, dx: dtype or SCOUT_DT_F32                */
    uint32_t weight_dtype;     /* of gate, post, norm and their gradients: the same two */
    float scale;               /* finite                                                */
    float eps;                 /* finite, >= 0                                          */
    uint32_t reserved;         /* 0                                                     */
    uint64_t rows;             /* below 2^32                                            */
    uint64_t dim;              /* 1..16384                                              */
    uint64_t groups;           /* divides rows; gate is [groups][dim], dense            */
    /* row strides of forward (x, b, y, n) and backward (dy, dn, b, y, dx, db), below 2^32 */
    uint64_t x_stride, b_stride, y_stride, n_stride, dy_stride, dn_stride, dx_stride, db_stride;
} scout_join_t;

SCOUT_API int scout_join_forward(const scout_join_t *j, const void *x, const void *b, const void *gate,
                                 const void *post, const void *norm, double p, uint64_t seed, uint64_t offset,
                                 const uint64_t *d_offset, void *y, void *n, float *stats, void *stream);

/* From dy and dn, the gradients of y and n (NULL: zero), over a row:
 *     t = dn * norm,   z = y * rms(y)
 *     g = dy + rms(y) (t - z mean(t z))            dx = g
 *     h = scale * g,   du = dropout(h * gate)      db = du without post, else with
 *     c = b * rms(b),  s = du * post               db = rms(b) (s - c mean(s c))
 * and over rows, fp32 sums in an order that the sizes fix:
 *     d_gate = sum over its rows of h * u,  d_post = sum of du * c,  d_norm = sum of dn * z
 * y and stats are the forward pass's.  dx, d_gate, d_post, d_norm: NULL where not wanted;
 * d_gate needs gate, d_post post, d_norm norm and dn. */
SCOUT_API int scout_join_backward_workspace(const scout_join_t *j, uint64_t *bytes);
SCOUT_API int scout_join_backward(const scout_join_t *j, const void *dy, const void *dn, const void *b, const void *y,
                                  const float *stats, const void *gate, const void *post, const void *norm, double p,
                                  uint64_t seed, uint64_t offset, const uint64_t *d_offset, void *dx, void *db,
                                  void *d_gate, void *d_post, void *d_norm, void *workspace, uint64_t workspace_bytes,
                                  void *stream);

/* ---- cross entropy over a vocabulary -----------------------------------------------------
 * With s_tv = x_t . w_v, for the rows t whose target is in 0..vocab-1:
 *     lse_t = ln sum_v exp s_tv,   loss_t = lse_t - s_{t,target}
 * Other rows do not count: loss and lse are 0 and their gradient is 0, whatever stands in x.
 *   dtype        of x and w: SCOUT_DT_BF16 or SCOUT_DT_F16
 *   x            device [rows][dim], row stride x_stride
 *   w            device [vocab][dim], row stride w_stride; 16-byte aligned, w_stride a multiple of 8
 *                (else SCOUT_ERR_ALIGN)
 *   targets      device [rows], SCOUT_DT_I32 or SCOUT_DT_I64
 *   loss, lse    device [rows] fp32
 * dim a multiple of 8 up to 65536, rows and vocab up to 2^24 and rows * vocab up to 2^45, else
 * SCOUT_ERR_UNSUPPORTED.  The scratch of the forward pass holds a copy of x and 8 bytes for each row and
 * 128 of the vocabulary (64 MB for 8192 rows and 128000).  The scratch of the backward pass holds a copy of x, dx in fp32, and G for a
 * piece of the vocabulary (in float16 in two forms): half a GiB each, more only where 8192 columns
 * take more. */
SCOUT_API int scout_loss_workspace(uint32_t dtype, uint64_t rows, uint64_t dim, uint64_t vocab,
                                   uint64_t *forward_bytes, uint64_t *backward_bytes);
SCOUT_API int scout_loss_forward(uint32_t dtype, uint32_t id_dtype, uint64_t rows, uint64_t dim, uint64_t vocab,
                                 const void *x, uint64_t x_stride, const void *w, uint64_t w_stride,
                                 const void *targets, float *loss, float *lse, void *workspace,
                                 uint64_t workspace_bytes, void *stream);

/* With g_t = d_loss[t * d_loss_stride] (stride 0: one number for all rows):
 *     G_tv = g_t (exp(s_tv - lse_t) - [v = target_t]),   dx_t = sum_v G_tv w_v
 *     dw_v = (accumulate ? dw_v : 0) + sum_t G_tv x_t
 * over the rows that count.  The scores are made again, in pieces of the vocabulary; G is
 * rounded to 16 bits for its products, which have fp32 sums: for dx before g_t is a factor in
 * float16, so that a row's dx does not depend on what others weigh; for dw relative to the
 * largest finite |g| (float16: entries below 2^-27 of that have fewer bits).  A row's entry
 * at its target enters with what that rounding took away: in dx always, in a row of dw for
 * two of its tokens (which two follows from the targets alone).  dx has x's type, dw
 * out_dtype (dtype or SCOUT_DT_F32).  Every row of dx and dw is written.
 *   dw           device [vocab][dim], row stride dw_stride */
SCOUT_API int scout_loss_backward(uint32_t dtype, uint32_t id_dtype, uint32_t out_dtype, uint64_t rows, uint64_t dim,
                                  uint64_t vocab, const void *x, uint64_t x_stride, const void *w, uint64_t w_stride,
                                  const void *targets, const float *lse, const float *d_loss, uint64_t d_loss_stride,
                                  void *dx, uint64_t dx_stride, void *dw, uint64_t dw_stride, uint32_t accumulate,
                                  void *workspace, uint64_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SCOUT_STEP_H */
