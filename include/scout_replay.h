/*
 * scout_replay.h - operators of one replayed transformer layer, on the device.
 *
 * In-situ replay (Sec. 6) runs a layer again on every peer from the same captured
 * inputs and lets exact consensus (Sec. 5.3) compare the surfaces it leaves: the
 * output and the gradients.  That comparison is of bits, so the operators that make
 * the surfaces must give the same bits wherever the hardware is healthy.  These do:
 * no floating-point atomics, and every sum has an order fixed by the sizes alone.
 *
 *   scout_attn_forward / scout_attn_backward    softmax attention and its gradient,
 *        which recomputes the probabilities from the saved row statistic
 *   scout_ckpt_pack / scout_ckpt_unpack         captured activations held in 8 bits
 *   scout_ckpt_wgrad                            a projection's weight gradient taken
 *        straight from such a checkpoint
 *
 * Conventions are those of scout.h (plain C, error codes, caller-owned memory, work
 * enqueued on `stream`).  Nothing here allocates: scratch is caller memory, of the
 * size the *_workspace calls return; it needs no initialisation, and two calls that may
 * run at the same time need one each.
 */
#ifndef SCOUT_REPLAY_H
#define SCOUT_REPLAY_H

#include "scout.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- attention -------------------------------------------------------------------
 * Row i of query head h of sequence b sees the keys j of head h / (q_heads / kv_heads)
 * with
 *     i < q_lens[b],  j < kv_lens[b],
 *     causal:        j <= p      where p = i + kv_lens[b] - q_lens[b]
 *     window w > 0:  j >  p - w  (the row's own position and the w - 1 before it)
 * so the last query stands at the last key.  With s_ij = scale * q_i . k_j over the
 * keys it sees:
 *     lse_i = ln sum_j exp s_ij,   o_i = sum_j exp(s_ij - lse_i) v_j
 * A row that sees nothing (past its length, or all its keys masked) has o = 0 and
 * lse = -inf, and contributes nothing to any gradient; one whose scores are all -Inf has
 * the same o and lse.  What stands in keys, values, queries or gradients that a row does
 * not see never reaches it, NaN and Inf included; a NaN that it sees always does.
 *
 * Sizes: batch * q_heads * q_len and batch * kv_heads * kv_len up to 2^30, batch * q_heads
 * up to 2^24, head_dim up to 128; beyond that SCOUT_ERR_UNSUPPORTED.  Element offsets are
 * 64-bit.
 *
 * Products are taken of the 16-bit inputs with fp32 sums; the probabilities (and in the
 * backward pass dS) are rounded to the inputs' type for their products; the softmax
 * statistics stay in fp32.  fp16 gradients should be loss-scaled as usual: dS below
 * 6e-8 vanishes. */
typedef struct {
    uint32_t dtype;            /* SCOUT_DT_BF16 or SCOUT_DT_F16                        */
    uint32_t batch;            /* >= 1                                                 */
    uint32_t q_len, kv_len;    /* tokens of the (padded) tensors; may be 0             */
    uint32_t q_heads, kv_heads;/* q_heads a multiple of kv_heads                       */
    uint32_t head_dim;         /* a multiple of 8, 8..128                              */
    uint32_t causal;           /* 0 or 1                                               */
    uint32_t window;           /* 0 = none; needs causal                               */
    float scale;               /* finite and > 0, e.g. 1 / sqrt(head_dim)              */
    /* Strides in elements of {sequence, token, head}; a head's elements are adjacent.
     * Multiples of 8, non-zero where the extent exceeds 1.  dq, dk, dv are laid out as
     * q, k, v. */
    uint64_t q_stride[3], k_stride[3], v_stride[3], o_stride[3], do_stride[3];
} scout_attn_t;

/* Bytes of scratch for one forward and one backward call. */
SCOUT_API int scout_attn_workspace(const scout_attn_t *a, uint64_t *forward_bytes, uint64_t *backward_bytes);

/*   q, k, v, o        device, 16-byte aligned (else SCOUT_ERR_ALIGN)
 *   q_lens, kv_lens   device [batch] int32, or NULL for q_len / kv_len; values outside
 *                     0..q_len / 0..kv_len are taken as the nearest end
 *   lse               device [batch][q_heads][q_len] fp32
 *   workspace         device, 256-byte aligned, at least forward_bytes (NULL if 0) */
SCOUT_API int scout_attn_forward(const scout_attn_t *a, const void *q, const void *k, const void *v,
                                 const int32_t *q_lens, const int32_t *kv_lens, void *o, float *lse,
                                 void *workspace, uint64_t workspace_bytes, void *stream);

/* With g = d_o (the gradient of o), all over the pairs (i, j) that see each other:
 *     P_ij = exp(s_ij - lse_i)   D_i = g_i . o_i   dS_ij = P_ij (g_i . v_j - D_i)
 *     dv_j = sum_i P_ij g_i      dq_i = scale sum_j dS_ij k_j
 *     dk_j = scale sum_i dS_ij q_i
 * dk and dv of a head that several query heads share are summed over those heads.
 * o and lse are the forward pass's.  Every element of dq, dk, dv is written. */
SCOUT_API int scout_attn_backward(const scout_attn_t *a, const void *q, const void *k, const void *v,
                                  const void *o, const float *lse, const void *d_o,
                                  const int32_t *q_lens, const int32_t *kv_lens, void *dq, void *dk, void *dv,
                                  void *workspace, uint64_t workspace_bytes, void *stream);

/* ---- activation checkpoints in 8 bits ---------------------------------------------
 * A row is cut into blocks of 32 elements (the last one short).  Per block, over its
 * finite elements: e = the smallest integer >= -126 with max |x| <= 127 * 2^e, and
 *     code = x / 2^e rounded to the nearest integer, ties to even,
 * so |code| <= 127 (<= 63 where 64 * 2^e would leave the source type's range).  A NaN or
 * Inf has code -128 and is restored as NaN; its block's other elements are unaffected.
 * The step is a power of two, so code * 2^e is exact in fp32 and bf16, and in fp16 for
 * checkpoints of fp16 data: restoring rounds nothing, and a checkpoint of the restored
 * tensor stands for the same values. */
#define SCOUT_CKPT_BLOCK 32

/*   dtype        of x: SCOUT_DT_F32, SCOUT_DT_BF16 or SCOUT_DT_F16
 *   x            device [rows][cols], row stride x_stride >= cols (elements), aligned to its
 *                element size
 *   codes        device [rows][cols] int8, row stride code_stride >= cols
 *   exps         device [rows][ceil(cols / 32)] int8 */
SCOUT_API int scout_ckpt_pack(uint32_t dtype, uint64_t rows, uint64_t cols, const void *x, uint64_t x_stride,
                              int8_t *codes, uint64_t code_stride, int8_t *exps, void *stream);
/* x = code * 2^e, rounded to `dtype` where that is needed (see above). */
SCOUT_API int scout_ckpt_unpack(uint32_t dtype, uint64_t rows, uint64_t cols, const int8_t *codes,
                                uint64_t code_stride, const int8_t *exps, void *x, uint64_t x_stride,
                                void *stream);

/* Weight gradient of y = x W^T, W [outs][ins], from the gradient of y and the checkpoint
 * of x:  dW[o][i] = (accumulate ? dW[o][i] : 0) + sum_t dy[t][o] * x[t][i]
 * with x restored in dy's type, fp32 sums, one rounding to out_dtype.
 *   dtype        of dy: SCOUT_DT_BF16 or SCOUT_DT_F16
 *   out_dtype    of dW: SCOUT_DT_F32 or dtype
 *   rows         tokens (0 gives a zero gradient, or leaves dW with accumulate)
 *   dy           device [rows][outs], row stride dy_stride
 *   codes, exps  the checkpoint: [rows][ins] and [rows][ceil(ins / 32)]
 *   dw           device [outs][ins], row stride dw_stride
 * dy and dw are aligned to their element sizes.  The result's bits depend on the values and
 * sizes alone: rows of dy that do not start on 16-byte boundaries are copied to scratch
 * first (the scratch has room for that). */
SCOUT_API int scout_ckpt_wgrad_workspace(uint32_t dtype, uint64_t rows, uint64_t outs, uint64_t ins, uint64_t *bytes);
SCOUT_API int scout_ckpt_wgrad(uint32_t dtype, uint32_t out_dtype, uint64_t rows, uint64_t outs, uint64_t ins,
                               const void *dy, uint64_t dy_stride, const int8_t *codes, uint64_t code_stride,
                               const int8_t *exps, void *dw, uint64_t dw_stride, uint32_t accumulate,
                               void *workspace, uint64_t workspace_bytes, void *stream);

/* The kernels' waits on their own copies and products are bounded (2 s).  Results of a call in which one gave up are not
 * valid and must not be voted on; on healthy hardware none does.  *total becomes the number that gave up on the current
 * device since the library was loaded.  It is never reset: two readings that differ say that one of the calls between them (on
 * whatever stream of the device) is not valid, whoever else reads.  Synchronises the device. */
SCOUT_API int scout_replay_waits(uint32_t *total /*host*/);
/* The same, counted since this function was last called in the process. */
SCOUT_API int scout_replay_error(uint32_t *count /*host*/);

/* Runs the end of a block of the backward pass in which the warps whose bits are set in `stuck` (0..255) wait on a barrier that
 * nothing arrives at, give up after 2 s (counted as above) and then agree with the others.  d_out: device uint32 [8][2], for every
 * warp the rows that it would make again and flags: 1 = some warp has such rows, 2 = no warp gave up. */
SCOUT_API int scout_selftest_give_up(uint32_t stuck, uint32_t *d_out /*device*/, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SCOUT_REPLAY_H */
