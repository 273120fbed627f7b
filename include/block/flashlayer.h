/*
 * flashlayer.h -- C ABI of the operators that complete a layer of an encoder or a
 * decoder around FlashSCA and the linear and norm operators (flashblock.h), for AMD
 * MI355X (gfx950): attention of queries to the states of an encoder of another length,
 * group norm with an activation on channels-last maps, and dropout from a counter-based
 * generator whose mask is never stored.  Each with its gradients.
 *
 * Attention.  For batch b, query i, head h and the head g = h / (H / Hk) of the states,
 *
 *   s[j]  = scale q[b,i,h,:] . k[b,j,g,:] + mask[b,h,i,j]      (j < key_lengths[b])
 *   out[b,i,h,:] = sum_j p[j] v[b,j,g,:],   p = softmax(s)
 *
 * A query all of whose s are -inf, or that has no keys, gets zeros, and its gradients
 * are zeros.
 *
 * Group norm.  For sample n, position r and channel c of group g = c / (C / groups),
 *
 *   y[n,r,c] = act((x[n,r,c] - mean[n,g]) rstd[n,g] weight[c] + bias[c])
 *
 * with the mean and 1 / sqrt(variance + eps) over all positions and the group's channels.
 *
 * Dropout.  With element e's word of the generator,
 *
 *   out[e] = residual[e] + (word[e] >= round(p 2^32) ? scale / (1 - p) x[e] : 0)
 *
 * Conventions are flashblock.h's: device memory, float32 statistics and sums, one rounding
 * for each output, optional tensors NULL, argument errors before any HIP call, calls
 * asynchronous on the stream, no state, no allocation, no atomics, bitwise reproducible
 * results, at most FLASHBLOCK_ROWS_MAX rows and strides between rows of at most
 * FLASHBLOCK_LD_MAX elements for group norm and dropout.  Attention's kernels may raise
 * their dynamic-LDS limit, as flashblock.h's do.
 */
#ifndef FLASHLAYER_H
#define FLASHLAYER_H

#include <stdint.h>

#include "flashblock.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Largest width of a head (D). */
#define FLASHLAYER_HEAD_MAX 128

typedef enum {
    FLASHLAYER_MASK_NONE = 0,
    FLASHLAYER_MASK_BOOL = 1,  /* bytes: 0 leaves the place out */
    FLASHLAYER_MASK_ADD = 2,   /* of the inputs' dtype, added to the scaled score */
    FLASHLAYER_MASK_ADD_F32 = 3
} flashlayer_mask;

/* An attention call's sizes, types and strides (in elements).  The channels of a head are
 * contiguous, and so are a mask's keys.  (Rows of q, k, v and grad_out may begin at any element; where all
 * begin at multiples of 16 bytes, long calls take up to half the time.)  Tiles, B Hk ((Lq H / Hk + 127) / 128) of
 * queries' heads and in the backward B Hk ((Lk + 127) / 128) of keys, at most 2^24 - 8. */
typedef struct {
    int64_t q_batch, q_row, q_head;        /* of q */
    int64_t k_batch, k_row, k_head;        /* of k */
    int64_t v_batch, v_row, v_head;        /* of v */
    int64_t o_batch, o_row, o_head;        /* of out; in the backward of grad_out */
    int64_t mask_batch, mask_head, mask_row; /* of the mask, 0 where it is the same for all */
    int32_t B, Lq, Lk, H, Hk, D;           /* H a multiple of Hk; D <= FLASHLAYER_HEAD_MAX */
    int32_t dtype;                         /* flashbev_dtype of q, k, v, out and gradients */
    int32_t mask;                          /* flashlayer_mask */
    float scale;                           /* finite, > 0 */
} flashlayer_attention;

/*
 * out = softmax(scale q k^T + mask) v.
 *
 *   q            [B, Lq, H, D], k and v [B, Lk, Hk, D], in dtype.
 *   mask         [B, H, Lq, Lk] by its strides, of args->mask's type, or NULL (MASK_NONE).
 *                Places left out by MASK_BOOL or by -inf get no weight.  A boolean mask
 *                that is the same for all queries and heads (mask_row and mask_head 0) leaves
 *                its keys out altogether, as key_lengths does: their k and v may hold anything.  (With
 *                other masks a NaN or infinite v reaches every query of its batch and head, a NaN or
 *                infinite k their grad_q, and an infinite score with -inf added is no number.)
 *   key_lengths  [B] int32, or NULL: keys from key_lengths[b] on are left out and not read.
 *                Values are taken as within 0 .. Lk.
 *   out          [B, Lq, H, D] in dtype; every element is written once.
 *   rest         [B, Lq, H, D] contiguous in dtype, or NULL: what the rounding took from
 *                out (out + rest has twice the digits), for the backward.
 *   stats        [B, H, Lq, 2] float32, or NULL: each row's largest score m (-inf for an
 *                empty one; where the scores grow slowly a value somewhat below it) and the
 *                logarithm of the sum of exp(s - m).
 *   workspace    device, flashlayer_attention_workspace_size bytes, 256-byte aligned; NULL
 *                where that is 0.
 */
int flashlayer_attention_forward(const flashlayer_attention *args, const void *q, const void *k,
                                 const void *v, const void *mask, const int32_t *key_lengths,
                                 void *out, void *rest, float *stats, void *workspace,
                                 uint64_t workspace_bytes, void *stream);

/* Workspace bytes of flashlayer_attention_forward: partial results where few queries leave
 * the keys to be split; copies of k and v where D is not a multiple of 16 bytes or a boolean
 * mask leaves keys out altogether (of over 32 rows).  Of the strides only mask_head and mask_row are
 * read, as zero or not.  No HIP call. */
int flashlayer_attention_workspace_size(const flashlayer_attention *args, uint64_t *bytes);

/*
 * The gradients of a loss, given grad_out = dL/d out.  With delta = grad_out . out of each row
 * and dS = p (grad_out v^T - delta),
 *
 *   grad_q = scale dS k,   grad_k = scale dS^T q,   grad_v = p^T grad_out
 *
 * (k's and v's summed over the query heads that share them).  p and dS are rounded to dtype
 * for the products; float16 ones first take powers of two by the largest |grad_out| and
 * 1 / sum exp(s - m), and above 2^11 by |v|, of a key for its own gradients and for grad_q the largest of a
 * batch's head of the states (keys that are left out altogether aside), so that none
 * overflows and small ones keep digits.  The mask gets no gradient.
 *
 *   args         as in the forward, with grad_out's strides as o_*.
 *   out, rest    the forward's, contiguous [B, Lq, H, D]; rest may be NULL: then delta is
 *                formed of the rounded out.
 *   stats        the forward's.
 *   grad_q       [B, Lq, H, D] contiguous, or NULL to skip it.
 *   grad_k, grad_v  [B, Lk, Hk, D] contiguous; both or neither.  Rows of keys that are left
 *                out are zeros, and so are all where there are no queries (no mask is read then).
 *   workspace    flashlayer_attention_backward_workspace_size bytes.
 */
int flashlayer_attention_backward(const flashlayer_attention *args, const void *grad_out,
                                  const void *q, const void *k, const void *v, const void *mask,
                                  const int32_t *key_lengths, const void *out, const void *rest,
                                  const float *stats, void *grad_q, void *grad_k, void *grad_v,
                                  void *workspace, uint64_t workspace_bytes, void *stream);

int flashlayer_attention_backward_workspace_size(const flashlayer_attention *args, int32_t want_q,
                                                 int32_t want_kv, uint64_t *bytes);

/* A group norm call's sizes, types and strides. */
typedef struct {
    int64_t N, R;          /* samples, and positions of each: N R rows */
    int64_t ldx, ldy;      /* row strides of x and y, in elements */
    int32_t C, groups;     /* channels (at most FLASHBLOCK_NORM_MAX), a multiple of groups */
    int32_t dtype;         /* flashbev_dtype of x and y */
    int32_t param_dtype;   /* of weight and bias: dtype, or FLASHBEV_F32 */
    int32_t act;           /* flashblock_act */
    float eps;             /* > 0 */
} flashlayer_group_norm;

/*
 * y = act(N(x) weight + bias).
 *
 *   x, y         [N R, C] in dtype.
 *   weight, bias [C] in param_dtype, each NULL where absent.
 *   stats        [N, groups, 2] float32, or NULL: the means and 1 / sqrt(variance + eps).
 *   workspace    flashlayer_group_norm_workspace_size bytes, 256-byte aligned.
 */
int flashlayer_group_norm_forward(const flashlayer_group_norm *args, const void *x,
                                  const void *weight, const void *bias, void *y, float *stats,
                                  void *workspace, uint64_t workspace_bytes, void *stream);

int flashlayer_group_norm_workspace_size(const flashlayer_group_norm *args, uint64_t *bytes);

/*
 * The gradients of a loss, given grad_y = dL/dy.  With xhat = (x - mean) rstd,
 * d = grad_y act'(xhat weight + bias) and means over the sample and group,
 *
 *   grad_x = rstd (d weight - mean(d weight) - xhat mean(d weight xhat))
 *   grad_weight = sum_{n,r} d xhat,   grad_bias = sum_{n,r} d
 *
 *   args        as in the forward; ldy is the stride of grad_y.
 *   stats       the forward's.
 *   grad_x      [N R, C] in dtype, contiguous rows (stride C), or NULL.
 *   grad_weight, grad_bias  [C] in param_dtype, each NULL where it is not asked for.
 */
int flashlayer_group_norm_backward(const flashlayer_group_norm *args, const void *grad_y,
                                   const void *x, const float *stats, const void *weight,
                                   const void *bias, void *grad_x, void *grad_weight,
                                   void *grad_bias, void *workspace, uint64_t workspace_bytes,
                                   void *stream);

int flashlayer_group_norm_backward_workspace_size(const flashlayer_group_norm *args,
                                                  uint64_t *bytes);

/* A dropout call's sizes, types, strides and generator.  The word of element e = m C + c is
 * number e % 4 of the block of Philox 4x32-10 (Salmon et al., "Parallel random numbers: as
 * easy as 1, 2, 3", 2011) whose counter is (e / 4, offset) and whose key is the seed, each of
 * 64 bits with the low word first. */
typedef struct {
    int64_t M;             /* rows */
    int64_t ldx, ldr, ldo; /* row strides of x, residual and out, in elements */
    uint64_t seed, offset;
    double p;              /* 0 <= p <= 1: the share that is dropped */
    int32_t C;             /* row width, at most FLASHBLOCK_WIDTH_MAX */
    int32_t dtype;         /* flashbev_dtype of x */
    int32_t stream_dtype;  /* of residual and out: dtype, or FLASHBEV_F32 */
    float scale;           /* finite */
} flashlayer_dropout;

/*
 * out = residual + scale / (1 - p) x where the element is kept, residual elsewhere.
 *
 *   x         [M, C] in dtype.  What is dropped may hold anything.
 *   residual  [M, C] in stream_dtype, or NULL.  It may be `out` itself (the same address and
 *             stride); no other overlap.
 *   state     device, two 64-bit words, seed and offset, read by the kernel in place of the
 *             arguments' (for captured graphs, whose arguments are fixed); or NULL.
 *   out       [M, C] in stream_dtype.
 */
int flashlayer_dropout_forward(const flashlayer_dropout *args, const void *x,
                               const void *residual, const uint64_t *state, void *out,
                               void *stream);

/* grad_x = scale / (1 - p) grad_out where the element was kept, 0 elsewhere: grad_out [M, C] in
 * stream_dtype at stride ldo, grad_x in dtype at stride ldx. */
int flashlayer_dropout_backward(const flashlayer_dropout *args, const void *grad_out,
                                const uint64_t *state, void *grad_x, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* FLASHLAYER_H */
