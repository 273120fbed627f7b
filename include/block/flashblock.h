/*
 * flashblock.h -- C ABI of the operators that stand around FlashSCA in an
 * encoder block, for AMD MI355X (gfx950): the matrix product with bias,
 * activation and residual in its epilogue (FlashSCA's value projection, its
 * sampling offsets and logits, its output projection onto the queries, a
 * block's feed-forward), and the norms before and after a block with its gate
 * and residual scale.  Both with their gradients.
 *
 * Linear.  For every row m and output channel n,
 *
 *   pre[m,n] = sum_k x[m,k] weight[n,k] + bias[n]
 *   out[m,n] = residual[m,n] + scale * act(pre[m,n])
 *
 * Norm.  For every row m of C channels, in sample m / (M / groups),
 *
 *   u = N_post(x) post_weight + post_bias          (u = x without a post norm)
 *   s = residual + (scale * gate) u                (rounded to the stream's type)
 *   y = N(s) weight + bias                         (not computed without a norm)
 *
 * where N is the layer norm (v - mean) / sqrt(variance + eps) or the RMS norm
 * v / sqrt(mean of squares + eps), reading s as it is stored.
 *
 * Conventions:
 *   - tensors are device memory, rows of contiguous elements at a stride `ld`
 *     (in elements, at least the row's width), aligned to the element size;
 *   - products accumulate in float32 (float32 inputs are multiplied as
 *     float32); statistics, gates and sums are float32; each output is rounded
 *     once, to nearest even;
 *   - widths (K, N) are at most FLASHBLOCK_WIDTH_MAX, a norm's (C)
 *     FLASHBLOCK_NORM_MAX, row strides at most FLASHBLOCK_LD_MAX elements, and
 *     rows at most FLASHBLOCK_ROWS_MAX;
 *   - an output must not overlap an input or another output, except where
 *     stated (byte ranges from a tensor's first to its last element are
 *     compared);
 *   - optional tensors are NULL where absent; a tensor without elements may be
 *     NULL.
 *
 * Results are bitwise reproducible: no atomics, sums in a fixed order that
 * depends on sizes, types, strides and alignment alone.
 *
 * Thread safety: no state; calls are asynchronous on the given stream and may
 * come from several threads.  No allocation, no printing, no abort.  Kernels
 * run on the calling thread's current HIP device, which must hold every buffer
 * of the call and the stream.  A product of large tiles needs more than 64 KiB of
 * LDS per workgroup and first raises that kernel's dynamic-LDS limit with
 * hipFuncSetAttribute, a per-process setting that is idempotent.  Status codes
 * are flashbev.h's; argument errors are reported before any HIP call.
 */
#ifndef FLASHBLOCK_H
#define FLASHBLOCK_H

#include <stdint.h>

#include "../flashbev.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Largest number of rows. */
#define FLASHBLOCK_ROWS_MAX 2147483392
/* Largest row width (K or N) and row stride, in elements. */
#define FLASHBLOCK_WIDTH_MAX 262144
#define FLASHBLOCK_LD_MAX 1048576
/* Largest row of a norm (C), in elements: a row stays in registers. */
#define FLASHBLOCK_NORM_MAX 16384

typedef enum {
    FLASHBLOCK_ACT_NONE = 0,
    FLASHBLOCK_ACT_RELU = 1,
    FLASHBLOCK_ACT_GELU = 2,       /* v (1 + erf(v / sqrt 2)) / 2 */
    FLASHBLOCK_ACT_GELU_TANH = 3,  /* v (1 + tanh(sqrt(2/pi) (v + 0.044715 v^3))) / 2 */
    FLASHBLOCK_ACT_SILU = 4        /* v / (1 + exp(-v)) */
} flashblock_act;

/* A linear call's sizes, types and strides. */
typedef struct {
    int64_t M;                       /* rows */
    int64_t ldx, ldw, ldr, ldo, ldp; /* row strides of x, weight, residual, out, pre */
    int32_t K, N;                    /* input and output channels */
    int32_t dtype;                   /* flashbev_dtype of x, weight, bias and pre */
    int32_t out_dtype;               /* of residual and out: dtype, or FLASHBEV_F32 */
    int32_t act;                     /* flashblock_act */
    float scale;                     /* finite */
} flashblock_linear;

/*
 * out = residual + scale * act(x weight^T + bias).
 *
 *   x          [M, K] in dtype.
 *   weight     [N, K] in dtype.
 *   bias       [N] in dtype, or NULL.
 *   residual   [M, N] in out_dtype, or NULL.  It may be `out` itself (the same
 *              address and stride); no other overlap.
 *   out        [M, N] in out_dtype; every element is written once.
 *   pre        [M, N] in dtype, or NULL: the sums before the activation, which
 *              the backward of an activation reads.
 *   workspace  device, at least flashblock_linear_workspace_size bytes, 256-byte
 *              aligned; NULL where that is 0.  Its contents on entry do not
 *              matter; calls that may overlap need one each.
 *   stream     hipStream_t; NULL means the default stream.
 *
 * Returns FLASHBEV_OK once enqueued or a negative flashbev_status;
 * FLASHBEV_ERR_SCRATCH for a workspace that is too small.  M or N zero enqueues
 * nothing; K zero leaves act(bias).
 */
int flashblock_linear_forward(const flashblock_linear *args, const void *x, const void *weight,
                              const void *bias, const void *residual, void *out, void *pre,
                              void *workspace, uint64_t workspace_bytes, void *stream);

/* Workspace bytes of flashblock_linear_forward (0 for most sizes): room for
 * float32 partial sums where few rows leave the K axis to be split.  No HIP
 * call. */
int flashblock_linear_workspace_size(const flashblock_linear *args, uint64_t *bytes);

/*
 * The gradients of a loss with respect to x, weight and bias, given
 * grad_out = dL/d out.  With d = scale * act'(pre) * grad_out,
 *
 *   grad_x = d weight,   grad_weight = d^T x,   grad_bias = sum_m d
 *
 * (the residual's gradient is grad_out itself).  The products read d in `dtype`
 * (rounded once where an activation or grad_out's type makes it another tensor
 * than grad_out; a scale alone multiplies the float32 sums); the bias gradient
 * sums it unrounded.
 *
 *   args        as in the forward; ldr is not read, ldo is grad_out's stride.
 *   grad_out    [M, N] in out_dtype.
 *   x, weight   as in the forward (x may be NULL without grad_weight, weight
 *               without grad_x).
 *   pre         the forward's, with args->ldp; not read without an activation.
 *   grad_x      [M, K] in dtype at stride ldgx, or NULL to skip it.
 *   grad_weight [N, K] in dtype at stride ldgw, or NULL.
 *   grad_bias   [N] in dtype, or NULL.
 *   workspace   as in the forward, flashblock_linear_backward_workspace_size
 *               bytes.
 *
 * At least one gradient must be asked for.  Every element is written once
 * (zeros where M is zero).
 */
int flashblock_linear_backward(const flashblock_linear *args, const void *grad_out, const void *x,
                               const void *weight, const void *pre, void *grad_x, int64_t ldgx,
                               void *grad_weight, int64_t ldgw, void *grad_bias, void *workspace,
                               uint64_t workspace_bytes, void *stream);

/* Workspace bytes of flashblock_linear_backward for the gradients that are
 * asked for (nonzero flags).  No HIP call. */
int flashblock_linear_backward_workspace_size(const flashblock_linear *args, int32_t want_x,
                                              int32_t want_weight, int32_t want_bias,
                                              uint64_t *bytes);

typedef enum {
    FLASHBLOCK_NORM_NONE = 0,
    FLASHBLOCK_NORM_LAYER = 1,
    FLASHBLOCK_NORM_RMS = 2
} flashblock_norm_kind;

/* A norm call's sizes, types and strides. */
typedef struct {
    int64_t M;                  /* rows */
    int64_t ldx, ldr, lds, ldy; /* row strides of x, residual, s, y */
    int64_t groups;             /* samples, of M / groups rows each: rows of gate, 1 without it */
    int32_t C;                  /* channels, at most FLASHBLOCK_NORM_MAX */
    int32_t dtype;              /* flashbev_dtype of x and y */
    int32_t stream_dtype;       /* of residual and s: dtype, or FLASHBEV_F32 */
    int32_t param_dtype;        /* of gate, weights and biases: dtype, or FLASHBEV_F32 */
    int32_t norm, post_norm;    /* flashblock_norm_kind; one at least is not NONE */
    float eps;                  /* > 0, of both norms */
    float scale;                /* finite */
} flashblock_norm;

/* The norms' vectors in param_dtype, each NULL where absent: gate [groups, C]
 * (contiguous), the others [C].  weight and bias need a norm, post_weight and
 * post_bias a post norm. */
typedef struct {
    const void *gate, *weight, *bias, *post_weight, *post_bias;
} flashblock_norm_params;

/*
 * s = residual + (scale * gate) N_post(x), y = N(s).
 *
 *   x         [M, C] in dtype.
 *   residual  [M, C] in stream_dtype, or NULL.  It may be `s` itself (the same
 *             address and stride); no other overlap.
 *   s         [M, C] in stream_dtype, or NULL where it is not wanted (then a
 *             norm must be).
 *   y         [M, C] in dtype; NULL without a norm.
 */
int flashblock_norm_forward(const flashblock_norm *args, const flashblock_norm_params *params,
                            const void *x, const void *residual, void *s, void *y, void *stream);

/* The gradients with respect to the vectors, in param_dtype, each NULL where
 * it is not asked for. */
typedef struct {
    void *gate, *weight, *bias, *post_weight, *post_bias;
} flashblock_norm_grads;

/*
 * The gradients of a loss, given grad_y = dL/dy and grad_s = dL/ds (the share
 * that reaches s past the norm).  With r = 1 / sqrt(variance + eps) and
 * shat = (s - mean) r of each row, and xhat, r_x those of x,
 *
 *   g  = grad_y weight
 *   ds = grad_s + r (g - mean(g) - shat mean(g shat))       (RMS: without mean(g))
 *   grad_residual = ds,   du = (scale * gate) ds
 *   h  = du post_weight,  grad_x = r_x (h - mean(h) - xhat mean(h xhat))
 *   grad_weight = sum_m grad_y shat,   grad_bias = sum_m grad_y
 *   grad_post_weight = sum_m du xhat,  grad_post_bias = sum_m du
 *   grad_gate = sum over a sample's rows of scale ds u
 *
 *   args          as in the forward, where ldy is the stride of grad_y and ldr
 *                 that of grad_s.
 *   grad_y        [M, C] in dtype, or NULL (no norm, or nothing reaches y).
 *   grad_s        [M, C] in stream_dtype, or NULL (nothing reaches s).
 *   x             the forward's; read with a post norm or for grad_gate, else
 *                 it may be NULL.
 *   s             the forward's; read where grad_y is given, else it may be NULL.
 *   grad_x        [M, C] in dtype at stride ldgx, or NULL.
 *   grad_residual [M, C] in stream_dtype at stride ldgr, or NULL.
 *   workspace     device, at least flashblock_norm_backward_workspace_size
 *                 bytes, 256-byte aligned (partial sums of the vectors'
 *                 gradients: for each vector a float32 row for every range of
 *                 rows, of which a sample has one or more); NULL where that is 0.
 *
 * At least one gradient must be asked for, and grad_y or grad_s given.
 */
int flashblock_norm_backward(const flashblock_norm *args, const flashblock_norm_params *params,
                             const void *grad_y, const void *grad_s, const void *x, const void *s,
                             void *grad_x, int64_t ldgx, void *grad_residual, int64_t ldgr,
                             const flashblock_norm_grads *grads, void *workspace,
                             uint64_t workspace_bytes, void *stream);

/* Workspace bytes of flashblock_norm_backward (the gradients asked for by
 * their pointers in `grads`, which are not dereferenced).  No HIP call. */
int flashblock_norm_backward_workspace_size(const flashblock_norm *args,
                                            const flashblock_norm_grads *grads, uint64_t *bytes);

#ifdef __cplusplus
}
#endif

#endif /* FLASHBLOCK_H */
