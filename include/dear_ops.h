/*
 * dear_ops.h -- C ABI of the training operators for MI355X (gfx950): what a transformer block
 * computes between two aggregations of its gradients.
 *
 *   attention     forward, and the backward pass that recomputes the probabilities
 *   norm          residual addition + root-mean-square norm, with a checkpoint of its output in
 *                 8 bits; backward pass
 *   checkpoints   activations kept in 8 bits for the backward pass, and the weight gradient of a
 *                 linear layer computed from the checkpoint of its input
 *
 * The library is libdear_ops.so.  Status codes and element types are those of dear.h
 * (dear_strerror describes a status).
 *
 * Conventions
 *   - Every function returns a status; nothing is printed, nothing aborts.  Arguments are checked
 *     before anything is launched; DEAR_EHIP means that a launch failed.
 *   - All pointers are DEVICE memory owned by the caller, except the argument structures and
 *     workspace sizes, which are host memory and read during the call.
 *   - Calls enqueue on the given HIP stream (hipStream_t as void *, NULL = default stream), do not
 *     synchronise, allocate nothing and keep nothing; they can be captured in a HIP graph.
 *   - Results do not depend on the order in which workgroups run: no atomics are used, and the
 *     same call on the same inputs gives the same bits.
 *   - Inputs and outputs must not overlap, unless stated.
 */
#ifndef DEAR_OPS_H
#define DEAR_OPS_H

#include <stdint.h>

#include "dear.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A [batch, token, head, head_dim] tensor: head_dim is contiguous, the other strides are in
 * elements.  A tensor that is read may have strides of 0 (broadcast); one that is written must
 * not map two elements to one place: in the order of their strides, each axis of several elements
 * has a stride of at least what head_dim and the axes before it span. */
typedef struct {
    void *data;
    int64_t batch_stride, token_stride, head_stride;
} dear_heads_t;

/* Attention of a batch of sequences.
 *
 *   s[i,j] = scale * q[i].k[j];  lse[i] = log(sum of exp(s[i,j]) over visible j)
 *   out[i] = sum of exp(s[i,j] - lse[i]) * v[j] over visible j
 *
 * Key j is visible to query i of sequence b where i < nq, j < nk and, if causal, j - nk <= i - nq
 * (the last query sees the last key), with nq = q_lens[b], nk = kv_lens[b] clamped to
 * 0 .. q_len, 0 .. kv_len.  A query that sees no key gets out = 0, lse = -inf and gradients of 0; a
 * key that no query sees gets gradients of 0.  What stands in tokens beyond the lengths is never
 * used.  Within them values are taken to be finite: a NaN or an infinity there may also reach rows of
 * its sequence that it is not visible to (0 * infinity).  Query head h reads key head h / (q_heads / kv_heads).
 * Products are taken of the inputs' type (fp32: fp32 matrix instructions); sums, the softmax and lse
 * are fp32.  In bf16 the probabilities and, in the backward pass, the gradients of s are rounded to
 * bf16 as operands of the second products.  */
typedef struct {
    int32_t batch;             /* >= 0                                                            */
    int32_t q_heads, kv_heads; /* >= 1, q_heads a multiple of kv_heads                            */
    int32_t head_dim;          /* 8 .. 128, a multiple of 8                                       */
    int64_t q_len, kv_len;     /* 0 .. 2^30: tokens that the tensors hold for each sequence       */
    int32_t dtype;             /* DEAR_F32 or DEAR_BF16, of all tensors except lse                */
    int32_t causal;            /* 0 or 1                                                          */
    float scale;               /* > 0, finite                                                     */
    int32_t reserved;          /* 0 */
    const int32_t *q_lens;     /* [batch] valid tokens, or NULL: q_len each                       */
    const int32_t *kv_lens;    /* [batch] valid tokens, or NULL: kv_len each                      */
    dear_heads_t q, k, v;      /* read                                                            */
    dear_heads_t out;          /* forward: written; backward: read                                */
    float *lse;                /* [batch, q_heads, q_len] contiguous; forward: written; backward: read */
    /* backward only */
    dear_heads_t dout;         /* read: gradient of out                                           */
    dear_heads_t dq, dk, dv;   /* written                                                         */
    void *workspace;           /* 256-byte aligned; NULL where its size is 0                      */
    int64_t workspace_bytes;
} dear_attention_t;

/* Base pointers must be 16-byte aligned and strides multiples of 16 bytes (DEAR_EALIGN otherwise).
 * Errors: DEAR_EINVAL, DEAR_EALIGN, DEAR_EHIP; DEAR_ETOOBIG where workspace_bytes is less than the call
 * needs, or where a launch would have 2^32 threads or more: 256 for every 128 queries of a head and, backward,
 * 256 (bf16 of more than 64 values 512) for every 64 keys of a key head. */
int dear_attention(const dear_attention_t *args, void *hip_stream);
int dear_attention_backward(const dear_attention_t *args, void *hip_stream);

/* Bytes of workspace that a call with these sizes needs (pointers and strides are not looked at): where
 * there are few rows, the sequence that they attend to is split, and the splits' results are joined.
 * Errors: DEAR_EINVAL, DEAR_ETOOBIG. */
int dear_attention_workspace(const dear_attention_t *args, int64_t *bytes);
int dear_attention_backward_workspace(const dear_attention_t *args, int64_t *bytes);

/* ---------------------------------------------------------------------------------
 * Checkpoints in 8 bits.  A row of `cols` values is cut into groups of DEAR_CHECKPOINT_GROUP
 * neighbours (the last one filled up with zeros).  With a = the group's largest magnitude, e = the
 * smallest integer >= -126 with a <= 127 * 2^e:
 *     code = x * 2^-e rounded to the nearest integer, halves to even;  exponent byte = e + 127
 *     value = code * 2^e
 * A group that holds a NaN or an infinity gets the exponent byte 255 and codes of 0, and its values
 * are NaN.  A value has at most 7 significant bits: it is exact in bf16 and in fp32.  (Of magnitudes
 * above 127 * 2^121 those that round to 2^128 become infinities, as they do when rounded to bf16.)
 *
 *   codes      int8, [rows, round_up(cols, DEAR_CHECKPOINT_GROUP)] contiguous, 16-byte aligned
 *   exponents  uint8, [rows, ceil(cols / DEAR_CHECKPOINT_GROUP)] contiguous
 *   rows >= 0, 1 <= cols <= 2^31 - 33; DEAR_ETOOBIG from 2^42 codes on
 */
#define DEAR_CHECKPOINT_GROUP 32

/* x: dtype, rows row_stride elements apart (>= cols where there are several rows), aligned to its element type. */
int dear_checkpoint_encode(const void *x, int32_t dtype, int64_t rows, int64_t cols, int64_t row_stride,
                           int8_t *codes, uint8_t *exponents, void *hip_stream);
/* out: dtype, [rows, cols] contiguous, aligned to its element type. */
int dear_checkpoint_decode(const int8_t *codes, const uint8_t *exponents, int64_t rows, int64_t cols,
                           int32_t dtype, void *out, void *hip_stream);

/* dw[n, k] = sum over rows m of dy[m, n] * value[m, k] -- the gradient of a linear layer's weight
 * [outs, ins] from the gradient of its output and the checkpoint of its input.  Products are exact
 * (dy in its type, the checkpoint's values as they are), sums fp32.
 *   dy         dtype, [rows, outs], rows dy_stride elements apart (>= outs where there are several),
 *              aligned to its element type
 *   codes, exponents   checkpoint of [rows, ins]
 *   dw         fp32, [outs, ins] contiguous, 16-byte aligned, written (0 where rows = 0)
 *   workspace  256-byte aligned, as many bytes as dear_checkpoint_weight_grad_workspace says; NULL
 *              where that is 0
 * outs, ins: 1 .. 2^24; rows: 0 .. 2^40.
 * Errors of the calls on checkpoints: DEAR_EINVAL, DEAR_EALIGN, DEAR_EHIP; DEAR_ETOOBIG as above, the weight
 * gradient's for 2^24 tiles of 128 x 128 outputs or more. */
int dear_checkpoint_weight_grad(const void *dy, int32_t dtype, int64_t dy_stride, const int8_t *codes,
                                const uint8_t *exponents, int64_t rows, int64_t outs, int64_t ins, float *dw,
                                void *workspace, int64_t workspace_bytes, void *hip_stream);
int dear_checkpoint_weight_grad_workspace(int32_t dtype, int64_t rows, int64_t outs, int64_t ins, int64_t *bytes);

/* ---------------------------------------------------------------------------------
 * Residual addition and root-mean-square norm.
 *     h = x + residual (rounded to dtype; h = x where residual is NULL)
 *     rstd = 1 / sqrt(mean of h^2 + eps);  y = h * rstd * weight (rounded to dtype)
 *     codes, exponents = checkpoint of y (of the rounded values: equal to dear_checkpoint_encode's of y)
 *
 *   x, residual  dtype, [rows, cols], rows x_stride / residual_stride elements apart
 *   weight       fp32, [cols]
 *   h            dtype, [rows, cols] contiguous, written; NULL where residual is NULL (x is h then)
 *   y            dtype, [rows, cols] contiguous, written; NULL if it is not wanted
 *   codes, exponents   written; both NULL if they are not wanted
 *   rstd         fp32, [rows], written
 * h may be x or residual itself (same address and strides).  rows >= 0, 1 <= cols <= DEAR_NORM_MAX_COLS.
 * Tensors are aligned to their element types, codes to 16 bytes.
 * Errors: DEAR_EINVAL, DEAR_EALIGN, DEAR_EHIP; DEAR_ETOOBIG for 2^31 rows or more (forward).
 */
#define DEAR_NORM_MAX_COLS 32768
int dear_add_rms_norm(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride,
                      const float *weight, int32_t dtype, int64_t rows, int64_t cols, float eps, void *h, void *y,
                      int8_t *codes, uint8_t *exponents, float *rstd, void *hip_stream);

/* Gradients:  g = dy * weight;  dx = rstd * g - h * rstd^3 * mean(g * h) + dh;
 *             dweight = sum over rows of dy * h * rstd
 *   dy, h, dh  dtype, [rows, cols], rows dy_stride / h_stride / dh_stride elements apart; dh (the gradient that
 *              reaches h by other ways) may be NULL
 *   dx         dtype, [rows, cols] contiguous, written: gradient of x and of residual alike
 *   dweight    fp32, [cols], written
 *   workspace  256-byte aligned, as many bytes as dear_add_rms_norm_backward_workspace says
 * dx may be dy, h or dh itself (same address and strides). */
int dear_add_rms_norm_backward(const void *dy, int64_t dy_stride, const void *h, int64_t h_stride, const void *dh,
                               int64_t dh_stride, const float *weight, const float *rstd, int32_t dtype,
                               int64_t rows, int64_t cols, void *dx, float *dweight, void *workspace,
                               int64_t workspace_bytes, void *hip_stream);
int dear_add_rms_norm_backward_workspace(int32_t dtype, int64_t rows, int64_t cols, int64_t *bytes);

#ifdef __cplusplus
}
#endif
#endif /* DEAR_OPS_H */
