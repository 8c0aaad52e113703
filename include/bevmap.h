/*
 * bevmap.h -- C ABI of libbevpool.so: operators of the model that reads a pooled
 * BEV map, on MI355X (gfx950). The pooling itself is in bevpool.h.
 *
 * Three operators, each with its gradients, channels last throughout:
 *  - bevmap_group_norm: group norm with an activation;
 *  - bevmap_attention: queries attend to an encoder's states of another length
 *    (the cells of a map, the pixels of the cameras);
 *  - bevmap_dropout: residual + dropout(x), the mask from a counter-based
 *    generator and never stored.
 *
 * The conventions of bevpool.h hold: return codes and bevpool_last_error, device
 * pointers on the current device, buffers owned by the caller, hip_stream a
 * hipStream_t passed as void* (NULL: the null stream). Every call is
 * asynchronous on hip_stream, allocates nothing, synchronises nothing, keeps
 * nothing after it returns, uses no atomics (equal inputs give equal bits) and
 * may be captured into a HIP graph. Temporaries go to a workspace of the
 * caller's, whose bytes the *_workspace calls return; calls that may overlap
 * need workspaces of their own. Outputs must not overlap inputs, other outputs or
 * the workspace. Pointers need the alignment of their elements; 16-byte aligned
 * rows are read and written 16 bytes at a time.
 * Sums, softmax statistics and norms are held in fp32; what an operator rounds
 * to 16 bits on the way is stated with it. dtype is a bevpool_dtype.
 */
#ifndef BEVMAP_H
#define BEVMAP_H

#include "bevpool.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Activation of bevmap_group_norm: z, max(z, 0), z / (1 + e^-z), z Phi(z) with
 * Phi the normal distribution function (through erf). */
typedef enum { BEVMAP_ACT_NONE = 0, BEVMAP_ACT_RELU = 1, BEVMAP_ACT_SILU = 2, BEVMAP_ACT_GELU = 3 } bevmap_act;

/*
 * Group norm over a map, channels last. Frame b has `pixels` rows; row s starts
 * at x + (b * pixels + s) * row_stride elements and holds `channels` elements,
 * channel c belonging to group c / (channels / groups). With mean and variance
 * (biased) over a frame's group, rstd = 1 / sqrt(variance + eps):
 *   z = weight[c] * (x - mean) * rstd + bias[c],  y = act(z).
 * The variance is formed from deviations, never as a difference of squares.
 */
typedef struct {
    int32_t batch, pixels, channels, groups;
    int64_t row_stride;    /* elements from row to row of x, >= channels */
    float eps;             /* >= 0 */
    int32_t act;           /* bevmap_act */
    int32_t x_dtype;       /* of x and grad_x */
    int32_t y_dtype;       /* of y and grad_y */
    int32_t weight_dtype;  /* of weight, bias and their gradients */
} bevmap_norm;

/* Bytes of workspace of bevmap_group_norm (backward = 0) or
 * bevmap_group_norm_backward (backward = 1); a negative error code if the
 * description is refused. Host only. */
BEVPOOL_API int64_t bevmap_group_norm_workspace(const bevmap_norm *norm, int32_t backward);

/*
 *  weight, bias: device [channels] of weight_dtype; NULL for ones and zeros.
 *  y:          device [batch][pixels][channels] of y_dtype, overwritten.
 *  mean, rstd: device float [batch][groups], overwritten: what the backward reads.
 * batch or pixels of 0 is a call that does nothing. An infinity or a NaN
 * reaches its frame's group alone.
 * Errors: INVALID_ARG (null pointer, a size below 0, channels or groups below 1,
 * channels not a multiple of groups, row_stride < channels, eps negative or not
 * finite, unknown act, workspace too small or not 16-byte aligned),
 * UNSUPPORTED_DTYPE, OVERFLOW (batch above 65535, batch * pixels reaching 2^30, row_stride reaching 2^31,
 * channels above 8192), HIP (launch failure).
 */
BEVPOOL_API int bevmap_group_norm(const bevmap_norm *norm, const void *x, const void *weight, const void *bias,
                                  void *y, float *mean, float *rstd, void *workspace,
                                  int64_t workspace_bytes, void *hip_stream);

/*
 * Gradients of bevmap_group_norm, with the mean and rstd that it wrote:
 *  grad_y:      device [batch][pixels][channels] of y_dtype.
 *  grad_x:      device [batch][pixels][channels] of x_dtype, overwritten.
 *  grad_weight, grad_bias: device [channels] of weight_dtype, overwritten
 *               (zeros for an empty map); NULL to skip.
 * Errors: those of bevmap_group_norm.
 */
BEVPOOL_API int bevmap_group_norm_backward(const bevmap_norm *norm, const void *grad_y, const void *x,
                                           const void *weight, const void *bias, const float *mean,
                                           const float *rstd, void *grad_x, void *grad_weight,
                                           void *grad_bias, void *workspace, int64_t workspace_bytes,
                                           void *hip_stream);

/*
 * Attention of queries to an encoder's states of another length. Query i of head
 * h reads key head h / (heads / key_heads):
 *   s_j = scale * q_i . k_j over the keys j in use, p = softmax(s),
 *   out_i = sum_j p_j v_j;  0 where no key is in use.
 * Key j of sample b is in use if j < key_lengths[b] and key_mask[b][j] is not 0.
 * Keys and values not in use are not read into any sum: they may hold anything,
 * NaN included, and their gradients are 0. Queries, and keys and values in use, must
 * be finite: where they are not, their sample's results are unspecified.
 * Element (b, i, h, c) of q is at q + b * q_batch + i * q_row + h * q_head + c,
 * strides in elements; k and v alike. out and the gradients are contiguous.
 */
typedef struct {
    int32_t batch, queries, keys, heads, key_heads, dim;
    int32_t dtype;         /* of q, k, v, out and the gradients */
    float scale;
    int64_t q_batch, q_row, q_head;
    int64_t k_batch, k_row, k_head;
    int64_t v_batch, v_row, v_head;
    int64_t mask_batch;    /* bytes from sample to sample of key_mask */
} bevmap_attend;

/* Bytes of workspace of bevmap_attention (backward = 0) or
 * bevmap_attention_backward (backward = 1); a negative error code if the
 * description is refused. Host only. */
BEVPOOL_API int64_t bevmap_attention_workspace(const bevmap_attend *attend, int32_t backward);

/*
 *  key_lengths: device int32 [batch], or NULL for all keys; clamped to
 *             [0, keys].
 *  key_mask:  device uint8 [batch][keys] (rows mask_batch bytes apart), or NULL.
 *  out:       device [batch][queries][heads][dim] of dtype, overwritten.
 *  out_low:   device, like out, or NULL; overwritten with what the rounding of
 *             out left over, for the backward (of 16-bit types; not written for fp32).
 *  lse:       device float [batch][heads][queries], or NULL; overwritten with
 *             log2 of the sum of e^s, -infinity where no key is in use.
 * Scores, softmax statistics and output sums are fp32; fp32 inputs are multiplied
 * as sums of three bf16 pieces each, which leaves out at most 2^-24 of a product. With 16-bit inputs the
 * probabilities, relative to a maximum of the row, are rounded to the inputs'
 * type for their product with v, which leaves out about 1.3 times as far off as
 * fp32 sums rounded once; of at most 32 rows, that is queries * heads /
 * key_heads, to two pieces of the type, which does not show in out.
 * A size of 0 is a call that writes zeros, or nothing.
 * Errors: INVALID_ARG (null pointer, a size below 0, heads, key_heads or dim
 * below 1, heads not a multiple of key_heads, scale not finite, a stride below
 * 0, workspace too small or not 16-byte aligned), UNSUPPORTED_DTYPE, OVERFLOW (dim above 128, batch * key_heads above
 * 65535, queries * heads / key_heads or keys reaching 2^30, k_row or v_row
 * reaching 2^22, batch * key_heads * the tiles of 128 that queries * heads /
 * key_heads make reaching 2^23), HIP (launch failure).
 */
BEVPOOL_API int bevmap_attention(const bevmap_attend *attend, const void *q, const void *k, const void *v,
                                 const int32_t *key_lengths, const uint8_t *key_mask, void *out,
                                 void *out_low, float *lse, void *workspace, int64_t workspace_bytes,
                                 void *hip_stream);

/*
 * Gradients of bevmap_attention, with the out, out_low and lse that it wrote:
 *  grad_out:  device [batch][queries][heads][dim] of dtype.
 *  grad_q:    device [batch][queries][heads][dim], grad_k, grad_v: device
 *             [batch][keys][key_heads][dim], of dtype, overwritten. A key head's
 *             gradients sum over the heads that share it.
 * out_low may be NULL (out is then taken as it is). Sums are fp32; with 16-bit types
 * the probabilities and the scores' gradients enter their products as two pieces
 * of the type.
 * Errors: those of bevmap_attention, and OVERFLOW where batch * key_heads * the tiles
 * of 128 that the keys make reach 2^23 (bevmap_attention_workspace says so as well).
 */
BEVPOOL_API int bevmap_attention_backward(const bevmap_attend *attend, const void *grad_out, const void *q,
                                          const void *k, const void *v, const int32_t *key_lengths,
                                          const uint8_t *key_mask, const void *out, const void *out_low,
                                          const float *lse, void *grad_q, void *grad_k, void *grad_v,
                                          void *workspace, int64_t workspace_bytes, void *hip_stream);

/*
 * y = residual + dropout(x) over rows * columns elements; element e = row *
 * columns + column is kept iff its draw, 16 bits, is >= threshold, and a kept x
 * is scaled by 65536 / (65536 - threshold), so that the expectation of y is
 * residual + x. threshold in 0..65536: 0 keeps all, 65536 none. The draw of e is
 * half e % 8 (low halves first) of the four 32-bit words that philox4x32-10
 * (Salmon et al., "Parallel random numbers: as easy as 1, 2, 3", 2011) gives for
 * the counter (e / 8, offset), low words first, and the key seed. The mask
 * depends on seed, offset and e alone: the backward draws it again.
 *  x, residual: device, rows x_stride and residual_stride elements apart (>=
 *             columns); residual NULL for none.
 *  y:         device [rows][columns], overwritten.
 * A dropped x does not reach y, whatever it holds. The gradient of x is the same
 * call on the gradient of y without a residual; the residual's is the gradient of y.
 * A graph that captured this call draws the same mask in each replay.
 * Errors: INVALID_ARG (null pointer, a size below 0, a stride < columns, threshold
 * outside 0..65536), UNSUPPORTED_DTYPE, OVERFLOW (rows * columns above 2^40;
 * with several rows, columns or a stride reaching 2^31), HIP (launch failure).
 */
BEVPOOL_API int bevmap_dropout(const void *x, int64_t x_stride, const void *residual,
                               int64_t residual_stride, void *y, int64_t rows, int64_t columns,
                               int32_t dtype, int32_t threshold, uint64_t seed, uint64_t offset,
                               void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* BEVMAP_H */
