/*
 * bevmap.h -- C ABI of libbevpool.so: operators of the model that reads a pooled
 * BEV map, on MI355X (gfx950). The pooling itself is in bevpool.h.
 *
 * Channels last throughout. With gradients:
 *  - bevmap_group_norm: group norm with an activation;
 *  - bevmap_attention: queries attend to an encoder's states of another length
 *    (the cells of a map, the pixels of the cameras);
 *  - bevmap_dropout: residual + dropout(x), the mask from a counter-based
 *    generator and never stored;
 *  - bevmap_rms_norm: root-mean-square norm of rows, of x + residual;
 *  - bevmap_rotary: pairs of channels turned by angles that go with a position;
 *  - bevmap_gated_act: act(gate) * value, what the backward needs kept in 8 bits.
 * For serving, in 8-bit integers:
 *  - bevmap_rms_norm_int8, bevmap_quantize_int8: rows as integers and a scale;
 *  - bevmap_linear_int8: their product with weights of a scale for each channel.
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

/*
 * Root-mean-square norm of rows. Row s starts at x + s * x_stride elements and holds
 * `channels` elements; residual alike. With h = x + residual (x without one):
 *   rstd = 1 / sqrt(mean of h^2 + eps),  y = weight[c] * h * rstd.
 * The sum is handed on rounded to x_dtype; y is formed from it before that.
 * Squares are summed in fp32, rows whose squares leave its range after a power of two is
 * taken out, so a row of any finite size is normed. An infinity or a NaN reaches its row
 * alone. (Gradients read rstd: through a row whose rstd is past fp32's range, of numbers below
 * 2^-127 with an eps of 0, they are not finite, and the weight's neither.)
 */
typedef struct {
    int64_t rows;
    int32_t channels;
    int32_t x_dtype;       /* of x, residual, sum and their gradients */
    int32_t y_dtype;       /* of y and grad_y */
    int32_t weight_dtype;  /* of weight and grad_weight */
    int64_t x_stride, residual_stride;   /* elements from row to row, >= channels */
    float eps;             /* >= 0 */
} bevmap_rms;

/*
 *  residual: NULL for none; sum is then not written (and may be NULL).
 *  weight:   device [channels] of weight_dtype; NULL for ones.
 *  sum:      device [rows][channels] of x_dtype, overwritten with x + residual.
 *  y:        device [rows][channels] of y_dtype, overwritten.
 *  rstd:     device float [rows], or NULL; overwritten: what the backward reads.
 * rows of 0 is a call that does nothing.
 * Errors: INVALID_ARG (null pointer, rows below 0, channels below 1, a stride <
 * channels, eps negative or not finite), UNSUPPORTED_DTYPE, OVERFLOW (rows or a stride
 * reaching 2^31, channels above 8192), HIP (launch failure).
 */
BEVPOOL_API int bevmap_rms_norm(const bevmap_rms *norm, const void *x, const void *residual, const void *weight,
                                void *sum, void *y, float *rstd, void *hip_stream);

/* Bytes of workspace of bevmap_rms_norm_backward; a negative error code if the
 * description is refused. Host only. */
BEVPOOL_API int64_t bevmap_rms_norm_backward_workspace(const bevmap_rms *norm);

/*
 * Gradients of bevmap_rms_norm, with the rstd that it wrote:
 *  grad_y:      device [rows][channels] of y_dtype.
 *  grad_sum:    device [rows][channels] of x_dtype: the gradient of sum, or NULL.
 *  x, residual: those of bevmap_rms_norm. Its sum in the place of x, with a NULL
 *               residual, does as well, but for what rounding it to x_dtype took away.
 *  grad_x:      device [rows][channels] of x_dtype, overwritten: the gradient of x, which
 *               is the residual's as well.
 *  grad_weight: device [channels] of weight_dtype, overwritten (zeros for no rows); NULL
 *               to skip.
 * Errors: those of bevmap_rms_norm, and INVALID_ARG for a workspace that is too small or
 * not 16-byte aligned.
 */
BEVPOOL_API int bevmap_rms_norm_backward(const bevmap_rms *norm, const void *grad_y, const void *grad_sum,
                                         const void *x, const void *residual, const void *weight,
                                         const float *rstd, void *grad_x, void *grad_weight, void *workspace,
                                         int64_t workspace_bytes, void *hip_stream);

/*
 * The norm's result in 8 bits, for a product that reads it: with top the largest
 * |weight * h| of a row,
 *   held = round(weight * h * (127 / top)), scale = top * rstd / 127,
 * so that held * scale is y to within half a scale; halves go to the even neighbour. A
 * row of zeros has scale 0 (eps of 0: NaN), one with an infinity or a NaN, its own, a
 * weight's or y's, has scale NaN and zeros.
 *  held:  device int8 [rows][channels], overwritten.  scale: device float [rows],
 *         overwritten.  The rest as for bevmap_rms_norm; y_dtype is not used.
 * Errors: those of bevmap_rms_norm.
 */
BEVPOOL_API int bevmap_rms_norm_int8(const bevmap_rms *norm, const void *x, const void *residual,
                                     const void *weight, void *sum, int8_t *held, float *scale, void *hip_stream);

/*
 * Rows as 8-bit integers: held = round(x * (127 / top)), scale = top / 127 with top the
 * row's largest |x|; rows of zeros, infinities and NaN as above.
 *  x: device, rows x_stride elements apart (>= columns).
 *  held: device int8 [rows][columns], scale: device float [rows], overwritten.
 * Errors: INVALID_ARG (null pointer, a size below 0, x_stride < columns),
 * UNSUPPORTED_DTYPE, OVERFLOW (rows or x_stride reaching 2^31, columns above 131071),
 * HIP (launch failure).
 */
BEVPOOL_API int bevmap_quantize_int8(const void *x, int64_t x_stride, int8_t *held, float *scale, int64_t rows,
                                     int32_t columns, int32_t dtype, void *hip_stream);

/*
 * Product of 8-bit integers with a scale for each row (token) and each feature:
 *   y[m][n] = x_scale[m] * w_scale[n] * (sum over k of x[m][k] * w[n][k]) + bias[n].
 * Sums are 32-bit integers, exact for all values of int8 up to 131071 channels; fp32
 * follows, in an order in which only results past its range are infinite, and one rounding
 * to y_dtype.
 */
typedef struct {
    int64_t rows;
    int32_t channels, features;          /* of the sum; of the result */
    int64_t x_stride, w_stride;          /* bytes from row to row, >= channels */
    int32_t y_dtype;
} bevmap_linear;

/*
 *  x: device int8, rows x_stride apart; x_scale: device float [rows].
 *  w: device int8 [features], rows w_stride apart; w_scale: device float [features].
 *  bias: device float [features], or NULL.
 *  y: device [rows][features] of y_dtype, overwritten.
 * Rows of 16-byte aligned addresses with channels a multiple of 16 are read past the
 * registers. rows or features of 0 is a call that does nothing.
 * Errors: INVALID_ARG (null pointer, rows or features below 0, channels below 1, a
 * stride < channels), UNSUPPORTED_DTYPE, OVERFLOW (channels above 131071, rows reaching
 * 2^30, a stride reaching 2^31, features above 2^20, rows * features reaching 2^37), HIP
 * (launch failure).
 */
BEVPOOL_API int bevmap_linear_int8(const bevmap_linear *linear, const int8_t *x, const float *x_scale,
                                   const int8_t *w, const float *w_scale, const float *bias, void *y,
                                   void *hip_stream);

/* Types of the positions of bevmap_rotary. */
typedef enum { BEVMAP_POSITION_I32 = 0, BEVMAP_POSITION_I64 = 1, BEVMAP_POSITION_F32 = 2 } bevmap_position;

/*
 * Rotary positions: the first 2 * pairs channels of each head are pairs (a, b), pair p
 * being channels (2 p, 2 p + 1) if interleaved, (p, p + pairs) otherwise, and
 *   (a, b) -> amplitude * (a cos t - b sin t, a sin t + b cos t),
 *   t = positions[token][p / (pairs / axes)] * frequencies[p].
 * Later channels keep their values. Positions have `axes` numbers a token: with two axes
 * the first half of the pairs turns with the first. Angles are formed and reduced in 64
 * bits, as exactly for positions up to 2^53 in magnitude as for near ones; the turn is fp32,
 * and its result is rounded once.
 * Element (b, n, h, c) of x is at x + b * x_batch + n * x_row + h * x_head + c, strides in
 * elements.
 */
typedef struct {
    int32_t batch, tokens, heads, dim, pairs, axes;
    int32_t interleaved;
    int32_t positions_type;              /* bevmap_position */
    int32_t dtype;                       /* of x and out */
    float amplitude;
    int64_t x_batch, x_row, x_head;
} bevmap_turn;

/*
 *  positions:   device [batch][tokens][axes] of positions_type. An infinity or a NaN gives
 *               NaN in the channels that turn with it.
 *  frequencies: device double [pairs], radians to a unit of position.
 *  out:         device [batch][tokens][heads][dim] of dtype, overwritten.
 *  backward:    not 0 turns by the negative angles: x is then the gradient of out, and out
 *               the gradient of x.
 * A size of 0 is a call that does nothing.
 * Errors: INVALID_ARG (null pointer, batch or tokens below 0, heads, dim, pairs or axes
 * below 1, 2 * pairs above dim, pairs not a multiple of axes, unknown position type,
 * amplitude not finite, a stride below 0), UNSUPPORTED_DTYPE, OVERFLOW (batch * tokens
 * reaching 2^31, heads above 65535, dim above 4096), HIP (launch failure).
 */
BEVPOOL_API int bevmap_rotary(const bevmap_turn *turn, const void *x, const void *positions,
                              const double *frequencies, void *out, int32_t backward, void *hip_stream);

/*
 * Gated activation: a row of x holds `features` gates and then as many values,
 *   y[f] = act(gate[f]) * value[f].
 * act is formed in fp32 to within 2^-15 of its value, far below 0 too (there silu is taken as
 * 0 where it is under 2^-118 in magnitude), and near 0 and above to within some 2^-22.
 */
typedef struct {
    int64_t rows;
    int32_t features;
    int32_t act;           /* bevmap_act */
    int32_t dtype;         /* of x, y and their gradients */
    int64_t x_stride;      /* elements from row to row of x, >= 2 * features */
} bevmap_gate;

/*
 *  x:     device [rows], rows x_stride apart.
 *  y:     device [rows][features], overwritten.
 *  held, exponents: NULL, or device int8 [rows][2][features] and uint8
 *         [rows][2][ceil(features / 32)], overwritten with x in 8 bits for the backward:
 *         32 neighbouring channels of a half share the least power of two 2^e whose 127-fold
 *         reaches their largest magnitude (e at least -127), held = round(x / 2^e) with
 *         halves to the even neighbour, exponents = e + 127; 255 and zeros for channels with
 *         an infinity or a NaN among them, which the backward takes as NaN.
 * rows of 0 is a call that does nothing.
 * Errors: INVALID_ARG (null pointer, one of held and exponents without the other, rows
 * below 0, features below 1, x_stride < 2 * features, unknown act), UNSUPPORTED_DTYPE,
 * OVERFLOW (rows or x_stride reaching 2^31, features reaching 2^24), HIP (launch failure).
 */
BEVPOOL_API int bevmap_gated_act(const bevmap_gate *gate, const void *x, void *y, int8_t *held, uint8_t *exponents,
                                 void *hip_stream);

/*
 * Gradients of bevmap_gated_act, from x (held and exponents NULL), or from what it held of
 * x (x may then be NULL):
 *  grad_y: device [rows][features].  grad_x: device [rows][2 * features], overwritten.
 * Errors: those of bevmap_gated_act.
 */
BEVPOOL_API int bevmap_gated_act_backward(const bevmap_gate *gate, const void *grad_y, const void *x,
                                          const int8_t *held, const uint8_t *exponents, void *grad_x,
                                          void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* BEVMAP_H */
