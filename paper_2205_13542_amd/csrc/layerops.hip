// C entries of the operators around attention (declared in include/bevmap.h): argument
// checks. The device work is in rms_norm.hip, rotary.hip, gated.hip and linear_int8.hip.
#include <math.h>

#include "mapops.h"

namespace {

constexpr int64_t kBig = int64_t(1) << 31;

bool known_dtype(int32_t d) { return d == BEVPOOL_F32 || d == BEVPOOL_BF16 || d == BEVPOOL_F16; }

int null_pointer() { return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "null pointer argument"); }

// residual: its stride counts too.
int check(const bevmap_rms *n, bool residual) {
    if (!n) return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "null description");
    if (n->rows < 0 || n->channels < 1)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "rows=%lld channels=%d", (long long)n->rows, n->channels);
    if (n->x_stride < n->channels || (residual && n->residual_stride < n->channels))
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "a row stride is below channels=%d", n->channels);
    if (!isfinite(n->eps) || n->eps < 0)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "eps=%g must be finite and >= 0", double(n->eps));
    if (!known_dtype(n->x_dtype) || !known_dtype(n->y_dtype) || !known_dtype(n->weight_dtype))
        return bevpool_fail(BEVPOOL_ERR_UNSUPPORTED_DTYPE, "dtypes %d, %d, %d", n->x_dtype, n->y_dtype,
                            n->weight_dtype);
    if (n->rows >= kBig || n->channels > kNormMaxChannels || n->x_stride >= kBig ||
        (residual && n->residual_stride >= kBig))
        return bevpool_fail(BEVPOOL_ERR_OVERFLOW, "rows=%lld channels=%d, or a row stride, is too large",
                            (long long)n->rows, n->channels);
    return BEVPOOL_OK;
}

int check(const bevmap_linear *n) {
    if (!n) return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "null description");
    if (n->rows < 0 || n->features < 0 || n->channels < 1)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "rows=%lld channels=%d features=%d", (long long)n->rows,
                            n->channels, n->features);
    if (n->x_stride < n->channels || n->w_stride < n->channels)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "a row stride is below channels=%d", n->channels);
    if (!known_dtype(n->y_dtype)) return bevpool_fail(BEVPOOL_ERR_UNSUPPORTED_DTYPE, "dtype %d", n->y_dtype);
    if (n->channels > kInt8MaxChannels || n->rows >= kBig / 2 || n->x_stride >= kBig || n->w_stride >= kBig ||
        n->features > (1 << 20) || n->rows * n->features >= int64_t(1) << 37)
        return bevpool_fail(BEVPOOL_ERR_OVERFLOW, "rows=%lld channels=%d features=%d, or a row stride, is too large",
                            (long long)n->rows, n->channels, n->features);
    return BEVPOOL_OK;
}

int check(const bevmap_turn *n) {
    if (!n) return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "null description");
    if (n->batch < 0 || n->tokens < 0 || n->heads < 1 || n->dim < 1 || n->pairs < 1 || n->axes < 1)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "batch=%d tokens=%d heads=%d dim=%d pairs=%d axes=%d", n->batch,
                            n->tokens, n->heads, n->dim, n->pairs, n->axes);
    if (int64_t(n->pairs) * 2 > n->dim || n->pairs % n->axes)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "pairs=%d: two channels each of dim=%d, a multiple of axes=%d",
                            n->pairs, n->dim, n->axes);
    if (n->positions_type < BEVMAP_POSITION_I32 || n->positions_type > BEVMAP_POSITION_F32)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "unknown position type %d", n->positions_type);
    if (!isfinite(n->amplitude)) return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "amplitude must be finite");
    if (n->x_batch < 0 || n->x_row < 0 || n->x_head < 0)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "strides must not be negative");
    if (!known_dtype(n->dtype)) return bevpool_fail(BEVPOOL_ERR_UNSUPPORTED_DTYPE, "dtype %d", n->dtype);
    if (int64_t(n->batch) * n->tokens >= kBig || n->heads > 65535 || n->dim > kTurnMaxDim)
        return bevpool_fail(BEVPOOL_ERR_OVERFLOW, "batch=%d tokens=%d heads=%d dim=%d: too large", n->batch, n->tokens,
                            n->heads, n->dim);
    return BEVPOOL_OK;
}

int check(const bevmap_gate *n, const int8_t *held, const uint8_t *exponents) {
    if (!n) return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "null description");
    if (n->rows < 0 || n->features < 1)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "rows=%lld features=%d", (long long)n->rows, n->features);
    if (n->x_stride < 2 * int64_t(n->features))
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "row stride %lld below twice features=%d", (long long)n->x_stride,
                            n->features);
    if (n->act < BEVMAP_ACT_NONE || n->act > BEVMAP_ACT_GELU)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "unknown activation %d", n->act);
    if (!held != !exponents)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "held and exponents go together");
    if (!known_dtype(n->dtype)) return bevpool_fail(BEVPOOL_ERR_UNSUPPORTED_DTYPE, "dtype %d", n->dtype);
    if (n->rows >= kBig || n->x_stride >= kBig || n->features >= (1 << 24))
        return bevpool_fail(BEVPOOL_ERR_OVERFLOW, "rows=%lld features=%d row stride %lld: too large",
                            (long long)n->rows, n->features, (long long)n->x_stride);
    return BEVPOOL_OK;
}

}  // namespace

extern "C" {

int bevmap_rms_norm(const bevmap_rms *norm, const void *x, const void *residual, const void *weight, void *sum,
                    void *y, float *rstd, void *hip_stream) {
    if (int rc = check(norm, residual != nullptr)) return rc;
    if (norm->rows > 0 && (!x || !y || (residual && !sum))) return null_pointer();
    return bevmap_launch_rms_norm(*norm, x, residual, weight, sum, y, rstd, nullptr, nullptr,
                                  static_cast<hipStream_t>(hip_stream));
}

int64_t bevmap_rms_norm_backward_workspace(const bevmap_rms *norm) {
    if (int rc = check(norm, false)) return rc;
    return bevmap_rms_workspace_bytes(*norm);
}

int bevmap_rms_norm_backward(const bevmap_rms *norm, const void *grad_y, const void *grad_sum, const void *x,
                             const void *residual, const void *weight, const float *rstd, void *grad_x,
                             void *grad_weight, void *workspace, int64_t workspace_bytes, void *hip_stream) {
    if (int rc = check(norm, residual != nullptr)) return rc;
    if (norm->rows > 0 && (!grad_y || !x || !rstd || !grad_x)) return null_pointer();
    const int64_t need = grad_weight ? bevmap_rms_workspace_bytes(*norm) : 0;
    if (need > 0 && (!workspace || workspace_bytes < need))
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "workspace of %lld bytes, needs %lld",
                            workspace ? (long long)workspace_bytes : 0ll, (long long)need);
    if (reinterpret_cast<uintptr_t>(workspace) % 16)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    return bevmap_launch_rms_norm_backward(*norm, grad_y, grad_sum, x, residual, weight, rstd, grad_x, grad_weight,
                                           workspace, static_cast<hipStream_t>(hip_stream));
}

int bevmap_rms_norm_int8(const bevmap_rms *norm, const void *x, const void *residual, const void *weight, void *sum,
                         int8_t *held, float *scale, void *hip_stream) {
    if (int rc = check(norm, residual != nullptr)) return rc;
    if (norm->rows > 0 && (!x || !held || !scale || (residual && !sum))) return null_pointer();
    return bevmap_launch_rms_norm(*norm, x, residual, weight, sum, nullptr, nullptr, held, scale,
                                  static_cast<hipStream_t>(hip_stream));
}

int bevmap_quantize_int8(const void *x, int64_t x_stride, int8_t *held, float *scale, int64_t rows, int32_t columns,
                         int32_t dtype, void *hip_stream) {
    if (rows < 0 || columns < 0)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "rows=%lld columns=%d", (long long)rows, columns);
    if (x_stride < columns)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "row stride %lld below columns=%d", (long long)x_stride, columns);
    if (!known_dtype(dtype)) return bevpool_fail(BEVPOOL_ERR_UNSUPPORTED_DTYPE, "dtype %d", dtype);
    if (rows >= kBig || x_stride >= kBig || columns > kInt8MaxChannels)
        return bevpool_fail(BEVPOOL_ERR_OVERFLOW, "rows=%lld columns=%d row stride %lld: too large", (long long)rows,
                            columns, (long long)x_stride);
    if (rows == 0) return BEVPOOL_OK;
    if (!scale || (columns > 0 && (!x || !held))) return null_pointer();
    return bevmap_launch_quantize(x, x_stride, held, scale, rows, columns, dtype,
                                  static_cast<hipStream_t>(hip_stream));
}

int bevmap_linear_int8(const bevmap_linear *linear, const int8_t *x, const float *x_scale, const int8_t *w,
                       const float *w_scale, const float *bias, void *y, void *hip_stream) {
    if (int rc = check(linear)) return rc;
    if (linear->rows > 0 && linear->features > 0 && (!x || !x_scale || !w || !w_scale || !y)) return null_pointer();
    return bevmap_launch_linear_int8(*linear, x, x_scale, w, w_scale, bias, y, static_cast<hipStream_t>(hip_stream));
}

int bevmap_rotary(const bevmap_turn *turn, const void *x, const void *positions, const double *frequencies, void *out,
                  int32_t backward, void *hip_stream) {
    if (int rc = check(turn)) return rc;
    if (turn->batch > 0 && turn->tokens > 0 && (!x || !positions || !frequencies || !out)) return null_pointer();
    return bevmap_launch_rotary(*turn, x, positions, frequencies, out, backward != 0,
                                static_cast<hipStream_t>(hip_stream));
}

int bevmap_gated_act(const bevmap_gate *gate, const void *x, void *y, int8_t *held, uint8_t *exponents,
                     void *hip_stream) {
    if (int rc = check(gate, held, exponents)) return rc;
    if (gate->rows > 0 && (!x || !y)) return null_pointer();
    return bevmap_launch_gate(*gate, x, y, held, exponents, static_cast<hipStream_t>(hip_stream));
}

int bevmap_gated_act_backward(const bevmap_gate *gate, const void *grad_y, const void *x, const int8_t *held,
                              const uint8_t *exponents, void *grad_x, void *hip_stream) {
    if (int rc = check(gate, held, exponents)) return rc;
    if (gate->rows > 0 && (!grad_y || !grad_x || (!x && !held))) return null_pointer();
    return bevmap_launch_gate_backward(*gate, grad_y, x, held, exponents, grad_x,
                                       static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
