// C entries of the map operators (declared in include/bevmap.h): argument checks.
// The device work is in norm.hip, attention.hip and dropout.hip.
#include <math.h>

#include "mapops.h"

namespace {

bool known_dtype(int32_t d) { return d == BEVPOOL_F32 || d == BEVPOOL_BF16 || d == BEVPOOL_F16; }

int check(const bevmap_norm *n) {
    if (!n) return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "null description");
    if (n->batch < 0 || n->pixels < 0 || n->channels < 1 || n->groups < 1)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "batch=%d pixels=%d channels=%d groups=%d", n->batch, n->pixels,
                            n->channels, n->groups);
    if (n->channels % n->groups)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "channels=%d is not a multiple of groups=%d", n->channels,
                            n->groups);
    if (n->row_stride < n->channels)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "row stride %lld below channels=%d", (long long)n->row_stride,
                            n->channels);
    if (!isfinite(n->eps) || n->eps < 0)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "eps=%g must be finite and >= 0", double(n->eps));
    if (n->act < BEVMAP_ACT_NONE || n->act > BEVMAP_ACT_GELU)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "unknown activation %d", n->act);
    if (!known_dtype(n->x_dtype) || !known_dtype(n->y_dtype) || !known_dtype(n->weight_dtype))
        return bevpool_fail(BEVPOOL_ERR_UNSUPPORTED_DTYPE, "dtypes %d, %d, %d", n->x_dtype, n->y_dtype,
                            n->weight_dtype);
    if (int64_t(n->batch) * n->pixels >= (int64_t(1) << 30) || n->channels > kNormMaxChannels || n->batch > 65535 ||
        n->row_stride >= (int64_t(1) << 31))
        return bevpool_fail(BEVPOOL_ERR_OVERFLOW, "batch=%d pixels=%d channels=%d row stride %lld: too large",
                            n->batch, n->pixels, n->channels, (long long)n->row_stride);
    return BEVPOOL_OK;
}

// backward: the tiles of keys are limited too.
int check(const bevmap_attend *a, bool backward) {
    if (!a) return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "null description");
    if (a->batch < 0 || a->queries < 0 || a->keys < 0 || a->heads < 1 || a->key_heads < 1 || a->dim < 1)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "batch=%d queries=%d keys=%d heads=%d key_heads=%d dim=%d",
                            a->batch, a->queries, a->keys, a->heads, a->key_heads, a->dim);
    if (a->heads % a->key_heads)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "heads=%d is not a multiple of key_heads=%d", a->heads,
                            a->key_heads);
    if (!isfinite(a->scale)) return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "scale must be finite");
    if (!known_dtype(a->dtype)) return bevpool_fail(BEVPOOL_ERR_UNSUPPORTED_DTYPE, "dtype %d", a->dtype);
    if (a->q_batch < 0 || a->q_row < 0 || a->q_head < 0 || a->k_batch < 0 || a->k_row < 0 || a->k_head < 0 ||
        a->v_batch < 0 || a->v_row < 0 || a->v_head < 0 || a->mask_batch < 0)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "strides must not be negative");
    if (a->dim > kAttendMaxDim || int64_t(a->batch) * a->key_heads > 65535 || a->keys >= (1 << 30) ||
        int64_t(a->queries) * (a->heads / a->key_heads) >= (int64_t(1) << 30) ||
        a->k_row >= (int64_t(1) << 22) || a->v_row >= (int64_t(1) << 22))
        return bevpool_fail(BEVPOOL_ERR_OVERFLOW,
                            "dim=%d batch=%d queries=%d keys=%d heads=%d key_heads=%d, or a key's or value's row "
                            "stride, is outside the limits", a->dim, a->batch, a->queries, a->keys, a->heads, a->key_heads);
    const int64_t rows = int64_t(a->queries) * (a->heads / a->key_heads);
    const int64_t owned = backward && a->keys > rows ? a->keys : rows;
    if (int64_t(a->batch) * a->key_heads * ((owned + kAttendTile - 1) / kAttendTile) >= kAttendMaxTiles)
        return bevpool_fail(BEVPOOL_ERR_OVERFLOW, "batch=%d queries=%d keys=%d heads=%d key_heads=%d: too many tiles of "
                            "%s", a->batch, a->queries, a->keys, a->heads, a->key_heads, owned > rows ? "keys" : "rows");
    return BEVPOOL_OK;
}

int check_workspace(const void *workspace, int64_t have, int64_t need) {
    if (need > 0 && (!workspace || have < need))
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "workspace of %lld bytes, needs %lld",
                            workspace ? (long long)have : 0ll, (long long)need);
    if (reinterpret_cast<uintptr_t>(workspace) % 16)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    return BEVPOOL_OK;
}

}  // namespace

extern "C" {

int64_t bevmap_group_norm_workspace(const bevmap_norm *norm, int32_t backward) {
    if (int rc = check(norm)) return rc;
    return bevmap_norm_workspace_bytes(*norm, backward != 0);
}

int bevmap_group_norm(const bevmap_norm *norm, const void *x, const void *weight, const void *bias, void *y,
                      float *mean, float *rstd, void *workspace, int64_t workspace_bytes, void *hip_stream) {
    if (int rc = check(norm)) return rc;
    const bool empty = norm->batch == 0 || norm->pixels == 0;
    if (!empty && (!x || !y || !mean || !rstd))
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "null pointer argument");
    if (int rc = check_workspace(workspace, workspace_bytes, bevmap_norm_workspace_bytes(*norm, false))) return rc;
    return bevmap_launch_norm(*norm, x, weight, bias, y, mean, rstd, workspace,
                              static_cast<hipStream_t>(hip_stream));
}

int bevmap_group_norm_backward(const bevmap_norm *norm, const void *grad_y, const void *x, const void *weight,
                               const void *bias, const float *mean, const float *rstd, void *grad_x,
                               void *grad_weight, void *grad_bias, void *workspace, int64_t workspace_bytes,
                               void *hip_stream) {
    if (int rc = check(norm)) return rc;
    const bool empty = norm->batch == 0 || norm->pixels == 0;
    if (!empty && (!grad_y || !x || !mean || !rstd || !grad_x))
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "null pointer argument");
    if (int rc = check_workspace(workspace, workspace_bytes, bevmap_norm_workspace_bytes(*norm, true))) return rc;
    return bevmap_launch_norm_backward(*norm, grad_y, x, weight, bias, mean, rstd, grad_x, grad_weight, grad_bias,
                                       workspace, static_cast<hipStream_t>(hip_stream));
}

int64_t bevmap_attention_workspace(const bevmap_attend *attend, int32_t backward) {
    if (int rc = check(attend, backward != 0)) return rc;
    return bevmap_attention_workspace_bytes(*attend, backward != 0);
}

int bevmap_attention(const bevmap_attend *attend, const void *q, const void *k, const void *v,
                     const int32_t *key_lengths, const uint8_t *key_mask, void *out, void *out_low, float *lse,
                     void *workspace, int64_t workspace_bytes, void *hip_stream) {
    if (int rc = check(attend, false)) return rc;
    const bool asked = attend->batch > 0 && attend->queries > 0;
    if (asked && (!q || !out || (attend->keys > 0 && (!k || !v))))
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "null pointer argument");
    if (int rc = check_workspace(workspace, workspace_bytes, bevmap_attention_workspace_bytes(*attend, false)))
        return rc;
    return bevmap_launch_attention(*attend, q, k, v, key_lengths, key_mask, out, out_low, lse, workspace,
                                   static_cast<hipStream_t>(hip_stream));
}

int bevmap_attention_backward(const bevmap_attend *attend, const void *grad_out, const void *q, const void *k,
                              const void *v, const int32_t *key_lengths, const uint8_t *key_mask, const void *out,
                              const void *out_low, const float *lse, void *grad_q, void *grad_k, void *grad_v,
                              void *workspace, int64_t workspace_bytes, void *hip_stream) {
    if (int rc = check(attend, true)) return rc;
    const bool asked = attend->batch > 0 && attend->queries > 0, stored = attend->batch > 0 && attend->keys > 0;
    if ((asked && (!grad_out || !q || !out || !lse || !grad_q)) || (stored && (!k || !v || !grad_k || !grad_v)))
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "null pointer argument");
    if (int rc = check_workspace(workspace, workspace_bytes, bevmap_attention_workspace_bytes(*attend, true)))
        return rc;
    return bevmap_launch_attention_backward(*attend, grad_out, q, k, v, key_lengths, key_mask, out, out_low, lse,
                                            grad_q, grad_k, grad_v, workspace,
                                            static_cast<hipStream_t>(hip_stream));
}

int bevmap_dropout(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, void *y,
                   int64_t rows, int64_t columns, int32_t dtype, int32_t threshold, uint64_t seed,
                   uint64_t offset, void *hip_stream) {
    if (rows < 0 || columns < 0)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "rows=%lld columns=%lld", (long long)rows, (long long)columns);
    if (threshold < 0 || threshold > 65536)
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "threshold=%d is outside 0..65536", threshold);
    if (!known_dtype(dtype)) return bevpool_fail(BEVPOOL_ERR_UNSUPPORTED_DTYPE, "dtype %d", dtype);
    if (rows == 0 || columns == 0) return BEVPOOL_OK;
    if (!x || !y) return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "null pointer argument");
    if (rows > 1 && (x_stride < columns || (residual && residual_stride < columns)))
        return bevpool_fail(BEVPOOL_ERR_INVALID_ARG, "a row stride is below columns=%lld", (long long)columns);
    const int64_t big = int64_t(1) << 31, most = int64_t(1) << 40;
    if (columns >= most || rows > most / columns || (rows > 1 && (columns >= big || x_stride >= big ||
                                                                 (residual && residual_stride >= big))))
        return bevpool_fail(BEVPOOL_ERR_OVERFLOW, "rows=%lld columns=%lld, or a row stride, is too large",
                            (long long)rows, (long long)columns);
    return bevmap_launch_dropout(x, x_stride, residual, residual_stride, y, rows, columns, dtype, threshold, seed,
                                 offset, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
