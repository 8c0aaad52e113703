// Declarations and device helpers shared by the map operators (include/bevmap.h):
// norm.hip, attention.hip and dropout.hip launch, mapops.hip checks.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "bevmap.h"
#include "internal.h"

// Limits that the kernels assume.
constexpr int kNormMaxChannels = 8192;  // two floats a channel in LDS
constexpr int kAttendMaxDim = 128;
constexpr int kAttendTile = 128;        // rows or keys that a workgroup owns
constexpr int64_t kAttendMaxTiles = int64_t(1) << 23;   // workgroups of a launch; more are never needed to split an axis

// Launches; arguments are checked by the caller (mapops.hip).
int64_t bevmap_norm_workspace_bytes(const bevmap_norm &n, bool backward);
int bevmap_launch_norm(const bevmap_norm &n, const void *x, const void *weight, const void *bias, void *y,
                       float *mean, float *rstd, void *workspace, hipStream_t stream);
int bevmap_launch_norm_backward(const bevmap_norm &n, const void *grad_y, const void *x, const void *weight,
                                const void *bias, const float *mean, const float *rstd, void *grad_x,
                                void *grad_weight, void *grad_bias, void *workspace, hipStream_t stream);
int64_t bevmap_attention_workspace_bytes(const bevmap_attend &a, bool backward);
int64_t bevmap_attention_backward_bytes(const bevmap_attend &a);
int bevmap_launch_attention(const bevmap_attend &a, const void *q, const void *k, const void *v,
                            const int32_t *lengths, const uint8_t *mask, void *out, void *out_low, float *lse,
                            void *workspace, hipStream_t stream);
int bevmap_launch_attention_backward(const bevmap_attend &a, const void *grad_out, const void *q, const void *k,
                                     const void *v, const int32_t *lengths, const uint8_t *mask, const void *out,
                                     const void *out_low, const float *lse, void *grad_q, void *grad_k,
                                     void *grad_v, void *workspace, hipStream_t stream);
int bevmap_launch_dropout(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, void *y,
                          int64_t rows, int64_t columns, int32_t dtype, int32_t threshold, uint64_t seed,
                          uint64_t offset, hipStream_t stream);

namespace bevmap {
namespace {

// Storage of a bevpool_dtype; conversions from float round to nearest even.
template <int DT>
struct Num;
template <>
struct Num<BEVPOOL_F32> {
    using T = float;
};
template <>
struct Num<BEVPOOL_BF16> {
    using T = __bf16;
};
template <>
struct Num<BEVPOOL_F16> {
    using T = _Float16;
};

template <class T, int N>
struct alignas(sizeof(T) * N > 16 ? 16 : sizeof(T) * N) Pack {
    T v[N];
};

// N consecutive elements, aligned to min(16, their bytes), as fp32.
template <class T, int N>
__device__ __forceinline__ void load_n(const T *p, float *out) {
    const Pack<T, N> q = *reinterpret_cast<const Pack<T, N> *>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = float(q.v[i]);
}

// STREAM: past the caches, for results that are larger than they are. (A constant:
// the compiler joins the two sides of a branch between such stores into a plain one.)
template <class T, int N, bool STREAM = false>
__device__ __forceinline__ void store_n(T *p, const float *in) {
    using Chunk = uint32_t __attribute__((ext_vector_type(4)));
    constexpr int kBytes = int(sizeof(T)) * N;
    Pack<T, N> q;
#pragma unroll
    for (int i = 0; i < N; ++i) q.v[i] = T(in[i]);
    if constexpr (STREAM && kBytes % 16 == 0) {
#pragma unroll
        for (int i = 0; i < kBytes / 16; ++i) {
            Chunk c;
            __builtin_memcpy(&c, reinterpret_cast<const char *>(&q) + 16 * i, 16);
            __builtin_nontemporal_store(c, reinterpret_cast<Chunk *>(p) + i);
        }
    } else {
        *reinterpret_cast<Pack<T, N> *>(p) = q;
    }
}

// The same with the type chosen at run time (uniform over the launch).
template <int N>
__device__ __forceinline__ void load_any(const void *p, int64_t at, int dtype, float *out) {
    if (dtype == BEVPOOL_F32)
        load_n<float, N>(static_cast<const float *>(p) + at, out);
    else if (dtype == BEVPOOL_BF16)
        load_n<__bf16, N>(static_cast<const __bf16 *>(p) + at, out);
    else
        load_n<_Float16, N>(static_cast<const _Float16 *>(p) + at, out);
}

template <int N, bool STREAM = false>
__device__ __forceinline__ void store_any(void *p, int64_t at, int dtype, const float *in) {
    if (dtype == BEVPOOL_F32)
        store_n<float, N, STREAM>(static_cast<float *>(p) + at, in);
    else if (dtype == BEVPOOL_BF16)
        store_n<__bf16, N, STREAM>(static_cast<__bf16 *>(p) + at, in);
    else
        store_n<_Float16, N, STREAM>(static_cast<_Float16 *>(p) + at, in);
}

inline int64_t dtype_bytes(int32_t dtype) { return dtype == BEVPOOL_F32 ? 4 : 2; }

// Whether address and strides (in elements) allow accesses of n elements at a time.
inline bool aligned_for(const void *p, int64_t stride, int32_t dtype, int n) {
    const int64_t bytes = n * dtype_bytes(dtype) > 16 ? 16 : n * dtype_bytes(dtype);
    return reinterpret_cast<uintptr_t>(p) % uintptr_t(bytes) == 0 && stride * dtype_bytes(dtype) % bytes == 0;
}

}  // namespace
}  // namespace bevmap
