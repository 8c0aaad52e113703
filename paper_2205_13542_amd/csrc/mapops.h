// Declarations and device helpers shared by the map operators (include/bevmap.h):
// norm.hip, attention.hip, dropout.hip, rms_norm.hip, rotary.hip, gated.hip and
// linear_int8.hip launch, mapops.hip and layerops.hip check.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "bevmap.h"
#include "internal.h"

// Limits that the kernels assume.
constexpr int kNormMaxChannels = 8192;  // two floats a channel in LDS; a row in a workgroup's registers
constexpr int kInt8MaxChannels = 131071;        // 128 * 128 * this stays below 2^31
constexpr int kTurnMaxDim = 4096;
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
// q, scale: the result in 8 bits, instead of y and rstd.
int bevmap_launch_rms_norm(const bevmap_rms &n, const void *x, const void *residual, const void *weight, void *sum,
                           void *y, float *rstd, int8_t *q, float *scale, hipStream_t stream);
int64_t bevmap_rms_workspace_bytes(const bevmap_rms &n);
int bevmap_launch_rms_norm_backward(const bevmap_rms &n, const void *grad_y, const void *grad_sum, const void *x,
                                    const void *residual, const void *weight, const float *rstd, void *grad_x,
                                    void *grad_weight, void *workspace, hipStream_t stream);
int bevmap_launch_quantize(const void *x, int64_t x_stride, int8_t *q, float *scale, int64_t rows, int32_t columns,
                           int32_t dtype, hipStream_t stream);
int bevmap_launch_linear_int8(const bevmap_linear &n, const int8_t *x, const float *x_scale, const int8_t *w,
                              const float *w_scale, const float *bias, void *y, hipStream_t stream);
int bevmap_launch_rotary(const bevmap_turn &n, const void *x, const void *positions, const double *frequencies,
                         void *out, bool backward, hipStream_t stream);
int bevmap_launch_gate(const bevmap_gate &n, const void *x, void *y, int8_t *q, uint8_t *e, hipStream_t stream);
int bevmap_launch_gate_backward(const bevmap_gate &n, const void *grad_y, const void *x, const int8_t *q,
                                const uint8_t *e, void *grad_x, hipStream_t stream);

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

// How rows lie. kUneven: their length is no multiple of N, or their addresses are not aligned to
// it. They are read and written 16 bytes at a time all the same, at the alignment of an
// element (100003 rows of 331 bf16 numbers one by one: a norm with a residual took 106 us,
// 8-bit integers from it 97). At c elements into a row that has `count` more, an access of less
// than N is the row's last 16 bytes, moved down by those before c; what lies behind the row
// is 0. It is written in pieces of 8, 4, 2 and 1 bytes. kShort: some row has less than N
// elements, and its end is read one by one. (No branch in the second: loads that follow each
// other are on their way together.)
enum { kEven, kUneven, kShort };
__device__ __forceinline__ void move_down(uint64_t (&v)[2], int bits) {     // by less than 128
    const uint64_t low = v[0] >> (bits & 63) | (v[1] << 1) << (63 - (bits & 63)), high = v[1] >> (bits & 63);
    v[0] = bits < 64 ? low : high;
    v[1] = bits < 64 ? high : 0;
}
template <class T, int N, int ROWS>
__device__ __forceinline__ void load_raw_part(const T *p, int count, T (&out)[N]) {
    static_assert(sizeof(T) * N <= 16 && sizeof(T) * N >= 4, "");
    constexpr int kBytes = sizeof(T) * N;
    if (ROWS == kUneven || count >= N) {
        const int back = count >= N ? 0 : N - count;
        uint64_t v[2] = {0, 0};
        __builtin_memcpy(v, p - back, kBytes);
        move_down(v, back * int(sizeof(T)) * 8);
        __builtin_memcpy(out, v, kBytes);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = T(0);
        for (int i = 0; i < count; ++i) {
            const T one = p[i];
#pragma unroll
            for (int k = 0; k < N; ++k) out[k] = k == i ? one : out[k];
        }
    }
}
template <class T, int N>
__device__ __forceinline__ void store_raw_part(T *p, int count, const T (&in)[N]) {
    constexpr int kBytes = sizeof(T) * N;
    if (count >= N) {
        __builtin_memcpy(p, in, kBytes);
        return;
    }
    uint64_t v[2] = {0, 0};
    __builtin_memcpy(v, in, kBytes);
    char *to = reinterpret_cast<char *>(p);
    const int bytes = count * int(sizeof(T));
    if (kBytes > 8 && bytes & 8) {
        __builtin_memcpy(to, v, 8);
        to += 8;
        v[0] = v[1];
    }
    if (kBytes > 4 && bytes & 4) {
        __builtin_memcpy(to, v, 4);
        to += 4;
        v[0] >>= 32;
    }
    if (sizeof(T) < 4 && bytes & 2) {
        __builtin_memcpy(to, v, 2);
        to += 2;
        v[0] >>= 16;
    }
    if (sizeof(T) < 2 && bytes & 1) __builtin_memcpy(to, v, 1);
}
template <class T, int N, int ROWS>
__device__ __forceinline__ void load_part(const T *p, int count, float *out) {
    if constexpr (ROWS == kEven) {
        load_n<T, N>(p, out);
    } else if constexpr (sizeof(T) * N > 16) {      // fp32 beside a 16-bit type: two accesses
        const bool more = count > N / 2;            // else the second is the first again, as zeros
        load_part<T, N / 2, ROWS>(p, count, out);
        load_part<T, N / 2, ROWS>(more ? p + N / 2 : p, more ? count - N / 2 : count, out + N / 2);
#pragma unroll
        for (int i = N / 2; i < N; ++i) out[i] = more ? out[i] : 0.0f;
    } else {
        T q[N];
        load_raw_part<T, N, ROWS>(p, count, q);
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = float(q[i]);
    }
}
template <class T, int N, int ROWS, bool STREAM = false>
__device__ __forceinline__ void store_part(T *p, int count, const float *in) {
    if constexpr (ROWS == kEven) {
        store_n<T, N, STREAM>(p, in);
    } else if constexpr (sizeof(T) * N > 16) {
        store_part<T, N / 2, ROWS>(p, count, in);
        if (count > N / 2) store_part<T, N / 2, ROWS>(p + N / 2, count - N / 2, in + N / 2);
    } else {
        T q[N];
#pragma unroll
        for (int i = 0; i < N; ++i) q[i] = T(in[i]);
        store_raw_part<T, N>(p, count, q);
    }
}
template <int N, int ROWS>
__device__ __forceinline__ void load_any_part(const void *p, int64_t at, int dtype, int count, float *out) {
    if (dtype == BEVPOOL_F32)
        load_part<float, N, ROWS>(static_cast<const float *>(p) + at, count, out);
    else if (dtype == BEVPOOL_BF16)
        load_part<__bf16, N, ROWS>(static_cast<const __bf16 *>(p) + at, count, out);
    else
        load_part<_Float16, N, ROWS>(static_cast<const _Float16 *>(p) + at, count, out);
}
template <int N, int ROWS, bool STREAM = false>
__device__ __forceinline__ void store_any_part(void *p, int64_t at, int dtype, int count, const float *in) {
    if (dtype == BEVPOOL_F32)
        store_part<float, N, ROWS, STREAM>(static_cast<float *>(p) + at, count, in);
    else if (dtype == BEVPOOL_BF16)
        store_part<__bf16, N, ROWS, STREAM>(static_cast<__bf16 *>(p) + at, count, in);
    else
        store_part<_Float16, N, ROWS, STREAM>(static_cast<_Float16 *>(p) + at, count, in);
}
// The same of 8-bit integers.
template <int N, int ROWS>
__device__ __forceinline__ void load_bytes(const int8_t *p, int count, int8_t (&out)[N]) {
    if constexpr (ROWS == kEven) __builtin_memcpy(out, __builtin_assume_aligned(p, N), N);
    else load_raw_part<int8_t, N, ROWS>(p, count, out);
}
template <int N, int ROWS>
__device__ __forceinline__ void store_bytes(int8_t *p, int count, const int8_t (&in)[N]) {
    if constexpr (ROWS == kEven) __builtin_memcpy(__builtin_assume_aligned(p, N), in, N);
    else store_raw_part<int8_t, N>(p, count, in);
}

// Elements of an access: what 16 bytes hold.
template <int DT>
constexpr int kWide = DT == BEVPOOL_F32 ? 4 : 8;

inline int64_t dtype_bytes(int32_t dtype) { return dtype == BEVPOOL_F32 ? 4 : 2; }

// Launches with a type and how rows lie as constants: body(type, rows).
template <int V>
struct Int {
    static constexpr int value = V;
};
template <class F>
void with_type_and_rows(int32_t dtype, int rows, F body) {
    auto go = [&](auto dt) {
        if (rows == kEven) body(dt, Int<kEven>());
        else if (rows == kUneven) body(dt, Int<kUneven>());
        else body(dt, Int<kShort>());
    };
    if (dtype == BEVPOOL_F32) go(Int<BEVPOOL_F32>());
    else if (dtype == BEVPOOL_BF16) go(Int<BEVPOOL_BF16>());
    else go(Int<BEVPOOL_F16>());
}

// Whether results of so many bytes go past the caches: more than half of what the XCDs' L2s
// hold together, of which little would be left for who reads them, and reads then share
// the caches with nothing (steps of a norm of 518400 x 80 169 -> 151 us, of a gated activation
// of 129600 x 640 120 -> 106; a turn of 8192 x 16 x 128 16.1 -> 12.5).
inline bool past_caches(int64_t bytes) { return bytes > (int64_t(16) << 20); }

// Whether address and strides (in elements) allow accesses of n elements at a time.
inline bool aligned_for(const void *p, int64_t stride, int32_t dtype, int n) {
    const int64_t bytes = n * dtype_bytes(dtype) > 16 ? 16 : n * dtype_bytes(dtype);
    return reinterpret_cast<uintptr_t>(p) % uintptr_t(bytes) == 0 && stride * dtype_bytes(dtype) % bytes == 0;
}

}  // namespace
}  // namespace bevmap
