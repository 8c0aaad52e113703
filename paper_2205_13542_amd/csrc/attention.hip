// Attention of queries to an encoder's states of another length, and its
// gradients (bevmap_attention, bevmap_attention_backward).
//
// The queries of the heads that share a key head are the rows of one problem:
// row r = query * group + head of the group, against that head's keys. This
// form gives one wave to a row (forward, gradient of q) or to a key (gradients
// of k and v): lanes are keys for the scores and channels for the sums.
#include "mapops.h"

namespace bevmap {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

struct AttendArgs {
    bevmap_attend a;
    const void *q, *k, *v, *dout, *out, *out_low;
    const int32_t *lengths;
    const uint8_t *mask;
    void *o, *o_low, *dq, *dk, *dv;
    float *lse, *delta;
    int32_t group, rows;      // heads that share a key head, queries * group
};

template <int DT>
struct At {
    using T = typename Num<DT>::T;
    const AttendArgs &g;
    int b, hk, len;
    __device__ At(const AttendArgs &g_, int bh) : g(g_) {
        b = bh / g.a.key_heads;
        hk = bh - b * g.a.key_heads;
        len = g.lengths ? min(max(g.lengths[b], 0), g.a.keys) : g.a.keys;
    }
    __device__ bool in_use(int j) const {
        return j < len && (!g.mask || g.mask[b * g.a.mask_batch + j]);
    }
    __device__ const T *q(int r) const {
        const int i = r / g.group, h = hk * g.group + r - i * g.group;
        return static_cast<const T *>(g.q) + b * g.a.q_batch + i * g.a.q_row + h * g.a.q_head;
    }
    __device__ const T *k(int j) const {
        return static_cast<const T *>(g.k) + b * g.a.k_batch + j * g.a.k_row + hk * g.a.k_head;
    }
    __device__ const T *v(int j) const {
        return static_cast<const T *>(g.v) + b * g.a.v_batch + j * g.a.v_row + hk * g.a.v_head;
    }
    __device__ int64_t row(int r) const {      // of out and its like, in elements
        const int i = r / g.group, h = hk * g.group + r - i * g.group;
        return ((int64_t(b) * g.a.queries + i) * g.a.heads + h) * g.a.dim;
    }
    __device__ int64_t stat(int r) const {     // of lse, delta
        const int i = r / g.group, h = hk * g.group + r - i * g.group;
        return (int64_t(b) * g.a.heads + h) * g.a.queries + i;
    }
    __device__ int64_t key(int j) const {      // of the gradients of k and v
        return ((int64_t(b) * g.a.keys + j) * g.a.key_heads + hk) * g.a.dim;
    }
};

__device__ __forceinline__ float wave_sum(float v) {
    for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
    return v;
}
__device__ __forceinline__ float wave_max(float v) {
    for (int m = 1; m < 64; m <<= 1) v = fmaxf(v, __shfl_xor(v, m));
    return v;
}

template <class T>
__device__ __forceinline__ float dot(const float *a, const T *b, int dim) {
    float s = 0.0f;
    for (int c = 0; c < dim; ++c) s = fmaf(a[c], float(b[c]), s);
    return s;
}

template <int DT>
__global__ __launch_bounds__(64) void k_attend(AttendArgs g) {
    using T = typename Num<DT>::T;
    __shared__ float q[128];
    const At<DT> at(g, blockIdx.y);
    const int lane = threadIdx.x, dim = g.a.dim, r = blockIdx.x;
    for (int c = lane; c < dim; c += 64) q[c] = float(at.q(r)[c]);
    __syncthreads();
    const float scale = g.a.scale * kLog2e;
    float top = -INFINITY, sum = 0.0f, o[2] = {0.0f, 0.0f};
    for (int j0 = 0; j0 < at.len; j0 += 64) {
        const int j = j0 + lane;
        const float s = at.in_use(j) ? dot(q, at.k(j), dim) * scale : -INFINITY;
        const float now = fmaxf(top, wave_max(s));
        if (now == -INFINITY) continue;
        const float old = exp2f(top - now), p = exp2f(s - now);
        sum = sum * old + wave_sum(p);
        for (int k = 0; k < 2; ++k) o[k] *= old;
        top = now;
        for (int i = 0; i < 64; ++i) {
            const float pi = __shfl(p, i);
            if (pi == 0.0f) continue;
            for (int k = 0; k < 2; ++k)
                if (lane + 64 * k < dim) o[k] = fmaf(pi, float(at.v(j0 + i)[lane + 64 * k]), o[k]);
        }
    }
    const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
    for (int k = 0; k < 2; ++k) {
        const int c = lane + 64 * k;
        if (c >= dim) continue;
        const float full = o[k] * inv;
        const T rounded = T(full);
        static_cast<T *>(g.o)[at.row(r) + c] = rounded;
        if (DT != BEVPOOL_F32 && g.o_low) static_cast<T *>(g.o_low)[at.row(r) + c] = T(full - float(rounded));
    }
    if (lane == 0 && g.lse) g.lse[at.stat(r)] = sum > 0.0f ? top + log2f(sum) : -INFINITY;
}

template <int DT>
__global__ __launch_bounds__(64) void k_attend_dq(AttendArgs g) {
    using T = typename Num<DT>::T;
    __shared__ float q[128], d[128];
    const At<DT> at(g, blockIdx.y);
    const int lane = threadIdx.x, dim = g.a.dim, r = blockIdx.x;
    float delta = 0.0f;
    for (int c = lane; c < dim; c += 64) {
        q[c] = float(at.q(r)[c]);
        d[c] = float(static_cast<const T *>(g.dout)[at.row(r) + c]);
        float o = float(static_cast<const T *>(g.out)[at.row(r) + c]);
        if (DT != BEVPOOL_F32 && g.out_low) o += float(static_cast<const T *>(g.out_low)[at.row(r) + c]);
        delta = fmaf(d[c], o, delta);
    }
    delta = wave_sum(delta);
    if (lane == 0) g.delta[at.stat(r)] = delta;
    __syncthreads();
    const float scale = g.a.scale * kLog2e, lse = g.lse[at.stat(r)];
    float acc[2] = {0.0f, 0.0f};
    for (int j0 = 0; j0 < at.len; j0 += 64) {
        const int j = j0 + lane;
        float ds = 0.0f;
        if (at.in_use(j)) {
            const float p = exp2f(dot(q, at.k(j), dim) * scale - lse);
            ds = p * (dot(d, at.v(j), dim) - delta) * g.a.scale;
        }
        for (int i = 0; i < 64; ++i) {
            const float di = __shfl(ds, i);
            if (di == 0.0f) continue;
            for (int k = 0; k < 2; ++k)
                if (lane + 64 * k < dim) acc[k] = fmaf(di, float(at.k(j0 + i)[lane + 64 * k]), acc[k]);
        }
    }
    for (int k = 0; k < 2; ++k)
        if (lane + 64 * k < dim) static_cast<T *>(g.dq)[at.row(r) + lane + 64 * k] = T(acc[k]);
}

template <int DT>
__global__ __launch_bounds__(64) void k_attend_dkv(AttendArgs g) {
    using T = typename Num<DT>::T;
    __shared__ float key[128], val[128];
    const At<DT> at(g, blockIdx.y);
    const int lane = threadIdx.x, dim = g.a.dim, j = blockIdx.x;
    const bool used = at.in_use(j);
    float dk[2] = {0.0f, 0.0f}, dv[2] = {0.0f, 0.0f};
    for (int c = lane; c < dim && used; c += 64) {
        key[c] = float(at.k(j)[c]);
        val[c] = float(at.v(j)[c]);
    }
    __syncthreads();
    const float scale = g.a.scale * kLog2e;
    for (int r0 = 0; r0 < g.rows && used; r0 += 64) {
        const int r = r0 + lane;
        float p = 0.0f, ds = 0.0f;
        if (r < g.rows) {
            p = exp2f(dot(key, at.q(r), dim) * scale - g.lse[at.stat(r)]);
            ds = p * (dot(val, static_cast<const T *>(g.dout) + at.row(r), dim) - g.delta[at.stat(r)]) * g.a.scale;
        }
        for (int i = 0; i < min(64, g.rows - r0); ++i) {
            const float pi = __shfl(p, i), di = __shfl(ds, i);
            for (int k = 0; k < 2; ++k)
                if (lane + 64 * k < dim) {
                    dv[k] = fmaf(pi, float(static_cast<const T *>(g.dout)[at.row(r0 + i) + lane + 64 * k]), dv[k]);
                    dk[k] = fmaf(di, float(at.q(r0 + i)[lane + 64 * k]), dk[k]);
                }
        }
    }
    for (int k = 0; k < 2; ++k)
        if (lane + 64 * k < dim) {
            static_cast<T *>(g.dk)[at.key(j) + lane + 64 * k] = T(dk[k]);
            static_cast<T *>(g.dv)[at.key(j) + lane + 64 * k] = T(dv[k]);
        }
}

AttendArgs fill(const bevmap_attend &a, const void *q, const void *k, const void *v, const int32_t *lengths,
                const uint8_t *mask) {
    AttendArgs g{};
    g.a = a;
    g.q = q;
    g.k = k;
    g.v = v;
    g.lengths = lengths;
    g.mask = mask;
    g.group = a.heads / a.key_heads;
    g.rows = a.queries * g.group;
    return g;
}

template <int DT>
int forward(const AttendArgs &g, hipStream_t stream) {
    if (g.rows > 0)
        hipLaunchKernelGGL((k_attend<DT>), dim3(g.rows, g.a.batch * g.a.key_heads), dim3(64), 0, stream, g);
    BEVPOOL_HIP(hipGetLastError());
    return BEVPOOL_OK;
}

template <int DT>
int backward(const AttendArgs &g, hipStream_t stream) {
    const uint32_t bh = g.a.batch * g.a.key_heads;
    if (g.rows > 0) hipLaunchKernelGGL((k_attend_dq<DT>), dim3(g.rows, bh), dim3(64), 0, stream, g);
    BEVPOOL_HIP(hipGetLastError());
    if (g.a.keys > 0) hipLaunchKernelGGL((k_attend_dkv<DT>), dim3(g.a.keys, bh), dim3(64), 0, stream, g);
    BEVPOOL_HIP(hipGetLastError());
    return BEVPOOL_OK;
}

}  // namespace
}  // namespace bevmap

using namespace bevmap;

int64_t bevmap_attention_workspace_bytes(const bevmap_attend &a, bool backward) {
    return backward ? int64_t(a.batch) * a.queries * a.heads * int64_t(sizeof(float)) : 0;
}

int bevmap_launch_attention(const bevmap_attend &a, const void *q, const void *k, const void *v,
                            const int32_t *lengths, const uint8_t *mask, void *out, void *out_low, float *lse,
                            void *, hipStream_t stream) {
    AttendArgs g = fill(a, q, k, v, lengths, mask);
    g.o = out;
    g.o_low = out_low;
    g.lse = lse;
    if (a.batch == 0) return BEVPOOL_OK;
    switch (a.dtype) {
        case BEVPOOL_F32: return forward<BEVPOOL_F32>(g, stream);
        case BEVPOOL_BF16: return forward<BEVPOOL_BF16>(g, stream);
        default: return forward<BEVPOOL_F16>(g, stream);
    }
}

int bevmap_launch_attention_backward(const bevmap_attend &a, const void *grad_out, const void *q, const void *k,
                                     const void *v, const int32_t *lengths, const uint8_t *mask, const void *out,
                                     const void *out_low, const float *lse, void *grad_q, void *grad_k,
                                     void *grad_v, void *workspace, hipStream_t stream) {
    AttendArgs g = fill(a, q, k, v, lengths, mask);
    g.dout = grad_out;
    g.out = out;
    g.out_low = out_low;
    g.lse = const_cast<float *>(lse);
    g.dq = grad_q;
    g.dk = grad_k;
    g.dv = grad_v;
    g.delta = static_cast<float *>(workspace);
    if (a.batch == 0) return BEVPOOL_OK;
    switch (a.dtype) {
        case BEVPOOL_F32: return backward<BEVPOOL_F32>(g, stream);
        case BEVPOOL_BF16: return backward<BEVPOOL_BF16>(g, stream);
        default: return backward<BEVPOOL_F16>(g, stream);
    }
}
