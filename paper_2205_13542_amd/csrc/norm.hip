// Group norm with an activation, channels last, and its gradients
// (bevmap_group_norm, bevmap_group_norm_backward).
//
// Both directions are two passes over the frame, a sum and an apply, and are
// bound by memory. In the sum pass a workgroup takes a chunk of rows of one frame;
// a thread keeps to V neighbouring channels and walks the chunk's rows, so that a
// wave reads whole stretches of rows whatever a group's width, and forms its
// channels' statistics in registers. Statistics travel as (mean, sum of squared
// deviations) and are joined by
//   mean = sum n_i mean_i / n,  M2 = sum M2_i + sum n_i (mean_i - mean)^2,
// so a large common offset costs no precision. A small kernel between the passes
// joins the chunks of each frame and group (and the weights' gradients): joined by
// each workgroup of the apply pass instead, the parts' latency stood in front of
// every one of them (360x360x80 fp32 to bf16: 33 us, now 28). The apply pass runs
// back to front, and the results of maps beyond the cache go past it, so that part of
// what it reads is still there.
// Eight frames of 360x360x80 in bf16 take 33 + 56 us forward and 80-84 + 94 backward: the
// 1.33 GB that two passes move, at 4.8 TB/s, what a large copy reaches.
#include "mapops.h"

namespace bevmap {
namespace {

constexpr int kNormBlock = 256;     // apply passes
constexpr int kSumBlock = kNormBlock;   // sum passes
constexpr int kJoinBlock = 256;
constexpr int kSumRows = 4;         // rows that a thread has in flight, in k_norm_sum
constexpr int kNormRows = 2;        // and elsewhere
constexpr int kMergeLanes = 16;     // lanes that join one group's channels
constexpr int kWgradChannels = 16;  // channels of a workgroup that sums weight gradients

struct NormArgs {
    const void *x, *dy, *weight, *bias;
    void *y, *dx, *dweight, *dbias;
    float *mean, *rstd;             // [B][G]
    float2 *parts;                  // [B][chunks][G]
    float2 *moments;                // backward: [B][G]
    float *channel_sums;            // backward: [B][chunks][2][C]
    int64_t ldx;
    int32_t batch, rows, C, G, per; // per: channels of a group
    int32_t chunk, n_chunks;        // rows of a chunk, chunks of a frame
    int32_t apply_rows, n_apply;    // the same for the apply pass
    int32_t y_dtype, w_dtype, act;
    bool stream;                    // results past the caches
    float eps;
};

template <int ACT>
__device__ __forceinline__ float activate(float z) {
    if constexpr (ACT == BEVMAP_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if constexpr (ACT == BEVMAP_ACT_SILU) return z * __builtin_amdgcn_rcpf(1.0f + __expf(-z));
    if constexpr (ACT == BEVMAP_ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678f));
    return z;
}

template <int ACT>
__device__ __forceinline__ float slope(float z) {
    if constexpr (ACT == BEVMAP_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if constexpr (ACT == BEVMAP_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.0f + __expf(-z));
        return s * (1.0f + z * (1.0f - s));
    }
    if constexpr (ACT == BEVMAP_ACT_GELU)
        return 0.5f * (1.0f + erff(z * 0.70710678f)) + z * __expf(-0.5f * z * z) * 0.39894228f;
    return 1.0f;
}

// body(constant) with the activation as a constant: one uniform branch for a batch
// of rows instead of one for an element.
template <int V>
struct Constant {
    static constexpr int value = V;
};
template <class F>
__device__ __forceinline__ void with_act(int act, F body) {
    switch (act) {
        case BEVMAP_ACT_RELU: body(Constant<BEVMAP_ACT_RELU>()); break;
        case BEVMAP_ACT_SILU: body(Constant<BEVMAP_ACT_SILU>()); break;
        case BEVMAP_ACT_GELU: body(Constant<BEVMAP_ACT_GELU>()); break;
        default: body(Constant<BEVMAP_ACT_NONE>()); break;
    }
}

__device__ __forceinline__ float weight_at(const void *w, int c, int dtype, float none) {
    float v = none;
    if (w) load_any<1>(w, c, dtype, &v);
    return v;
}

__device__ __forceinline__ float lane_sum(float v) {     // over kMergeLanes lanes
#pragma unroll
    for (int m = 1; m < kMergeLanes; m <<= 1) v += __shfl_xor(v, m);
    return v;
}

// Columns of a block of vectors: thread -> (row lane, vector).
struct Columns {
    int vectors, lanes;   // vectors of this block, row lanes that walk it
    int lane, vec;        // of this thread; lane >= lanes: idle
};
template <int BLOCK>
__device__ __forceinline__ Columns columns(int first, int n_vec) {
    Columns c;
    c.vectors = min(BLOCK, n_vec - first);
    c.lanes = BLOCK / c.vectors;
    c.lane = threadIdx.x / c.vectors;
    c.vec = first + threadIdx.x - c.lane * c.vectors;
    return c;
}

// Sums v over the row lanes, in halves; every lane gets the sums. th: a float for each
// thread's channels, free on entry and exit.
template <int V>
__device__ __forceinline__ void add_lanes(const Columns &c, int first, int width, float *v, float *th) {
    float *mine = th + c.lane * width + (c.vec - first) * V;
    if (c.lane < c.lanes)
#pragma unroll
        for (int i = 0; i < V; ++i) mine[i] = v[i];
    for (int n = c.lanes; n > 1; n = (n + 1) / 2) {
        const int half = (n + 1) / 2;
        __syncthreads();
        if (c.lane < n - half)
#pragma unroll
            for (int i = 0; i < V; ++i) mine[i] += mine[half * width + i];
    }
    __syncthreads();
    if (c.lane < c.lanes)
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = th[(c.vec - first) * V + i];
    __syncthreads();
}

// Statistics of a chunk of rows: parts[b][chunk][g] = (mean, M2).
template <int DT, int V>
__global__ __launch_bounds__(kSumBlock) void k_norm_sum(NormArgs a) {
    using T = typename Num<DT>::T;
    extern __shared__ float lds[];
    float *ch_mean = lds, *ch_m2 = lds + a.C;             // [C] each
    float *th = lds + 2 * a.C;                            // [lanes][V * vectors]
    const int b = blockIdx.y, r0 = blockIdx.x * a.chunk, r1 = min(r0 + a.chunk, a.rows);
    const int n_vec = a.C / V;
    const T *x = static_cast<const T *>(a.x) + int64_t(b) * a.rows * a.ldx;
    for (int first = 0; first < n_vec; first += kSumBlock) {
        const Columns c = columns<kSumBlock>(first, n_vec);
        float mean[V], m2[V];
#pragma unroll
        for (int i = 0; i < V; ++i) mean[i] = m2[i] = 0.0f;
        int n = 0;
        if (c.lane < c.lanes) {
            const T *p = x + c.vec * V;
            for (int r = r0 + c.lane; r < r1; r += kSumRows * c.lanes) {
                float v[kSumRows][V];
                int more = 0;                             // rows of this batch
#pragma unroll
                for (int k = 0; k < kSumRows; ++k) {
#pragma unroll
                    for (int i = 0; i < V; ++i) v[k][i] = 0.0f;
                    if (r + k * c.lanes < r1) {
                        load_n<T, V>(p + int64_t(r + k * c.lanes) * a.ldx, v[k]);
                        ++more;
                    }
                }
                // join them to the n rows before
                const float inv = 1.0f / float(more), share = float(more) / float(n + more), both = float(n) * share;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float m = 0.0f, q = 0.0f;
#pragma unroll
                    for (int k = 0; k < kSumRows; ++k) m += v[k][i];
                    m *= inv;
#pragma unroll
                    for (int k = 0; k < kSumRows; ++k) {
                        const float d = k < more ? v[k][i] - m : 0.0f;
                        q = fmaf(d, d, q);
                    }
                    const float d = m - mean[i];
                    mean[i] = fmaf(d, share, mean[i]);
                    m2[i] += fmaf(d * d, both, q);
                }
                n += more;
            }
        }
        const int width = c.vectors * V;                  // channels of this block of columns
        // join the row lanes: lane l walked ceil((rows - l) / lanes) rows
        const float rows = float(r1 - r0), mine = c.lane < c.lanes ? float(n) : 0.0f;
        float total[V];
#pragma unroll
        for (int i = 0; i < V; ++i) total[i] = mean[i] * mine;
        add_lanes<V>(c, first, width, total, th);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            total[i] /= rows;
            const float d = mean[i] - total[i];
            m2[i] = mine > 0.0f ? fmaf(d * d, mine, m2[i]) : 0.0f;
        }
        if (c.lane == 0)
#pragma unroll
            for (int i = 0; i < V; ++i) ch_mean[c.vec * V + i] = total[i];
        add_lanes<V>(c, first, width, m2, th);
        if (c.lane == 0)
#pragma unroll
            for (int i = 0; i < V; ++i) ch_m2[c.vec * V + i] = m2[i];
        __syncthreads();
    }
    // join a group's channels, all of equal counts
    const int lane = threadIdx.x % kMergeLanes;
    for (int g0 = 0; g0 < a.G; g0 += kSumBlock / kMergeLanes) {
        const int g = g0 + threadIdx.x / kMergeLanes;
        float m = 0.0f, q = 0.0f;
        if (g < a.G)
            for (int c = lane; c < a.per; c += kMergeLanes) m += ch_mean[g * a.per + c];
        m = lane_sum(m) / float(a.per);
        if (g < a.G)
            for (int c = lane; c < a.per; c += kMergeLanes) {
                const float d = ch_mean[g * a.per + c] - m;
                q += ch_m2[g * a.per + c] + d * d * float(r1 - r0);
            }
        q = lane_sum(q);
        if (g < a.G && lane == 0) a.parts[(int64_t(b) * a.n_chunks + blockIdx.x) * a.G + g] = make_float2(m, q);
    }
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
    return v;
}

// Joins the chunks of a frame's group, a wave to a group: mean and rstd. A lane
// keeps its first kJoin parts in registers, all of them on the way at once.
constexpr int kJoin = 16;
__global__ __launch_bounds__(64) void k_norm_join(NormArgs a) {
    const int g = blockIdx.x, b = blockIdx.y, lane = threadIdx.x;
    const float2 *parts = a.parts + int64_t(b) * a.n_chunks * a.G + g;
    const float total = float(a.rows);
    auto rows_of = [&](int k) { return float(min(a.chunk, a.rows - k * a.chunk)); };
    float2 p[kJoin];
#pragma unroll
    for (int i = 0; i < kJoin; ++i) {
        const int k = lane + 64 * i;
        p[i] = k < a.n_chunks ? parts[int64_t(k) * a.G] : make_float2(0.0f, 0.0f);
    }
    float m = 0.0f, q = 0.0f;
#pragma unroll
    for (int i = 0; i < kJoin; ++i)
        if (lane + 64 * i < a.n_chunks) m = fmaf(p[i].x, rows_of(lane + 64 * i), m);
    m = wave_sum(m) / total;
#pragma unroll
    for (int i = 0; i < kJoin; ++i)
        if (lane + 64 * i < a.n_chunks) {
            const float d = p[i].x - m;
            q += fmaf(d * d, rows_of(lane + 64 * i) * float(a.per), p[i].y);
        }
    q = wave_sum(q);
    if (lane == 0) {
        a.mean[int64_t(b) * a.G + g] = m;
        a.rstd[int64_t(b) * a.G + g] = 1.0f / sqrtf(q / (total * float(a.per)) + a.eps);
    }
}

template <int DT, int V, bool STREAM>
__global__ __launch_bounds__(kNormBlock) void k_norm_apply(NormArgs a) {
    using T = typename Num<DT>::T;
    // back to front: what the sum pass read last is still in cache
    const int b = gridDim.y - 1 - blockIdx.y;
    const int r0 = (a.n_apply - 1 - blockIdx.x) * a.apply_rows, r1 = min(r0 + a.apply_rows, a.rows);
    const float *mean = a.mean + int64_t(b) * a.G, *rstd = a.rstd + int64_t(b) * a.G;
    const int n_vec = a.C / V;
    const T *x = static_cast<const T *>(a.x) + int64_t(b) * a.rows * a.ldx;
    const int64_t out0 = int64_t(b) * a.rows * a.C;
    for (int first = 0; first < n_vec; first += kNormBlock) {
        const Columns c = columns<kNormBlock>(first, n_vec);
        if (c.lane >= c.lanes) continue;
        float mu[V], mul[V], add[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int ch = c.vec * V + i, g = ch / a.per;
            mu[i] = mean[g];
            mul[i] = rstd[g] * weight_at(a.weight, ch, a.w_dtype, 1.0f);
            add[i] = weight_at(a.bias, ch, a.w_dtype, 0.0f);
        }
        for (int r = r0 + c.lane; r < r1; r += kNormRows * c.lanes) {
            float v[kNormRows][V];
#pragma unroll
            for (int k = 0; k < kNormRows; ++k)
                if (r + k * c.lanes < r1) load_n<T, V>(x + int64_t(r + k * c.lanes) * a.ldx + c.vec * V, v[k]);
            with_act(a.act, [&](auto act) {
#pragma unroll
                for (int k = 0; k < kNormRows; ++k) {
                    if (r + k * c.lanes >= r1) break;
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        v[k][i] = activate<act.value>(fmaf(v[k][i] - mu[i], mul[i], add[i]));
                    store_any<V, STREAM>(a.y, out0 + int64_t(r + k * c.lanes) * a.C + c.vec * V, a.y_dtype, v[k]);
                }
            });
        }
    }
}

// Per channel sums over a chunk of dz and dz * xh, with dz = dy act'(z); and per
// group those sums with the channels' weights: parts = (sum e, sum e xh), e = dz w.
template <int DT, int V>
__global__ __launch_bounds__(kSumBlock) void k_norm_grad_sum(NormArgs a) {
    using T = typename Num<DT>::T;
    extern __shared__ float lds[];
    float *ch_sum = lds, *ch_dot = lds + a.C;
    float *th = lds + 2 * a.C;
    const int b = blockIdx.y, r0 = blockIdx.x * a.chunk, r1 = min(r0 + a.chunk, a.rows);
    const int n_vec = a.C / V;
    const T *x = static_cast<const T *>(a.x) + int64_t(b) * a.rows * a.ldx;
    const int64_t dy0 = int64_t(b) * a.rows * a.C;
    float *sums = a.channel_sums + (int64_t(b) * a.n_chunks + blockIdx.x) * 2 * a.C;
    for (int first = 0; first < n_vec; first += kSumBlock) {
        const Columns c = columns<kSumBlock>(first, n_vec);
        const int width = c.vectors * V;
        float w[V], sum[V], dot[V];
#pragma unroll
        for (int i = 0; i < V; ++i) w[i] = sum[i] = dot[i] = 0.0f;
        if (c.lane < c.lanes) {
            float mu[V], rs[V], add[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int ch = c.vec * V + i, g = ch / a.per;
                mu[i] = a.mean[int64_t(b) * a.G + g];
                rs[i] = a.rstd[int64_t(b) * a.G + g];
                w[i] = weight_at(a.weight, ch, a.w_dtype, 1.0f);
                add[i] = weight_at(a.bias, ch, a.w_dtype, 0.0f);
            }
            for (int r = r0 + c.lane; r < r1; r += kNormRows * c.lanes) {
                float v[kNormRows][V], d[kNormRows][V];
#pragma unroll
                for (int k = 0; k < kNormRows; ++k)
                    if (r + k * c.lanes < r1) {
                        load_n<T, V>(x + int64_t(r + k * c.lanes) * a.ldx + c.vec * V, v[k]);
                        load_any<V>(a.dy, dy0 + int64_t(r + k * c.lanes) * a.C + c.vec * V, a.y_dtype, d[k]);
                    }
                with_act(a.act, [&](auto act) {
#pragma unroll
                    for (int k = 0; k < kNormRows; ++k) {
                        if (r + k * c.lanes >= r1) break;
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            const float xh = (v[k][i] - mu[i]) * rs[i];
                            const float dz = d[k][i] * slope<act.value>(fmaf(xh, w[i], add[i]));
                            sum[i] += dz;
                            dot[i] = fmaf(dz, xh, dot[i]);
                        }
                    }
                });
            }
        }
        add_lanes<V>(c, first, width, sum, th);
        add_lanes<V>(c, first, width, dot, th);
        if (c.lane == 0)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int ch = c.vec * V + i;
                sums[ch] = sum[i];
                sums[a.C + ch] = dot[i];
                ch_sum[ch] = sum[i] * w[i];
                ch_dot[ch] = dot[i] * w[i];
            }
        __syncthreads();
    }
    const int lane = threadIdx.x % kMergeLanes;
    for (int g0 = 0; g0 < a.G; g0 += kSumBlock / kMergeLanes) {
        const int g = g0 + threadIdx.x / kMergeLanes;
        float s = 0.0f, d = 0.0f;
        if (g < a.G)
            for (int c = lane; c < a.per; c += kMergeLanes) {
                s += ch_sum[g * a.per + c];
                d += ch_dot[g * a.per + c];
            }
        s = lane_sum(s);
        d = lane_sum(d);
        if (g < a.G && lane == 0) a.parts[(int64_t(b) * a.n_chunks + blockIdx.x) * a.G + g] = make_float2(s, d);
    }
}

// Weight gradients of kWgradChannels channels: the chunks' sums of all frames.
__device__ __forceinline__ void weight_gradients(const NormArgs &a, int block, float *lds) {
    const int ch = block * kWgradChannels + threadIdx.x % kWgradChannels;
    const int lane = threadIdx.x / kWgradChannels, lanes = kJoinBlock / kWgradChannels;
    const int64_t n = int64_t(a.batch) * a.n_chunks;
    float s = 0.0f, d = 0.0f;
    if (ch < a.C)
#pragma unroll 8
        for (int64_t k = lane; k < n; k += lanes) {
            s += a.channel_sums[k * 2 * a.C + ch];
            d += a.channel_sums[k * 2 * a.C + a.C + ch];
        }
    lds[threadIdx.x] = s;
    lds[kJoinBlock + threadIdx.x] = d;
    __syncthreads();
    if (lane == 0 && ch < a.C) {
        s = d = 0.0f;
        for (int l = 0; l < lanes; ++l) {
            s += lds[l * kWgradChannels + threadIdx.x];
            d += lds[kJoinBlock + l * kWgradChannels + threadIdx.x];
        }
        if (a.dbias) store_any<1>(a.dbias, ch, a.w_dtype, &s);
        if (a.dweight) store_any<1>(a.dweight, ch, a.w_dtype, &d);
    }
}

// Joins the chunks: per frame and group, a wave to a group, the means of e and e xh
// (to moments [B][G]); and, in the grid's columns from n_join on, the weight
// gradients.
__global__ __launch_bounds__(kJoinBlock) void k_norm_grad_join(NormArgs a, int n_join) {
    __shared__ float lds[2 * kJoinBlock];
    if (int(blockIdx.x) >= n_join) {
        if (blockIdx.y == 0) weight_gradients(a, blockIdx.x - n_join, lds);
        return;
    }
    const int g = blockIdx.x * (kJoinBlock / 64) + threadIdx.x / 64, b = blockIdx.y, lane = threadIdx.x & 63;
    if (g >= a.G) return;
    const float2 *parts = a.parts + int64_t(b) * a.n_chunks * a.G + g;
    float s = 0.0f, d = 0.0f;
#pragma unroll 16
    for (int k = lane; k < a.n_chunks; k += 64) {
        const float2 p = parts[int64_t(k) * a.G];
        s += p.x;
        d += p.y;
    }
    s = wave_sum(s);
    d = wave_sum(d);
    const float inv = 1.0f / (float(a.rows) * float(a.per));
    if (lane == 0) a.moments[int64_t(b) * a.G + g] = make_float2(s * inv, d * inv);
}

// dx = rstd (e - mean(e) - xh mean(e xh)).
template <int DT, int V, bool STREAM>
__global__ __launch_bounds__(kNormBlock) void k_norm_grad_apply(NormArgs a) {
    using T = typename Num<DT>::T;
    const int b = gridDim.y - 1 - blockIdx.y;      // back to front, as k_norm_apply
    const int r0 = (a.n_apply - 1 - blockIdx.x) * a.apply_rows, r1 = min(r0 + a.apply_rows, a.rows);
    const int n_vec = a.C / V;
    const T *x = static_cast<const T *>(a.x) + int64_t(b) * a.rows * a.ldx;
    T *dx = static_cast<T *>(a.dx) + int64_t(b) * a.rows * a.C;
    const int64_t dy0 = int64_t(b) * a.rows * a.C;
    for (int first = 0; first < n_vec; first += kNormBlock) {
        const Columns c = columns<kNormBlock>(first, n_vec);
        if (c.lane >= c.lanes) continue;
        float mu[V], rs[V], w[V], add[V], e1[V], e2[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int ch = c.vec * V + i, g = ch / a.per;
            mu[i] = a.mean[int64_t(b) * a.G + g];
            rs[i] = a.rstd[int64_t(b) * a.G + g];
            w[i] = weight_at(a.weight, ch, a.w_dtype, 1.0f);
            add[i] = weight_at(a.bias, ch, a.w_dtype, 0.0f);
            const float2 m = a.moments[int64_t(b) * a.G + g];
            e1[i] = m.x;
            e2[i] = m.y;
        }
        for (int r = r0 + c.lane; r < r1; r += kNormRows * c.lanes) {
            float v[kNormRows][V], d[kNormRows][V];
#pragma unroll
            for (int k = 0; k < kNormRows; ++k)
                if (r + k * c.lanes < r1) {
                    load_n<T, V>(x + int64_t(r + k * c.lanes) * a.ldx + c.vec * V, v[k]);
                    load_any<V>(a.dy, dy0 + int64_t(r + k * c.lanes) * a.C + c.vec * V, a.y_dtype, d[k]);
                }
            with_act(a.act, [&](auto act) {
#pragma unroll
                for (int k = 0; k < kNormRows; ++k) {
                    if (r + k * c.lanes >= r1) break;
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float xh = (v[k][i] - mu[i]) * rs[i];
                        const float e = d[k][i] * slope<act.value>(fmaf(xh, w[i], add[i])) * w[i];
                        v[k][i] = rs[i] * (e - e1[i] - xh * e2[i]);
                    }
                    store_n<T, V, STREAM>(dx + int64_t(r + k * c.lanes) * a.C + c.vec * V, v[k]);
                }
            });
        }
    }
}

// Small maps: a launch costs the host about 3.3 us, more than the work, so a group
// that one workgroup holds in registers takes one kernel in each direction instead of three,
// where small() does not expect that to take longer.
constexpr int kSmallBlock = 1024;
constexpr int kSmallRows = 8;       // values of a thread (16 spill in the backward)
constexpr int kSmallFrames = 4;     // of the backward, whose workgroup takes a group of all frames in turn

// Sum over the workgroup; red: kSmallBlock / 64 floats, free on entry and exit.
__device__ __forceinline__ float block_sum(float v, float *red) {
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = (threadIdx.x & 63) < kSmallBlock / 64 ? red[threadIdx.x & 63] : 0.0f;
    v = wave_sum(v);
    __syncthreads();
    return v;
}

// Thread -> (row lane, channel of the group); row lanes past the last are idle.
struct SmallPlace {
    int lanes, lane, ch;
};
__device__ __forceinline__ SmallPlace small_place(int per) {
    SmallPlace p;
    p.lanes = kSmallBlock / per;
    p.lane = threadIdx.x / per;
    p.ch = threadIdx.x - p.lane * per;
    return p;
}

template <int DT>
__global__ __launch_bounds__(kSmallBlock) void k_norm_small(NormArgs a) {
    using T = typename Num<DT>::T;
    __shared__ float red[kSmallBlock / 64];
    const int g = blockIdx.x, b = blockIdx.y, n = a.rows * a.per;
    const SmallPlace p = small_place(a.per);
    const int ch = g * a.per + p.ch;
    const T *x = static_cast<const T *>(a.x) + int64_t(b) * a.rows * a.ldx + ch;
    auto in = [&](int k) { return p.lane < p.lanes && p.lane + k * p.lanes < a.rows; };
    float v[kSmallRows], sum = 0.0f, m2 = 0.0f;
#pragma unroll
    for (int k = 0; k < kSmallRows; ++k) v[k] = in(k) ? float(x[int64_t(p.lane + k * p.lanes) * a.ldx]) : 0.0f;
#pragma unroll
    for (int k = 0; k < kSmallRows; ++k) sum += v[k];
    const float mean = block_sum(sum, red) / float(n);
#pragma unroll
    for (int k = 0; k < kSmallRows; ++k) {
        const float d = in(k) ? v[k] - mean : 0.0f;
        m2 = fmaf(d, d, m2);
    }
    const float rstd = 1.0f / sqrtf(block_sum(m2, red) / float(n) + a.eps);
    if (threadIdx.x == 0) {
        a.mean[int64_t(b) * a.G + g] = mean;
        a.rstd[int64_t(b) * a.G + g] = rstd;
    }
    if (p.lane >= p.lanes) return;
    const float mul = rstd * weight_at(a.weight, ch, a.w_dtype, 1.0f), add = weight_at(a.bias, ch, a.w_dtype, 0.0f);
    with_act(a.act, [&](auto act) {
#pragma unroll
        for (int k = 0; k < kSmallRows; ++k) {
            if (!in(k)) continue;
            const float y = activate<act.value>(fmaf(v[k] - mean, mul, add));
            store_any<1>(a.y, (int64_t(b) * a.rows + p.lane + k * p.lanes) * a.C + ch, a.y_dtype, &y);
        }
    });
}

template <int DT>
__global__ __launch_bounds__(kSmallBlock) void k_norm_small_grad(NormArgs a) {
    using T = typename Num<DT>::T;
    __shared__ float red[kSmallBlock / 64], meet[2][kSmallBlock];
    const int g = blockIdx.x;
    const SmallPlace p = small_place(a.per);
    const int ch = min(g * a.per + p.ch, a.C - 1);
    const float w = weight_at(a.weight, ch, a.w_dtype, 1.0f), add = weight_at(a.bias, ch, a.w_dtype, 0.0f);
    const float inv = 1.0f / (float(a.rows) * float(a.per));
    float all = 0.0f, all_dot = 0.0f;              // of this thread's channel, over the frames
    for (int b = 0; b < a.batch; ++b) {
        const T *x = static_cast<const T *>(a.x) + int64_t(b) * a.rows * a.ldx + ch;
        const int64_t to = int64_t(b) * a.rows * a.C + ch;
        const float mean = a.mean[int64_t(b) * a.G + g], rstd = a.rstd[int64_t(b) * a.G + g];
        auto in = [&](int k) { return p.lane < p.lanes && p.lane + k * p.lanes < a.rows; };
        float xh[kSmallRows], dz[kSmallRows], sum = 0.0f, dot = 0.0f;
#pragma unroll
        for (int k = 0; k < kSmallRows; ++k) {
            const int r = p.lane + k * p.lanes;
            xh[k] = mean;
            dz[k] = 0.0f;
            if (in(k)) {
                xh[k] = float(x[int64_t(r) * a.ldx]);
                load_any<1>(a.dy, to + int64_t(r) * a.C, a.y_dtype, &dz[k]);
            }
        }
        with_act(a.act, [&](auto act) {
#pragma unroll
            for (int k = 0; k < kSmallRows; ++k) {
                if (!in(k)) continue;
                xh[k] = (xh[k] - mean) * rstd;
                dz[k] *= slope<act.value>(fmaf(xh[k], w, add));
                sum += dz[k];
                dot = fmaf(dz[k], xh[k], dot);
            }
        });
        all += sum;
        all_dot += dot;
        const float m1 = block_sum(sum * w, red) * inv, m2 = block_sum(dot * w, red) * inv;
        T *dx = static_cast<T *>(a.dx) + to;
#pragma unroll
        for (int k = 0; k < kSmallRows; ++k)
            if (in(k)) dx[int64_t(p.lane + k * p.lanes) * a.C] = T(rstd * (dz[k] * w - m1 - xh[k] * m2));
    }
    // the row lanes' upper halves go to the lower ones
    meet[0][threadIdx.x] = all;
    meet[1][threadIdx.x] = all_dot;
    for (int n = p.lanes; n > 1; n = (n + 1) / 2) {
        const int half = (n + 1) / 2, from = threadIdx.x + half * a.per;
        __syncthreads();
        if (p.lane < n - half) {
            meet[0][threadIdx.x] = all += meet[0][from];
            meet[1][threadIdx.x] = all_dot += meet[1][from];
        }
    }
    if (p.lane != 0) return;
    if (a.dbias) store_any<1>(a.dbias, ch, a.w_dtype, &all);
    if (a.dweight) store_any<1>(a.dweight, ch, a.w_dtype, &all_dot);
}

constexpr int kSumGrid = 1024;      // workgroups of a sum pass, about
constexpr int kApplyGrid = 2048;    // workgroups of an apply pass, about
constexpr int kThreadRows = 8;      // rows of a thread, about, at least,
constexpr int kLeastGrid = 512;     // unless fewer workgroups than this were left: two to a compute unit
// Maps that together exceed the 256 MB of cache behind the L2s: results are then
// written past it, and more of x is still there for the second read.
constexpr int64_t kCacheBytes = int64_t(256) << 20;
static_assert(kSumGrid <= 64 * kJoin, "k_norm_join holds a group's parts in registers");

int ceil_div(int64_t a, int64_t b) { return int((a + b - 1) / b); }

int64_t elements(const bevmap_norm &n) { return int64_t(n.batch) * n.pixels * n.channels; }

// A workgroup to a group reads a piece of every row, and a cache line for it, so many groups
// ask for the same lines again and again; and workgroups of 16 waves start at 7 ns each (11
// of the backward, one frame after the other). So one kernel is taken where that costs less
// than the three, which depend little on the sizes as long as a launch is most of their time,
// but join every group. Microseconds, fitted to both forms of 654 shapes (fp32 and bf16, 1 to 80
// channels of a group, 32 to 1024 channels, 16 to 8100 rows, 1 to 64 frames). Of the faster
// form's time the rule costs 0.5% forward and 1.2% backward on average; one kernel for all
// would cost 34% and 15%: 64 frames of 8100 rows and 80 groups of one channel in fp32, 714 us
// and 88; four frames of 8100 rows and 32 such groups, backward, 99 and 18.
bool small(const bevmap_norm &n, bool backward) {
    const int per = n.channels / n.groups;
    if (per > kSmallBlock || ceil_div(n.pixels, kSmallBlock / per) > kSmallRows ||
        (backward && n.batch > kSmallFrames))
        return false;
    const double rows = double(n.batch) * n.pixels, groups = double(n.batch) * n.groups;
    const double lines = rows * n.groups;
    const double one = backward ? 15e-6 * lines + 11e-3 * groups + 2e-3 * rows : 12.5e-6 * lines + 6.7e-3 * groups;
    return one <= 12.0 + 0.03 * n.groups;
}

void split(const bevmap_norm &n, NormArgs *a) {
    // row lanes of a workgroup with the widest accesses (by the sizes alone: the workspace goes by this)
    int vec = n.x_dtype == BEVPOOL_F32 ? 4 : 8;
    while (n.channels % vec) vec >>= 1;
    const int vectors = n.channels / vec, lanes = vectors < kNormBlock ? kNormBlock / vectors : 1;
    const int spread = ceil_div(int64_t(n.batch) * n.pixels, kLeastGrid);
    const int least = kThreadRows * lanes < spread ? kThreadRows * lanes : spread;
    a->chunk = ceil_div(n.pixels, ceil_div(kSumGrid, n.batch));
    if (a->chunk < least) a->chunk = least;
    a->n_chunks = ceil_div(n.pixels, a->chunk);
    a->apply_rows = ceil_div(n.pixels, ceil_div(kApplyGrid, n.batch));
    if (a->apply_rows < least) a->apply_rows = least;
    a->n_apply = ceil_div(n.pixels, a->apply_rows);
}

NormArgs fill(const bevmap_norm &n, const void *x, const void *weight, const void *bias, void *workspace) {
    NormArgs a{};
    a.x = x;
    a.weight = weight;
    a.bias = bias;
    a.ldx = n.row_stride;
    a.batch = n.batch;
    a.rows = n.pixels;
    a.C = n.channels;
    a.G = n.groups;
    a.per = n.channels / n.groups;
    a.y_dtype = n.y_dtype;
    a.w_dtype = n.weight_dtype;
    a.act = n.act;
    a.eps = n.eps;
    split(n, &a);
    a.parts = static_cast<float2 *>(workspace);
    a.moments = a.parts + int64_t(n.batch) * a.n_chunks * n.groups;
    a.channel_sums = reinterpret_cast<float *>(a.moments + int64_t(n.batch) * n.groups);
    return a;
}

// Elements of an access: the widest of 16 bytes of x and less that divides the
// channels and that every tensor's alignment allows.
int vector_of(const bevmap_norm &n, const void *x, const void *y, const void *dx) {
    for (int v = n.x_dtype == BEVPOOL_F32 ? 4 : 8; v > 1; v >>= 1)
        if (n.channels % v == 0 && aligned_for(x, n.row_stride, n.x_dtype, v) && aligned_for(y, 0, n.y_dtype, v) &&
            (!dx || aligned_for(dx, 0, n.x_dtype, v)))
            return v;
    return 1;
}

// Bytes of LDS: two floats a channel, and one for each thread's V channels.
size_t sum_lds(const NormArgs &a, int v) { return (2 * size_t(a.C) + size_t(kSumBlock) * v) * sizeof(float); }

// Raises a kernel's limit of dynamic LDS where it needs more than the default.
template <class K>
int allow_lds(K kernel, size_t bytes) {
    if (bytes > 64 * 1024)
        BEVPOOL_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                        hipFuncAttributeMaxDynamicSharedMemorySize, int(bytes)));
    return BEVPOOL_OK;
}

template <int DT, int V>
int forward(const NormArgs &a, hipStream_t stream) {
    const size_t lds = sum_lds(a, V);
    if (int rc = allow_lds(k_norm_sum<DT, V>, lds)) return rc;
    hipLaunchKernelGGL((k_norm_sum<DT, V>), dim3(a.n_chunks, a.batch), dim3(kSumBlock), lds, stream, a);
    BEVPOOL_HIP(hipGetLastError());
    hipLaunchKernelGGL(k_norm_join, dim3(a.G, a.batch), dim3(64), 0, stream, a);
    BEVPOOL_HIP(hipGetLastError());
    if (V >= 4 && a.stream)
        hipLaunchKernelGGL((k_norm_apply<DT, V, (V >= 4)>), dim3(a.n_apply, a.batch), dim3(kNormBlock), 0, stream, a);
    else
        hipLaunchKernelGGL((k_norm_apply<DT, V, false>), dim3(a.n_apply, a.batch), dim3(kNormBlock), 0, stream, a);
    BEVPOOL_HIP(hipGetLastError());
    return BEVPOOL_OK;
}

template <int DT, int V>
int backward(const NormArgs &a, hipStream_t stream) {
    const size_t lds = sum_lds(a, V);
    if (int rc = allow_lds(k_norm_grad_sum<DT, V>, lds)) return rc;
    hipLaunchKernelGGL((k_norm_grad_sum<DT, V>), dim3(a.n_chunks, a.batch), dim3(kSumBlock), lds, stream, a);
    BEVPOOL_HIP(hipGetLastError());
    const int n_join = ceil_div(a.G, kJoinBlock / 64), extra = a.dweight || a.dbias ? ceil_div(a.C, kWgradChannels) : 0;
    hipLaunchKernelGGL(k_norm_grad_join, dim3(n_join + extra, a.batch), dim3(kJoinBlock), 0, stream, a, n_join);
    BEVPOOL_HIP(hipGetLastError());
    if (V >= 4 && a.stream)
        hipLaunchKernelGGL((k_norm_grad_apply<DT, V, (V >= 4)>), dim3(a.n_apply, a.batch), dim3(kNormBlock), 0, stream, a);
    else
        hipLaunchKernelGGL((k_norm_grad_apply<DT, V, false>), dim3(a.n_apply, a.batch), dim3(kNormBlock), 0, stream, a);
    BEVPOOL_HIP(hipGetLastError());
    return BEVPOOL_OK;
}

template <int DT>
int dispatch(const NormArgs &a, int v, bool back, hipStream_t stream) {
    switch (v) {
        case 0:
            if (back)
                hipLaunchKernelGGL((k_norm_small_grad<DT>), dim3(a.G), dim3(kSmallBlock), 0, stream, a);
            else
                hipLaunchKernelGGL((k_norm_small<DT>), dim3(a.G, a.batch), dim3(kSmallBlock), 0, stream, a);
            BEVPOOL_HIP(hipGetLastError());
            return BEVPOOL_OK;
        case 8:
            if constexpr (DT != BEVPOOL_F32) return back ? backward<DT, 8>(a, stream) : forward<DT, 8>(a, stream);
        case 4: return back ? backward<DT, 4>(a, stream) : forward<DT, 4>(a, stream);
        case 2: return back ? backward<DT, 2>(a, stream) : forward<DT, 2>(a, stream);
        default: return back ? backward<DT, 1>(a, stream) : forward<DT, 1>(a, stream);
    }
}

// v: elements of an access; 0 for the kernels of small maps.
int dispatch(int dtype, const NormArgs &a, int v, bool back, hipStream_t stream) {
    switch (dtype) {
        case BEVPOOL_F32: return dispatch<BEVPOOL_F32>(a, v, back, stream);
        case BEVPOOL_BF16: return dispatch<BEVPOOL_BF16>(a, v, back, stream);
        default: return dispatch<BEVPOOL_F16>(a, v, back, stream);
    }
}

__global__ void k_zero_weights(void *a, void *b, int n, int dtype) {
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    const float zero = 0.0f;
    if (i < n && a) store_any<1>(a, i, dtype, &zero);
    if (i < n && b) store_any<1>(b, i, dtype, &zero);
}

}  // namespace
}  // namespace bevmap

using namespace bevmap;

int64_t bevmap_norm_workspace_bytes(const bevmap_norm &n, bool backward) {
    if (n.batch == 0 || n.pixels == 0 || small(n, backward)) return 0;
    NormArgs a{};
    split(n, &a);
    const int64_t chunks = int64_t(n.batch) * a.n_chunks;
    const int64_t parts = chunks * n.groups * int64_t(sizeof(float2));
    if (!backward) return parts;
    return parts + int64_t(n.batch) * n.groups * int64_t(sizeof(float2)) +
           chunks * 2 * n.channels * int64_t(sizeof(float));
}

int bevmap_launch_norm(const bevmap_norm &n, const void *x, const void *weight, const void *bias, void *y,
                       float *mean, float *rstd, void *workspace, hipStream_t stream) {
    if (n.batch == 0 || n.pixels == 0) return BEVPOOL_OK;
    NormArgs a = fill(n, x, weight, bias, workspace);
    a.y = y;
    a.stream = elements(n) * (dtype_bytes(n.x_dtype) + dtype_bytes(n.y_dtype)) > kCacheBytes;
    a.mean = mean;
    a.rstd = rstd;
    return dispatch(n.x_dtype, a, small(n, false) ? 0 : vector_of(n, x, y, nullptr), false, stream);
}

int bevmap_launch_norm_backward(const bevmap_norm &n, const void *grad_y, const void *x, const void *weight,
                                const void *bias, const float *mean, const float *rstd, void *grad_x,
                                void *grad_weight, void *grad_bias, void *workspace, hipStream_t stream) {
    if (n.batch == 0 || n.pixels == 0) {
        if (grad_weight || grad_bias) {
            hipLaunchKernelGGL(k_zero_weights, dim3(ceil_div(n.channels, kNormBlock)), dim3(kNormBlock), 0, stream,
                               grad_weight, grad_bias, n.channels, n.weight_dtype);
            BEVPOOL_HIP(hipGetLastError());
        }
        return BEVPOOL_OK;
    }
    NormArgs a = fill(n, x, weight, bias, workspace);
    a.dy = grad_y;
    a.stream = elements(n) * (2 * dtype_bytes(n.x_dtype) + dtype_bytes(n.y_dtype)) > kCacheBytes;
    a.dx = grad_x;
    a.dweight = grad_weight;
    a.dbias = grad_bias;
    a.mean = const_cast<float *>(mean);
    a.rstd = const_cast<float *>(rstd);
    return dispatch(n.x_dtype, a, small(n, true) ? 0 : vector_of(n, x, grad_y, grad_x), true, stream);
}
