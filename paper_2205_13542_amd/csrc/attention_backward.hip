// Gradients of the attention (bevmap_attention_backward); the layout of the
// products is in attention.h.
//
// With p = 2^(log2 scores - lse) formed again from the forward's lse, delta_r =
// dout_r . out_r and ds = p (dout v^T - delta):
//   dq = scale ds k,  dk = scale ds^T q,  dv = p^T dout.
// Two kernels, each of which keeps its sums in registers, so nothing is added up in
// memory and equal inputs give equal bits: k_attend_dq owns a tile of rows and
// walks the keys, k_attend_dkv owns a tile of keys and walks the rows of all heads
// that share them. Scores are formed in both, seven products in place of
// five. An axis that is too short to fill the chip has the walk of the other
// split, and k_attend_add joins the parts.
#include "attention.h"

namespace bevmap {
namespace {

constexpr int kOwn = 128;           // rows or keys that a workgroup owns, 32 a wave
constexpr int kWalk = 32;           // keys or rows of a tile that it walks

template <int DT, int DB>
struct Walk {
    using S = Shape<DT, DB>;
    static constexpr int kTileBytes = kWalk * S::kRowBytes;
    static constexpr int kLoads = (kWalk * S::kUsed + kAttendBlock - 1) / kAttendBlock;
};

template <int DT>
__device__ __forceinline__ float pair_dot(u32x4 a, u32x4 b, u32x4 low) {
    using T = typename Num<DT>::T;
    using Vec = T __attribute__((ext_vector_type(Mma<DT>::kElems)));
    const Vec x = __builtin_bit_cast(Vec, a), y = __builtin_bit_cast(Vec, b), z = __builtin_bit_cast(Vec, low);
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < Mma<DT>::kElems; ++i)
        s = fmaf(float(x[i]), DT == BEVPOOL_F32 ? float(y[i]) : float(y[i]) + float(z[i]), s);
    return s;
}

// A lane's row or key of a gradient: 16 channels of each block, whole or to a part.
template <int DT, int DB>
__device__ __forceinline__ void write_row(const f32x16 *acc, bool on, float mul, typename Num<DT>::T *to,
                                          float *part, int dim, int half) {
    using T = typename Num<DT>::T;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int ch = 32 * d + 8 * (i >> 2) + 4 * half + (i & 3);
            if (ch >= dim) continue;
            const float v = on ? acc[d][i] * mul : 0.0f;
            if (part)
                part[ch] = v;
            else
                to[ch] = T(v);
        }
}

template <int DT, int DB, bool VEC>
__global__ __launch_bounds__(kAttendBlock, 2) void k_attend_dq(AttendArgs g) {
    using S = Shape<DT, DB>;
    using T = typename S::T;
    using M = typename S::M;
    using W = Walk<DT, DB>;
    extern __shared__ __attribute__((aligned(16))) char lds[];       // [2][k, v][tile]
    const int n_bh = g.a.batch * g.a.key_heads;
    int bh, tile;
    work_of(n_bh, g.n_split * g.n_tiles, bh, tile);
    const int split = tile / g.n_tiles;
    tile -= split * g.n_tiles;
    const Problem<DT> at(g, bh);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, dim = g.a.dim;
    const int row = tile * kOwn + 32 * wave + (lane & 31);
    const bool in = row < g.rows;

    u32x4 q[S::kSteps], d[S::kSteps];
    float delta = 0.0f, lse = INFINITY;
#pragma unroll
    for (int s = 0; s < S::kSteps; ++s) q[s] = d[s] = u32x4{0, 0, 0, 0};
    if (in) {
        const T *p = at.q(row);
        const int64_t to = at.row(row);
#pragma unroll
        for (int s = 0; s < S::kSteps; ++s) {
            q[s] = load_chunk<DT, VEC>(p, 2 * s + half, dim);
            d[s] = load_chunk<DT, VEC>(static_cast<const T *>(g.dout) + to, 2 * s + half, dim);
            const u32x4 o = load_chunk<DT, VEC>(static_cast<const T *>(g.out) + to, 2 * s + half, dim);
            u32x4 low = {0, 0, 0, 0};
            if (DT != BEVPOOL_F32 && g.out_low)
                low = load_chunk<DT, VEC>(static_cast<const T *>(g.out_low) + to, 2 * s + half, dim);
            delta += pair_dot<DT>(d[s], o, low);
        }
        lse = g.lse[at.stat(row)];
    }
    delta = both_sum(delta);
    if (in && half == 0 && split == 0) g.delta[at.stat(row)] = delta;
    if (lse == -INFINITY) lse = INFINITY;        // a row without keys: every p is 0

    const int tiles = (at.len + kWalk - 1) / kWalk, per = (tiles + g.n_split - 1) / g.n_split;
    const int t0 = split * per, t1 = min(t0 + per, tiles);
    u32x4 next_k[W::kLoads], next_v[W::kLoads];
    int used;
    auto fetch = [&](int t) {
        const int j0 = t * kWalk;
        used = lane < kWalk ? at.ask(j0 + lane) : 0;
#pragma unroll
        for (int i = 0; i < W::kLoads; ++i) {
            const int n = threadIdx.x + i * kAttendBlock, r = n / S::kUsed, c = n - r * S::kUsed;
            next_k[i] = next_v[i] = u32x4{0, 0, 0, 0};
            if (r < kWalk && j0 + r < at.len) {
                next_k[i] = load_chunk<DT, VEC>(at.k(j0 + r), c, dim);
                next_v[i] = load_chunk<DT, VEC>(at.v(j0 + r), c, dim);
            }
        }
    };
    auto put = [&](int buffer) {
        const uint32_t word = uint32_t(__ballot(used != 0));
        char *k = lds + buffer * 2 * W::kTileBytes, *v = k + W::kTileBytes;
#pragma unroll
        for (int i = 0; i < W::kLoads; ++i) {
            const int n = threadIdx.x + i * kAttendBlock, r = n / S::kUsed, c = n - r * S::kUsed;
            if (r >= kWalk) break;
            const bool use = (word >> r) & 1;
            *reinterpret_cast<u32x4 *>(k + chunk_at<S::kChunks>(r, c)) = use ? next_k[i] : u32x4{0, 0, 0, 0};
            *reinterpret_cast<u32x4 *>(v + chunk_at<S::kChunks>(r, c)) = use ? next_v[i] : u32x4{0, 0, 0, 0};
        }
        return word;
    };
    f32x16 dq[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) dq[i] = zeros();
    const float c = g.sign * g.log2_scale;
    uint32_t word = 0;
    if (t0 < t1) {
        fetch(t0);
        word = put(0);
        if (t0 + 1 < t1) fetch(t0 + 1);
    }
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
        const char *k = lds + ((t - t0) & 1) * 2 * W::kTileBytes, *v = k + W::kTileBytes;
        if (word != 0) {
            f32x16 s = S::scores(k, 0, q, zeros());
            const f32x16 dp = S::scores(v, 0, d, zeros());
            const uint32_t bits = word >> (4 * half);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float p = __builtin_amdgcn_exp2f(fmaf(s[i], c, -lse));
                s[i] = bits & (1u << (8 * (i >> 2) + (i & 3))) ? p * (dp[i] - delta) : 0.0f;
            }
            S::sums(k, 0, M::rows(s), dq);
        }
        if (t + 1 < t1) {
            word = put((t + 1 - t0) & 1);
            if (t + 2 < t1) fetch(t + 2);
        }
        __syncthreads();
    }
    if (!in) return;
    float *part = nullptr;
    if (g.n_split > 1) part = g.part + ((int64_t(split) * n_bh + bh) * g.rows + row) * dim;
    write_row<DT, DB>(dq, true, g.a.scale, static_cast<T *>(g.dq) + at.row(row), part, dim, half);
}

template <int DT, int DB, bool VEC>
__global__ __launch_bounds__(kAttendBlock, 2) void k_attend_dkv(AttendArgs g) {
    using S = Shape<DT, DB>;
    using T = typename S::T;
    using M = typename S::M;
    using W = Walk<DT, DB>;
    extern __shared__ __attribute__((aligned(16))) char lds[];       // [2][q, dout][tile], then [2][lse, delta][kWalk]
    float *stats = reinterpret_cast<float *>(lds + 4 * W::kTileBytes);
    const int n_bh = g.a.batch * g.a.key_heads;
    int bh, tile;
    work_of(n_bh, g.n_split * g.n_tiles, bh, tile);
    const int split = tile / g.n_tiles;
    tile -= split * g.n_tiles;
    const Problem<DT> at(g, bh);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, dim = g.a.dim;
    const int key = tile * kOwn + 32 * wave + (lane & 31);
    const bool in = key < g.a.keys, use = in && at.ask(key) != 0;

    u32x4 k[S::kSteps], v[S::kSteps];
#pragma unroll
    for (int s = 0; s < S::kSteps; ++s) k[s] = v[s] = u32x4{0, 0, 0, 0};
    if (use) {
#pragma unroll
        for (int s = 0; s < S::kSteps; ++s) {
            k[s] = load_chunk<DT, VEC>(at.k(key), 2 * s + half, dim);
            v[s] = load_chunk<DT, VEC>(at.v(key), 2 * s + half, dim);
        }
    }
    const int tiles = (g.rows + kWalk - 1) / kWalk, per = (tiles + g.n_split - 1) / g.n_split;
    // a tile of keys past the sample's length has nothing to walk
    const int t0 = split * per, t1 = tile * kOwn < at.len ? min(t0 + per, tiles) : t0;
    u32x4 next_q[W::kLoads], next_d[W::kLoads];
    float next_stat = 0.0f;
    auto fetch = [&](int t) {
        const int r0 = t * kWalk;
#pragma unroll
        for (int i = 0; i < W::kLoads; ++i) {
            const int n = threadIdx.x + i * kAttendBlock, r = n / S::kUsed, c = n - r * S::kUsed;
            next_q[i] = next_d[i] = u32x4{0, 0, 0, 0};
            if (r < kWalk && r0 + r < g.rows) {
                next_q[i] = load_chunk<DT, VEC>(at.q(r0 + r), c, dim);
                next_d[i] = load_chunk<DT, VEC>(static_cast<const T *>(g.dout) + at.row(r0 + r), c, dim);
            }
        }
        if (threadIdx.x < 2 * kWalk) {
            const int r = r0 + (threadIdx.x & (kWalk - 1));
            const float none = threadIdx.x < kWalk ? INFINITY : 0.0f;       // lse, delta of rows past the last
            next_stat = r < g.rows ? (threadIdx.x < kWalk ? g.lse : g.delta)[at.stat(r)] : none;
            if (next_stat == -INFINITY) next_stat = INFINITY;
        }
    };
    auto put = [&](int buffer) {
        char *q = lds + buffer * 2 * W::kTileBytes, *d = q + W::kTileBytes;
#pragma unroll
        for (int i = 0; i < W::kLoads; ++i) {
            const int n = threadIdx.x + i * kAttendBlock, r = n / S::kUsed, c = n - r * S::kUsed;
            if (r >= kWalk) break;
            *reinterpret_cast<u32x4 *>(q + chunk_at<S::kChunks>(r, c)) = next_q[i];
            *reinterpret_cast<u32x4 *>(d + chunk_at<S::kChunks>(r, c)) = next_d[i];
        }
        if (threadIdx.x < 2 * kWalk) stats[buffer * 2 * kWalk + threadIdx.x] = next_stat;
    };
    f32x16 dk[DB], dv[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) dk[i] = dv[i] = zeros();
    const float c = g.sign * g.log2_scale;
    if (t0 < t1) {
        fetch(t0);
        put(0);
        if (t0 + 1 < t1) fetch(t0 + 1);
    }
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
        const int buffer = (t - t0) & 1;
        const char *q = lds + buffer * 2 * W::kTileBytes, *d = q + W::kTileBytes;
        const float *lse = stats + buffer * 2 * kWalk, *delta = lse + kWalk;
        f32x16 p = S::scores(q, 0, k, zeros());
        f32x16 ds = S::scores(d, 0, v, zeros());
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int r = 8 * (i >> 2) + 4 * half + (i & 3);
            p[i] = __builtin_amdgcn_exp2f(fmaf(p[i], c, -lse[r]));
            ds[i] = p[i] * (ds[i] - delta[r]);
        }
        S::sums(d, 0, M::rows(p), dv);
        S::sums(q, 0, M::rows(ds), dk);
        if (t + 1 < t1) {
            put((t + 1 - t0) & 1);
            if (t + 2 < t1) fetch(t + 2);
        }
        __syncthreads();
    }
    if (!in) return;
    float *part_k = nullptr, *part_v = nullptr;
    if (g.n_split > 1) {
        const int64_t all = int64_t(n_bh) * g.a.keys * dim;
        part_k = g.part + split * 2 * all + (int64_t(bh) * g.a.keys + key) * dim;
        part_v = part_k + all;
    }
    // a key out of use is a zero key here, whose sums are not its gradients
    write_row<DT, DB>(dk, use, g.a.scale, static_cast<T *>(g.dk) + at.key(key), part_k, dim, half);
    write_row<DT, DB>(dv, use, 1.0f, static_cast<T *>(g.dv) + at.key(key), part_v, dim, half);
}

// Joins parts, one thread to an element. KEYS: of the gradients of k (grid z 0)
// and v (1), else of q.
template <int DT, bool KEYS>
__global__ __launch_bounds__(kAttendBlock) void k_attend_add(AttendArgs g) {
    using T = typename Num<DT>::T;
    const int per_bh = KEYS ? g.a.keys : g.rows, dim = g.a.dim;
    const int64_t total = int64_t(g.a.batch) * g.a.key_heads * per_bh * dim;
    const int64_t n = int64_t(blockIdx.x) * kAttendBlock + threadIdx.x;
    if (n >= total) return;
    const int64_t slot = n / dim;
    const int ch = int(n - slot * dim), bh = int(slot / per_bh), i = int(slot - int64_t(bh) * per_bh);
    const Problem<DT> at(g, bh);
    const float *part = g.part + (KEYS ? int64_t(blockIdx.z) * total : 0) + n;
    const int64_t step = KEYS ? 2 * total : total;
    float sum = 0.0f;
#pragma unroll 4
    for (int s = 0; s < g.n_split; ++s) sum += part[s * step];
    T *to = static_cast<T *>(!KEYS ? g.dq : blockIdx.z ? g.dv : g.dk);
    to[(KEYS ? at.key(i) : at.row(i)) + ch] = T(sum);
}

constexpr int kFill = 512;          // workgroups that fill the chip, two to a compute unit

// Workgroups that own `own` rows or keys, and parts of the `walk` others; a part
// has at least kPartTiles tiles.
constexpr int kPartTiles = 4;
void partition(const bevmap_attend &a, int64_t own, int64_t walk, int32_t *n_tiles, int32_t *n_split) {
    *n_tiles = attend_ceil(own, kOwn);
    const int64_t whole = int64_t(a.batch) * a.key_heads * *n_tiles;
    int64_t split = whole ? (kFill + whole - 1) / whole : 1;
    const int64_t most = attend_ceil(walk, kWalk * kPartTiles);
    if (split > most) split = most;
    *n_split = split < 1 ? 1 : int32_t(split);
}

int64_t rows_of(const bevmap_attend &a) { return int64_t(a.queries) * (a.heads / a.key_heads); }

template <int DT, int DB, bool VEC>
int launch(AttendArgs g, hipStream_t stream) {
    using W = Walk<DT, DB>;
    const size_t lds = 4 * size_t(W::kTileBytes) + 4 * kWalk * sizeof(float);
    if (lds > 64 * 1024) {
        BEVPOOL_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(k_attend_dq<DT, DB, VEC>),
                                        hipFuncAttributeMaxDynamicSharedMemorySize, int(lds)));
        BEVPOOL_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(k_attend_dkv<DT, DB, VEC>),
                                        hipFuncAttributeMaxDynamicSharedMemorySize, int(lds)));
    }
    const int64_t bh = int64_t(g.a.batch) * g.a.key_heads;
    const auto blocks = [](int64_t n) { return uint32_t((n + kAttendBlock - 1) / kAttendBlock); };
    if (g.rows > 0) {
        partition(g.a, g.rows, g.a.keys, &g.n_tiles, &g.n_split);
        hipLaunchKernelGGL((k_attend_dq<DT, DB, VEC>), dim3(uint32_t(bh * g.n_split * g.n_tiles)),
                           dim3(kAttendBlock), lds, stream, g);
        BEVPOOL_HIP(hipGetLastError());
        if (g.n_split > 1)
            hipLaunchKernelGGL((k_attend_add<DT, false>), dim3(blocks(bh * g.rows * g.a.dim)), dim3(kAttendBlock), 0,
                               stream, g);
        BEVPOOL_HIP(hipGetLastError());
    }
    if (g.a.keys > 0) {
        partition(g.a, g.a.keys, g.rows, &g.n_tiles, &g.n_split);
        hipLaunchKernelGGL((k_attend_dkv<DT, DB, VEC>), dim3(uint32_t(bh * g.n_split * g.n_tiles)),
                           dim3(kAttendBlock), lds, stream, g);
        BEVPOOL_HIP(hipGetLastError());
        if (g.n_split > 1)
            hipLaunchKernelGGL((k_attend_add<DT, true>), dim3(blocks(bh * g.a.keys * g.a.dim), 1, 2),
                               dim3(kAttendBlock), 0, stream, g);
        BEVPOOL_HIP(hipGetLastError());
    }
    return BEVPOOL_OK;
}

template <int DT, int DB>
int launch(const AttendArgs &g, bool vec, hipStream_t stream) {
    return vec ? launch<DT, DB, true>(g, stream) : launch<DT, DB, false>(g, stream);
}

template <int DT>
int backward(const AttendArgs &g, bool vec, hipStream_t stream) {
    switch ((g.a.dim + 31) / 32) {
        case 1: return launch<DT, 1>(g, vec, stream);
        case 2: return launch<DT, 2>(g, vec, stream);
        case 3: return launch<DT, 3>(g, vec, stream);
        default: return launch<DT, 4>(g, vec, stream);
    }
}

}  // namespace
}  // namespace bevmap

using namespace bevmap;

int64_t bevmap_attention_backward_bytes(const bevmap_attend &a) {
    int32_t tiles, split_q, split_k;
    partition(a, rows_of(a), a.keys, &tiles, &split_q);
    partition(a, a.keys, rows_of(a), &tiles, &split_k);
    const int64_t rows = int64_t(a.batch) * a.queries * a.heads, keys = int64_t(a.batch) * a.keys * a.key_heads;
    const int64_t parts_q = split_q > 1 ? split_q * rows * a.dim : 0;
    const int64_t parts_k = split_k > 1 ? 2 * split_k * keys * a.dim : 0;
    // delta, then the parts of one gradient at a time
    return (rows + (parts_q > parts_k ? parts_q : parts_k)) * int64_t(sizeof(float));
}

int bevmap_launch_attention_backward(const bevmap_attend &a, const void *grad_out, const void *q, const void *k,
                                     const void *v, const int32_t *lengths, const uint8_t *mask, const void *out,
                                     const void *out_low, const float *lse, void *grad_q, void *grad_k,
                                     void *grad_v, void *workspace, hipStream_t stream) {
    if (a.batch == 0) return BEVPOOL_OK;
    const int64_t bh = int64_t(a.batch) * a.key_heads, most = int64_t(1) << 23;
    int32_t tiles, split;
    partition(a, rows_of(a), a.keys, &tiles, &split);
    const bool wide = bh * tiles * split >= most;
    partition(a, a.keys, rows_of(a), &tiles, &split);
    if (wide || bh * tiles * split >= most)
        return bevpool_fail(BEVPOOL_ERR_OVERFLOW, "batch=%d queries=%d keys=%d heads=%d: too many tiles", a.batch,
                            a.queries, a.keys, a.heads);
    AttendArgs g = attend_fill(a, q, k, v, lengths, mask);
    g.dout = grad_out;
    g.out = out;
    g.out_low = out_low;
    g.lse = const_cast<float *>(lse);
    g.dq = grad_q;
    g.dk = grad_k;
    g.dv = grad_v;
    g.delta = static_cast<float *>(workspace);
    g.part = g.delta + int64_t(a.batch) * a.queries * a.heads;
    const int e = a.dtype == BEVPOOL_F32 ? 4 : 8;
    const bool vec = attend_vec(a, q, k, v) && aligned_for(grad_out, 0, a.dtype, e) && aligned_for(out, 0, a.dtype, e) &&
                     (!out_low || aligned_for(out_low, 0, a.dtype, e));
    switch (a.dtype) {
        case BEVPOOL_F32: return backward<BEVPOOL_F32>(g, vec, stream);
        case BEVPOOL_BF16: return backward<BEVPOOL_BF16>(g, vec, stream);
        default: return backward<BEVPOOL_F16>(g, vec, stream);
    }
}
