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
// split, and k_attend_add joins the parts. Few rows take k_attend_dkv_few.
//
// fp16's p and ds are held scaled by powers of two (attention.h): unscaled they end at
// 2^-24, which probabilities of 10^5 keys are near (dv 5 times as far off as its own
// rounding; dq of small gradients 37 times). It costs 7 to 10% of the pair's time.
//
// p and ds enter their products as two pieces of a 16-bit type: rounded once they
// left dq, dk and dv of bf16 up to 1.55 times as far off as gradients in fp32 rounded
// at the end; the pieces cost a quarter of the pair of kernels at large sizes.
//
// 4 x 600 queries of 8 heads over 8100 masked keys, ragged, 64 channels: dq 62 us and
// its joining 9, dk and dv 75, two waves a SIMD that wait for LDS and for each other. 4096
// rows, 8192 keys, 8 heads of 32, 64 and 128 channels: bf16 105 + 150, 149 + 216 and 260 +
// 539 us (340, 470 and 430 TFLOP/s, five products counted), fp16 6 to 11% more, fp32
// 316 + 455, 540 + 837 and 1126 + 2491 (111, 125 and 95). dk and dv of 128 channels hold both
// sums and both operands: one wave a SIMD, and in fp32 166 to 170 registers spilled (of
// three blocks in 16 bits 6 to 17, and up to 6 of dq).
#include "attention.h"

namespace bevmap {
namespace {

constexpr int kOwn = kAttendTile;   // rows or keys that a workgroup owns, 32 a wave

// Rows or keys of a tile that is walked, and what a thread moves of it.
template <int DT, int DB>
struct Walk {
    using S = Shape<DT, DB>;
    static constexpr int kBlocks = DT != BEVPOOL_F32 && DB <= 2 ? 2 : 1;        // of 32
    static constexpr int kSize = 32 * kBlocks;
    static constexpr int kBytes = kSize * S::kRowBytes;
    static constexpr int kLds = 4 * kBytes + 4 * kSize * int(sizeof(float));
    static_assert(kLds >= 4 * 32 * 32 * DB * int(sizeof(typename S::T)), "write_rows() of four waves");
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
template <int DT, int DB, bool VEC>
__device__ __forceinline__ void write_row(const f32x16 *acc, bool on, float mul, typename Num<DT>::T *to,
                                          float *part, int dim, int half) {
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int ch = 32 * d + 2 * i + 4 * half;
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = on ? acc[d][i + e] * mul : 0.0f;
            if (part)
                write4<VEC>(part, ch, dim, v);
            else
                write4<VEC>(to, ch, dim, v);
        }
}

template <int DT, int DB, bool VEC>
__global__ __launch_bounds__(kAttendBlock, waves_dq(DT, DB)) void k_attend_dq(AttendArgs g) {
    using S = Shape<DT, DB>;
    using T = typename S::T;
    using M = typename S::M;
    using W = Walk<DT, DB>;
    static_assert(W::kLds * waves_dq(DT, DB) <= kLdsBytes, "workgroups that partition_q() counts");
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

    u32x4 q[S::kOperand], d[S::kOperand];
    float delta = 0.0f, lse = INFINITY;
#pragma unroll
    for (int s = 0; s < S::kOperand; ++s) q[s] = d[s] = u32x4{0, 0, 0, 0};
    if (in) {
        const int64_t to = at.row(row);
        const T *dout = static_cast<const T *>(g.dout) + to, *out = static_cast<const T *>(g.out) + to;
        S::template operand<VEC>(at.q(row), half, dim, g.pairs, q);
        S::template operand<VEC>(dout, half, dim, g.pairs, d);
#pragma unroll
        for (int c = 0; c < S::kUsed / 2; ++c) {
            u32x4 low = {0, 0, 0, 0};
            if (DT != BEVPOOL_F32 && g.out_low)
                low = load_chunk<DT, VEC>(static_cast<const T *>(g.out_low) + to, 2 * c + half, dim, g.pairs);
            delta += pair_dot<DT>(load_chunk<DT, VEC>(dout, 2 * c + half, dim, g.pairs), load_chunk<DT, VEC>(out, 2 * c + half, dim, g.pairs),
                                  low);
        }
        lse = g.lse[at.stat(row)];
    }
    delta = both_sum(delta);
    if (in && half == 0 && split == 0) g.delta[at.stat(row)] = delta;
    if (lse == -INFINITY) lse = INFINITY;        // a row without keys: every p is 0

    const int tiles = (at.len + W::kSize - 1) / W::kSize, per = (tiles + g.n_split - 1) / g.n_split;
    const int t0 = split * per, t1 = min(t0 + per, tiles);
    using Used = InUse<W::kSize>;
    Stage<DT, DB, VEC, W::kSize> next_k(uint32_t(g.a.k_row * int(sizeof(T))), dim), next_v(uint32_t(g.a.v_row * int(sizeof(T))), dim);
    Mask<W::kSize> mask;
    auto key_rows = [&](int t) { return reinterpret_cast<const char *>(at.k(t * W::kSize)); };
    auto value_rows = [&](int t) { return reinterpret_cast<const char *>(at.v(t * W::kSize)); };
    f32x16 dq[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) dq[i] = zeros();
    const float c = g.sign * g.log2_scale;
    float lift = DT == BEVPOOL_F16 ? kFirstLift : 0.0f;
    Used use = {}, next = {};
    if (t0 < t1) {
        mask.ask(at, t0 * W::kSize);
        use = mask.count(at, t0 * W::kSize);
        next_k.load(key_rows(t0), use.words, use.all, dim, g.pairs);
        next_v.load(value_rows(t0), use.words, use.all, dim, g.pairs);
        mask.ask(at, (t0 + 1) * W::kSize);
        next_k.store(lds);
        next_v.store(lds + W::kBytes);
    }
    for (int t2 = t0; t2 < t1; t2 += 2) {
#pragma unroll
        for (int buffer = 0; buffer < 2; ++buffer) {
            const int t = t2 + buffer;
            if (t >= t1) break;
            const char *k = lds + buffer * 2 * W::kBytes, *v = k + W::kBytes;
            if (t + 1 < t1) {
                next = mask.count(at, (t + 1) * W::kSize);
                next_k.load(key_rows(t + 1), next.words, next.all, dim, g.pairs);
                next_v.load(value_rows(t + 1), next.words, next.all, dim, g.pairs);
                mask.ask(at, (t + 2) * W::kSize);
            }
            __syncthreads();
#pragma unroll
            for (int n = 0; n < W::kBlocks; ++n) {
                const uint32_t word = uint32_t(use.words[0] >> (32 * n));
                if (__builtin_expect(word == 0, 0)) continue;
                f32x16 s = S::scores(k, 32 * n, q, zeros());
                const f32x16 dp = S::scores(v, 32 * n, d, zeros());
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c, lift - lse)) * (dp[i] - delta);
                if (__builtin_expect(word != 0xFFFFFFFFu, 0)) {
                    const uint32_t bits = word >> (4 * half);
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] = bits & (1u << (8 * (i >> 2) + (i & 3))) ? s[i] : 0.0f;
                }
                typename M::Rows high, low;
                M::rows_of_two(s, high, low);
                if constexpr (DT == BEVPOOL_F16)
                    if (__builtin_expect(__any(high.reaches_two()), 0)) {
                        const float mul = lower(s, lift);
#pragma unroll
                        for (int b = 0; b < DB; ++b)
#pragma unroll
                            for (int i = 0; i < 16; ++i) dq[b][i] *= mul;
                        M::rows_of_two(s, high, low);
                    }
                S::sums(k, 32 * n, high, dq, DT == BEVPOOL_F32 ? nullptr : &low);
            }
            if (t + 1 < t1) {
                char *to = lds + (1 - buffer) * 2 * W::kBytes;
                next_k.store(to);
                next_v.store(to + W::kBytes);
                use = next;
            }
        }
    }
    if (!in) return;
    float *part = nullptr;
    if (g.n_split > 1) part = g.part + ((int64_t(split) * n_bh + bh) * g.rows + row) * dim;
    write_row<DT, DB, VEC>(dq, true, g.a.scale * power_of_two(-lift), static_cast<T *>(g.dq) + at.row(row), part, dim, half);
}

// What a wave's lanes wrote to LDS, its others may now read, and the other way round.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Chunk c of row r of a wave's 32 rows in LDS.
template <int DT, int DB>
__device__ __forceinline__ int wave_chunk(int r, int c) {
    return (r * (DB * 32 * int(sizeof(typename Num<DT>::T)) / 16) + (c ^ (r & 3))) * 16;
}

// The same for a wave's 32 rows from `first` on, through LDS (32 rows of 32 DB elements,
// the wave's own): a lane holds pieces of its row, and rows are written 16 bytes a lane
// one after the other. With few queries the gradients of k and v are mostly this.
template <int DT, int DB, class Unit, class Row>
__device__ __forceinline__ void write_rows(const f32x16 *acc, bool on, float mul, char *lds, int dim, int rows, Row to) {
    using T = typename Num<DT>::T;
    const int lane = threadIdx.x & 63, row = lane & 31, half = lane >> 5;
    const auto at = [&](int r, int c) { return lds + wave_chunk<DT, DB>(r, c); };
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int byte = (32 * d + 2 * i + 4 * half) * int(sizeof(T));
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = on ? acc[d][i + e] * mul : 0.0f;
            store_n<T, 4>(reinterpret_cast<T *>(at(row, byte / 16) + byte % 16), v);
        }
    wave_sync();
    constexpr int kUnit = int(sizeof(Unit));
    const int used = dim * int(sizeof(T)) / kUnit;
    for (int n = lane; n < rows * used; n += 64) {
        const int r = n / used, byte = (n - r * used) * kUnit;
        Unit x;
        __builtin_memcpy(&x, at(r, byte / 16) + byte % 16, kUnit);
        *reinterpret_cast<Unit *>(reinterpret_cast<char *>(to(r)) + byte) = x;
    }
    wave_sync();
}
// And the other way: a lane's row as an operand of scores(), read by the wave a unit a lane.
template <int DT, int DB, class Unit, class Row>
__device__ __forceinline__ void read_rows(u32x4 *y, bool use, char *lds, int dim, int rows, Row from) {
    using S = Shape<DT, DB>;
    const int lane = threadIdx.x & 63, row = lane & 31, half = lane >> 5;
    constexpr int kUnit = int(sizeof(Unit)), kUnits = S::kUsed * 16 / kUnit;
    const int used = dim * int(sizeof(typename S::T)) / kUnit;
    for (int n = lane; n < 32 * kUnits; n += 64) {
        const int r = n / kUnits, c = n - r * kUnits, byte = c * kUnit;
        Unit x = 0;
        if (r < rows && c < used) x = *reinterpret_cast<const Unit *>(reinterpret_cast<const char *>(from(r)) + byte);
        __builtin_memcpy(lds + wave_chunk<DT, DB>(r, byte / 16) + byte % 16, &x, kUnit);
    }
    wave_sync();
#pragma unroll
    for (int s = 0; s < S::kSteps; ++s) {
        u32x4 x = {0, 0, 0, 0};
        if (use) x = *reinterpret_cast<const u32x4 *>(lds + wave_chunk<DT, DB>(row, 2 * s + half));
        y[s] = x;
    }
    wave_sync();
}

template <int DT, int DB, bool VEC>
__global__ __launch_bounds__(kAttendBlock, waves_dkv(DT, DB)) void k_attend_dkv(AttendArgs g) {
    using S = Shape<DT, DB>;
    using T = typename S::T;
    using M = typename S::M;
    using W = Walk<DT, DB>;
    static_assert(W::kLds * waves_dkv(DT, DB) <= kLdsBytes, "workgroups that partition_k() counts");
    extern __shared__ __attribute__((aligned(16))) char lds[];       // [2][q, dout][tile], then [2][lse, delta][row]
    float *stats = reinterpret_cast<float *>(lds + 4 * W::kBytes);
    const int n_bh = g.a.batch * g.a.key_heads;
    int bh, tile;
    work_of(n_bh, g.n_split * g.n_tiles, bh, tile);
    const int split = tile / g.n_tiles;
    tile -= split * g.n_tiles;
    const Problem<DT> at(g, bh);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, dim = g.a.dim;
    const int key = tile * kOwn + 32 * wave + (lane & 31);
    const bool in = key < g.a.keys, use = in && at.ask(key) != 0;

    u32x4 k[S::kOperand], v[S::kOperand];
#pragma unroll
    for (int s = 0; s < S::kOperand; ++s) k[s] = v[s] = u32x4{0, 0, 0, 0};
    if (use) {
        S::template operand<VEC>(at.k(key), half, dim, g.pairs, k);
        S::template operand<VEC>(at.v(key), half, dim, g.pairs, v);
    }
    const int tiles = (g.rows + W::kSize - 1) / W::kSize, per = (tiles + g.n_split - 1) / g.n_split;
    // a tile of keys past the sample's length has nothing to walk
    const int t0 = split * per, t1 = tile * kOwn < at.len ? min(t0 + per, tiles) : t0;
    using Rows = Stage<DT, DB, VEC, W::kSize>;
    u32x4 next_q[Rows::kLoads], next_d[Rows::kLoads];
    float next_stat = 0.0f;
    auto fetch = [&](int t) {
        const int r0 = t * W::kSize;
#pragma unroll
        for (int i = 0; i < Rows::kLoads; ++i) {
            const int r = Rows::row(i), c = Rows::chunk(i);
            next_q[i] = next_d[i] = u32x4{0, 0, 0, 0};
            if ((Rows::kEven || r < W::kSize) && r0 + r < g.rows) {
                int query, head;
                at.split_row(r0 + r, query, head);
                next_q[i] = load_chunk<DT, VEC>(at.q(query, head), c, dim, g.pairs);
                next_d[i] = load_chunk<DT, VEC>(static_cast<const T *>(g.dout) + at.row(query, head), c, dim, g.pairs);
            }
        }
        if (threadIdx.x < 2 * W::kSize) {
            const int r = r0 + (threadIdx.x & (W::kSize - 1));
            const float none = threadIdx.x < W::kSize ? INFINITY : 0.0f;     // lse, delta of rows past the last
            next_stat = r < g.rows ? (threadIdx.x < W::kSize ? g.lse : g.delta)[at.stat(r)] : none;
            if (next_stat == -INFINITY) next_stat = INFINITY;
            if (threadIdx.x < W::kSize) next_stat -= kRaised<DT>;
        }
    };
    auto put = [&](char *q, float *stat) {
#pragma unroll
        for (int i = 0; i < Rows::kLoads; ++i) {
            const int r = Rows::row(i);
            if (!Rows::kEven && r >= W::kSize) break;
            S::put(q, r, Rows::chunk(i), next_q[i]);
            S::put(q + W::kBytes, r, Rows::chunk(i), next_d[i]);
        }
        if (threadIdx.x < 2 * W::kSize) stat[threadIdx.x] = next_stat;
    };
    f32x16 dk[DB], dv[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) dk[i] = dv[i] = zeros();
    const float c = g.sign * g.log2_scale;
    float lift = DT == BEVPOOL_F16 ? kFirstLift - kRaised<DT> : 0.0f;       // beyond kRaised
    if (t0 < t1) {
        fetch(t0);
        put(lds, stats);
    }
    for (int t2 = t0; t2 < t1; t2 += 2) {
#pragma unroll
        for (int buffer = 0; buffer < 2; ++buffer) {
            const int t = t2 + buffer;
            if (t >= t1) break;
            const char *q = lds + buffer * 2 * W::kBytes, *d = q + W::kBytes;
            const float *lse = stats + buffer * 2 * W::kSize + 4 * half, *delta = lse + W::kSize;
            if (t + 1 < t1) fetch(t + 1);
            __syncthreads();
#pragma unroll
            for (int n = 0; n < W::kBlocks; ++n) {
                if (n > 0 && t * W::kSize + 32 * n >= g.rows) break;       // a block past the last row
                f32x16 p = S::scores(q, 32 * n, k, zeros());
                f32x16 ds = S::scores(d, 32 * n, v, zeros());
                const float up = power_of_two(lift);
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const float4 l = *reinterpret_cast<const float4 *>(lse + 32 * n + 2 * i);
                    const float4 m = *reinterpret_cast<const float4 *>(delta + 32 * n + 2 * i);
                    const float ls[4] = {l.x, l.y, l.z, l.w}, de[4] = {m.x, m.y, m.z, m.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        p[i + e] = __builtin_amdgcn_exp2f(fmaf(p[i + e], c, -ls[e]));
                        ds[i + e] = p[i + e] * (ds[i + e] - de[e]);
                        if constexpr (DT == BEVPOOL_F16) ds[i + e] *= up;
                    }
                }
                typename M::Rows high, low;         // two pieces of each, as in k_attend_dq
                M::rows_of_two(p, high, low);
                S::sums(d, 32 * n, high, dv, DT == BEVPOOL_F32 ? nullptr : &low);
                M::rows_of_two(ds, high, low);
                if constexpr (DT == BEVPOOL_F16)
                    if (__builtin_expect(__any(high.reaches_two()), 0)) {
                        const float mul = lower(ds, lift);
#pragma unroll
                        for (int b = 0; b < DB; ++b)
#pragma unroll
                            for (int i = 0; i < 16; ++i) dk[b][i] *= mul;
                        M::rows_of_two(ds, high, low);
                    }
                S::sums(q, 32 * n, high, dk, DT == BEVPOOL_F32 ? nullptr : &low);
            }
            if (t + 1 < t1) put(lds + (1 - buffer) * 2 * W::kBytes, stats + (1 - buffer) * 2 * W::kSize);
        }
    }
    // a key out of use is a zero key here, whose sums are not its gradients
    const float of_k = g.a.scale * power_of_two(-lift - kRaised<DT>), of_v = power_of_two(-kRaised<DT>);
    if (VEC && sizeof(T) == 2 && g.n_split == 1) {
        const int first = tile * kOwn + 32 * wave, rows = min(32, g.a.keys - first);
        char *mine = lds + wave * (32 * 32 * DB * int(sizeof(T)));
        __syncthreads();                       // the last tile may still be read
        if (rows <= 0) return;
        write_rows<DT, DB, u32x4>(dk, use, of_k, mine, dim, rows, [&](int r) { return static_cast<T *>(g.dk) + at.key(first + r); });
        write_rows<DT, DB, u32x4>(dv, use, of_v, mine, dim, rows, [&](int r) { return static_cast<T *>(g.dv) + at.key(first + r); });
        return;
    }
    if (!in) return;
    float *part_k = nullptr, *part_v = nullptr;
    if (g.n_split > 1) {
        const int64_t all = int64_t(n_bh) * g.a.keys * dim;
        part_k = g.part + split * 2 * all + (int64_t(bh) * g.a.keys + key) * dim;
        part_v = part_k + all;
    }
    write_row<DT, DB, VEC>(dk, use, of_k, static_cast<T *>(g.dk) + at.key(key), part_k, dim, half);
    write_row<DT, DB, VEC>(dv, use, of_v, static_cast<T *>(g.dv) + at.key(key), part_v, dim, half);
}

// The same for few rows, one block of them: nothing is walked, so the sums of dv and dk
// are formed and written one after the other in half the registers, and with two or
// three waves to a SIMD where k_attend_dkv has one, the memory, which bounds it, is kept
// busy: 2 x 4 queries over 40000 keys of 8 heads in bf16, 64 channels 61 us, 128 channels 137
// (656 MB read and written, 4.8 TB/s; k_attend_dkv took 72 and 220); fp32 153 and 379 (220
// and 552). 16-bit rows that do not start on 16 bytes go through LDS both ways (84
// channels: 262 us, 400 without).
constexpr int kFewRows = 32;
template <int DT, int DB>
struct Few {
    using S = Shape<DT, DB>;
    static constexpr int kBytes = kFewRows * S::kRowBytes;
    static constexpr int kRead = 2 * kBytes + 2 * kFewRows * int(sizeof(float));          // q, dout, lse, delta
    static constexpr int kWrite = DT == BEVPOOL_F32 ? 0 : 4 * 32 * 32 * DB * int(sizeof(typename S::T));   // write_rows()
    static constexpr int kLds = kRead + kWrite;
    static_assert(kLds <= 64 * 1024, "more has to be asked for");
    static constexpr int kWaves = DT == BEVPOOL_F32 ? (DB <= 2 ? 2 : 1) : DB <= 2 ? 4 : 3;
};
template <int DT, int DB, bool VEC>
__global__ __launch_bounds__(kAttendBlock, (Few<DT, DB>::kWaves)) void k_attend_dkv_few(AttendArgs g) {
    using S = Shape<DT, DB>;
    using T = typename S::T;
    using M = typename S::M;
    using F = Few<DT, DB>;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    char *q = lds, *d = lds + F::kBytes;
    float *lse = reinterpret_cast<float *>(lds + 2 * F::kBytes), *delta = lse + kFewRows;
    int bh, tile;
    work_of(g.a.batch * g.a.key_heads, g.n_tiles, bh, tile);
    const Problem<DT> at(g, bh);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, dim = g.a.dim;
    const int key = tile * kOwn + 32 * wave + (lane & 31);
    const bool in = key < g.a.keys, use = in && at.ask(key) != 0;

    u32x4 k[S::kOperand], v[S::kOperand];
#pragma unroll
    for (int s = 0; s < S::kOperand; ++s) k[s] = v[s] = u32x4{0, 0, 0, 0};
    const int first = tile * kOwn + 32 * wave, rows = min(32, g.a.keys - first);
    char *mine = lds + F::kRead + wave * (F::kWrite / 4);
    if constexpr (VEC || DT == BEVPOOL_F32) {
        if (use) {
            S::template operand<VEC>(at.k(key), half, dim, g.pairs, k);
            S::template operand<VEC>(at.v(key), half, dim, g.pairs, v);
        }
    } else {
        const auto key_row = [&](int r) { return at.k(first + r); };
        const auto value_row = [&](int r) { return at.v(first + r); };
        if (g.pairs) {
            read_rows<DT, DB, uint32_t>(k, use, mine, dim, rows, key_row);
            read_rows<DT, DB, uint32_t>(v, use, mine, dim, rows, value_row);
        } else {
            read_rows<DT, DB, uint16_t>(k, use, mine, dim, rows, key_row);
            read_rows<DT, DB, uint16_t>(v, use, mine, dim, rows, value_row);
        }
    }
    for (int n = threadIdx.x; n < kFewRows * S::kUsed; n += kAttendBlock) {
        const int r = n / S::kUsed, c = n % S::kUsed;
        u32x4 x = {0, 0, 0, 0}, y = {0, 0, 0, 0};
        if (r < g.rows) {
            int query, head;
            at.split_row(r, query, head);
            x = load_chunk<DT, VEC>(at.q(query, head), c, dim, g.pairs);
            y = load_chunk<DT, VEC>(static_cast<const T *>(g.dout) + at.row(query, head), c, dim, g.pairs);
        }
        S::put(q, r, c, x);
        S::put(d, r, c, y);
    }
    if (threadIdx.x < kFewRows) {
        float l = INFINITY, e = 0.0f;            // rows past the last, and rows without keys: every p is 0
        if (int(threadIdx.x) < g.rows) {
            l = g.lse[at.stat(threadIdx.x)];
            e = g.delta[at.stat(threadIdx.x)];
        }
        lse[threadIdx.x] = (l == -INFINITY ? INFINITY : l) - kRaised<DT>;
        delta[threadIdx.x] = e;
    }
    __syncthreads();
    const float c = g.sign * g.log2_scale;
    float lift = DT == BEVPOOL_F16 ? kFirstLift - kRaised<DT> : 0.0f;       // beyond kRaised
    f32x16 p = S::scores(q, 0, k, zeros());
    f32x16 ds = S::scores(d, 0, v, zeros());
    const float up = power_of_two(lift);
#pragma unroll
    for (int i = 0; i < 16; i += 4)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            p[i + e] = __builtin_amdgcn_exp2f(fmaf(p[i + e], c, -lse[4 * half + 2 * i + e]));
            ds[i + e] = p[i + e] * (ds[i + e] - delta[4 * half + 2 * i + e]);
            if constexpr (DT == BEVPOOL_F16) ds[i + e] *= up;
        }
    f32x16 sum[DB];
    auto write = [&](void *to, float mul) {
        T *rows_of = static_cast<T *>(to);
        if constexpr (VEC && DT != BEVPOOL_F32)
            write_rows<DT, DB, u32x4>(sum, use, mul, mine, dim, rows, [&](int r) { return rows_of + at.key(first + r); });
        else if constexpr (DT != BEVPOOL_F32) {
            if (g.pairs)
                write_rows<DT, DB, uint32_t>(sum, use, mul, mine, dim, rows, [&](int r) { return rows_of + at.key(first + r); });
            else
                write_rows<DT, DB, uint16_t>(sum, use, mul, mine, dim, rows, [&](int r) { return rows_of + at.key(first + r); });
        } else if (in)
            write_row<DT, DB, VEC>(sum, use, mul, rows_of + at.key(key), nullptr, dim, half);
    };
    typename M::Rows high, low;
#pragma unroll
    for (int i = 0; i < DB; ++i) sum[i] = zeros();
    M::rows_of_two(p, high, low);
    S::sums(d, 0, high, sum, DT == BEVPOOL_F32 ? nullptr : &low);
    write(g.dv, power_of_two(-kRaised<DT>));
#pragma unroll
    for (int i = 0; i < DB; ++i) sum[i] = zeros();
    M::rows_of_two(ds, high, low);
    if constexpr (DT == BEVPOOL_F16)
        if (__any(high.reaches_two())) {
            lower(ds, lift);
            M::rows_of_two(ds, high, low);
        }
    S::sums(q, 0, high, sum, DT == BEVPOOL_F32 ? nullptr : &low);
    write(g.dk, g.a.scale * power_of_two(-lift - kRaised<DT>));
}

// Joins parts, one thread to an element: of the gradient of q (grid z 0), k (1) and v (2).
struct Parts {
    const float *q, *k;       // of k, then of v, for each part
    int32_t split_q, split_k; // 1: written whole, nothing to join
};
template <int DT>
__global__ __launch_bounds__(kAttendBlock) void k_attend_add(AttendArgs g, Parts parts) {
    using T = typename Num<DT>::T;
    const bool keys = blockIdx.z != 0;
    const int split = keys ? parts.split_k : parts.split_q, per_bh = keys ? g.a.keys : g.rows, dim = g.a.dim;
    const int64_t total = int64_t(g.a.batch) * g.a.key_heads * per_bh * dim;
    const int64_t n = int64_t(blockIdx.x) * kAttendBlock + threadIdx.x;
    if (split <= 1 || n >= total) return;
    const int64_t slot = n / dim;
    const int ch = int(n - slot * dim), bh = int(slot / per_bh), i = int(slot - int64_t(bh) * per_bh);
    const Problem<DT> at(g, bh);
    const float *part = (keys ? parts.k + int64_t(blockIdx.z - 1) * total : parts.q) + n;
    const int64_t step = keys ? 2 * total : total;
    float sum = 0.0f;
#pragma unroll 4
    for (int s = 0; s < split; ++s) sum += part[s * step];
    T *to = static_cast<T *>(!keys ? g.dq : blockIdx.z == 1 ? g.dk : g.dv);
    to[(keys ? at.key(i) : at.row(i)) + ch] = T(sum);
}

int64_t rows_of(const bevmap_attend &a) { return int64_t(a.queries) * (a.heads / a.key_heads); }

// Workgroups that own kOwn rows (of q) or keys, and parts of the others, of at least
// kPartSize each. More workgroups even out samples of unequal length where rows walk
// the keys; where keys walk the rows, parts are as large as all keys, and not for that.
constexpr int kPartSize = 128;
void partition_q(const bevmap_attend &a, bool lengths, int32_t *n_tiles, int32_t *n_split) {
    *n_tiles = attend_ceil(rows_of(a), kOwn);
    int slots = kUnits * waves_dq(a.dtype, (a.dim + 31) / 32);
    if (lengths) slots += slots / 2;
    *n_split = pick_split(int64_t(a.batch) * a.key_heads * *n_tiles, slots, a.keys, attend_ceil(a.keys, kPartSize),
                          lengths ? 600.0 : 300.0, a.dtype);       // twice the forward's work for the same parts
}
void partition_k(const bevmap_attend &a, int32_t *n_tiles, int32_t *n_split) {
    *n_tiles = attend_ceil(a.keys, kOwn);
    *n_split = pick_split(int64_t(a.batch) * a.key_heads * *n_tiles, kUnits * waves_dkv(a.dtype, (a.dim + 31) / 32),
                          rows_of(a), attend_ceil(rows_of(a), kPartSize), 480.0, a.dtype);     // two parts, 2.5 times the work
}

// Floats of the workspace: delta, ahead of the parts, and parts, which start on 16 bytes.
int64_t delta_floats(const bevmap_attend &a) { return (int64_t(a.batch) * a.queries * a.heads + 3) / 4 * 4; }
int64_t part_floats(int64_t parts, int64_t floats) { return (parts * floats + 3) / 4 * 4; }

template <int DT, int DB, bool VEC>
int launch(AttendArgs g, hipStream_t stream) {
    using W = Walk<DT, DB>;
    const size_t lds = W::kLds;
    if (lds > 64 * 1024) {
        BEVPOOL_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(k_attend_dq<DT, DB, VEC>),
                                        hipFuncAttributeMaxDynamicSharedMemorySize, int(lds)));
        BEVPOOL_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(k_attend_dkv<DT, DB, VEC>),
                                        hipFuncAttributeMaxDynamicSharedMemorySize, int(lds)));
    }
    const int64_t bh = int64_t(g.a.batch) * g.a.key_heads;
    Parts parts{g.part, nullptr, 1, 1};
    if (g.rows > 0) {
        partition_q(g.a, g.lengths != nullptr, &g.n_tiles, &g.n_split);
        parts.split_q = g.n_split;
        hipLaunchKernelGGL((k_attend_dq<DT, DB, VEC>), dim3(uint32_t(bh * g.n_split * g.n_tiles)),
                           dim3(kAttendBlock), lds, stream, g);
        BEVPOOL_HIP(hipGetLastError());
    }
    if (g.a.keys > 0) {
        if (parts.split_q > 1) g.part += part_floats(parts.split_q, bh * g.rows * g.a.dim);
        partition_k(g.a, &g.n_tiles, &g.n_split);
        parts.k = g.part;
        parts.split_k = g.n_split;
        if (g.rows <= kFewRows)
            hipLaunchKernelGGL((k_attend_dkv_few<DT, DB, VEC>), dim3(uint32_t(bh * g.n_tiles)), dim3(kAttendBlock),
                               (Few<DT, DB>::kLds), stream, g);
        else
            hipLaunchKernelGGL((k_attend_dkv<DT, DB, VEC>), dim3(uint32_t(bh * g.n_split * g.n_tiles)),
                               dim3(kAttendBlock), lds, stream, g);
        BEVPOOL_HIP(hipGetLastError());
    }
    const int64_t of_q = parts.split_q > 1 ? bh * g.rows * g.a.dim : 0;
    const int64_t of_k = parts.split_k > 1 ? bh * g.a.keys * g.a.dim : 0;
    if (of_q || of_k) {
        const int64_t most = of_q > of_k ? of_q : of_k;
        hipLaunchKernelGGL((k_attend_add<DT>), dim3(uint32_t((most + kAttendBlock - 1) / kAttendBlock), 1, of_k ? 3 : 1),
                           dim3(kAttendBlock), 0, stream, g, parts);
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
    int32_t tiles, split_q, split_lengths, split_k;
    partition_q(a, false, &tiles, &split_q);
    partition_q(a, true, &tiles, &split_lengths);
    if (split_lengths > split_q) split_q = split_lengths;
    partition_k(a, &tiles, &split_k);
    const int64_t rows = int64_t(a.batch) * a.queries * a.heads, keys = int64_t(a.batch) * a.keys * a.key_heads;
    const int64_t parts_q = split_q > 1 ? part_floats(split_q, rows * a.dim) : 0;
    const int64_t parts_k = split_k > 1 ? part_floats(2 * int64_t(split_k), keys * a.dim) : 0;
    return (delta_floats(a) + parts_q + parts_k) * int64_t(sizeof(float));
}

int bevmap_launch_attention_backward(const bevmap_attend &a, const void *grad_out, const void *q, const void *k,
                                     const void *v, const int32_t *lengths, const uint8_t *mask, const void *out,
                                     const void *out_low, const float *lse, void *grad_q, void *grad_k,
                                     void *grad_v, void *workspace, hipStream_t stream) {
    if (a.batch == 0) return BEVPOOL_OK;
    AttendArgs g = attend_fill(a, q, k, v, lengths, mask);
    g.dout = grad_out;
    g.out = out;
    g.out_low = out_low;
    g.lse = const_cast<float *>(lse);
    g.dq = grad_q;
    g.dk = grad_k;
    g.dv = grad_v;
    g.delta = static_cast<float *>(workspace);
    g.part = g.delta + delta_floats(a);
    const int e = a.dtype == BEVPOOL_F32 ? 4 : 8;
    const auto by = [&](int n) {
        const auto ok = [&](const void *p) { return !p || aligned_for(p, 0, a.dtype, n); };
        return attend_by(a, q, k, v, n) && ok(grad_out) && ok(out) && ok(out_low) && ok(grad_q) && ok(grad_k) &&
               ok(grad_v);
    };
    const bool vec = by(e);
    g.pairs = by(2);
    switch (a.dtype) {
        case BEVPOOL_F32: return backward<BEVPOOL_F32>(g, vec, stream);
        case BEVPOOL_BF16: return backward<BEVPOOL_BF16>(g, vec, stream);
        default: return backward<BEVPOOL_F16>(g, vec, stream);
    }
}
