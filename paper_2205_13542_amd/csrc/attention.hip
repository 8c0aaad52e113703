// Attention of queries to an encoder's states of another length, forward
// (bevmap_attention); the layout of the products is in attention.h.
//
// A workgroup takes a tile of rows and walks the keys tile by tile: keys and values
// go through registers to LDS one tile ahead of the products, every lane holds the
// scores of one row against 16 of 32 keys, and a softmax with a running maximum
// and sum joins the tiles in one pass over the keys. Few rows leave the chip idle,
// so the keys are then split over workgroups, and a second kernel joins the parts.
//
// A block of 32 rows and 32 keys takes a SIMD 278, 377 and 645 ns for 32, 64 and 128
// channels of bf16 (4096 rows, 8192 keys, 8 heads: 480, 710 and 830 TFLOP/s; a library
// product of 8192^3 reaches 1100), and 222 ns for 32 channels at 32400 rows and 16896
// keys. Of that 16 exponentials of 3.5 ns and 47 other vector instructions of 1.3 to 2 ns
// fill 117 to 150 ns, and beside them 4 matrix instructions of 16 ns; the rest is waiting,
// for LDS, at barriers and for each other (28% of the waves' cycles). 128 channels are
// bound by the matrix cores and the LDS reads that feed them. Scores of the next
// block formed ahead of a block's exponentials, the usual order and one block held
// back were within 5% of each other. One query over 129600 keys in bf16, 8 heads on 2:
// 17 us of 64 channels, whether all 66 MB are in use or, by a mask, 46; 30 us of 128,
// 133 MB (4.0 and 4.5 TB/s; joining 5 each); of fp32 37 and 123. 32400 queries over
// 16896 keys, 4 heads of 32: 464.
#include "attention.h"

namespace bevmap {
namespace {

// Exponentials are taken relative to a maximum that is not kept up to date: a
// tile whose sum for some row passes this (log2: 12) forms the rows' maxima, rescales
// what is summed and takes its exponentials again. The first tile always does. In
// between, a tile costs no maximum, and what is lost is nothing: the exponentials
// keep their relative precision. Those of fp16, from 2^-24 to 2^16, are taken relative to
// 2^-7 of the maximum, so that many small ones beside a large one are not lost.
template <int DT>
constexpr float kMaxTileSum = DT == BEVPOOL_F16 ? 32768.0f : 4096.0f;
template <int DT>
constexpr float kBelowTop = DT == BEVPOOL_F16 ? 7.0f : 0.0f;

// WR waves side by side have rows of their own (4), or all share the tile's rows
// and split each tile's keys (1).
template <int DT, int DB, int WR>
struct Tile {
    static constexpr int kBlocks = WR == 1 || DT == BEVPOOL_F32 ? 1 : 2;    // 32-key blocks of a wave
    static constexpr int kKeys = 32 * kBlocks * (4 / WR);       // of a tile
    static constexpr int kRows = 32 * WR;
    static constexpr int kBytes = kKeys * Shape<DT, DB>::kRowBytes;
    // pairs of tiles, keys and values, in LDS: two where they fit
    static constexpr int kPairs = 4 * kBytes <= 128 * 1024 ? 2 : 1;
    static constexpr int kLds = 2 * kPairs * kBytes;
    // Waves of a SIMD, or workgroups of a compute unit: by the registers, which the launch bound holds them to, and by
    // the LDS as well. fp32 of three blocks has one by its LDS, but in the registers of two it is faster (4096 rows,
    // 8192 keys, 8 heads of 96: 646 us) than with accumulation registers to move to and from (694).
    static constexpr int kWaves = WR == 1 ? waves_few(DT, DB) : waves_forward(DT, DB);
    static constexpr int kResident = kWaves * kLds <= kLdsBytes ? kWaves : kLdsBytes / kLds;
    static_assert(kResident > 0, "no workgroup fits");
};

template <int DT>
int resident_forward(int db, bool few) {
    if (few) {
        if constexpr (DT != BEVPOOL_F32) {
            if (db == 3) return Tile<DT, 3, 1>::kResident;
            if (db == 4) return Tile<DT, 4, 1>::kResident;
        }
        return db == 1 ? Tile<DT, 1, 1>::kResident : Tile<DT, 2, 1>::kResident;
    }
    return db == 1   ? Tile<DT, 1, 4>::kResident
           : db == 2 ? Tile<DT, 2, 4>::kResident
           : db == 3 ? Tile<DT, 3, 4>::kResident
                     : Tile<DT, 4, 4>::kResident;
}
// Workgroups of k_attend that a compute unit holds, by blocks of 32 channels.
int resident_forward(int dt, int db, bool few) {
    return dt == BEVPOOL_F32 ? resident_forward<BEVPOOL_F32>(db, few) : resident_forward<BEVPOOL_BF16>(db, few);
}

// What a part of a row with this maximum and sum counts where the whole row's
// maximum is `most`: nothing without keys; a sum that is NaN without a maximum
// (every score was NaN) stays one.
__device__ __forceinline__ float part_weight(float top, float sum, float most) {
    if (sum == 0.0f) return 0.0f;
    return top == -INFINITY ? 1.0f : exp2f(top - most);
}

template <int DT, int DB, bool VEC, int WR>
__global__ __launch_bounds__(kAttendBlock, (Tile<DT, DB, WR>::kWaves)) void k_attend(AttendArgs g) {
    using S = Shape<DT, DB>;
    using T = typename S::T;
    using M = typename S::M;
    using W = Tile<DT, DB, WR>;
    extern __shared__ __attribute__((aligned(16))) char lds[];

    const int n_bh = g.a.batch * g.a.key_heads;
    int bh, tile;
    work_of(n_bh, g.n_split * g.n_tiles, bh, tile);
    const int split = tile / g.n_tiles;
    tile -= split * g.n_tiles;
    const Problem<DT> at(g, bh);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const int row = tile * W::kRows + (WR == 1 ? 0 : 32 * wave) + (lane & 31);
    const int dim = g.a.dim;

    u32x4 q[S::kOperand];
#pragma unroll
    for (int s = 0; s < S::kOperand; ++s) q[s] = u32x4{0, 0, 0, 0};
    if (row < g.rows) S::template operand<VEC>(at.q(row), half, dim, g.pairs, q);
    if (g.sign != 1.0f) {
#pragma unroll
        for (int s = 0; s < S::kOperand; ++s) q[s] = g.sign == 0.0f ? u32x4{0, 0, 0, 0} : q[s] ^ 0x80008000u;
    }

    // this part's tiles of keys
    const int tiles = (at.len + W::kKeys - 1) / W::kKeys;
    const int per = (tiles + g.n_split - 1) / g.n_split;
    const int t0 = split * per, t1 = min(t0 + per, tiles);

    const uint32_t k_step = uint32_t(g.a.k_row * int(sizeof(T))), v_step = uint32_t(g.a.v_row * int(sizeof(T)));
    using Used = InUse<W::kKeys>;
    Stage<DT, DB, VEC, W::kKeys> next_k(k_step, dim), next_v(v_step, dim);
    Mask<W::kKeys> mask;
    auto key_rows = [&](int t) { return reinterpret_cast<const char *>(at.k(t * W::kKeys)); };
    auto value_rows = [&](int t) { return reinterpret_cast<const char *>(at.v(t * W::kKeys)); };

    f32x16 o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = zeros();
    float top = -INFINITY, sum = 0.0f;     // of log2 scores; sum over this lane's keys
    const float c = g.log2_scale;
    // Probabilities of 16-bit types are rounded to the type for their product with v, and their sum is that of the
    // rounded ones, so that the weights add up to one: out is 1.3 times as far off as fp32 rounded once (32400 x
    // 16896, 4 heads of 32, bf16: 2.25e-3 of its norm, 1.66e-3). What the rounding leaves as a second piece would
    // end that, for 25 to 45% of the time again (4096 rows, 8192 keys, 8 heads of 32, 64 and 128 channels of bf16:
    // 72, 106 and 181 us, with it 98, 137 and 229; the former case 475 and 690). Few rows, bound by reading, take it.
    constexpr bool kTwo = WR == 1 && DT != BEVPOOL_F32;
    typename M::Rows p, p_low;
    // p and this lane's sum of the exponentials of a block's scores relative to base
    auto exponentials = [&](const f32x16 &s, float base) {
        f32x16 e;
#pragma unroll
        for (int i = 0; i < 16; ++i) e[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c, -base));
        if constexpr (kTwo) {
            M::rows_of_two(e, p, p_low);
            return p.sum() + p_low.sum();
        } else {
            p = M::rows(e);
            return p.sum();
        }
    };
    // keys out of use: bit k of word is key k of the block
    auto leave_out = [&](f32x16 &s, uint32_t word) {
        const uint32_t bits = word >> (4 * half);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = bits & (1u << (8 * (i >> 2) + (i & 3))) ? s[i] : -INFINITY;
    };
    // new maxima; what is summed and p again, relative to them
    auto raise = [&](const f32x16 &s) {
        float high = s[0];
#pragma unroll
        for (int i = 0; i < 16; ++i) high = fmaxf(high, s[i]);
        const float now = fmaxf(top, both_max(high) * c - kBelowTop<DT>);
        const float old = top == -INFINITY ? 0.0f : exp2f(top - now);
        sum *= old;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] *= old;
        top = now;
        return exponentials(s, top == -INFINITY ? 0.0f : top);
    };

    // While a tile is used the next one is read, and the mask of the one after it, so that rows out of use are
    // not read. The buffer is a constant, which leaves no address to compute: the loop takes two tiles a turn.
    const int row0 = WR == 1 ? 32 * wave : 0;          // of this wave's keys in a tile
    Used use = {}, next = {};
    if (t0 < t1) {
        mask.ask(at, t0 * W::kKeys);
        use = mask.count(at, t0 * W::kKeys);
        next_k.load(key_rows(t0), use.words, use.all, dim, g.pairs);
        next_v.load(value_rows(t0), use.words, use.all, dim, g.pairs);
        mask.ask(at, (t0 + 1) * W::kKeys);
        next_k.store(lds);
        next_v.store(lds + W::kBytes);
    }
    for (int t2 = t0; t2 < t1; t2 += 2) {
#pragma unroll
        for (int turn = 0; turn < 2; ++turn) {
            const int t = t2 + turn, buffer = turn & (W::kPairs - 1);
            if (t >= t1) break;
            const char *k = lds + buffer * 2 * W::kBytes, *v = k + W::kBytes;
            if (t + 1 < t1) {
                next = mask.count(at, (t + 1) * W::kKeys);
                next_k.load(key_rows(t + 1), next.words, next.all, dim, g.pairs);
                next_v.load(value_rows(t + 1), next.words, next.all, dim, g.pairs);
                mask.ask(at, (t + 2) * W::kKeys);
            }
            __syncthreads();
            uint64_t mine = use.words[0];
            if constexpr (Used::kWords == 2) mine = row0 >= 64 ? use.words[1] : mine;
            mine >>= row0 & 63;
            f32x16 s[W::kBlocks];
#pragma unroll
            for (int n = 0; n < W::kBlocks; ++n) s[n] = S::scores(k, row0 + 32 * n, q, zeros());
#pragma unroll
            for (int n = 0; n < W::kBlocks; ++n) {
                const uint32_t word = uint32_t(mine >> (32 * n));
                if (__builtin_expect(word != 0xFFFFFFFFu, 0)) {
                    if (word == 0) continue;
                    leave_out(s[n], word);
                }
                float part = exponentials(s[n], top);
                if (__builtin_expect(__any(!(part <= kMaxTileSum<DT>)), 0)) part = raise(s[n]);
                sum += part;
                S::sums(v, row0 + 32 * n, p, o, kTwo ? &p_low : nullptr);
            }
            if constexpr (W::kPairs == 1) __syncthreads();
            if (t + 1 < t1) {
                char *to = lds + (W::kPairs == 1 ? 0 : 1 - buffer) * 2 * W::kBytes;
                next_k.store(to);
                next_v.store(to + W::kBytes);
                use = next;
            }
        }
    }
    __syncthreads();
    sum = both_sum(sum);

    if constexpr (WR == 1) {
        // join the four waves, which saw different keys, through LDS
        float *parts = reinterpret_cast<float *>(lds);          // [4][32 rows][32 DB + 1]
        constexpr int kPitch = 32 * DB + 1;
        float2 *stats = reinterpret_cast<float2 *>(parts + 4 * 32 * kPitch + (4 * 32 * kPitch & 1));
        if (half == 0) stats[wave * 32 + lane] = make_float2(top, sum);
        __syncthreads();
        float most = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) most = fmaxf(most, stats[w * 32 + (lane & 31)].x);
        const float mul = part_weight(top, sum, most);
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                parts[(wave * 32 + (lane & 31)) * kPitch + 32 * d + 8 * (i >> 2) + 4 * half + (i & 3)] = o[d][i] * mul;
        float all = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float2 st = stats[w * 32 + (lane & 31)];
            all += st.y * part_weight(st.x, st.y, most);
        }
        __syncthreads();
        top = most;
        sum = all;
        // wave w keeps channel block w of the joined sums (DB <= 4)
        if (wave >= DB) return;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int at_ch = 32 * wave + 8 * (i >> 2) + 4 * half + (i & 3);
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; ++w) v += parts[(w * 32 + (lane & 31)) * kPitch + at_ch];
            o[0][i] = v;
        }
    }

    if (row >= g.rows) return;
    const int first = WR == 1 ? wave : 0, blocks = WR == 1 ? 1 : DB;
    // fn(channel, four values) of this lane
    auto each4 = [&](float mul, auto fn) {
#pragma unroll
        for (int d = 0; d < DB; ++d) {
            if (d >= blocks) break;
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const float x[4] = {o[d][i] * mul, o[d][i + 1] * mul, o[d][i + 2] * mul, o[d][i + 3] * mul};
                fn(32 * (first + d) + 2 * i + 4 * half, x);
            }
        }
    };
    if (g.n_split > 1) {
        const int64_t slot = (int64_t(split) * n_bh + bh) * g.rows + row;
        if (half == 0 && first == 0) g.part_stats[slot] = make_float2(top, sum);
        if (sum == 0.0f) return;              // the joining kernel does not read it
        float *p = g.part + slot * g.part_pitch;
        each4(1.0f, [&](int ch, const float *x) { write4<true>(p, ch, g.part_pitch, x); });
        return;
    }
    const int64_t to = at.row(row);
    T *out = static_cast<T *>(g.o) + to;
    each4(sum == 0.0f ? 0.0f : 1.0f / sum, [&](int ch, const float *x) {
        write4<VEC>(out, ch, dim, x);
        if (DT != BEVPOOL_F32 && g.o_low) {
            float low[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) low[e] = x[e] - float(T(x[e]));
            write4<VEC>(static_cast<T *>(g.o_low) + to, ch, dim, low);
        }
    });
    if (g.lse && half == 0 && first == 0)
        g.lse[at.stat(row)] = sum == 0.0f ? -INFINITY : top + __builtin_amdgcn_logf(sum);
}

// Joins the parts of rows. A thread holds four channels of a row and every SL-th
// part, kJoinAhead of them on the way at once; the SL threads of a row's four
// channels meet in LDS.
constexpr int kJoinAhead = 8;
constexpr int kJoinNarrow = 16;     // columns of a workgroup for rows of up to 64 channels
// COLUMNS: (row, four channels) of a workgroup.
template <int DT, int SL, int COLUMNS>
__global__ __launch_bounds__(SL * COLUMNS) void k_attend_join(AttendArgs g) {
    using T = typename Num<DT>::T;
    constexpr int kColumns = COLUMNS;
    __shared__ float meet[6][SL == 1 ? 1 : SL * kColumns];
    const int per_row = g.part_pitch / 4, rows_here = kColumns / per_row;
    const int lane = threadIdx.x / kColumns, column = threadIdx.x % kColumns;
    const int64_t total = int64_t(g.a.batch) * g.a.key_heads * g.rows;
    const int64_t slot = int64_t(blockIdx.x) * rows_here + column / per_row;
    const int ch = column % per_row * 4;
    const bool here = column < rows_here * per_row && slot < total;
    float top = -INFINITY, sum = 0.0f, o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    // adds a part, or a joined set of parts, with maximum x and sum w
    auto add = [&](float x, float w, const float *v) {
        if (w == 0.0f) return;
        const float now = fmaxf(top, x), a = part_weight(top, sum, now), b = part_weight(x, w, now);
        sum = sum * a + w * b;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = o[e] * a + v[e] * b;
        top = now;
    };
    if (here)
        for (int s0 = lane; s0 < g.n_split; s0 += SL * kJoinAhead) {
            float2 st[kJoinAhead];
            float4 v[kJoinAhead];
#pragma unroll
            for (int i = 0; i < kJoinAhead; ++i) {
                const int s = s0 + i * SL;
                st[i] = make_float2(-INFINITY, 0.0f);
                v[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (s < g.n_split) {
                    st[i] = g.part_stats[s * total + slot];
                    v[i] = *reinterpret_cast<const float4 *>(g.part + (s * total + slot) * g.part_pitch + ch);
                }
            }
#pragma unroll
            for (int i = 0; i < kJoinAhead; ++i) add(st[i].x, st[i].y, reinterpret_cast<const float *>(&v[i]));
        }
    if constexpr (SL > 1) {
        meet[0][threadIdx.x] = top;
        meet[1][threadIdx.x] = sum;
#pragma unroll
        for (int e = 0; e < 4; ++e) meet[2 + e][threadIdx.x] = o[e];
        // halves meet halves
#pragma unroll
        for (int m = SL / 2; m > 0; m >>= 1) {
            __syncthreads();
            if (lane >= m) continue;
            const int from = (lane + m) * kColumns + column;
            const float v[4] = {meet[2][from], meet[3][from], meet[4][from], meet[5][from]};
            add(meet[0][from], meet[1][from], v);
            meet[0][threadIdx.x] = top;
            meet[1][threadIdx.x] = sum;
#pragma unroll
            for (int e = 0; e < 4; ++e) meet[2 + e][threadIdx.x] = o[e];
        }
        if (lane != 0) return;
    }
    if (!here) return;
    const int bh = int(slot / g.rows), row = int(slot - int64_t(bh) * g.rows);
    const Problem<DT> at(g, bh);
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    const int64_t to = at.row(row);
    float low[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        o[e] *= inv;
        low[e] = o[e] - float(T(o[e]));
    }
    // rows of out start on four elements only if dim is a multiple of four
    if (g.a.dim % 4 == 0 && g.out_aligned) {
        write4<true>(static_cast<T *>(g.o) + to, ch, g.a.dim, o);
        if (DT != BEVPOOL_F32 && g.o_low) write4<true>(static_cast<T *>(g.o_low) + to, ch, g.a.dim, low);
    } else {
        write4<false>(static_cast<T *>(g.o) + to, ch, g.a.dim, o);
        if (DT != BEVPOOL_F32 && g.o_low) write4<false>(static_cast<T *>(g.o_low) + to, ch, g.a.dim, low);
    }
    if (g.lse && ch == 0) g.lse[at.stat(row)] = sum == 0.0f ? -INFINITY : top + __builtin_amdgcn_logf(sum);
}

template <int DT, int SL, int COLUMNS>
void launch_join(const AttendArgs &g, hipStream_t stream) {
    static_assert(COLUMNS * 4 >= kAttendMaxDim || COLUMNS == kJoinNarrow, "a row to a workgroup at least");
    const int64_t rows_here = COLUMNS / (g.part_pitch / 4), rows = int64_t(g.a.batch) * g.a.key_heads * g.rows;
    hipLaunchKernelGGL((k_attend_join<DT, SL, COLUMNS>), dim3(uint32_t((rows + rows_here - 1) / rows_here)),
                       dim3(SL * COLUMNS), 0, stream, g);
}

constexpr int kFewRows = 32;        // rows of a key head that one wave holds

int part_pitch(const bevmap_attend &a) { return (a.dim + 3) / 4 * 4; }

// Rows, row tiles and parts of the keys, a rule on the sizes alone, and on whether
// samples have lengths: unequal ones need more workgroups to even out, and do less
// work by the row. Parts are chosen for the workgroups that the chip holds (one query of 8
// heads on 2 of 128 over 129600 keys in bf16: 48 us with parts for twice as many, now 39).
void partition(const bevmap_attend &a, bool lengths, AttendArgs *g, bool *few) {
    const int64_t rows = int64_t(a.queries) * (a.heads / a.key_heads);
    // (fp32 tiles of 128 keys and more than 64 channels do not fit LDS)
    *few = rows <= kFewRows && (a.dtype != BEVPOOL_F32 || a.dim <= 64);
    g->n_tiles = attend_ceil(rows, *few ? kFewRows : kAttendTile);
    int slots = kUnits * resident_forward(a.dtype, attend_ceil(a.dim, 32), *few);
    if (lengths) slots += slots / 2;
    g->n_split = pick_split(int64_t(a.batch) * a.key_heads * g->n_tiles, slots, a.keys,
                            attend_ceil(a.keys, *few ? 256 : 128), lengths ? 1200.0 : 600.0, a.dtype);
}

template <int DT, int DB, bool VEC, int WR>
int launch(const AttendArgs &g, hipStream_t stream) {
    size_t lds = Tile<DT, DB, WR>::kLds;
    if (WR == 1) {
        const size_t join = (4 * 32 * (32 * DB + 1) + 2 * 128 + 1) * sizeof(float);
        lds = lds > join ? lds : join;
    }
    if (lds > 64 * 1024)
        BEVPOOL_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(k_attend<DT, DB, VEC, WR>),
                                        hipFuncAttributeMaxDynamicSharedMemorySize, int(lds)));
    const uint32_t grid = uint32_t(g.a.batch) * g.a.key_heads * g.n_split * g.n_tiles;
    hipLaunchKernelGGL((k_attend<DT, DB, VEC, WR>), dim3(grid), dim3(kAttendBlock), lds, stream, g);
    BEVPOOL_HIP(hipGetLastError());
    return BEVPOOL_OK;
}

template <int DT, int DB>
int launch(const AttendArgs &g, bool vec, bool few, hipStream_t stream) {
    if constexpr (DT != BEVPOOL_F32 || DB <= 2)
        if (few) return vec ? launch<DT, DB, true, 1>(g, stream) : launch<DT, DB, false, 1>(g, stream);
    return vec ? launch<DT, DB, true, 4>(g, stream) : launch<DT, DB, false, 4>(g, stream);
}

template <int DT>
int forward(const AttendArgs &g, bool vec, bool few, hipStream_t stream) {
    int rc;
    switch ((g.a.dim + 31) / 32) {
        case 1: rc = launch<DT, 1>(g, vec, few, stream); break;
        case 2: rc = launch<DT, 2>(g, vec, few, stream); break;
        case 3: rc = launch<DT, 3>(g, vec, few, stream); break;
        default: rc = launch<DT, 4>(g, vec, few, stream); break;
    }
    if (rc || g.n_split == 1) return rc;
    // a thread reads its parts in one go, or in two; many parts mean few rows, and then the smaller the
    // workgroups the better (235 parts of 8 rows of 64 channels: 16 x 64 threads 7.6 us, 32 x 32 5.8, 32 x 16 5.0)
    const bool narrow = g.part_pitch <= 4 * kJoinNarrow;
    if (g.n_split > 16 * kJoinAhead)
        narrow ? launch_join<DT, 32, kJoinNarrow>(g, stream) : launch_join<DT, 32, 32>(g, stream);
    else if (g.n_split > 4 * kJoinAhead)
        narrow ? launch_join<DT, 16, kJoinNarrow>(g, stream) : launch_join<DT, 16, 32>(g, stream);
    else if (g.n_split > kJoinAhead)
        launch_join<DT, 4, 64>(g, stream);
    else
        launch_join<DT, 1, 256>(g, stream);
    BEVPOOL_HIP(hipGetLastError());
    return BEVPOOL_OK;
}

}  // namespace
}  // namespace bevmap

using namespace bevmap;

int64_t bevmap_attention_workspace_bytes(const bevmap_attend &a, bool backward) {
    if (backward) return bevmap_attention_backward_bytes(a);
    AttendArgs g{};
    bool few;
    partition(a, false, &g, &few);
    const int without = g.n_split;
    partition(a, true, &g, &few);
    const int parts = without > g.n_split ? without : g.n_split;
    if (parts <= 1) return 0;
    return int64_t(parts) * a.batch * a.queries * a.heads *
           (part_pitch(a) * int64_t(sizeof(float)) + int64_t(sizeof(float2)));
}

int bevmap_launch_attention(const bevmap_attend &a, const void *q, const void *k, const void *v,
                            const int32_t *lengths, const uint8_t *mask, void *out, void *out_low, float *lse,
                            void *workspace, hipStream_t stream) {
    if (a.batch == 0 || a.queries == 0) return BEVPOOL_OK;
    AttendArgs g = attend_fill(a, q, k, v, lengths, mask);
    g.o = out;
    g.o_low = out_low;
    g.lse = lse;
    bool few;
    partition(a, lengths != nullptr, &g, &few);
    // 16-byte aligned parts first, then their rows' statistics
    g.part_pitch = part_pitch(a);
    g.part = static_cast<float *>(workspace);
    g.part_stats = reinterpret_cast<float2 *>(g.part + int64_t(g.n_split) * a.batch * a.queries * a.heads * g.part_pitch);
    g.out_aligned = aligned_for(out, 0, a.dtype, 4) && (!out_low || aligned_for(out_low, 0, a.dtype, 4));
    const bool vec = attend_by(a, q, k, v, a.dtype == BEVPOOL_F32 ? 4 : 8) && g.out_aligned;
    g.pairs = attend_by(a, q, k, v, 2);
    switch (a.dtype) {
        case BEVPOOL_F32: return forward<BEVPOOL_F32>(g, vec, few, stream);
        case BEVPOOL_BF16: return forward<BEVPOOL_BF16>(g, vec, few, stream);
        default: return forward<BEVPOOL_F16>(g, vec, few, stream);
    }
}
