// Device pieces shared by the attention kernels (attention.hip, attention_backward.hip).
//
// The queries of the heads that share a key head are the rows of one problem:
// row r = query * group + head of the group, against that key head's keys. All
// products run on the matrix cores in 32x32 blocks, held so that no result has
// to change lanes to become the next product's operand:
//
// - A block of scores is formed as keys x rows (or rows x keys): with x the tile
//   in LDS and y in registers, mma gives lane l column l % 32 (one row of y) and
//   the 16 tile rows 8 (i / 4) + 4 (l / 32) + i % 4, i = 0..15.
// - The second product contracts over those tile rows. Its order of summation is
//   free, so step s takes the rows that a lane already holds, and only the
//   tile's operand has to follow that order: read transposed from LDS,
//   four tile rows at a time.
#pragma once

#include <math.h>

#include "mapops.h"

namespace bevmap {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kAttendBlock = 256;       // four waves

struct AttendArgs {
    bevmap_attend a;
    const void *q, *k, *v, *dout, *out, *out_low;
    const int32_t *lengths;
    const uint8_t *mask;
    void *o, *o_low, *dq, *dk, *dv;
    float *lse, *delta;
    float *part;                  // fp32 parts of a split axis
    float2 *part_stats;           // forward: (maximum, sum) of a part's rows
    int32_t part_pitch;           // floats from row to row of a part
    bool pairs;                   // rows can be read two elements at a time
    bool out_aligned;             // four elements of out and out_low can be written at a time
    int32_t group, rows;          // heads that share a key head, queries * group
    bevpool::FastDiv by_group;
    int32_t n_tiles, n_split;     // tiles of the axis that a workgroup owns, parts of the other
    float scale, log2_scale;      // |scale|, |scale| log2(e); 1 and log2(e) where scale is 0
    float sign;                   // of scale, 0 where it is 0: q is multiplied by it
};

namespace {

using f32x16 = float __attribute__((ext_vector_type(16)));
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
using u32x2 = uint32_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ f32x16 zeros() {
    f32x16 z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.0f;
    return z;
}

// fp32 goes through the bf16 matrix cores: x is the sum of three bf16 pieces, exactly
// (8 + 8 + 8 of its 24 bits), each what the ones before leave rounded to nearest, so that
// a second piece is at most 2^-8 of its number and a third 2^-17. Six of the nine products
// of pieces are formed; the others together are at most 2^-24 of the product, of either
// sign. (Pieces cut off towards zero take 3 to 7% less time, but leave out up to 2^-21,
// all with the product's own sign.) That takes 6 / 16 of the time of the fp32 matrix
// instructions (32x32x16 in 32 cycles, 32x32x2 in 64): 143, 181 and 150 TFLOP/s forward
// at 32, 64 and 128 channels (4096 rows, 8192 keys, 8 heads), where those reached 118,
// 127 and 112.
//
// A chunk is 16 bytes of a row in memory: 8 elements of a 16-bit type, 4 of fp32. In
// step s of a product, K = 16, the two half waves hold elements 16 s + 8 half ..
// Two fp32 numbers cut off to bf16, and what is left of one.
__device__ __forceinline__ uint32_t cut_pair(float x, float y) {
    return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302);
}
__device__ __forceinline__ float left_of(float x) { return x - __uint_as_float(__float_as_uint(x) & 0xFFFF0000u); }

template <int DT>
struct Mma {
    using T = typename Num<DT>::T;
    static constexpr int kElems = 8;
    using Vec = T __attribute__((ext_vector_type(8)));
    // a block's 16 values of a lane as the second product's operand, rounded to T
    struct Rows {
        u32x4 half[2];
        // their sum, as rounded
        __device__ __forceinline__ float sum() const {
            float a = 0.0f, b = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                a = pair_sum(half[0][i], a);
                b = pair_sum(half[1][i], b);
            }
            return a + b;
        }
        // whether some value of fp16 is 2 or more: the exponent's highest bit
        __device__ __forceinline__ bool reaches_two() const {
            const u32x4 any = half[0] | half[1];
            return ((any[0] | any[1] | any[2] | any[3]) & 0x40004000u) != 0;
        }
    };
    // What rows(p) left over: p - rows(p) to another 8 or 11 bits. rows of such a pair cut p off instead of rounding it.
    static __device__ __forceinline__ void rows_of_two(const f32x16 &p, Rows &high, Rows &low) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            Vec l;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const float x = p[8 * s + e], y = p[8 * s + e + 1];
                uint32_t both;
                if constexpr (DT == BEVPOOL_BF16) {
                    both = cut_pair(x, y);
                    l[e] = T(left_of(x));
                    l[e + 1] = T(left_of(y));
                } else {
                    const auto cut = __builtin_amdgcn_cvt_pkrtz(x, y);
                    both = __builtin_bit_cast(uint32_t, cut);
                    l[e] = T(x - float(cut[0]));
                    l[e + 1] = T(y - float(cut[1]));
                }
                high.half[s][e / 2] = both;
            }
            low.half[s] = __builtin_bit_cast(u32x4, l);
        }
    }
    static __device__ __forceinline__ float pair_sum(uint32_t v, float c) {
        using Two = T __attribute__((ext_vector_type(2)));
        const Two ones = {T(1.0f), T(1.0f)};
        if constexpr (DT == BEVPOOL_BF16)
            return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(Two, v), ones, c, false);
        else
            return __builtin_amdgcn_fdot2(__builtin_bit_cast(Two, v), ones, c, false);
    }
    static __device__ __forceinline__ f32x16 mul(u32x4 a, u32x4 b, f32x16 c) {
        if constexpr (DT == BEVPOOL_BF16)
            return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(Vec, a), __builtin_bit_cast(Vec, b), c,
                                                           0, 0, 0);
        else
            return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(Vec, a), __builtin_bit_cast(Vec, b), c, 0,
                                                          0, 0);
    }
    static __device__ __forceinline__ Rows rows(const f32x16 &p) {
        Rows r;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            Vec v;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = T(p[8 * s + e]);
            r.half[s] = __builtin_bit_cast(u32x4, v);
        }
        return r;
    }
};
// The three pieces of a pair of fp32 numbers. ANY: the numbers may be so large that
// bf16 would round them to infinity, and are held to its largest there.
template <bool ANY>
__device__ __forceinline__ void three_pieces(float x, float y, uint32_t *piece) {
    using Two = __bf16 __attribute__((ext_vector_type(2)));
    constexpr float kMost = 0x1.FEp127f;
    Two p = {__bf16(ANY ? __builtin_amdgcn_fmed3f(x, -kMost, kMost) : x),
             __bf16(ANY ? __builtin_amdgcn_fmed3f(y, -kMost, kMost) : y)};
    piece[0] = __builtin_bit_cast(uint32_t, p);
#pragma unroll
    for (int k = 1; k < 3; ++k) {
        x -= __uint_as_float(piece[k - 1] << 16);
        y -= __uint_as_float(piece[k - 1] & 0xFFFF0000u);
        p = Two{__bf16(x), __bf16(y)};
        piece[k] = __builtin_bit_cast(uint32_t, p);
    }
}
template <>
struct Mma<BEVPOOL_F32> {
    using T = float;
    static constexpr int kElems = 4;
    struct Rows {
        u32x4 piece[3][2];
        float total;
        __device__ __forceinline__ float sum() const { return total; }
    };
    using Piece = Mma<BEVPOOL_BF16>;
    // c += a b, the least products first; a[i], b[i]: the pieces of a step's operands
    static __device__ __forceinline__ f32x16 mul(const u32x4 *a, u32x4 b0, u32x4 b1, u32x4 b2, f32x16 c) {
        c = Piece::mul(a[2], b0, c);
        c = Piece::mul(a[0], b2, c);
        c = Piece::mul(a[1], b1, c);
        c = Piece::mul(a[1], b0, c);
        c = Piece::mul(a[0], b1, c);
        return Piece::mul(a[0], b0, c);
    }
    // ANY: p may be of any size (three_pieces)
    template <bool ANY = false>
    static __device__ __forceinline__ Rows rows(const f32x16 &p) {
        Rows r;
        float a[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < 16; ++i) a[i & 3] += p[i];
        r.total = (a[0] + a[1]) + (a[2] + a[3]);
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            uint32_t piece[3];
            three_pieces<ANY>(p[i], p[i + 1], piece);
#pragma unroll
            for (int k = 0; k < 3; ++k) r.piece[k][i >> 3][(i & 7) >> 1] = piece[k];
        }
        return r;
    }
    static __device__ __forceinline__ void rows_of_two(const f32x16 &p, Rows &high, Rows &) { high = rows<true>(p); }
};

// Layout of a tile in LDS: rows of CH chunks (a power of two; of fp32 one such row
// for each piece, side by side), chunk c of row r at chunk c ^ turn(r). Sixteen
// consecutive rows read at one chunk, and four consecutive rows read along 64 bytes,
// then fall into distinct banks.
template <int CH>
__device__ __forceinline__ int turn(int row) {
    if constexpr (CH <= 4) return (row >> 2) & 3;
    if constexpr (CH == 8) return ((row >> 1) & 1) << 2 | ((row >> 2) & 3);
    return (row & 3) << 2 | ((row >> 2) & 3);
}

constexpr int pow2_chunks(int n) { return n <= 4 ? 4 : n <= 8 ? 8 : 16; }

// One chunk of a row: elements c * kElems.. of dim, zeros past dim. VEC: rows
// start on 16-byte boundaries and dim is a multiple of the chunk. Else elements are
// read one by one, or, with 16-bit types, by twos where rows start on 4 bytes and dim
// is even (pairs, uniform).
template <int DT, bool VEC>
__device__ __forceinline__ u32x4 load_chunk(const typename Num<DT>::T *row, int c, int dim, bool pairs) {
    using T = typename Num<DT>::T;
    constexpr int E = Mma<DT>::kElems;
    u32x4 out = {0, 0, 0, 0};
    if constexpr (VEC) {
        if (c * E < dim) out = *reinterpret_cast<const u32x4 *>(row + c * E);
    } else if (DT != BEVPOOL_F32 && pairs) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c * E + 2 * e < dim) out[e] = *reinterpret_cast<const uint32_t *>(row + c * E + 2 * e);
    } else {
        T v[E];
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = c * E + e < dim ? row[c * E + e] : T(0.0f);
        out = __builtin_bit_cast(u32x4, v);
    }
    return out;
}

// DB blocks of 32 channels of type DT.
template <int DT, int DB>
struct Shape {
    using M = Mma<DT>;
    using T = typename M::T;
    static constexpr int kPieces = DT == BEVPOOL_F32 ? 3 : 1;
    static constexpr int kUsed = DB * 32 / M::kElems;        // chunks of a row in memory
    static constexpr int kChunks = pow2_chunks(DB * 4);      // of a row's piece in LDS
    static constexpr int kPieceBytes = kChunks * 16;
    static constexpr int kRowBytes = kPieces * kPieceBytes;
    static constexpr int kSteps = 2 * DB;
    static constexpr int kOperand = kPieces * kSteps;        // registers of a row as an operand: [piece][step]

    // Bytes of 8 elements from 8 c of a row's first piece in LDS.
    static __device__ __forceinline__ int chunk_at(int row, int c) {
        return row * kRowBytes + (c ^ turn<kChunks>(row)) * 16;
    }
    // Chunk c of a row, as it was in memory, to LDS.
    static __device__ __forceinline__ void put(char *tile, int row, int c, u32x4 v) {
        if constexpr (DT != BEVPOOL_F32) {
            *reinterpret_cast<u32x4 *>(tile + chunk_at(row, c)) = v;
        } else {
            uint32_t piece[2][3];
#pragma unroll
            for (int i = 0; i < 2; ++i)
                three_pieces<true>(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]), piece[i]);
            char *to = tile + chunk_at(row, c >> 1) + (c & 1) * 8;
#pragma unroll
            for (int k = 0; k < 3; ++k)
                *reinterpret_cast<u32x2 *>(to + k * kPieceBytes) = u32x2{piece[0][k], piece[1][k]};
        }
    }
    // A row in memory as an operand of scores().
    template <bool VEC>
    static __device__ __forceinline__ void operand(const T *row, int half, int dim, bool pairs, u32x4 *y) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            if constexpr (DT != BEVPOOL_F32) {
                y[s] = load_chunk<DT, VEC>(row, 2 * s + half, dim, pairs);
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const u32x4 v = load_chunk<DT, VEC>(row, 4 * s + 2 * half + i, dim, pairs);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        uint32_t piece[3];
                        three_pieces<true>(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]), piece);
#pragma unroll
                        for (int k = 0; k < 3; ++k) y[k * kSteps + s][2 * i + j] = piece[k];
                    }
                }
            }
        }
    }

    // acc[32 tile rows from row0][32 columns] += tile x y^T over the channels.
    static __device__ __forceinline__ f32x16 scores(const char *tile, int row0, const u32x4 *y, f32x16 acc) {
        const int lane = threadIdx.x & 63, row = row0 + (lane & 31), half = lane >> 5;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const char *at = tile + chunk_at(row, 2 * s + half);
            u32x4 x[kPieces];
#pragma unroll
            for (int k = 0; k < kPieces; ++k) x[k] = *reinterpret_cast<const u32x4 *>(at + k * kPieceBytes);
            if constexpr (DT != BEVPOOL_F32)
                acc = M::mul(x[0], y[s], acc);
            else
                acc = M::mul(x, y[s], y[kSteps + s], y[2 * kSteps + s], acc);
        }
        return acc;
    }

    // acc[d][32 channels from 32 d][32 columns] += tile^T x p over the 32 tile rows from row0; with low, += tile^T x low.
    static __device__ __forceinline__ void sums(const char *tile, int row0, const typename M::Rows &p, f32x16 *acc,
                                                const typename M::Rows *low = nullptr) {
        using s4 = short __attribute__((ext_vector_type(4)));
        using lds4 = __attribute__((address_space(3))) s4;
        // ds_read_b64_tr_b16: in 16 lanes, lane t names 4 elements of row t / 4 at columns 4 (t % 4) and
        // gets column t of the four rows
        const int lane = threadIdx.x & 63, half = lane >> 5, t = lane & 15, sub = (lane >> 4) & 1;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                u32x4 x[kPieces];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int row = row0 + 16 * s + 8 * e + 4 * half + (t >> 2);
                    const int col = 4 * d + 2 * sub + ((t & 3) >> 1);       // in chunks
                    const char *at = tile + chunk_at(row, col) + (t & 1) * 8;
#pragma unroll
                    for (int k = 0; k < kPieces; ++k) {
                        const u32x2 r = __builtin_bit_cast(
                            u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(at + k * kPieceBytes)));
                        x[k][2 * e] = r[0];
                        x[k][2 * e + 1] = r[1];
                    }
                }
                if constexpr (DT != BEVPOOL_F32) {
                    acc[d] = M::mul(x[0], p.half[s], acc[d]);
                    if (low) acc[d] = M::mul(x[0], low->half[s], acc[d]);
                } else {
                    acc[d] = M::mul(x, p.piece[0][s], p.piece[1][s], p.piece[2][s], acc[d]);
                }
            }
        }
    }
};

// The largest of a lane and the lane 32 away, and their sum.
__device__ __forceinline__ float both_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float both_sum(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// fp16 ends at 2^-24, so its probabilities and their gradients are held multiplied by
// powers of two: probabilities by 2^kRaised, and a row's or key's gradients by one of its
// own, 2^lift, that starts too large and is lowered when a value reaches 2.
template <int DT>
constexpr float kRaised = DT == BEVPOOL_F16 ? 12.0f : 0.0f;
constexpr float kFirstLift = 60.0f;
__device__ __forceinline__ float power_of_two(float n) { return ldexpf(1.0f, int(n)); }

// Lowers the lifts of the lanes' columns where x, of them and in both half waves, reaches 2;
// returns what to multiply the column's sums by, x being multiplied here. To 1/8: what
// comes is seldom 16 times the largest so far.
__device__ __forceinline__ float lower(f32x16 &x, float &lift) {
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) most = fmaxf(most, fabsf(x[i]));
    most = both_max(most);
    const int by = most >= 2.0f ? -3 - __builtin_amdgcn_frexp_expf(most) : 0;
    lift += float(by);
    const float mul = ldexpf(1.0f, by);
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] *= mul;
    return mul;
}

// Four consecutive channels of a row from channel ch, of dim; VEC: they are
// aligned and dim is a multiple of four.
template <bool VEC, class T>
__device__ __forceinline__ void write4(T *row, int ch, int dim, const float *v) {
    if constexpr (VEC) {
        if (ch < dim) store_n<T, 4>(row + ch, v);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (ch + e < dim) row[ch + e] = T(v[e]);
    }
}

// Sample, key head and its addresses.
template <int DT>
struct Problem {
    using T = typename Num<DT>::T;
    const AttendArgs &g;
    int b, hk, len;
    __device__ __forceinline__ Problem(const AttendArgs &g_, int bh) : g(g_) {
        b = bh / g.a.key_heads;
        hk = bh - b * g.a.key_heads;
        len = g.lengths ? min(max(g.lengths[b], 0), g.a.keys) : g.a.keys;
    }
    __device__ __forceinline__ void split_row(int r, int &i, int &h) const {
        i = int(bevpool::fdiv(uint32_t(r), g.by_group));
        h = hk * g.group + r - i * g.group;
    }
    __device__ __forceinline__ const T *q(int i, int h) const {
        return static_cast<const T *>(g.q) + b * g.a.q_batch + i * g.a.q_row + h * g.a.q_head;
    }
    __device__ __forceinline__ const T *q(int r) const {
        int i, h;
        split_row(r, i, h);
        return q(i, h);
    }
    __device__ __forceinline__ const T *k(int j) const {
        return static_cast<const T *>(g.k) + b * g.a.k_batch + hk * g.a.k_head + j * g.a.k_row;
    }
    __device__ __forceinline__ const T *v(int j) const {
        return static_cast<const T *>(g.v) + b * g.a.v_batch + hk * g.a.v_head + j * g.a.v_row;
    }
    __device__ __forceinline__ int64_t row(int i, int h) const {      // of out and its like, in elements
        return ((int64_t(b) * g.a.queries + i) * g.a.heads + h) * g.a.dim;
    }
    __device__ __forceinline__ int64_t row(int r) const {
        int i, h;
        split_row(r, i, h);
        return row(i, h);
    }
    __device__ __forceinline__ int64_t stat(int r) const {     // of lse, delta
        int i, h;
        split_row(r, i, h);
        return (int64_t(b) * g.a.heads + h) * g.a.queries + i;
    }
    __device__ __forceinline__ int64_t key(int j) const {      // of the gradients of k and v
        return ((int64_t(b) * g.a.keys + j) * g.a.key_heads + hk) * g.a.dim;
    }
    // Which of 64 keys are in use, bit by bit; every lane of a wave asks for its own key.
    __device__ __forceinline__ int ask(int j) const {
        return j < len ? (g.mask ? g.mask[b * g.a.mask_batch + j] : 1) : 0;
    }
};

// Work of a workgroup: item n of `per` of problem bh (sample, key head). Workgroups are
// dealt to the 8 XCDs round-robin, and a problem's workgroups share its keys and
// values, so problem bh's all go to XCD bh % 8, which also spreads samples of
// unequal length; what is left of the last 8 problems is cut into eighths.
__device__ __forceinline__ void work_of(int n_bh, int per, int &bh, int &n) {
    int id = blockIdx.x;
    const int whole = (n_bh & ~7) * per;
    if (id < whole) {
        const int k = id >> 3, round = k / per;
        bh = 8 * round + (id & 7);
        n = k - round * per;
        return;
    }
    id -= whole;
    const int left = (n_bh & 7) * per, q = left >> 3, r = left & 7, x = id & 7, k = id >> 3;
    id = x < r ? x * (q + 1) + k : r * (q + 1) + (x - r) * q + k;
    const int p = id / per;
    bh = (n_bh & ~7) + p;
    n = id - p * per;
}

// Rows of a tile on their way from memory to LDS, a few chunks to a thread; rows are
// `stride` bytes apart. Chunks past the last channel are copies of the last one:
// they meet zeros in the other operand, or their results are not written.
template <int DT, int DB, bool VEC, int ROWS>
struct Stage {
    using S = Shape<DT, DB>;
    using T = typename S::T;
    static constexpr int kLoads = (ROWS * S::kUsed + kAttendBlock - 1) / kAttendBlock;
    static constexpr bool kEven = ROWS * S::kUsed % kAttendBlock == 0;      // no thread is left over
    u32x4 reg[kLoads];
    uint32_t at[kLoads];        // bytes from the tile's first row

    static __device__ __forceinline__ int row(int i) { return (threadIdx.x + i * kAttendBlock) / S::kUsed; }
    static __device__ __forceinline__ int chunk(int i) { return (threadIdx.x + i * kAttendBlock) % S::kUsed; }

    __device__ __forceinline__ Stage(uint32_t stride, int dim) {
        const int last = (dim - 1) / S::M::kElems;
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            at[i] = uint32_t(row(i)) * stride + (VEC ? uint32_t(min(chunk(i), last)) * 16 : 0);
    }
    // base: the tile's first row (uniform). words: its rows in use, the others are
    // not read and count as zeros; all: whether every row is.
    template <int WORDS>
    __device__ __forceinline__ void load(const char *base, const uint64_t (&words)[WORDS], bool all, int dim,
                                         bool pairs) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = row(i);
            const bool there = kEven || r < ROWS;
            uint64_t word = words[0];
            if constexpr (WORDS == 2) word = r >= 64 ? words[1] : word;
            if constexpr (VEC) {
                if (all) {
                    if (there) reg[i] = *reinterpret_cast<const u32x4 *>(base + at[i]);
                } else {
                    reg[i] = u32x4{0, 0, 0, 0};
                    if (there && (word >> (r & 63)) & 1) reg[i] = *reinterpret_cast<const u32x4 *>(base + at[i]);
                }
            } else {
                reg[i] = u32x4{0, 0, 0, 0};
                if (there && (word >> (r & 63)) & 1)
                    reg[i] = load_chunk<DT, false>(reinterpret_cast<const T *>(base + at[i]), chunk(i), dim, pairs);
            }
        }
    }
    __device__ __forceinline__ void store(char *tile) const {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = row(i);
            if (!kEven && r >= ROWS) break;
            S::put(tile, r, chunk(i), reg[i]);
        }
    }
};

// The keys in use of a tile of KEYS keys, a bit to a key.
template <int KEYS>
struct InUse {
    static constexpr int kWords = KEYS <= 64 ? 1 : KEYS / 64;
    static constexpr uint64_t kFull = KEYS >= 64 ? ~0ull : (1ull << (KEYS & 63)) - 1;
    uint64_t words[kWords];
    bool all;
};
// ask() sends for the mask of the tile at key j0, count() makes the tile's words of it.
template <int KEYS>
struct Mask {
    using Tile = InUse<KEYS>;
    int used[Tile::kWords];
    template <class P>
    __device__ __forceinline__ void ask(const P &at, int j0) {
        const int lane = threadIdx.x & 63;
        if (at.g.mask)
#pragma unroll
            for (int w = 0; w < Tile::kWords; ++w) used[w] = KEYS >= 64 || lane < KEYS ? at.ask(j0 + 64 * w + lane) : 0;
    }
    template <class P>
    __device__ __forceinline__ Tile count(const P &at, int j0) const {
        Tile t;
        t.all = true;
#pragma unroll
        for (int w = 0; w < Tile::kWords; ++w) {
            const int there = at.len - j0 - 64 * w;
            t.words[w] = at.g.mask ? __ballot(used[w] != 0)
                                   : there >= 64 ? Tile::kFull : there <= 0 ? 0ull : Tile::kFull & ((1ull << there) - 1);
            t.all = t.all && t.words[w] == Tile::kFull;
        }
        return t;
    }
};

inline int attend_ceil(int64_t a, int64_t b) { return int((a + b - 1) / b); }

// Parts that `walk` keys or rows are split into for `whole` workgroups that own the
// others, where `slots` run at once: the fewest rounds of workgroups by parts of the
// work, against the writing and joining of parts. A part's are `join` / walk of all the
// work: it moves 8 bytes of a row and channel (at 3 TB/s), where the forward takes
// about 150 ns of a SIMD for 32 rows, 32 keys and 32 channels, which makes join 600;
// fp32 takes four times as long.
inline int pick_split(int64_t whole, int slots, int64_t walk, int64_t most, double join, int dtype) {
    if (whole <= 0 || walk <= 0) return 1;
    if (dtype == BEVPOOL_F32) join *= 0.25;
    const double part = join / double(walk) * double(whole) / slots;
    int64_t best = 1;
    double least = double((whole + slots - 1) / slots);
    for (int rounds = 1; rounds <= 3; ++rounds) {
        // the most parts of so many rounds, or fewer where rounds / s + s * part is least
        int64_t s = rounds * int64_t(slots) / whole, fewer = int64_t(sqrt(rounds / part) + 0.5);
        if (s > fewer) s = fewer;
        if (s > most) s = most;
        if (s < 2) continue;
        const double cost = double((whole * s + slots - 1) / slots) / double(s) + double(s) * part;
        if (cost < least * 0.98) {
            least = cost;
            best = s;
        }
    }
    return int(best);
}
constexpr int kUnits = 256;     // compute units

// Waves of a SIMD, which is workgroups of a compute unit, that the registers allow by
// blocks of 32 channels; the kernels' launch bounds hold them to it. Those of the forward
// may be fewer by their LDS (resident_forward()).
constexpr int kLdsBytes = 160 * 1024;   // of a compute unit
constexpr int waves_forward(int dt, int db) { return db == 1 ? 4 : db == 2 ? 3 : db == 3 || dt != BEVPOOL_F32 ? 2 : 1; }
constexpr int waves_few(int dt, int db) { return db == 4 || (db == 3 && dt == BEVPOOL_F32) ? 1 : 2; }
constexpr int waves_dq(int dt, int db) {
    return dt == BEVPOOL_F32 ? (db == 1 ? 3 : db == 2 ? 2 : 1) : (db == 1 ? 4 : db == 2 ? 3 : 2);
}
constexpr int waves_dkv(int dt, int db) { return dt == BEVPOOL_F32 ? (db == 1 ? 2 : 1) : db == 1 ? 3 : db <= 3 ? 2 : 1; }

AttendArgs attend_fill(const bevmap_attend &a, const void *q, const void *k, const void *v, const int32_t *lengths,
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
    g.by_group = bevpool::make_fastdiv(uint32_t(g.group));
    g.scale = a.scale == 0.0f ? 1.0f : a.scale < 0.0f ? -a.scale : a.scale;
    g.log2_scale = g.scale * kLog2e;
    g.sign = a.scale == 0.0f ? 0.0f : a.scale < 0.0f ? -1.0f : 1.0f;
    return g;
}

// Whether rows can be read n elements at a time.
bool attend_by(const bevmap_attend &a, const void *q, const void *k, const void *v, int e) {
    auto ok = [&](const void *p, int64_t batch, int64_t row, int64_t head, int rows, int heads) {
        return aligned_for(p, a.batch > 1 ? batch : 0, a.dtype, e) && aligned_for(p, rows > 1 ? row : 0, a.dtype, e) &&
               aligned_for(p, heads > 1 ? head : 0, a.dtype, e);
    };
    return a.dim % e == 0 && ok(q, a.q_batch, a.q_row, a.q_head, a.queries, a.heads) &&
           ok(k, a.k_batch, a.k_row, a.k_head, a.keys, a.key_heads) &&
           ok(v, a.v_batch, a.v_row, a.v_head, a.keys, a.key_heads);
}

}  // namespace
}  // namespace bevmap
