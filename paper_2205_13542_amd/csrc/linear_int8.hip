// Product of 8-bit integers with a scale for each token and each output channel
// (bevmap_linear_int8):
//
//   y[m][n] = x_scale[m] * w_scale[n] * sum_k x[m][k] w[n][k] + bias[n].
//
// Sums are 32-bit integers and exact; fp32 and one rounding follow. Both operands lie
// along k, so 16 bytes of a row are what a lane of the matrix cores takes
// (v_mfma_i32_32x32x32_i8, 16x16x64). The weights are the instruction's rows and the
// tokens its columns: a lane then holds neighbouring channels of one token, in the order
// in which y lies.
//
// Two forms. Tiles: a workgroup stages kStep bytes of its rows and channels in LDS, two
// stages in turn, the next on its way (past the registers, where rows are 16-byte
// aligned) while the matrix cores work: 16896 x 2048 x 4096 (tokens, k, channels) takes 150
// to 161 us, 8192^3 468, 2350 TOP/s (a library product without scales 170 and 445). Rows of
// any other alignment go through the registers, with no branch of a lane's own on the way, so
// that all loads of a stage are under way at a time: 16390 x 1025 x 1021 takes 38 to 42 us. Few
// tokens: the weights are what is read, so a workgroup takes 16 channels, its waves share out
// k and join their sums in LDS: 64 x 4096 x 2048 takes 5.1 us.
#include "mapops.h"

namespace bevmap {
namespace {

using i32x4 = int32_t __attribute__((ext_vector_type(4)));
using i32x16 = int32_t __attribute__((ext_vector_type(16)));

constexpr int kRun = 128;               // bytes of k that a wave of the form for few tokens takes at once
constexpr int kUnits = 256;             // compute units
constexpr int kGroup = 4;               // tiles of tokens that are walked before the next tile of features

struct LinearArgs {
    const int8_t *x, *w;
    const float *x_scale, *w_scale, *bias;
    void *y;
    int64_t ldx, ldw;
    int32_t M, N, K;
    int32_t m_tiles, n_tiles, y_dtype;
    bool wide;                          // rows of y lie at 16 bytes, in whole accesses
};

__device__ const uint4 kNothing = {0, 0, 0, 0};     // what lies past the end of k

// 16 bytes of a row of K from k on, at any alignment; where the row ends before them, its
// last 16 (all of a row shorter than that, and zeros), which settle_chunk then moves.
__device__ __forceinline__ i32x4 load_chunk(const int8_t *row, int k, int K) {
    i32x4 v = {0, 0, 0, 0};
    if (K >= 16) {
        __builtin_memcpy(&v, row + min(k, K - 16), 16);
    } else {
        int8_t b[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) b[i] = i < K ? row[i] : int8_t(0);
        __builtin_memcpy(&v, b, 16);
    }
    return v;
}
// What load_chunk brought, moved down by the bytes before k, zeros behind it.
__device__ __forceinline__ i32x4 settle_chunk(i32x4 v, int k, int K) {
    const int down = 8 * (k - max(K - 16, 0));
    if (down <= 0) return v;
    uint64_t part[2];
    __builtin_memcpy(part, &v, 16);
    const bool far = down >= 64;
    const uint64_t low = far ? part[1] : part[0], high = far ? 0 : part[1];
    const int by = down % 64;
    part[0] = down >= 128 ? 0 : low >> by | high << 1 << (63 - by);
    part[1] = high >> by;
    __builtin_memcpy(&v, part, 16);
    return v;
}

__device__ __forceinline__ float scaled(int32_t sum, float xs, float ws, float bias) {
    return fmaf(float(sum) * xs, ws, bias);
}
// From a token's scale of kLoud on its product with a sum of 2^31 may leave fp32's range where
// that with the channel's scale as well does not: the channel's comes first then.
constexpr float kLoud = 0x1p96f;
__device__ __forceinline__ float scaled_any(int32_t sum, float xs, float ws, float bias) {
    return xs > kLoud ? scaled(sum, ws, xs, bias) : scaled(sum, xs, ws, bias);
}

// MW x NW waves of BM x BN blocks of 32 x 32, kStep bytes of k in a stage. DIRECT: every
// row starts on 16 bytes and K is a multiple of 16.
template <int MW, int NW, int BM, int BN, int KS, bool DIRECT>
struct Tile {
    static constexpr int kStep = KS, kChunks = KS / 16;         // 16-byte chunks of a row in a stage
    // Row r of a stage holds chunk c of its bytes at place c ^ bank_of(r): the sixteen lanes
    // that read at once, each 16 bytes of a row of its own, then cover all banks.
    static __device__ __forceinline__ int bank_of(int r) { return r / (256 / kStep) % kChunks; }
    static constexpr int kThreads = 64 * MW * NW;
    static_assert(kThreads / kChunks % 16 == 0, "a thread's rows of a stage share their bank_of");
    static constexpr int kM = 32 * MW * BM, kN = 32 * NW * BN;
    static constexpr int kStage = (kM + kN) * kStep;            // tokens, then channels
    static constexpr int kLoads = (kM + kN) * kChunks / kThreads;   // chunks of a thread
    static constexpr int kScales = (kM + 2 * kN) * 4;
    static constexpr int kOutPitch = 4 * 32 * BN + 16;          // bytes of a row of a wave's results, fp32
    static constexpr int kOut = MW * NW * 32 * kOutPitch;
    static constexpr int lds(int steps) {
        const int stages = kStage * (steps > 1 ? 2 : 1);
        return kScales + (stages > kOut ? stages : kOut);
    }
};

// body(constant) with the type of y
template <class F>
__device__ __forceinline__ void with_dtype(int dtype, F body) {
    if (dtype == BEVPOOL_F32) body(Int<BEVPOOL_F32>());
    else if (dtype == BEVPOOL_BF16) body(Int<BEVPOOL_BF16>());
    else body(Int<BEVPOOL_F16>());
}

// The channel that row r of a wave's 32 * BN rows of weights stands for: lane l of a
// block holds rows 8 (i / 4) + 4 (l / 32) + i % 4, and these are to be neighbours, over
// the wave's blocks too.
template <int BN>
__device__ __forceinline__ int channel_of(int r) {
    const int block = r / 32, g = r % 32 / 8, half = r / 4 % 2;
    return half * 16 * BN + block * 16 + g * 4 + r % 4;
}

// A tile of the product, its first token and channel m0 and n0.
template <int MW, int NW, int BM, int BN, int KS, bool DIRECT>
__device__ __forceinline__ void multiply_tile(const LinearArgs &a, char *lds, int m0, int n0) {
    using G = Tile<MW, NW, BM, BN, KS, DIRECT>;
    constexpr int kStep = G::kStep, kChunks = G::kChunks;
    float *xs = reinterpret_cast<float *>(lds), *ws = xs + G::kM, *bias = ws + G::kN;
    char *stages = lds + G::kScales;
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const int steps = (a.K + kStep - 1) / kStep;

    // A thread's chunks: row i * (threads / 8) + tid / 8 of the stage, its place tid % 8
    // holding the chunk of k that makes lanes of a column read different banks.
    const int place = tid % kChunks, k_at = (place ^ G::bank_of(tid / kChunks)) * 16;
    const int8_t *from[G::kLoads];
#pragma unroll
    for (int i = 0; i < G::kLoads; ++i) {
        const int r = i * (G::kThreads / kChunks) + tid / kChunks;
        if (r < G::kM) {
            from[i] = a.x + int64_t(min(m0 + r, a.M - 1)) * a.ldx;
        } else {
            const int c = r - G::kM, n = n0 + c / (32 * BN) * (32 * BN) + channel_of<BN>(c % (32 * BN));
            from[i] = a.w + int64_t(min(n, a.N - 1)) * a.ldw;
        }
    }
    i32x4 held[DIRECT ? 1 : G::kLoads];
    // Chunks i0 .. i1 - 1 of a thread for a step, on their way to the stage or into registers.
    auto fetch = [&](int step, char *stage, int i0, int i1) {
        const int k = step * kStep + k_at;
        if constexpr (DIRECT) {
            const bool whole = (step + 1) * kStep <= a.K;
#pragma unroll
            for (int i = i0; i < i1; ++i) {
                const void *p = from[i] + k;
                if (!whole && k >= a.K) p = &kNothing;
                // lands at the wave's first place and 16 bytes further for each lane
                __builtin_amdgcn_global_load_lds(
                    (const __attribute__((address_space(1))) void *)p,
                    (__attribute__((address_space(3))) void *)(stage + (i * G::kThreads + wave * 64) * 16), 16, 0, 0);
            }
        } else {
#pragma unroll
            for (int i = i0; i < i1; ++i) held[i] = load_chunk(from[i], k, a.K);
        }
    };
    auto place_held = [&](int step, char *stage) {
        if constexpr (!DIRECT) {
            if ((step + 1) * kStep > a.K)
#pragma unroll
                for (int i = 0; i < G::kLoads; ++i) held[i] = settle_chunk(held[i], step * kStep + k_at, a.K);
#pragma unroll
            for (int i = 0; i < G::kLoads; ++i)
                *reinterpret_cast<i32x4 *>(stage + (i * G::kThreads + tid) * 16) = held[i];
        }
    };

    const int wm = wave % MW, wn = wave / MW, half = lane / 32, col = lane % 32;
    i32x16 acc[BN][BM];
#pragma unroll
    for (int i = 0; i < BN; ++i)
#pragma unroll
        for (int j = 0; j < BM; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;

    // Operands of a quarter of a stage, 32 bytes of k, for all of the wave's blocks. Two sets in
    // turn: while one is multiplied the next is on its way.
    struct Operands {
        i32x4 x[BM], w[BN];
    } set[2];
    const int x_row = (wm * BM * 32 + col) * kStep, w_row = (G::kM + wn * BN * 32 + col) * kStep;
    auto read = [&](const char *stage, int k, Operands &o) {
        const int chunk = ((2 * k + half) ^ G::bank_of(col)) * 16;
#pragma unroll
        for (int j = 0; j < BM; ++j) o.x[j] = *reinterpret_cast<const i32x4 *>(stage + x_row + j * 32 * kStep + chunk);
#pragma unroll
        for (int i = 0; i < BN; ++i) o.w[i] = *reinterpret_cast<const i32x4 *>(stage + w_row + i * 32 * kStep + chunk);
    };
    // between(i) runs after the products of the i-th blocks of channels: reads that are begun
    // there have the other products' time, and wait for nothing that is still to be multiplied.
    auto multiply = [&](const Operands &o, auto between) {
#pragma unroll
        for (int i = 0; i < BN; ++i) {
#pragma unroll
            for (int j = 0; j < BM; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(o.w[i], o.x[j], acc[i][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
            between(i);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    constexpr int kQuarters = kStep / 32, kSpread = BN > 1 ? BN - 1 : 1;

    fetch(0, stages, 0, G::kLoads);
    for (int i = tid; i < G::kM; i += G::kThreads) xs[i] = a.x_scale[min(m0 + i, a.M - 1)];
    for (int i = tid; i < G::kN; i += G::kThreads) {
        const int n = min(n0 + i, a.N - 1);
        ws[i] = a.w_scale[n];
        bias[i] = a.bias ? a.bias[n] : 0.0f;
    }
    place_held(0, stages);
    __syncthreads();
    read(stages, 0, set[0]);
    if (steps > 1) fetch(1, stages + G::kStage, 0, G::kLoads);
    for (int s = 0; s + 1 < steps; ++s) {
        char *now = stages + (s & 1) * G::kStage, *next = stages + ((s + 1) & 1) * G::kStage;
#pragma unroll
        for (int k = 0; k + 1 < kQuarters; ++k)
            multiply(set[k & 1], [&](int i) {
                if (i == 0) read(now, k + 1, set[(k + 1) & 1]);
            });
        // all that this stage holds is in registers: the one after next may overwrite it
        place_held(s + 1, next);
        __syncthreads();
        multiply(set[(kQuarters - 1) & 1], [&](int i) {
            if (i == 0) read(next, 0, set[0]);
            if (s + 2 < steps && (i > 0 || BN == 1)) {
                const int at = BN == 1 ? 0 : i - 1;
                fetch(s + 2, now, G::kLoads * at / kSpread, G::kLoads * (at + 1) / kSpread);
            }
        });
    }
    const char *last = stages + ((steps - 1) & 1) * G::kStage;
    const int left = a.K - (steps - 1) * kStep;
#pragma unroll
    for (int k = 0; k < kQuarters; ++k) {
        if (k * 32 >= left) break;
        multiply(set[k & 1], [&](int i) {
            if (i == 0 && k + 1 < kQuarters) read(last, k + 1, set[(k + 1) & 1]);
        });
    }
    __syncthreads();

    // Sums go through LDS, 32 tokens of a wave at a time, so that whole rows are written. A
    // lane then keeps to its channels, whose scales stay in registers.
    char *mine = stages + wave * 32 * G::kOutPitch;
    constexpr int kCols = 32 * BN, kPer = kCols / 8;    // lanes of a row, eight channels each
    const int nw = n0 + wn * kCols, mw = wm * BM * 32, mine_at = lane % kPer * 8;
    auto place_sums = [&](int j) {
#pragma unroll
        for (int i = 0; i < BN; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int c = half * 16 * BN + i * 16 + g * 4;
                *reinterpret_cast<i32x4 *>(mine + col * G::kOutPitch + c * 4) =
                    i32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
            }
        // a wave's own rows: no other wave to wait for
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    // (apart from the rest: a branch among its stores made whole products 2 to 7% slower)
    if (__builtin_expect(__any(xs[mw + lane % (32 * BM)] > kLoud), 0)) {
#pragma unroll
        for (int j = 0; j < BM; ++j) {
            place_sums(j);
#pragma unroll 1
            for (int at = lane; at < 32 * kCols; at += 64) {
                const int r = at / kCols, c = at % kCols, m = m0 + mw + j * 32 + r, n = nw + c;
                if (m >= a.M || n >= a.N) continue;
                const float v = scaled_any(*reinterpret_cast<const int32_t *>(mine + r * G::kOutPitch + c * 4),
                                           xs[mw + j * 32 + r], ws[wn * kCols + c], bias[wn * kCols + c]);
                store_any<1>(a.y, int64_t(m) * a.N + n, a.y_dtype, &v);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
        return;
    }
    float w_scale[8], b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        w_scale[e] = ws[wn * kCols + mine_at + e];
        b[e] = bias[wn * kCols + mine_at + e];
    }
#pragma unroll
    for (int j = 0; j < BM; ++j) {
        place_sums(j);
        const int m_first = m0 + mw + j * 32;
        with_dtype(a.y_dtype, [&](auto dt) {
            using T = typename Num<decltype(dt)::value>::T;
            T *y = static_cast<T *>(a.y);
            const int n = nw + mine_at;
#pragma unroll 4
            for (int r = lane / kPer; r < 32; r += 64 / kPer) {
                const i32x4 *p = reinterpret_cast<const i32x4 *>(mine + r * G::kOutPitch + mine_at * 4);
                const i32x4 low = p[0], high = p[1];
                const float scale = xs[mw + j * 32 + r];
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = scaled(e < 4 ? low[e] : high[e - 4], scale, w_scale[e], b[e]);
                if (m_first + r >= a.M || n >= a.N) continue;
                T *to = y + int64_t(m_first + r) * a.N + n;
                if (a.wide) store_n<T, 8>(to, v);
                else store_part<T, 8, kUneven>(to, a.N - n, v);
            }
        });
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// Tiles in the order in which they are taken: kGroup down before the next of the features,
// so that those that run at a time share their rows in a cache.
__device__ __forceinline__ void place_of(int tile, int m_tiles, int n_tiles, int *m, int *n) {
    const int group = tile / (kGroup * n_tiles), in = tile - group * kGroup * n_tiles;
    const int tall = min(kGroup, m_tiles - group * kGroup);
    *m = group * kGroup + in % tall;
    *n = in / tall;
}
// Neighbouring workgroups go to different XCDs: each XCD gets a run of tiles of its own
// (8192^3: 564 us, with tiles row by row 596).
__device__ __forceinline__ int run_of(int block, int tiles) {
    const int xcd = block % 8;
    return xcd * (tiles / 8) + min(xcd, tiles % 8) + block / 8;
}

template <int MW, int NW, int BM, int BN, int KS, bool DIRECT>
__global__ __launch_bounds__(64 * MW * NW) void k_linear(LinearArgs a) {
    using G = Tile<MW, NW, BM, BN, KS, DIRECT>;
    extern __shared__ __align__(16) char lds[];
    int m, n;
    place_of(run_of(blockIdx.x, gridDim.x), a.m_tiles, a.n_tiles, &m, &n);
    multiply_tile<MW, NW, BM, BN, KS, DIRECT>(a, lds, m * G::kM, n * G::kN);
}

// Tiles of 256 x 256, the last ones in eighths: a few tiles that are left over a whole
// round of workgroups would take as long as a round.
template <bool DIRECT>
__global__ __launch_bounds__(512) void k_linear_eighths(LinearArgs a, int whole) {
    extern __shared__ __align__(16) char lds[];
    const int block = blockIdx.x, left = a.m_tiles * a.n_tiles - whole;
    int m, n;
    if (block < whole) {
        place_of(run_of(block, whole), a.m_tiles, a.n_tiles, &m, &n);
        multiply_tile<4, 2, 2, 4, 128, DIRECT>(a, lds, m * 256, n * 256);
        return;
    }
    const int part = (block - whole) / left;
    place_of(whole + (block - whole) % left, a.m_tiles, a.n_tiles, &m, &n);
    multiply_tile<4, 2, 1, 1, 128, DIRECT>(a, lds, m * 256 + part / 4 * 128, n * 256 + part % 4 * 64);
}

// Few tokens: 16 channels and 16 * MB tokens of a workgroup, whose waves share out k in
// runs of kRun bytes. A wave reads eight rows of a run at a time, whole cache lines, and
// turns them in LDS of its own into the operands' order, 16 rows of 16 bytes. (Read in that
// order, a wave's load of 16 half lines takes a compute unit some 70 cycles: 64 x 4096 x
// 2048 7.8 us.)
template <int MB, int WAVES, bool DIRECT>
__global__ __launch_bounds__(64 * WAVES) void k_linear_few(LinearArgs a) {
    constexpr int kBlocks = 1 + MB;         // of 16 rows: channels, then tokens
    constexpr int kMine = kBlocks * 16 * kRun;
    __shared__ __align__(16) char lds[WAVES * kMine];
    i32x4(*sums)[MB][64] = reinterpret_cast<i32x4(*)[MB][64]>(lds);
    static_assert(sizeof(i32x4) * MB * 64 <= kMine, "");
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, quarter = lane / 16, col = lane % 16;
    const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * MB;
    const int line = lane / 8, chunk = lane % 8;
    const int8_t *from[kBlocks][2];         // rows line and line + 8 of a block
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        from[0][h] = a.w + int64_t(min(n0 + 8 * h + line, a.N - 1)) * a.ldw;
#pragma unroll
        for (int j = 0; j < MB; ++j)
            from[1 + j][h] = a.x + int64_t(min(m0 + 16 * j + 8 * h + line, a.M - 1)) * a.ldx;
    }
    i32x4 way[kBlocks][2];                  // a run on its way
    auto fetch = [&](int first) {
        const int k = first + 16 * chunk;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if constexpr (DIRECT) {
                    way[b][h] = i32x4{0, 0, 0, 0};
                    if (k < a.K) way[b][h] = *reinterpret_cast<const i32x4 *>(from[b][h] + k);
                } else {
                    way[b][h] = load_chunk(from[b][h], k, a.K);
                }
            }
    };
    // row r's chunk c lies at place c ^ r / 2: sixteen rows at one chunk cover all banks
    char *mine = lds + wave * kMine;
    i32x4 acc[MB];
#pragma unroll
    for (int j = 0; j < MB; ++j) acc[j] = i32x4{0, 0, 0, 0};
    fetch(wave * kRun);
    for (int first = wave * kRun; first < a.K; first += WAVES * kRun) {
        if (!DIRECT && first + kRun > a.K)
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int h = 0; h < 2; ++h) way[b][h] = settle_chunk(way[b][h], first + 16 * chunk, a.K);
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = 8 * h + line;
                *reinterpret_cast<i32x4 *>(mine + (b * 16 + r) * kRun + (chunk ^ r / 2) * 16) = way[b][h];
            }
        if (first + WAVES * kRun < a.K) fetch(first + WAVES * kRun);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int s = 0; s < kRun / 64; ++s) {
            i32x4 v[kBlocks];
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
                v[b] = *reinterpret_cast<const i32x4 *>(mine + (b * 16 + col) * kRun + ((4 * s + quarter) ^ col / 2) * 16);
#pragma unroll
            for (int j = 0; j < MB; ++j) acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v[0], v[1 + j], acc[j], 0, 0, 0);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < MB; ++j) sums[wave][j][lane] = acc[j];
    __syncthreads();
    // sums[..][j][l][e]: token 16 j + l % 16, channel 4 (l / 16) + e
    for (int t = threadIdx.x; t < 256 * MB; t += 64 * WAVES) {
        const int c = t % 16, row = t / 16, m = m0 + row, n = n0 + c;
        if (m >= a.M || n >= a.N) continue;
        int32_t sum = 0;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) sum += sums[v][row / 16][c / 4 * 16 + row % 16][c % 4];
        const float y = scaled_any(sum, a.x_scale[m], a.w_scale[n], a.bias ? a.bias[n] : 0.0f);
        store_any<1>(a.y, int64_t(m) * a.N + n, a.y_dtype, &y);
    }
}

template <int MB, int WAVES, bool DIRECT>
int launch_few(const LinearArgs &a, hipStream_t stream) {
    hipLaunchKernelGGL((k_linear_few<MB, WAVES, DIRECT>),
                       dim3(uint32_t((a.N + 15) / 16), uint32_t((a.M + 16 * MB - 1) / (16 * MB))), dim3(64 * WAVES), 0,
                       stream, a);
    BEVPOOL_HIP(hipGetLastError());
    return BEVPOOL_OK;
}

template <int MW, int NW, int BM, int BN, int KS, bool DIRECT>
int launch_tiles(LinearArgs a, hipStream_t stream) {
    using G = Tile<MW, NW, BM, BN, KS, DIRECT>;
    a.m_tiles = (a.M + G::kM - 1) / G::kM;
    a.n_tiles = (a.N + G::kN - 1) / G::kN;
    const int lds = G::lds((a.K + KS - 1) / KS);
    auto kernel = k_linear<MW, NW, BM, BN, KS, DIRECT>;
    if (lds > 65536)
        BEVPOOL_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                        hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    hipLaunchKernelGGL(kernel, dim3(uint32_t(a.m_tiles * a.n_tiles)), dim3(G::kThreads), lds, stream, a);
    BEVPOOL_HIP(hipGetLastError());
    return BEVPOOL_OK;
}

template <bool DIRECT>
int launch_eighths(LinearArgs a, int left, hipStream_t stream) {
    using G = Tile<4, 2, 2, 4, 128, DIRECT>;
    a.m_tiles = (a.M + 255) / 256;
    a.n_tiles = (a.N + 255) / 256;
    const int tiles = a.m_tiles * a.n_tiles, lds = G::lds((a.K + 127) / 128);
    BEVPOOL_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(k_linear_eighths<DIRECT>),
                                    hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    hipLaunchKernelGGL((k_linear_eighths<DIRECT>), dim3(uint32_t(tiles + 7 * left)), dim3(512), lds, stream, a,
                       tiles - left);
    BEVPOOL_HIP(hipGetLastError());
    return BEVPOOL_OK;
}

// A launch has fewer than 2^32 threads.
bool fits(int64_t tiles, int threads) { return tiles * threads < int64_t(1) << 32; }

template <bool DIRECT>
int launch(const LinearArgs &a, hipStream_t stream) {
    auto tiles = [&](int m, int n) { return int64_t((a.M + m - 1) / m) * ((a.N + n - 1) / n); };
    // Few tokens. The time of this form goes with its workgroups and with k, that of tiles of
    // 64 x 64 that all run at once with k alone, and the two meet at about 1100 workgroups
    // (256 x 2048, K 2048, 1024 of them: 7.0 against 8.3 us; 1111 x 520, K 336, 1155: 4.3
    // against 3.8). Eight waves where a compute unit holds one workgroup (64 x 2048, K 4096:
    // 5.1 against 5.8 us), four where it holds more (256 x 2048, K 2048: 7.0 against 7.4).
    // Blocks of 16 tokens where they make no more workgroups than there are compute units (32 x
    // 1024, K 4096: 3.8 against 4.4 us; 64 x 2048, twice as many: 5.6 against 5.1).
    if (a.M <= 16 || tiles(16, 16) <= kUnits) return launch_few<1, 8, DIRECT>(a, stream);
    if (const int64_t groups = tiles(32, 16); groups <= 1100)
        return groups <= kUnits ? launch_few<2, 8, DIRECT>(a, stream) : launch_few<2, 4, DIRECT>(a, stream);
    // Tiles of 64 x 64 where those of 128 x 128 leave compute units without work, and, two to a
    // unit, for the shortest k, whose rows are not read often enough to repay larger tiles
    // (5120 x 1024, K 128: 5.9 against 7.0 us, K 512: 10.8 against 10.0).
    if (tiles(128, 128) < (a.K < 256 ? 2 * kUnits : kUnits)) return launch_tiles<2, 2, 1, 1, 128, DIRECT>(a, stream);
    // Rounds of workgroups, in units of a round of 256 x 256 tiles, one to a compute unit (38
    // us at K 2048): a round of 128 x 128, two to a unit, takes 22 us, one of eighths 10.
    const int64_t big = tiles(256, 256), left = big % kUnits;
    const bool eighths = big >= kUnits && left > 0 && left <= kUnits / 4;
    const double big_time = double(big / kUnits) + (left == 0 ? 0.0 : eighths ? 0.27 * double((8 * left + kUnits - 1) / kUnits) : 1.0);
    const double small_time = 0.58 * double((tiles(128, 128) + 2 * kUnits - 1) / (2 * kUnits));
    // Short rows that go through the registers: 128 x 64 by eight waves (100000 x 250, K 120:
    // 19.2 us against 20.6 by 128 x 128; 3000 x 2000, K 331: 11.6 against 12.7; 33000 x 509, K
    // 443: 33.3 against 31.5).
    if constexpr (!DIRECT)
        if (a.K <= 384 && fits(tiles(128, 64), 512)) return launch_tiles<4, 2, 1, 1, 128, DIRECT>(a, stream);
    if (a.K < 512 || small_time < big_time) return launch_tiles<2, 2, 2, 2, 128, DIRECT>(a, stream);
    return eighths ? launch_eighths<DIRECT>(a, int(left), stream) : launch_tiles<4, 2, 2, 4, 128, DIRECT>(a, stream);
}

}  // namespace
}  // namespace bevmap

using namespace bevmap;

int bevmap_launch_linear_int8(const bevmap_linear &n, const int8_t *x, const float *x_scale, const int8_t *w,
                              const float *w_scale, const float *bias, void *y, hipStream_t stream) {
    if (n.rows == 0 || n.features == 0) return BEVPOOL_OK;
    LinearArgs a{};
    a.x = x;
    a.w = w;
    a.x_scale = x_scale;
    a.w_scale = w_scale;
    a.bias = bias;
    a.y = y;
    a.ldx = n.rows == 1 ? 0 : n.x_stride;
    a.ldw = n.features == 1 ? 0 : n.w_stride;
    a.M = int32_t(n.rows);
    a.N = n.features;
    a.K = n.channels;
    a.y_dtype = n.y_dtype;
    a.wide = n.features % 8 == 0 && aligned_for(y, 0, n.y_dtype, 8);
    const bool direct = n.channels % 16 == 0 && a.ldx % 16 == 0 && a.ldw % 16 == 0 &&
                        reinterpret_cast<uintptr_t>(x) % 16 == 0 && reinterpret_cast<uintptr_t>(w) % 16 == 0;
    return direct ? launch<true>(a, stream) : launch<false>(a, stream);
}
