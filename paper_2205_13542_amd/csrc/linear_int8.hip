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
// aligned) while the matrix cores work. Few tokens: the weights are what is read, so a
// workgroup takes 16 channels, its waves share out k, and operands go straight to
// registers; the waves' sums are joined in LDS.
#include "mapops.h"

namespace bevmap {
namespace {

using i32x4 = int32_t __attribute__((ext_vector_type(4)));
using i32x16 = int32_t __attribute__((ext_vector_type(16)));

constexpr int kStep = 128;              // bytes of k in a stage
constexpr int kChunks = kStep / 16;     // 16-byte chunks of a row in a stage

struct LinearArgs {
    const int8_t *x, *w;
    const float *x_scale, *w_scale, *bias;
    void *y;
    int64_t ldx, ldw;
    int32_t M, N, K;
    int32_t m_tiles, n_tiles, y_dtype;
    bool wide;                          // rows of y can be written 16 bytes at a time
};

__device__ const uint4 kNothing = {0, 0, 0, 0};     // what lies past the end of k

// 16 bytes of a row of K from k on, zeros past its end; any alignment.
__device__ __forceinline__ i32x4 load_chunk(const int8_t *row, int k, int K) {
    i32x4 v = {0, 0, 0, 0};
    if (k + 16 <= K) {
        __builtin_memcpy(&v, row + k, 16);
    } else if (k < K) {
        int8_t b[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) b[i] = k + i < K ? row[k + i] : int8_t(0);
        __builtin_memcpy(&v, b, 16);
    }
    return v;
}

__device__ __forceinline__ float scaled(int32_t sum, float xs, float ws, float bias) {
    return fmaf(float(sum) * xs, ws, bias);
}

// MW x NW waves of BM x BN blocks of 32 x 32. DIRECT: every row starts on 16 bytes and K
// is a multiple of 16.
template <int MW, int NW, int BM, int BN, bool DIRECT>
struct Tile {
    static constexpr int kThreads = 64 * MW * NW;
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

// The channel that row r of a wave's 32 * BN rows of weights stands for: lane l of a
// block holds rows 8 (i / 4) + 4 (l / 32) + i % 4, and these are to be neighbours, over
// the wave's blocks too.
template <int BN>
__device__ __forceinline__ int channel_of(int r) {
    const int block = r / 32, g = r % 32 / 8, half = r / 4 % 2;
    return half * 16 * BN + block * 16 + g * 4 + r % 4;
}

template <int MW, int NW, int BM, int BN, bool DIRECT>
__global__ __launch_bounds__(64 * MW * NW) void k_linear(LinearArgs a) {
    using G = Tile<MW, NW, BM, BN, DIRECT>;
    extern __shared__ __align__(16) char lds[];
    float *xs = reinterpret_cast<float *>(lds), *ws = xs + G::kM, *bias = ws + G::kN;
    char *stages = lds + G::kScales;
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    // neighbouring workgroups go to different XCDs: each gets a run of tiles of its own,
    // which share their rows in its cache
    const int tiles = a.m_tiles * a.n_tiles, xcd = blockIdx.x % 8, at = blockIdx.x / 8;
    const int tile = xcd * (tiles / 8) + (xcd < tiles % 8 ? xcd : tiles % 8) + at;
    const int m0 = tile / a.n_tiles * G::kM, n0 = tile % a.n_tiles * G::kN;
    const int steps = (a.K + kStep - 1) / kStep;

    for (int i = tid; i < G::kM; i += G::kThreads) xs[i] = a.x_scale[min(m0 + i, a.M - 1)];
    for (int i = tid; i < G::kN; i += G::kThreads) {
        const int n = min(n0 + i, a.N - 1);
        ws[i] = a.w_scale[n];
        bias[i] = a.bias ? a.bias[n] : 0.0f;
    }

    // A thread's chunks: row i * (threads / 8) + tid / 8 of the stage, its place tid % 8
    // holding the chunk of k that makes lanes of a column read different banks.
    const int place = tid % kChunks, k_at = (place ^ (tid / kChunks % kChunks)) * 16;
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
    auto fetch = [&](int step, char *stage) {
        const int k = step * kStep + k_at;
#pragma unroll
        for (int i = 0; i < G::kLoads; ++i) {
            if constexpr (DIRECT) {
                const void *p = k < a.K ? static_cast<const void *>(from[i] + k) : static_cast<const void *>(&kNothing);
                // lands at the wave's first place and 16 bytes further for each lane
                __builtin_amdgcn_global_load_lds(
                    (const __attribute__((address_space(1))) void *)p,
                    (__attribute__((address_space(3))) void *)(stage + (i * G::kThreads + wave * 64) * 16), 16, 0, 0);
            } else {
                held[i] = load_chunk(from[i], k, a.K);
            }
        }
    };
    auto place_held = [&](char *stage) {
        if constexpr (!DIRECT)
#pragma unroll
            for (int i = 0; i < G::kLoads; ++i)
                *reinterpret_cast<i32x4 *>(stage + (i * G::kThreads + tid) * 16) = held[i];
    };

    const int wm = wave % MW, wn = wave / MW, half = lane / 32, col = lane % 32;
    i32x16 acc[BN][BM];
#pragma unroll
    for (int i = 0; i < BN; ++i)
#pragma unroll
        for (int j = 0; j < BM; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;

    fetch(0, stages);
    place_held(stages);
    __syncthreads();
    for (int s = 0; s < steps; ++s) {
        const char *now = stages + (s & 1) * G::kStage;
        char *next = stages + ((s + 1) & 1) * G::kStage;
        if (s + 1 < steps) fetch(s + 1, next);
        const char *xt = now + (wm * BM * 32 + col) * kStep, *wt = now + (G::kM + wn * BN * 32 + col) * kStep;
#pragma unroll
        for (int k = 0; k < kStep / 32; ++k) {
            if (s * kStep + k * 32 >= a.K) break;
            const int chunk = ((2 * k + half) ^ (col % kChunks)) * 16;
            i32x4 xv[BM], wv[BN];
#pragma unroll
            for (int j = 0; j < BM; ++j) xv[j] = *reinterpret_cast<const i32x4 *>(xt + j * 32 * kStep + chunk);
#pragma unroll
            for (int i = 0; i < BN; ++i) wv[i] = *reinterpret_cast<const i32x4 *>(wt + i * 32 * kStep + chunk);
#pragma unroll
            for (int i = 0; i < BN; ++i)
#pragma unroll
                for (int j = 0; j < BM; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wv[i], xv[j], acc[i][j], 0, 0, 0);
        }
        if (s + 1 < steps) place_held(next);
        __syncthreads();
    }

    // Results go through LDS, 32 tokens of a wave at a time, so that whole rows are written.
    char *mine = stages + wave * 32 * G::kOutPitch;
    constexpr int kCols = 32 * BN;
    const int nw = n0 + wn * kCols;         // the wave's first channel
#pragma unroll
    for (int j = 0; j < BM; ++j) {
        const int m_first = m0 + (wm * BM + j) * 32;
        const float scale = xs[(wm * BM + j) * 32 + col];
#pragma unroll
        for (int i = 0; i < BN; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int c = half * 16 * BN + i * 16 + g * 4;
                float4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    (&v.x)[e] = scaled(acc[i][j][4 * g + e], scale, ws[wn * kCols + c + e], bias[wn * kCols + c + e]);
                *reinterpret_cast<float4 *>(mine + col * G::kOutPitch + c * 4) = v;
            }
        // a wave's own rows: no other wave to wait for
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (a.wide) {
            constexpr int kPer = kCols / 8;     // lanes of a row, eight channels each
            for (int r = lane / kPer; r < 32; r += 64 / kPer) {
                const int m = m_first + r, n = nw + lane % kPer * 8;
                if (m < a.M && n < a.N) {
                    float v[8];
                    const float4 *p = reinterpret_cast<const float4 *>(mine + r * G::kOutPitch + lane % kPer * 32);
                    *reinterpret_cast<float4 *>(v) = p[0];
                    *reinterpret_cast<float4 *>(v + 4) = p[1];
                    store_any<8>(a.y, int64_t(m) * a.N + n, a.y_dtype, v);
                }
            }
        } else {
            for (int t = lane; t < 32 * kCols; t += 64) {
                const int m = m_first + t / kCols, n = nw + t % kCols;
                if (m < a.M && n < a.N)
                    store_any<1>(a.y, int64_t(m) * a.N + n, a.y_dtype,
                                 reinterpret_cast<const float *>(mine + t / kCols * G::kOutPitch) + t % kCols);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// Few tokens: 16 channels and 16 * MB tokens of a workgroup, whose waves share out k in
// runs of kStep bytes.
constexpr int kFewWaves = 8;
template <int MB, bool DIRECT>
__global__ __launch_bounds__(64 * kFewWaves) void k_linear_few(LinearArgs a) {
    __shared__ i32x4 sums[kFewWaves][MB][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, quarter = lane / 16, col = lane % 16;
    const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * MB;
    const int8_t *w = a.w + int64_t(min(n0 + col, a.N - 1)) * a.ldw, *x[MB];
#pragma unroll
    for (int j = 0; j < MB; ++j) x[j] = a.x + int64_t(min(m0 + 16 * j + col, a.M - 1)) * a.ldx;
    auto load = [&](const int8_t *row, int k) {
        if constexpr (DIRECT) {
            i32x4 v = {0, 0, 0, 0};
            if (k < a.K) v = *reinterpret_cast<const i32x4 *>(row + k);
            return v;
        } else {
            return load_chunk(row, k, a.K);
        }
    };
    i32x4 acc[MB];
#pragma unroll
    for (int j = 0; j < MB; ++j) acc[j] = i32x4{0, 0, 0, 0};
    for (int first = wave * kStep; first < a.K; first += kFewWaves * kStep) {
        i32x4 wv[kStep / 64], xv[kStep / 64][MB];
#pragma unroll
        for (int s = 0; s < kStep / 64; ++s) {
            const int k = first + 64 * s + 16 * quarter;
            wv[s] = load(w, k);
#pragma unroll
            for (int j = 0; j < MB; ++j) xv[s][j] = load(x[j], k);
        }
#pragma unroll
        for (int s = 0; s < kStep / 64; ++s)
#pragma unroll
            for (int j = 0; j < MB; ++j) acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[s], xv[s][j], acc[j], 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < MB; ++j) sums[wave][j][lane] = acc[j];
    __syncthreads();
    // sums[..][j][l][e]: token 16 j + l % 16, channel 4 (l / 16) + e
    for (int t = threadIdx.x; t < 256 * MB; t += 64 * kFewWaves) {
        const int c = t % 16, row = t / 16, m = m0 + row, n = n0 + c;
        if (m >= a.M || n >= a.N) continue;
        int32_t sum = 0;
#pragma unroll
        for (int v = 0; v < kFewWaves; ++v) sum += sums[v][row / 16][c / 4 * 16 + row % 16][c % 4];
        const float y = scaled(sum, a.x_scale[m], a.w_scale[n], a.bias ? a.bias[n] : 0.0f);
        store_any<1>(a.y, int64_t(m) * a.N + n, a.y_dtype, &y);
    }
}

template <int MW, int NW, int BM, int BN, bool DIRECT>
int launch_tiles(LinearArgs a, hipStream_t stream) {
    using G = Tile<MW, NW, BM, BN, DIRECT>;
    a.m_tiles = (a.M + G::kM - 1) / G::kM;
    a.n_tiles = (a.N + G::kN - 1) / G::kN;
    const int lds = G::lds((a.K + kStep - 1) / kStep);
    auto kernel = k_linear<MW, NW, BM, BN, DIRECT>;
    if (lds > 65536)
        BEVPOOL_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                        hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    hipLaunchKernelGGL(kernel, dim3(uint32_t(a.m_tiles * a.n_tiles)), dim3(G::kThreads), lds, stream, a);
    BEVPOOL_HIP(hipGetLastError());
    return BEVPOOL_OK;
}

template <bool DIRECT>
int launch(const LinearArgs &a, hipStream_t stream) {
    auto tiles = [&](int m, int n) { return int64_t((a.M + m - 1) / m) * ((a.N + n - 1) / n); };
    if (a.M <= 16) {
        hipLaunchKernelGGL((k_linear_few<1, DIRECT>), dim3(uint32_t((a.N + 15) / 16)), dim3(64 * kFewWaves), 0, stream,
                           a);
        BEVPOOL_HIP(hipGetLastError());
        return BEVPOOL_OK;
    }
    if (tiles(64, 64) < 128) {
        hipLaunchKernelGGL((k_linear_few<4, DIRECT>), dim3(uint32_t((a.N + 15) / 16), uint32_t((a.M + 63) / 64)),
                           dim3(64 * kFewWaves), 0, stream, a);
        BEVPOOL_HIP(hipGetLastError());
        return BEVPOOL_OK;
    }
    if (tiles(128, 128) < 512) return launch_tiles<2, 2, 1, 1, DIRECT>(a, stream);
    if (tiles(256, 256) < 512 || a.K <= 512) return launch_tiles<2, 2, 2, 2, DIRECT>(a, stream);
    return launch_tiles<4, 2, 2, 4, DIRECT>(a, stream);
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
