// Root-mean-square norm of rows, of x + residual where there is one, with its gradients
// (bevmap_rms_norm, bevmap_rms_norm_backward), and rows held in 8-bit integers
// (bevmap_rms_norm_int8, bevmap_quantize_int8).
//
//   h = x + residual,  r = 1 / sqrt(mean h^2 + eps),  y = w h r
//   u = h r, e = dy w:  dh = dsum + r (e - u mean(e u)),  dw = sum over rows of dy u
//   z = h w, top = max |z|:  q = round(z (127 / top)),  scale = top r / 127
// r cancels in q, so the integers do not depend on the order in which the squares are
// summed, and one pass over the row in registers gives both.
//
// Bound by memory: a row stays in the registers of the lanes that share it, and each
// tensor is read or written once. Lanes: the least power of two that holds a row at V
// elements a lane, up to a wave; longer rows take several accesses a lane, or a whole
// workgroup. Workgroups stay and walk the rows, so that the weights are read once into
// registers and the backward sums dw there; its parts are joined in a fixed order by a
// small kernel. 518400 x 80 in bf16 takes 58 us forward with a residual (332 MB, 5.7 TB/s;
// a copy of 4 GiB reaches 4.75), 84 + 6 backward (415 MB); 129600 x 80 in 8 bits 15.9.
#include <initializer_list>

#include "mapops.h"

namespace bevmap {
namespace {

constexpr int kRmsBlock = 256;
constexpr int kRmsWave = 64;
constexpr int kRmsJoinChannels = 16;   // channels of a workgroup that joins parts of dw
constexpr int kRmsJoinBlock = 1024;

struct RmsArgs {
    const void *x, *residual, *weight, *dy, *dsum;
    void *sum, *y;                  // backward: sum is dx
    int8_t *q;
    float *rstd, *scale, *parts;    // parts: [workgroups][C]
    int64_t ldx, ldr, rows, chunk;  // chunk: rows of a workgroup of the backward
    int32_t C, y_dtype, w_dtype;
    float eps;
};

enum { kFloat, kInt8Norm, kInt8 };      // what a forward kernel writes

// Sum, or the largest of unsigned numbers, over the LANES lanes that share a row. Over a
// workgroup: through LDS, two slots in turn, so that one barrier a row is enough.
template <class F, class T>
__device__ __forceinline__ T over_wave(T v, int lanes, F f) {
#pragma unroll
    for (int m = 1; m < lanes; m <<= 1) v = f(v, __shfl_xor(v, m));
    return v;
}
template <int LANES, class F, class T>
__device__ __forceinline__ T over_lanes(T v, F f, T *slots, int turn) {
    if constexpr (LANES <= kRmsWave) return over_wave(v, LANES, f);
    constexpr int kWaves = kRmsBlock / kRmsWave;
    v = over_wave(v, kRmsWave, f);
    T *s = slots + (turn & 1) * kWaves;
    if (threadIdx.x % kRmsWave == 0) s[threadIdx.x / kRmsWave] = v;
    __syncthreads();
    return f(f(s[0], s[1]), f(s[2], s[3]));
}

__device__ __forceinline__ float plus(float a, float b) { return a + b; }
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }

constexpr uint32_t kInfBits = 0x7F800000u;
// |v| as an unsigned number: in the order of magnitudes, with NaN above infinity
__device__ __forceinline__ uint32_t size_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// How z becomes q: q = round(z * up * mul), scale = top * rstd / 127.
struct Steps {
    float up, mul, scale;
    bool none;      // a row with an infinity or a NaN: q = 0, scale NaN
};
__device__ __forceinline__ Steps steps_of(uint32_t top_bits, float rstd) {
    const float top = __uint_as_float(top_bits);
    Steps s;
    s.none = top_bits >= kInfBits;
    s.up = top < 0x1p-100f ? 0x1p64f : 1.0f;            // 127 / top would be infinite
    s.mul = top > 0.0f && !s.none ? 127.0f / (top * s.up) : 0.0f;
    s.scale = s.none ? __uint_as_float(0x7FC00000u) : top * rstd / 127.0f;
    return s;
}
__device__ __forceinline__ int8_t held(float z, const Steps &s) {
    return int8_t(s.none ? 0.0f : rintf(z * s.up * s.mul));
}

// Waves of a SIMD that the registers are to leave room for, where they are next to that: all
// of the workgroups that stay then run at a time (8 bits of 100003 x 331: 48 us, by seven 54).
constexpr int rms_waves(int lanes, int iter, int out, int rows) {
    return out == kInt8Norm && lanes <= kRmsWave && (iter == 1 || rows == kEven) ? 8 : 1;
}

template <int DT, int LANES, int ITER, int OUT, int ROWS, bool STREAM>
__global__ __launch_bounds__(kRmsBlock, rms_waves(LANES, ITER, OUT, ROWS)) void k_rms(RmsArgs a) {
    using T = typename Num<DT>::T;
    constexpr int V = kWide<DT>, kRows = kRmsBlock / LANES;
    __shared__ float add[8];
    __shared__ uint32_t most[8];
    const int lane = threadIdx.x % LANES, n_vec = (a.C + V - 1) / V;
    const T *x = static_cast<const T *>(a.x), *res = static_cast<const T *>(a.residual);
    T *sum = static_cast<T *>(a.sum);
    float w[ITER][V];
#pragma unroll
    for (int k = 0; k < ITER; ++k) {
#pragma unroll
        for (int i = 0; i < V; ++i) w[k][i] = 1.0f;
        if (OUT != kInt8 && a.weight && lane + k * LANES < n_vec)
            load_any_part<V, ROWS>(a.weight, (lane + k * LANES) * V, a.w_dtype, a.C - (lane + k * LANES) * V, w[k]);
    }
    const float per = 1.0f / float(a.C);
    int turn = 0;
    for (int64_t first = int64_t(blockIdx.x) * kRows; first < a.rows; first += int64_t(gridDim.x) * kRows, ++turn) {
        const int64_t row = first + threadIdx.x / LANES;
        const bool live = row < a.rows;
        float h[ITER][V];
#pragma unroll
        for (int k = 0; k < ITER; ++k) {
            const int at = lane + k * LANES;
#pragma unroll
            for (int i = 0; i < V; ++i) h[k][i] = 0.0f;
            if (live && at < n_vec) {
                const int count = a.C - at * V;
                load_part<T, V, ROWS>(x + row * a.ldx + at * V, count, h[k]);
                if (OUT != kInt8 && res) {
                    float r[V];
                    load_part<T, V, ROWS>(res + row * a.ldr + at * V, count, r);
#pragma unroll
                    for (int i = 0; i < V; ++i) h[k][i] += r[i];
                    store_part<T, V, ROWS, STREAM>(sum + row * a.C + at * V, count, h[k]);
                }
            }
        }
        float rstd = 1.0f, s = 1.0f, ss = 0.0f;     // y = w h rstd, h times s by then
        if constexpr (OUT != kInt8) {
#pragma unroll
            for (int k = 0; k < ITER; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) ss = fmaf(h[k][i], h[k][i], ss);
            ss = over_lanes<LANES>(ss, plus, add, turn);
            // Squares that leave fp32's range: the row's numbers times a power of two, squared again, and
            // normed as they are then (1 / rms itself may be no fp32 number).
            // (A sum of 0 is a row of zeros, or of numbers so small that only an eps of nothing shows them.)
            const bool large = !(ss < 0x1p120f), small = ss < 0x1p-90f && a.eps < 0x1p-60f;
            if (LANES > kRmsWave ? large || small : __any(large || small)) {
                s = large ? 0x1p-80f : small ? 0x1p93f : 1.0f;
                float again = 0.0f;
#pragma unroll
                for (int k = 0; k < ITER; ++k)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        h[k][i] *= s;
                        again = fmaf(h[k][i], h[k][i], again);
                    }
                if constexpr (LANES > kRmsWave) __syncthreads();    // the slots are read
                ss = over_lanes<LANES>(again, plus, add, turn);
            }
            rstd = 1.0f / sqrtf(ss * per + a.eps * s * s);
        }
        if constexpr (OUT == kFloat) {
            if (a.rstd && live && lane == 0) a.rstd[row] = rstd * s;
#pragma unroll
            for (int k = 0; k < ITER; ++k) {
                const int at = lane + k * LANES;
#pragma unroll
                for (int i = 0; i < V; ++i) h[k][i] = h[k][i] * rstd * w[k][i];
                if (live && at < n_vec)
                    store_any_part<V, ROWS, STREAM>(a.y, row * a.C + at * V, a.y_dtype, a.C - at * V, h[k]);
            }
        } else {
            auto largest = [&] {
                uint32_t top = 0;
#pragma unroll
                for (int k = 0; k < ITER; ++k)
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        if (lane + k * LANES < n_vec) top = larger(top, size_bits(OUT == kInt8Norm ? h[k][i] * w[k][i] : h[k][i]));
                return over_lanes<LANES>(top, larger, most, turn);
            };
            uint32_t top = largest();
            if constexpr (OUT == kInt8Norm) {
                // Products with the weights that leave fp32's range where the norm does not: once more, of
                // the row times the power of two next to 1 / rms, which leaves q as it would be.
                const bool far = top >= kInfBits || (top < __float_as_uint(0x1p-100f) && ss > 0.0f);
                if (LANES > kRmsWave ? far : __any(far)) {
                    const uint32_t power = __float_as_uint(rstd) & kInfBits;
                    const float p = far && power > 0 && power < kInfBits ? __uint_as_float(power) : 1.0f;
                    rstd /= p;
#pragma unroll
                    for (int k = 0; k < ITER; ++k)
#pragma unroll
                        for (int i = 0; i < V; ++i) h[k][i] *= p;
                    if constexpr (LANES > kRmsWave) __syncthreads();    // the slots are read
                    top = largest();
                }
            }
            const Steps steps = steps_of(top, rstd);
            if (live && lane == 0) a.scale[row] = steps.scale;
#pragma unroll
            for (int k = 0; k < ITER; ++k) {
                const int at = lane + k * LANES;
                int8_t q[V];
#pragma unroll
                for (int i = 0; i < V; ++i) q[i] = held(OUT == kInt8Norm ? h[k][i] * w[k][i] : h[k][i], steps);
                if (live && at < n_vec) store_bytes<V, ROWS>(a.q + row * a.C + at * V, a.C - at * V, q);
            }
        }
    }
}

// Rows too long for registers, a workgroup to a row: read twice, the second time from cache.
// (4096 x 16384 in bf16 takes 50 us, 201 MB at 4.0 TB/s; fp32 91.)
template <int DT, int ROWS>
__global__ __launch_bounds__(kRmsBlock) void k_quantize_long(RmsArgs a) {
    using T = typename Num<DT>::T;
    constexpr int V = kWide<DT>;
    __shared__ uint32_t most[8];
    const int n_vec = (a.C + V - 1) / V;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, ++turn) {
        const T *x = static_cast<const T *>(a.x) + row * a.ldx;
        uint32_t top = 0;
        for (int at = threadIdx.x; at < n_vec; at += kRmsBlock) {
            float v[V];
            load_part<T, V, ROWS>(x + int64_t(at) * V, a.C - at * V, v);
#pragma unroll
            for (int i = 0; i < V; ++i) top = larger(top, size_bits(v[i]));
        }
        const Steps steps = steps_of(over_lanes<kRmsBlock>(top, larger, most, turn), 1.0f);
        if (threadIdx.x == 0) a.scale[row] = steps.scale;
        for (int at = threadIdx.x; at < n_vec; at += kRmsBlock) {
            float v[V];
            int8_t q[V];
            load_part<T, V, ROWS>(x + int64_t(at) * V, a.C - at * V, v);
#pragma unroll
            for (int i = 0; i < V; ++i) q[i] = held(v[i], steps);
            store_bytes<V, ROWS>(a.q + row * a.C + int64_t(at) * V, a.C - at * V, q);
        }
    }
}

template <int DT, int LANES, int ITER, int ROWS, bool STREAM>
__global__ __launch_bounds__(kRmsBlock) void k_rms_grad(RmsArgs a) {
    using T = typename Num<DT>::T;
    constexpr int V = kWide<DT>, kRows = kRmsBlock / LANES;
    extern __shared__ float joined[];       // [n_vec * V], rows shared by a wave or less
    __shared__ float add[8];
    const int lane = threadIdx.x % LANES, n_vec = (a.C + V - 1) / V;
    const T *x = static_cast<const T *>(a.x), *res = static_cast<const T *>(a.residual);
    const T *dsum = static_cast<const T *>(a.dsum);
    T *dx = static_cast<T *>(a.sum);
    float w[ITER][V], dw[ITER][V];
#pragma unroll
    for (int k = 0; k < ITER; ++k) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            w[k][i] = 1.0f;
            dw[k][i] = 0.0f;
        }
        if (a.weight && lane + k * LANES < n_vec)
            load_any_part<V, ROWS>(a.weight, (lane + k * LANES) * V, a.w_dtype, a.C - (lane + k * LANES) * V, w[k]);
    }
    const float per = 1.0f / float(a.C);
    const int64_t begin = int64_t(blockIdx.x) * a.chunk, end = min(begin + a.chunk, a.rows);
    int turn = 0;
    for (int64_t first = begin; first < end; first += kRows, ++turn) {
        const int64_t row = first + threadIdx.x / LANES;
        const bool live = row < end;
        const float rstd = live ? a.rstd[row] : 0.0f;
        float u[ITER][V], other[ITER][V], e[ITER][V], more[ITER][V], dot = 0.0f;
#pragma unroll
        for (int k = 0; k < ITER; ++k) {
            const int at = lane + k * LANES;
#pragma unroll
            for (int i = 0; i < V; ++i) u[k][i] = other[k][i] = e[k][i] = more[k][i] = 0.0f;
            if (live && at < n_vec) {
                const int count = a.C - at * V;
                load_part<T, V, ROWS>(x + row * a.ldx + at * V, count, u[k]);
                if (res) load_part<T, V, ROWS>(res + row * a.ldr + at * V, count, other[k]);
                load_any_part<V, ROWS>(a.dy, row * a.C + at * V, a.y_dtype, count, e[k]);
                if (dsum) load_part<T, V, ROWS>(dsum + row * a.C + at * V, count, more[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < ITER; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                u[k][i] = (u[k][i] + other[k][i]) * rstd;
                dw[k][i] = fmaf(e[k][i], u[k][i], dw[k][i]);
                e[k][i] *= w[k][i];
                dot = fmaf(e[k][i], u[k][i], dot);
            }
        const float mean = over_lanes<LANES>(dot, plus, add, turn) * per;
#pragma unroll
        for (int k = 0; k < ITER; ++k) {
            const int at = lane + k * LANES;
#pragma unroll
            for (int i = 0; i < V; ++i) e[k][i] = fmaf(rstd, fmaf(-u[k][i], mean, e[k][i]), more[k][i]);
            if (live && at < n_vec) store_part<T, V, ROWS, STREAM>(dx + row * a.C + at * V, a.C - at * V, e[k]);
        }
    }
    if (!a.parts) return;
    float *part = a.parts + int64_t(blockIdx.x) * a.C;
    if constexpr (LANES > kRmsWave) {
#pragma unroll
        for (int k = 0; k < ITER; ++k)
            if (lane + k * LANES < n_vec)
                store_part<float, V, ROWS>(part + (lane + k * LANES) * V, a.C - (lane + k * LANES) * V, dw[k]);
    } else {
        // over the rows of a wave, then one wave after the other
#pragma unroll
        for (int k = 0; k < ITER; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int m = LANES; m < kRmsWave; m <<= 1) dw[k][i] += __shfl_xor(dw[k][i], m);
        constexpr int kWaves = kRmsBlock / kRmsWave;
        const int wave = threadIdx.x / kRmsWave;
        for (int turns = 0; turns < kWaves; ++turns) {
            if (wave == turns && threadIdx.x % kRmsWave < LANES)
#pragma unroll
                for (int k = 0; k < ITER; ++k) {
                    const int at = lane + k * LANES;
                    if (at >= n_vec) continue;
#pragma unroll
                    for (int i = 0; i < V; ++i) {       // of whole vectors: joined has their room
                        if (turns > 0) dw[k][i] += joined[at * V + i];
                        joined[at * V + i] = dw[k][i];
                    }
                    if (turns == kWaves - 1) store_part<float, V, ROWS>(part + at * V, a.C - at * V, dw[k]);
                }
            __syncthreads();
        }
    }
}

// dw = the sum of the parts, in halves over the lanes that share a channel.
__global__ __launch_bounds__(kRmsJoinBlock) void k_rms_join(const float *parts, int n, int C, void *dw, int dtype) {
    constexpr int kLanes = kRmsJoinBlock / kRmsJoinChannels;
    __shared__ float th[kLanes][kRmsJoinChannels + 1];
    const int i = threadIdx.x % kRmsJoinChannels, lane = threadIdx.x / kRmsJoinChannels;
    const int c = blockIdx.x * kRmsJoinChannels + i;
    float sum = 0.0f;
    if (c < C)
#pragma unroll 8
        for (int p = lane; p < n; p += kLanes) sum += parts[int64_t(p) * C + c];
    th[lane][i] = sum;
    for (int half = kLanes / 2; half > 0; half /= 2) {
        __syncthreads();
        if (lane < half) th[lane][i] += th[lane + half][i];
    }
    if (lane == 0 && c < C) store_any<1>(dw, c, dtype, &th[0][i]);
}

// A form: lanes that share a row, accesses of a lane.
struct Form {
    int lanes, iter;
};

constexpr int64_t kRmsGroups = 2048;    // workgroups that stay: eight to a compute unit

// How rows of C elements lie that start at p and are so many elements apart.
int rows_lie(int32_t dtype, int32_t C, std::initializer_list<const void *> p, std::initializer_list<int64_t> strides) {
    const int v = dtype == BEVPOOL_F32 ? 4 : 8;
    if (C < v) return kShort;
    bool even = C % v == 0;
    for (const void *q : p) even = even && aligned_for(q, 0, dtype, v);
    for (int64_t s : strides) even = even && aligned_for(nullptr, s, dtype, v);
    return even ? kEven : kUneven;
}
// The same where something of another type, which starts at p, has rows beside them.
int beside(int lie, int32_t dtype, const void *p) {
    return lie == kEven && !aligned_for(p, 0, dtype, 8) ? kUneven : lie;
}
int beside_bytes(int lie, const void *p) { return lie == kEven && reinterpret_cast<uintptr_t>(p) % 8 ? kUneven : lie; }

// A row of up to a wave's accesses takes the fewest lanes; a longer one a wave, two accesses
// a lane, where rows are many, else a workgroup. (Four and eight accesses of a wave were
// slower than a workgroup: steps of 16896 x 2048 157 us against 115, of 8192 x 4096 172
// against 137; two were not: 33000 x 1024 129 against 136.)
Form form_of(int32_t dtype, int32_t C, int64_t rows) {
    const int v = dtype == BEVPOOL_F32 ? 4 : 8, n = (C + v - 1) / v;
    if (n <= 64) return {n <= 8 ? 8 : n <= 16 ? 16 : n <= 32 ? 32 : 64, 1};
    if (n <= 128 && rows >= 4 * kRmsGroups) return {64, 2};
    return {256, n <= 256 ? 1 : n <= 512 ? 2 : n <= 1024 ? 4 : 8};
}

// body(constants LANES, ITER) of a form
template <int DT, int ROWS, class F>
void with_form(const Form &f, F body) {
    if (ROWS == kShort || f.lanes == 8) return body(Int<8>(), Int<1>());
    if constexpr (ROWS != kShort) {
        if (f.lanes == 16) return body(Int<16>(), Int<1>());
        if (f.lanes == 32) return body(Int<32>(), Int<1>());
        if (f.lanes == 64) return f.iter == 1 ? body(Int<64>(), Int<1>()) : body(Int<64>(), Int<2>());
        if (f.iter == 1) return body(Int<256>(), Int<1>());
        if (f.iter == 2) return body(Int<256>(), Int<2>());
        if (f.iter == 4) return body(Int<256>(), Int<4>());
        if constexpr (kWide<DT> == 4) body(Int<256>(), Int<8>());
    }
}

template <int OUT>
int launch_rows(const RmsArgs &a, int32_t dtype, int lie, hipStream_t stream) {
    const Form f = form_of(dtype, a.C, a.rows);
    const bool past = OUT != kInt8 && past_caches(a.rows * a.C * dtype_bytes(dtype));
    const int64_t each = kRmsBlock / f.lanes, all = (a.rows + each - 1) / each;
    const dim3 grid{uint32_t(all < kRmsGroups ? all : kRmsGroups)}, wg(kRmsBlock);
    with_type_and_rows(dtype, lie, [&](auto dt, auto how) {
        constexpr int DT = decltype(dt)::value;
        constexpr int ROWS = decltype(how)::value;
        constexpr bool kMay = ROWS == kEven && OUT != kInt8;    // writes whole 16 bytes
        with_form<DT, ROWS>(f, [&](auto lanes, auto iter) {
            constexpr int L = decltype(lanes)::value, I = decltype(iter)::value;
            if (kMay && past) hipLaunchKernelGGL((k_rms<DT, L, I, OUT, ROWS, kMay>), grid, wg, 0, stream, a);
            else hipLaunchKernelGGL((k_rms<DT, L, I, OUT, ROWS, false>), grid, wg, 0, stream, a);
        });
    });
    BEVPOOL_HIP(hipGetLastError());
    return BEVPOOL_OK;
}

// Rows of a workgroup of the backward, a multiple of those it takes at once.
int64_t chunk_of(int64_t rows, int64_t each) {
    // eight rows or more to a lane, so that parts of dw cost little beside the rows, if that
    // leaves two workgroups to a compute unit
    const int64_t share = (rows + kRmsGroups - 1) / kRmsGroups, half = (rows + 511) / 512;
    int64_t chunk = half < 8 * each ? half : 8 * each;
    if (share > chunk) chunk = share;
    return (chunk + each - 1) / each * each;
}

}  // namespace
}  // namespace bevmap

using namespace bevmap;

// Parts of dw: as many as any form of these sizes makes.
int64_t bevmap_rms_workspace_bytes(const bevmap_rms &n) {
    if (n.rows == 0) return 0;
    int64_t most = 0;
    for (int64_t each : {1, 4, 8, 16, 32}) {    // rows that the forms take at once
        const int64_t chunk = chunk_of(n.rows, each), groups = (n.rows + chunk - 1) / chunk;
        if (groups > most) most = groups;
    }
    return most * n.channels * int64_t(sizeof(float));
}

int bevmap_launch_rms_norm(const bevmap_rms &n, const void *x, const void *residual, const void *weight, void *sum,
                           void *y, float *rstd, int8_t *q, float *scale, hipStream_t stream) {
    if (n.rows == 0) return BEVPOOL_OK;
    RmsArgs a{};
    a.x = x;
    a.residual = residual;
    a.weight = weight;
    a.sum = sum;
    a.y = y;
    a.rstd = rstd;
    a.q = q;
    a.scale = scale;
    a.ldx = n.x_stride;
    a.ldr = n.residual_stride;
    a.rows = n.rows;
    a.C = n.channels;
    a.y_dtype = n.y_dtype;
    a.w_dtype = n.weight_dtype;
    a.eps = n.eps;
    const bool one = n.rows == 1;
    int lie = rows_lie(n.x_dtype, n.channels, {x, residual, sum},
                       {one ? 0 : n.x_stride, one || !residual ? 0 : n.residual_stride});
    lie = beside(lie, n.weight_dtype, weight);
    if (q) return launch_rows<kInt8Norm>(a, n.x_dtype, beside_bytes(lie, q), stream);
    return launch_rows<kFloat>(a, n.x_dtype, beside(lie, n.y_dtype, y), stream);
}

int bevmap_launch_quantize(const void *x, int64_t x_stride, int8_t *q, float *scale, int64_t rows, int32_t columns,
                           int32_t dtype, hipStream_t stream) {
    if (rows == 0) return BEVPOOL_OK;
    RmsArgs a{};
    a.x = x;
    a.q = q;
    a.scale = scale;
    a.ldx = x_stride;
    a.rows = rows;
    a.C = columns;
    const int lie = beside_bytes(rows_lie(dtype, columns, {x}, {rows == 1 ? 0 : x_stride}), q);
    if (columns <= kNormMaxChannels) return launch_rows<kInt8>(a, dtype, lie, stream);
    const dim3 grid{uint32_t(rows < kRmsGroups ? rows : kRmsGroups)}, wg(kRmsBlock);
    with_type_and_rows(dtype, lie, [&](auto dt, auto how) {
        hipLaunchKernelGGL((k_quantize_long<decltype(dt)::value, decltype(how)::value>), grid, wg, 0, stream, a);
    });
    BEVPOOL_HIP(hipGetLastError());
    return BEVPOOL_OK;
}

int bevmap_launch_rms_norm_backward(const bevmap_rms &n, const void *grad_y, const void *grad_sum, const void *x,
                                    const void *residual, const void *weight, const float *rstd, void *grad_x,
                                    void *grad_weight, void *workspace, hipStream_t stream) {
    int64_t groups = 0;
    float *parts = grad_weight ? static_cast<float *>(workspace) : nullptr;
    if (n.rows > 0) {
        RmsArgs a{};
        a.x = x;
        a.residual = residual;
        a.weight = weight;
        a.dy = grad_y;
        a.dsum = grad_sum;
        a.sum = grad_x;
        a.rstd = const_cast<float *>(rstd);
        a.parts = parts;
        a.ldx = n.x_stride;
        a.ldr = n.residual_stride;
        a.rows = n.rows;
        a.C = n.channels;
        a.y_dtype = n.y_dtype;
        a.w_dtype = n.weight_dtype;
        const bool one = n.rows == 1;
        int lie = rows_lie(n.x_dtype, n.channels, {x, residual, grad_sum, grad_x},
                           {one ? 0 : n.x_stride, one || !residual ? 0 : n.residual_stride});
        lie = beside(beside(lie, n.weight_dtype, weight), n.y_dtype, grad_y);
        const Form f = form_of(n.x_dtype, n.channels, n.rows);
        const int64_t each = kRmsBlock / f.lanes;
        a.chunk = chunk_of(n.rows, each);
        groups = (n.rows + a.chunk - 1) / a.chunk;
        const dim3 grid{uint32_t(groups)}, wg(kRmsBlock);
        const bool past = past_caches(n.rows * n.channels * dtype_bytes(n.x_dtype));
        with_type_and_rows(n.x_dtype, lie, [&](auto dt, auto how) {
            constexpr int DT = decltype(dt)::value;
            constexpr int ROWS = decltype(how)::value;
            with_form<DT, ROWS>(f, [&](auto lanes, auto iter) {
                constexpr int L = decltype(lanes)::value, I = decltype(iter)::value;
                const size_t lds = L <= kRmsWave ? size_t(L) * I * kWide<DT> * sizeof(float) : 0;
                if (ROWS == kEven && past) hipLaunchKernelGGL((k_rms_grad<DT, L, I, ROWS, ROWS == kEven>), grid, wg, lds, stream, a);
                else hipLaunchKernelGGL((k_rms_grad<DT, L, I, ROWS, false>), grid, wg, lds, stream, a);
            });
        });
        BEVPOOL_HIP(hipGetLastError());
    }
    if (grad_weight) {
        const dim3 grid{uint32_t((n.channels + kRmsJoinChannels - 1) / kRmsJoinChannels)}, wg(kRmsJoinBlock);
        hipLaunchKernelGGL(k_rms_join, grid, wg, 0, stream, parts, int(groups), n.channels, grad_weight,
                           n.weight_dtype);
        BEVPOOL_HIP(hipGetLastError());
    }
    return BEVPOOL_OK;
}
