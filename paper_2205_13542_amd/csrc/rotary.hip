// Rotary positions (bevmap_rotary): pair p of a head's channels is turned by the angle
// position[axis(p)] * frequency[p],
//   (a, b) -> amplitude (a cos - b sin, a sin + b cos).
// The gradient is the turn by the negative angle of the same amplitude.
//
// A workgroup takes a tile of tokens. It forms the sines and cosines of the tile's
// (token, pair) once into LDS, since all heads share them, and then walks the tile's
// channels 16 bytes at a time in the order in which they lie in memory: bound by memory.
// 8192 tokens of 16 heads of 128, 67 MB, take 12 us; 129600 of 4 of 32 in halves, 66 MB, 16.
//
// The angle is reduced in 64 bits, as turns: position * frequency / (2 pi) with what each
// product rounds off kept, less whole turns and the nearest quarter, so that a position
// far into a context is turned as exactly as a near one.
#include "mapops.h"

namespace bevmap {
namespace {

constexpr int kTurnBlock = 256;
constexpr int kTurnAhead = 2;           // units of a thread that are on their way at once
constexpr int kTurnEntries = 2048;      // (cos, sin) of a tile, 16 KB
constexpr int64_t kTurnGroups = 1 << 16;

struct TurnArgs {
    const void *x, *positions;
    const double *frequencies;
    void *out;
    int64_t x_batch, x_row, x_head, tokens;     // tokens: batch * tokens of a sample
    int32_t per_sample, heads, dim, pairs, axes, positions_type;
    int32_t tile;                               // tokens of a workgroup's turn
    bevpool::FastDiv by_sample, by_pairs, by_axis, by_head, by_units;
    float amplitude, sign;
};

__device__ __forceinline__ double position_at(const TurnArgs &a, int64_t i) {
    if (a.positions_type == BEVMAP_POSITION_I32) return double(static_cast<const int32_t *>(a.positions)[i]);
    if (a.positions_type == BEVMAP_POSITION_I64) return double(static_cast<const int64_t *>(a.positions)[i]);
    return double(static_cast<const float *>(a.positions)[i]);
}

// (cos, sin) of position * frequency. Within an eighth of a turn either way, the series
// of the two, the first term left out below 2^-28.
__device__ __forceinline__ float2 turn_of(double position, double frequency) {
    constexpr double kHigh = 0x1.45f306dc9c883p-3, kLow = -0x1.6b01ec5417056p-57;     // 1 / (2 pi) in two pieces
    const double angle = position * frequency, rest = fma(position, frequency, -angle);
    const double turns = angle * kHigh, fine = fma(angle, kHigh, -turns) + fma(angle, kLow, rest * kHigh);
    const double part = (turns - rint(turns)) + fine, quarter = rint(4.0 * part);
    const float y = float((part - 0.25 * quarter) * 6.283185307179586);
    const float s = y * y;
    float sine = fmaf(s, fmaf(s, fmaf(s, fmaf(s, 1.0f / 362880.0f, -1.0f / 5040.0f), 1.0f / 120.0f), -1.0f / 6.0f), 0.0f);
    sine = fmaf(y, sine, y);
    const float cosine =
        fmaf(s, fmaf(s, fmaf(s, fmaf(s, fmaf(s, -1.0f / 3628800.0f, 1.0f / 40320.0f), -1.0f / 720.0f), 1.0f / 24.0f),
                     -0.5f), 1.0f);
    const int k = int(quarter) & 3;
    const float c = k & 1 ? sine : cosine, d = k & 1 ? cosine : sine;
    return make_float2(k == 1 || k == 2 ? -c : c, k >= 2 ? -d : d);
}

// V: elements of an access. A unit is V pairs in halves (two accesses), V / 2 pairs
// interleaved (one access; with V = 1 one pair in two), or V channels that keep their place.
template <int DT, int V, bool MIXED, bool STREAM>
__global__ __launch_bounds__(kTurnBlock) void k_turn(TurnArgs a) {
    using T = typename Num<DT>::T;
    extern __shared__ float2 turns[];            // [tile][pairs]
    const T *x = static_cast<const T *>(a.x);
    T *out = static_cast<T *>(a.out);
    constexpr int kEach = MIXED ? (V > 1 ? V / 2 : 1) : V;      // pairs of a unit
    constexpr bool kOne = MIXED && V > 1;                       // one access to a unit
    const int turned = a.pairs / kEach, units = turned + (a.dim - 2 * a.pairs) / V;
    const int apart = MIXED ? 1 : a.pairs;
    for (int64_t first = int64_t(blockIdx.x) * a.tile; first < a.tokens; first += int64_t(gridDim.x) * a.tile) {
        const int n = int(min(int64_t(a.tile), a.tokens - first)), all = n * a.heads * units;
        for (int begin = 0; begin < all; begin += kTurnAhead * kTurnBlock) {
            // a thread's units are on their way while it forms the tile's sines and cosines
            Pack<T, V> low[kTurnAhead], high[kTurnAhead];
            T *to[kTurnAhead];
            int turn[kTurnAhead];           // first of the unit's pairs among the tile's; -1: channels that stay
#pragma unroll
            for (int j = 0; j < kTurnAhead; ++j) {
                const int i = begin + j * kTurnBlock + threadIdx.x;
                to[j] = nullptr;
                if (i >= all) continue;
                const uint32_t th = bevpool::fdiv(i, a.by_units), u = i - th * units;
                const uint32_t t = bevpool::fdiv(th, a.by_head), head = th - t * a.heads;
                const uint32_t token = uint32_t(first + t), b = bevpool::fdiv(token, a.by_sample);
                const bool turns_it = int(u) < turned;
                const int c = !turns_it ? 2 * a.pairs + int(u - turned) * V : MIXED && V == 1 ? 2 * u : u * V;
                const T *from = x + int64_t(b) * a.x_batch + int64_t(token - b * a.per_sample) * a.x_row +
                                head * a.x_head + c;
                low[j] = *reinterpret_cast<const Pack<T, V> *>(from);
                if (!kOne && turns_it) high[j] = *reinterpret_cast<const Pack<T, V> *>(from + apart);
                turn[j] = turns_it ? int(t * a.pairs + u * kEach) : -1;
                to[j] = out + (int64_t(token) * a.heads + head) * a.dim + c;
            }
            if (begin == 0) {
                for (int i = threadIdx.x; i < n * a.pairs; i += kTurnBlock) {
                    const uint32_t t = bevpool::fdiv(i, a.by_pairs), p = i - t * a.pairs;
                    const int64_t at = (first + t) * a.axes + bevpool::fdiv(p, a.by_axis);
                    const float2 cs = turn_of(position_at(a, at), a.frequencies[p]);
                    turns[i] = make_float2(cs.x * a.amplitude, cs.y * a.amplitude * a.sign);
                }
                __syncthreads();
            }
#pragma unroll
            for (int j = 0; j < kTurnAhead; ++j) {
                if (!to[j]) continue;
                float v[V];
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] = float(low[j].v[e]);
                if (turn[j] >= 0) {
                    const float2 *cs = turns + turn[j];
                    if constexpr (kOne) {
#pragma unroll
                        for (int e = 0; e < V / 2; ++e) {
                            const float p = v[2 * e], q = v[2 * e + 1];
                            v[2 * e] = fmaf(p, cs[e].x, -q * cs[e].y);
                            v[2 * e + 1] = fmaf(p, cs[e].y, q * cs[e].x);
                        }
                    } else {
                        float w[V];
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            const float p = v[e], q = float(high[j].v[e]);
                            v[e] = fmaf(p, cs[e].x, -q * cs[e].y);
                            w[e] = fmaf(p, cs[e].y, q * cs[e].x);
                        }
                        store_n<T, V, STREAM>(to[j] + apart, w);
                    }
                }
                store_n<T, V, STREAM>(to[j], v);
            }
        }
        __syncthreads();
    }
}

template <int DT, int V, bool MIXED>
void launch(const TurnArgs &a, hipStream_t stream) {
    const int64_t all = (a.tokens + a.tile - 1) / a.tile;
    const dim3 grid{uint32_t(all < kTurnGroups ? all : kTurnGroups)}, wg(kTurnBlock);
    const size_t lds = size_t(a.tile) * a.pairs * sizeof(float2);
    if (V > 2 && past_caches(a.tokens * a.heads * a.dim * dtype_bytes(DT)))
        hipLaunchKernelGGL((k_turn<DT, V, MIXED, (V > 2)>), grid, wg, lds, stream, a);
    else
        hipLaunchKernelGGL((k_turn<DT, V, MIXED, false>), grid, wg, lds, stream, a);
}

template <int DT, int V>
void launch(const TurnArgs &a, bool mixed, hipStream_t stream) {
    if (mixed) launch<DT, V, true>(a, stream);
    else launch<DT, V, false>(a, stream);
}

template <int DT>
void launch(const TurnArgs &a, int v, bool mixed, hipStream_t stream) {
    constexpr int kWide = DT == BEVPOOL_F32 ? 4 : 8;
    if (v == kWide) launch<DT, kWide>(a, mixed, stream);
    else if (v == 2) launch<DT, 2>(a, mixed, stream);
    else launch<DT, 1>(a, mixed, stream);
}

}  // namespace
}  // namespace bevmap

using namespace bevmap;

int bevmap_launch_rotary(const bevmap_turn &n, const void *x, const void *positions, const double *frequencies,
                         void *out, bool backward, hipStream_t stream) {
    TurnArgs a{};
    a.tokens = int64_t(n.batch) * n.tokens;
    if (a.tokens == 0) return BEVPOOL_OK;
    a.x = x;
    a.positions = positions;
    a.frequencies = frequencies;
    a.out = out;
    a.x_batch = n.x_batch;
    a.x_row = n.x_row;
    a.x_head = n.x_head;
    a.per_sample = n.tokens;
    a.heads = n.heads;
    a.dim = n.dim;
    a.pairs = n.pairs;
    a.axes = n.axes;
    a.positions_type = n.positions_type;
    a.amplitude = n.amplitude;
    a.sign = backward ? -1.0f : 1.0f;
    const bool mixed = n.interleaved != 0;
    int v = 1;
    for (int wide : {n.dtype == BEVPOOL_F32 ? 4 : 8, 2}) {
        const bool fits = n.dim % wide == 0 && (mixed ? 2 * n.pairs : n.pairs) % wide == 0 &&
                          aligned_for(x, n.heads > 1 ? n.x_head : 0, n.dtype, wide) &&
                          aligned_for(x, n.tokens > 1 ? n.x_row : 0, n.dtype, wide) &&
                          aligned_for(x, n.batch > 1 ? n.x_batch : 0, n.dtype, wide) &&
                          aligned_for(out, 0, n.dtype, wide);
        if (fits) {
            v = wide;
            break;
        }
    }
    const int each = mixed ? (v > 1 ? v / 2 : 1) : v;
    const int units = n.pairs / each + (n.dim - 2 * n.pairs) / v;
    // Tokens of a tile: a unit and a pair to every thread, less where that leaves compute units
    // without work. (129600 tokens, 4 heads of 32: 36 us a step; two units to a thread 44, four 52.)
    auto per = [](int64_t of, int64_t each) { return (of + each - 1) / each; };
    const int64_t by_unit = per(kTurnBlock, int64_t(n.heads) * units), by_pair = per(kTurnBlock, n.pairs);
    int64_t tile = by_unit > by_pair ? by_unit : by_pair;
    if (tile > kTurnEntries / n.pairs) tile = kTurnEntries / n.pairs;
    const int64_t spread = (a.tokens + 1023) / 1024;     // a tile's units are 2^31 only where out is 2^41
    if (tile > spread) tile = spread;
    a.tile = int32_t(tile < 1 ? 1 : tile);
    a.by_sample = bevpool::make_fastdiv(uint32_t(n.tokens));
    a.by_pairs = bevpool::make_fastdiv(uint32_t(n.pairs));
    a.by_axis = bevpool::make_fastdiv(uint32_t(n.pairs / n.axes));
    a.by_head = bevpool::make_fastdiv(uint32_t(n.heads));
    a.by_units = bevpool::make_fastdiv(uint32_t(units));
    if (n.dtype == BEVPOOL_F32) launch<BEVPOOL_F32>(a, v, mixed, stream);
    else if (n.dtype == BEVPOOL_BF16) launch<BEVPOOL_BF16>(a, v, mixed, stream);
    else launch<BEVPOOL_F16>(a, v, mixed, stream);
    BEVPOOL_HIP(hipGetLastError());
    return BEVPOOL_OK;
}
