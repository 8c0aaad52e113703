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

// An access has V elements. A unit is V pairs in halves (two accesses), V / 2 pairs
// interleaved (one access), or V channels that keep their place. Short rows (kShort) go pair
// by pair.
template <int DT, bool MIXED, int ROWS, bool STREAM>
__global__ __launch_bounds__(kTurnBlock) void k_turn(TurnArgs a) {
    using T = typename Num<DT>::T;
    constexpr int V = ROWS != kShort ? kWide<DT> : MIXED ? 2 : 1;
    extern __shared__ float2 turns[];            // [tile][pairs]
    const T *x = static_cast<const T *>(a.x);
    T *out = static_cast<T *>(a.out);
    constexpr int kEach = MIXED ? V / 2 : V;                    // pairs of a unit
    const int turned = (a.pairs + kEach - 1) / kEach, rest = a.dim - 2 * a.pairs, units = turned + (rest + V - 1) / V;
    for (int64_t first = int64_t(blockIdx.x) * a.tile; first < a.tokens; first += int64_t(gridDim.x) * a.tile) {
        const int n = int(min(int64_t(a.tile), a.tokens - first)), all = n * a.heads * units;
        for (int begin = 0; begin < all; begin += kTurnAhead * kTurnBlock) {
            // a thread's units are on their way while it forms the tile's sines and cosines
            float low[kTurnAhead][V], high[kTurnAhead][V];
            T *to[kTurnAhead];
            int count[kTurnAhead];          // elements of an access
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
                const int c = turns_it ? u * V : 2 * a.pairs + int(u - turned) * V;
                const T *from = x + int64_t(b) * a.x_batch + int64_t(token - b * a.per_sample) * a.x_row +
                                head * a.x_head + c;
                count[j] = !turns_it ? a.dim - c : MIXED ? 2 * a.pairs - c : a.pairs - c;
                if constexpr (ROWS == kShort) {
#pragma unroll
                    for (int e = 0; e < V; ++e) low[j][e] = e < count[j] ? float(from[e]) : 0.0f;
                    if (!MIXED && turns_it) high[j][0] = float(from[a.pairs]);
                } else {        // a window over the end of the channels that stay begins among the others
                    load_part<T, V, ROWS>(from, count[j], low[j]);
                    if (!MIXED && turns_it) load_part<T, V, ROWS>(from + a.pairs, count[j], high[j]);
                }
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
                float(&v)[V] = low[j];
                if (turn[j] >= 0) {
                    // (an uneven unit's last angles are another's, for elements that are not written)
                    const float2 *cs = turns + turn[j];
                    if constexpr (MIXED) {
#pragma unroll
                        for (int e = 0; e < V / 2; ++e) {
                            const float p = v[2 * e], q = v[2 * e + 1];
                            v[2 * e] = fmaf(p, cs[e].x, -q * cs[e].y);
                            v[2 * e + 1] = fmaf(p, cs[e].y, q * cs[e].x);
                        }
                    } else {
                        float(&w)[V] = high[j];
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            const float p = v[e], q = w[e];
                            v[e] = fmaf(p, cs[e].x, -q * cs[e].y);
                            w[e] = fmaf(p, cs[e].y, q * cs[e].x);
                        }
                        if constexpr (ROWS == kShort) to[j][a.pairs] = T(w[0]);
                        else store_part<T, V, ROWS, STREAM>(to[j] + a.pairs, count[j], w);
                    }
                }
                if constexpr (ROWS == kShort) {
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        if (e < count[j]) to[j][e] = T(v[e]);
                } else {
                    store_part<T, V, ROWS, STREAM>(to[j], count[j], v);
                }
            }
        }
        __syncthreads();
    }
}

template <int DT, bool MIXED, int ROWS>
void launch(const TurnArgs &a, hipStream_t stream) {
    const int64_t all = (a.tokens + a.tile - 1) / a.tile;
    const dim3 grid{uint32_t(all < kTurnGroups ? all : kTurnGroups)}, wg(kTurnBlock);
    // room for the angles that an uneven unit reads and does not use
    const size_t lds = (size_t(a.tile) * a.pairs + kWide<DT>) * sizeof(float2);
    // (not in halves: their accesses write parts of cache lines, which only a cache joins: 50000 x 8
    // heads of 64 with 20 pairs, fp32, 81 us past the caches and 44 through them)
    if (MIXED && ROWS == kEven && past_caches(a.tokens * a.heads * a.dim * dtype_bytes(DT)))
        hipLaunchKernelGGL((k_turn<DT, MIXED, ROWS, MIXED && ROWS == kEven>), grid, wg, lds, stream, a);
    else
        hipLaunchKernelGGL((k_turn<DT, MIXED, ROWS, false>), grid, wg, lds, stream, a);
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
    int v = n.dtype == BEVPOOL_F32 ? 4 : 8;
    const int part = mixed ? 2 * n.pairs : n.pairs, rest = n.dim - 2 * n.pairs;     // what is read as a row
    const bool even = rest % v == 0 && part % v == 0 && aligned_for(x, n.heads > 1 ? n.x_head : 0, n.dtype, v) &&
                      aligned_for(x, n.tokens > 1 ? n.x_row : 0, n.dtype, v) &&
                      aligned_for(x, n.batch > 1 ? n.x_batch : 0, n.dtype, v) && aligned_for(out, 0, n.dtype, v);
    // Pair by pair where an access is longer than a row, and where few accesses of a half are whole
    // (129600 x 4 x 32 with 15 pairs in halves: bf16 26 us against 34, fp32 27 against 36; 42 of
    // 84 channels: bf16 24 by wide accesses).
    const bool few = !mixed && (n.dtype == BEVPOOL_F32 || part < 2 * v);
    const int lie = even ? kEven : part < v || few ? kShort : kUneven;
    if (lie == kShort) v = mixed ? 2 : 1;
    const int each = mixed ? v / 2 : v, units = (n.pairs + each - 1) / each + (rest + v - 1) / v;
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
    with_type_and_rows(n.dtype, lie, [&](auto dt, auto how) {
        constexpr int DT = decltype(dt)::value, ROWS = decltype(how)::value;
        if (mixed) launch<DT, true, ROWS>(a, stream);
        else launch<DT, false, ROWS>(a, stream);
    });
    BEVPOOL_HIP(hipGetLastError());
    return BEVPOOL_OK;
}
