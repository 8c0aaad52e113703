// Gated activation y = act(g) v, the halves of a row, and its gradients
// (bevmap_gated_act, bevmap_gated_act_backward). What the backward needs of the row
// is the row itself, or a copy in 8 bits.
//
//   dg = dy v act'(g),  dv = dy act(g)
//
// The copy: kBlock neighbouring channels of a half share the least power of two 2^e
// whose 127-fold reaches their largest magnitude, and are held as q = round(x / 2^e).
// Products with powers of two are exact, so q depends on x alone (no rounding stands
// before the one that is meant), and is off by at most 1 / 127 of the block's largest.
// 8.25 bits an element; the exponent is stored with a bias of 127.
//
// Bound by memory. A thread takes V neighbouring channels of both halves, and
// neighbouring lanes the rest of their blocks, whose largest goes through the lanes.
// 129600 x 640 in bf16 takes 54-56 us with the copy (335 MB, 6.0 TB/s), 52 backward from it.
#include "activation.h"
#include "mapops.h"

namespace bevmap {
namespace {

constexpr int kGateBlock = 256;
constexpr int kHeld = 32;               // channels that share an exponent
constexpr int kNanExponent = 255;       // of a block with an infinity or a NaN
constexpr int64_t kGateGroups = 1 << 16;

struct GateArgs {
    const void *x, *dy;
    void *y, *dx;
    int8_t *q;                  // [rows][2][F]
    uint8_t *e;                 // [rows][2][blocks]
    int64_t ldx, rows, units;   // units: threads' worth of work, whole blocks of every row
    int32_t F, blocks, act;
    bool held;                  // write q and e
};

// The largest magnitude's bits over the lanes that share a block.
template <int V>
__device__ __forceinline__ uint32_t block_top(const float *v) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const uint32_t b = __float_as_uint(v[i]) & 0x7FFFFFFFu;
        top = b > top ? b : top;
    }
#pragma unroll
    for (int m = 1; m < kHeld / V; m <<= 1) {
        const uint32_t b = __shfl_xor(top, m);
        top = b > top ? b : top;
    }
    return top;
}

// The least e with 127 * 2^e >= top, held to what a byte with a bias of 127 says; what is
// then below half of 2^-127 is 0. 127 is 1.984375 * 2^6.
__device__ __forceinline__ int exponent_of(uint32_t top) {
    const int e = int(top >> 23) - 127 - 6 + ((top & 0x7FFFFFu) > 0x7E0000u);
    return e > -127 ? e : -127;
}

// count: channels of the unit, 0 of one past the row's end.
template <int V, int ROWS>
__device__ __forceinline__ void hold(const float *v, int8_t *q, uint8_t *e, int count, bool first) {
    const uint32_t top = block_top<V>(v);
    const bool none = top >= 0x7F800000u;
    const int ex = exponent_of(top);
    int8_t b[V];
#pragma unroll
    for (int i = 0; i < V; ++i) b[i] = int8_t(none ? 0.0f : rintf(ldexpf(v[i], -ex)));
    if (count > 0) store_bytes<V, ROWS>(q, count, b);
    if (first) *e = uint8_t(none ? kNanExponent : ex + 127);
}

template <int V, int ROWS>
__device__ __forceinline__ void release(const int8_t *q, uint8_t e, int count, float *v) {
    int8_t b[V];
    load_bytes<V, ROWS>(q, count, b);
#pragma unroll
    for (int i = 0; i < V; ++i)
        v[i] = e == kNanExponent ? __uint_as_float(0x7FC00000u) : ldexpf(float(b[i]), int(e) - 127);
}

// Unit n of a pass: row and first channel; whole blocks of kHeld / V units each.
struct Place {
    int64_t row;
    int32_t c;
};
template <int V>
__device__ __forceinline__ Place place_of(int64_t n, int32_t blocks) {
    const int32_t per = blocks * (kHeld / V);
    Place p;
    p.row = n / per;
    p.c = int32_t(n - p.row * per) * V;
    return p;
}

template <int DT, int ROWS, bool STREAM>
__global__ __launch_bounds__(kGateBlock) void k_gate(GateArgs a) {
    using T = typename Num<DT>::T;
    constexpr int V = kWide<DT>;
    const T *x = static_cast<const T *>(a.x);
    T *y = static_cast<T *>(a.y);
    // whole waves stay together, for the lanes that share a block
    for (int64_t n0 = int64_t(blockIdx.x) * kGateBlock; n0 < a.units; n0 += int64_t(gridDim.x) * kGateBlock) {
        const int64_t n = n0 + threadIdx.x;
        const Place p = place_of<V>(n, a.blocks);
        const int count = n < a.units && p.c < a.F ? a.F - p.c : 0;
        float g[V], v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] = v[i] = 0.0f;
        if (count > 0) {
            load_part<T, V, ROWS>(x + p.row * a.ldx + p.c, count, g);
            load_part<T, V, ROWS>(x + p.row * a.ldx + a.F + p.c, count, v);
        }
        if (a.held) {
            int8_t *q = a.q + p.row * 2 * a.F + p.c;
            uint8_t *e = a.e + p.row * 2 * a.blocks + p.c / kHeld;
            const bool first = count > 0 && p.c % kHeld == 0;
            hold<V, ROWS>(g, q, e, count, first);
            hold<V, ROWS>(v, q + a.F, e + a.blocks, count, first);
        }
        with_act(a.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] *= activate<act.value>(g[i]);
        });
        if (count > 0) store_part<T, V, ROWS, STREAM>(y + p.row * a.F + p.c, count, v);
    }
}

template <int DT, int ROWS, bool HELD, bool STREAM>
__global__ __launch_bounds__(kGateBlock) void k_gate_grad(GateArgs a) {
    using T = typename Num<DT>::T;
    constexpr int V = kWide<DT>;
    const T *x = static_cast<const T *>(a.x), *dy = static_cast<const T *>(a.dy);
    T *dx = static_cast<T *>(a.dx);
    for (int64_t n = int64_t(blockIdx.x) * kGateBlock + threadIdx.x; n < a.units;
         n += int64_t(gridDim.x) * kGateBlock) {
        const Place p = place_of<V>(n, a.blocks);
        const int count = a.F - p.c;
        if (count <= 0) continue;
        float g[V], v[V], d[V];
        load_part<T, V, ROWS>(dy + p.row * a.F + p.c, count, d);
        if constexpr (HELD) {
            const int8_t *q = a.q + p.row * 2 * a.F + p.c;
            const uint8_t *e = a.e + p.row * 2 * a.blocks + p.c / kHeld;
            release<V, ROWS>(q, e[0], count, g);
            release<V, ROWS>(q + a.F, e[a.blocks], count, v);
        } else {
            load_part<T, V, ROWS>(x + p.row * a.ldx + p.c, count, g);
            load_part<T, V, ROWS>(x + p.row * a.ldx + a.F + p.c, count, v);
        }
        with_act(a.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float gate = g[i];
                g[i] = d[i] * v[i] * slope<act.value>(gate);
                v[i] = d[i] * activate<act.value>(gate);
            }
        });
        store_part<T, V, ROWS, STREAM>(dx + p.row * 2 * a.F + p.c, count, g);
        store_part<T, V, ROWS, STREAM>(dx + p.row * 2 * a.F + a.F + p.c, count, v);
    }
}

// How the halves of rows lie.
int halves_lie(const bevmap_gate &n, const void *x, const void *y, const void *dx, const void *q) {
    const int v = n.dtype == BEVPOOL_F32 ? 4 : 8;
    if (n.features < v) return kShort;
    const bool even = n.features % v == 0 && aligned_for(x, n.rows == 1 ? 0 : n.x_stride, n.dtype, v) &&
                      aligned_for(y, 0, n.dtype, v) && aligned_for(dx, 0, n.dtype, v) &&
                      reinterpret_cast<uintptr_t>(q) % 8 == 0;
    return even ? kEven : kUneven;
}

GateArgs args_of(const bevmap_gate &n) {
    GateArgs a{};
    a.ldx = n.x_stride;
    a.rows = n.rows;
    a.F = n.features;
    a.blocks = (n.features + kHeld - 1) / kHeld;
    a.units = n.rows * a.blocks * (kHeld / (n.dtype == BEVPOOL_F32 ? 4 : 8));
    a.act = n.act;
    return a;
}

dim3 grid_of(const GateArgs &a) {
    const int64_t all = (a.units + kGateBlock - 1) / kGateBlock;
    return dim3{uint32_t(all < kGateGroups ? all : kGateGroups)};
}

}  // namespace
}  // namespace bevmap

using namespace bevmap;

int bevmap_launch_gate(const bevmap_gate &n, const void *x, void *y, int8_t *q, uint8_t *e, hipStream_t stream) {
    if (n.rows == 0) return BEVPOOL_OK;
    GateArgs a = args_of(n);
    a.x = x;
    a.y = y;
    a.q = q;
    a.e = e;
    a.held = q != nullptr;
    const bool past = past_caches(n.rows * n.features * dtype_bytes(n.dtype));
    with_type_and_rows(n.dtype, halves_lie(n, x, y, nullptr, q), [&](auto dt, auto how) {
        constexpr int DT = decltype(dt)::value;
        constexpr int ROWS = decltype(how)::value;
        if (ROWS == kEven && past) hipLaunchKernelGGL((k_gate<DT, ROWS, ROWS == kEven>), grid_of(a), dim3(kGateBlock), 0, stream, a);
        else hipLaunchKernelGGL((k_gate<DT, ROWS, false>), grid_of(a), dim3(kGateBlock), 0, stream, a);
    });
    BEVPOOL_HIP(hipGetLastError());
    return BEVPOOL_OK;
}

int bevmap_launch_gate_backward(const bevmap_gate &n, const void *grad_y, const void *x, const int8_t *q,
                                const uint8_t *e, void *grad_x, hipStream_t stream) {
    if (n.rows == 0) return BEVPOOL_OK;
    GateArgs a = args_of(n);
    a.x = x;
    a.dy = grad_y;
    a.dx = grad_x;
    a.q = const_cast<int8_t *>(q);
    a.e = const_cast<uint8_t *>(e);
    const bool past = past_caches(n.rows * 2 * n.features * dtype_bytes(n.dtype));
    with_type_and_rows(n.dtype, halves_lie(n, q ? nullptr : x, grad_y, grad_x, q), [&](auto dt, auto how) {
        constexpr int DT = decltype(dt)::value;
        constexpr int ROWS = decltype(how)::value;
        auto go = [&](auto held) {
            constexpr bool kHeldRow = decltype(held)::value;
            if (ROWS == kEven && past)
                hipLaunchKernelGGL((k_gate_grad<DT, ROWS, kHeldRow, ROWS == kEven>), grid_of(a), dim3(kGateBlock), 0, stream, a);
            else
                hipLaunchKernelGGL((k_gate_grad<DT, ROWS, kHeldRow, false>), grid_of(a), dim3(kGateBlock), 0, stream, a);
        };
        if (q) go(Int<1>());
        else go(Int<0>());
    });
    BEVPOOL_HIP(hipGetLastError());
    return BEVPOOL_OK;
}
