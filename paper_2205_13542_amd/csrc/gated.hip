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

template <int V>
struct alignas(V) Bytes {
    int8_t v[V];
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

template <int V>
__device__ __forceinline__ void hold(const float *v, int8_t *q, uint8_t *e, bool live, bool first) {
    const uint32_t top = block_top<V>(v);
    const bool none = top >= 0x7F800000u;
    const int ex = exponent_of(top);
    Bytes<V> b;
#pragma unroll
    for (int i = 0; i < V; ++i) b.v[i] = int8_t(none ? 0.0f : rintf(ldexpf(v[i], -ex)));
    if (live) *reinterpret_cast<Bytes<V> *>(q) = b;
    if (first) *e = uint8_t(none ? kNanExponent : ex + 127);
}

template <int V>
__device__ __forceinline__ void release(const int8_t *q, uint8_t e, float *v) {
    const Bytes<V> b = *reinterpret_cast<const Bytes<V> *>(q);
#pragma unroll
    for (int i = 0; i < V; ++i)
        v[i] = e == kNanExponent ? __uint_as_float(0x7FC00000u) : ldexpf(float(b.v[i]), int(e) - 127);
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

template <int DT, int V, bool STREAM>
__global__ __launch_bounds__(kGateBlock) void k_gate(GateArgs a) {
    using T = typename Num<DT>::T;
    const T *x = static_cast<const T *>(a.x);
    T *y = static_cast<T *>(a.y);
    // whole waves stay together, for the lanes that share a block
    for (int64_t n0 = int64_t(blockIdx.x) * kGateBlock; n0 < a.units; n0 += int64_t(gridDim.x) * kGateBlock) {
        const int64_t n = n0 + threadIdx.x;
        const Place p = place_of<V>(n, a.blocks);
        const bool live = n < a.units && p.c < a.F;
        float g[V], v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] = v[i] = 0.0f;
        if (live) {
            load_n<T, V>(x + p.row * a.ldx + p.c, g);
            load_n<T, V>(x + p.row * a.ldx + a.F + p.c, v);
        }
        if (a.held) {
            int8_t *q = a.q + p.row * 2 * a.F + p.c;
            uint8_t *e = a.e + p.row * 2 * a.blocks + p.c / kHeld;
            const bool first = live && p.c % kHeld == 0;
            hold<V>(g, q, e, live, first);
            hold<V>(v, q + a.F, e + a.blocks, live, first);
        }
        with_act(a.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] *= activate<act.value>(g[i]);
        });
        if (live) store_n<T, V, STREAM>(y + p.row * a.F + p.c, v);
    }
}

template <int DT, int V, bool HELD, bool STREAM>
__global__ __launch_bounds__(kGateBlock) void k_gate_grad(GateArgs a) {
    using T = typename Num<DT>::T;
    const T *x = static_cast<const T *>(a.x), *dy = static_cast<const T *>(a.dy);
    T *dx = static_cast<T *>(a.dx);
    for (int64_t n = int64_t(blockIdx.x) * kGateBlock + threadIdx.x; n < a.units;
         n += int64_t(gridDim.x) * kGateBlock) {
        const Place p = place_of<V>(n, a.blocks);
        if (p.c >= a.F) continue;
        float g[V], v[V], d[V];
        load_n<T, V>(dy + p.row * a.F + p.c, d);
        if constexpr (HELD) {
            const int8_t *q = a.q + p.row * 2 * a.F + p.c;
            const uint8_t *e = a.e + p.row * 2 * a.blocks + p.c / kHeld;
            release<V>(q, e[0], g);
            release<V>(q + a.F, e[a.blocks], v);
        } else {
            load_n<T, V>(x + p.row * a.ldx + p.c, g);
            load_n<T, V>(x + p.row * a.ldx + a.F + p.c, v);
        }
        with_act(a.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float gate = g[i];
                g[i] = d[i] * v[i] * slope<act.value>(gate);
                v[i] = d[i] * activate<act.value>(gate);
            }
        });
        store_n<T, V, STREAM>(dx + p.row * 2 * a.F + p.c, g);
        store_n<T, V, STREAM>(dx + p.row * 2 * a.F + a.F + p.c, v);
    }
}

// Elements of an access: as many as 16 bytes hold where both halves of every row allow it, two, or one.
int access(const bevmap_gate &n, const void *x, const void *y, const void *dx, const void *q) {
    for (int v : {n.dtype == BEVPOOL_F32 ? 4 : 8, 2})
        if (n.features % v == 0 && (!x || aligned_for(x, n.rows == 1 ? 0 : n.x_stride, n.dtype, v)) &&
            aligned_for(y, 0, n.dtype, v) && aligned_for(dx, 0, n.dtype, v) &&
            reinterpret_cast<uintptr_t>(q) % uintptr_t(v) == 0)
            return v;
    return 1;
}

template <int V>
struct Int {
    static constexpr int value = V;
};
template <class F>
void with_type(int32_t dtype, int v, F body) {
    auto go = [&](auto dt) {
        constexpr int kWide = decltype(dt)::value == BEVPOOL_F32 ? 4 : 8;
        if (v == kWide) body(dt, Int<kWide>());
        else if (v == 2) body(dt, Int<2>());
        else body(dt, Int<1>());
    };
    if (dtype == BEVPOOL_F32) go(Int<BEVPOOL_F32>());
    else if (dtype == BEVPOOL_BF16) go(Int<BEVPOOL_BF16>());
    else go(Int<BEVPOOL_F16>());
}

GateArgs args_of(const bevmap_gate &n, int v) {
    GateArgs a{};
    a.ldx = n.x_stride;
    a.rows = n.rows;
    a.F = n.features;
    a.blocks = (n.features + kHeld - 1) / kHeld;
    a.units = n.rows * a.blocks * (kHeld / v);
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
    const int v = access(n, x, y, nullptr, q);
    GateArgs a = args_of(n, v);
    a.x = x;
    a.y = y;
    a.q = q;
    a.e = e;
    a.held = q != nullptr;
    const bool past = past_caches(n.rows * n.features * dtype_bytes(n.dtype));
    with_type(n.dtype, v, [&](auto dt, auto width) {
        constexpr int DT = decltype(dt)::value, V = decltype(width)::value;
        if (V > 2 && past) hipLaunchKernelGGL((k_gate<DT, V, (V > 2)>), grid_of(a), dim3(kGateBlock), 0, stream, a);
        else hipLaunchKernelGGL((k_gate<DT, V, false>), grid_of(a), dim3(kGateBlock), 0, stream, a);
    });
    BEVPOOL_HIP(hipGetLastError());
    return BEVPOOL_OK;
}

int bevmap_launch_gate_backward(const bevmap_gate &n, const void *grad_y, const void *x, const int8_t *q,
                                const uint8_t *e, void *grad_x, hipStream_t stream) {
    if (n.rows == 0) return BEVPOOL_OK;
    const int v = access(n, q ? nullptr : x, grad_y, grad_x, q);
    GateArgs a = args_of(n, v);
    a.x = x;
    a.dy = grad_y;
    a.dx = grad_x;
    a.q = const_cast<int8_t *>(q);
    a.e = const_cast<uint8_t *>(e);
    const bool past = past_caches(n.rows * 2 * n.features * dtype_bytes(n.dtype));
    with_type(n.dtype, v, [&](auto dt, auto width) {
        constexpr int DT = decltype(dt)::value, V = decltype(width)::value;
        auto go = [&](auto held) {
            constexpr bool kHeldRow = decltype(held)::value != 0;
            if (V > 2 && past)
                hipLaunchKernelGGL((k_gate_grad<DT, V, kHeldRow, (V > 2)>), grid_of(a), dim3(kGateBlock), 0, stream, a);
            else
                hipLaunchKernelGGL((k_gate_grad<DT, V, kHeldRow, false>), grid_of(a), dim3(kGateBlock), 0, stream, a);
        };
        if (q) go(Int<1>());
        else go(Int<0>());
    });
    BEVPOOL_HIP(hipGetLastError());
    return BEVPOOL_OK;
}
