// Residual + dropout with a mask that is drawn where it is used (bevmap_dropout).
//
// Philox4x32-10 (Salmon et al., "Parallel random numbers: as easy as 1, 2, 3",
// 2011) maps a 128-bit counter under a 64-bit key to 128 random bits: ten rounds
// of two 32 x 32 -> 64-bit products each. One counter serves eight elements, 16
// bits each, which is one 16-byte access of a 16-bit type; 16 bits place the keep
// probability to 1 / 65536, and the scale is that of the placed probability.
// Bound by memory: 41.5 M bf16 elements with a residual, 249 MB, take 45 us, and
// without one, 166 MB, 30 us, 5.5 TB/s (a copy of 4 GiB reaches 4.8). The draws, 20
// products for eight elements, hide behind it.
#include "mapops.h"

namespace bevmap {
namespace {

constexpr int kDropBlock = 256;
constexpr int kDraws = 8;      // elements of one counter
constexpr int64_t kDropGrid = 1 << 20;   // workgroups at most

struct DropArgs {
    const void *x, *residual;
    void *y;
    int64_t x_stride, residual_stride, columns, n;   // n elements in all
    uint32_t threshold;
    float scale;
    uint32_t key0, key1, offset0, offset1;
};

__device__ __forceinline__ void philox(uint64_t block, const DropArgs &a, uint32_t (&w)[4]) {
    uint32_t c0 = uint32_t(block), c1 = uint32_t(block >> 32), c2 = a.offset0, c3 = a.offset1;
    uint32_t k0 = a.key0, k1 = a.key1;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p0 = uint64_t(c0) * 0xD2511F53u, p1 = uint64_t(c2) * 0xCD9E8D57u;
        c0 = uint32_t(p1 >> 32) ^ c1 ^ k0;
        c1 = uint32_t(p1);
        c2 = uint32_t(p0 >> 32) ^ c3 ^ k1;
        c3 = uint32_t(p0);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    w[0] = c0;
    w[1] = c1;
    w[2] = c2;
    w[3] = c3;
}

// VEC: a counter's eight elements lie side by side on 16-byte boundaries in
// every tensor. FLAT: rows follow each other without a gap, one index for all.
template <int DT, bool VEC, bool FLAT>
__global__ __launch_bounds__(kDropBlock) void k_dropout(DropArgs a) {
    using T = typename Num<DT>::T;
    const T *x = static_cast<const T *>(a.x), *res = static_cast<const T *>(a.residual);
    T *y = static_cast<T *>(a.y);
    const int64_t step = int64_t(gridDim.x) * kDropBlock;
    for (int64_t block = int64_t(blockIdx.x) * kDropBlock + threadIdx.x; block * kDraws < a.n; block += step) {
        const int64_t e0 = block * kDraws;
        int64_t row = 0, col = e0;
        if constexpr (!FLAT) {
            row = e0 / a.columns;
            col = e0 - row * a.columns;
        }
        uint32_t w[4];
        if (VEC && e0 + kDraws <= a.n) {
            float v[kDraws], r[kDraws];
            load_n<T, kDraws>(x + row * a.x_stride + col, v);
            if (res) load_n<T, kDraws>(res + row * a.residual_stride + col, r);
            philox(uint64_t(block), a, w);
#pragma unroll
            for (int i = 0; i < kDraws; ++i) {
                const uint32_t draw = i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xFFFFu;
                v[i] = draw >= a.threshold ? v[i] * a.scale : 0.0f;
                if (res) v[i] += r[i];
            }
            store_n<T, kDraws>(y + e0, v);
            continue;
        }
        philox(uint64_t(block), a, w);
        for (int i = 0; i < kDraws && e0 + i < a.n; ++i) {
            const uint32_t word = i < 4 ? (i < 2 ? w[0] : w[1]) : (i < 6 ? w[2] : w[3]);
            const uint32_t draw = i & 1 ? word >> 16 : word & 0xFFFFu;
            float v = draw >= a.threshold ? float(x[row * a.x_stride + col]) * a.scale : 0.0f;
            if (res) v += float(res[row * a.residual_stride + col]);
            y[e0 + i] = T(v);
            if (++col == a.columns && !FLAT) {
                col = 0;
                ++row;
            }
        }
    }
}

template <int DT>
void launch(const DropArgs &a, bool vec, bool flat, hipStream_t stream) {
    const int64_t blocks = (a.n + kDraws * kDropBlock - 1) / (kDraws * kDropBlock);
    const dim3 grid{uint32_t(blocks < kDropGrid ? blocks : kDropGrid)}, wg(kDropBlock);
    if (vec && flat)
        hipLaunchKernelGGL((k_dropout<DT, true, true>), grid, wg, 0, stream, a);
    else if (vec)
        hipLaunchKernelGGL((k_dropout<DT, true, false>), grid, wg, 0, stream, a);
    else if (flat)
        hipLaunchKernelGGL((k_dropout<DT, false, true>), grid, wg, 0, stream, a);
    else
        hipLaunchKernelGGL((k_dropout<DT, false, false>), grid, wg, 0, stream, a);
}

}  // namespace
}  // namespace bevmap

using namespace bevmap;

int bevmap_launch_dropout(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, void *y,
                          int64_t rows, int64_t columns, int32_t dtype, int32_t threshold, uint64_t seed,
                          uint64_t offset, hipStream_t stream) {
    if (rows == 0 || columns == 0) return BEVPOOL_OK;
    DropArgs a;
    a.x = x;
    a.residual = residual;
    a.y = y;
    a.x_stride = x_stride;
    a.residual_stride = residual ? residual_stride : x_stride;
    a.columns = columns;
    a.n = rows * columns;
    a.threshold = uint32_t(threshold);
    a.scale = threshold < 65536 ? 65536.0f / float(65536 - threshold) : 0.0f;
    a.key0 = uint32_t(seed);
    a.key1 = uint32_t(seed >> 32);
    a.offset0 = uint32_t(offset);
    a.offset1 = uint32_t(offset >> 32);
    const bool flat = rows == 1 || (x_stride == columns && a.residual_stride == columns);
    bool vec = aligned_for(x, flat ? 0 : x_stride, dtype, kDraws) && aligned_for(y, 0, dtype, kDraws) &&
               (!residual || aligned_for(residual, flat ? 0 : residual_stride, dtype, kDraws));
    vec = vec && (flat || columns % kDraws == 0);
    switch (dtype) {
        case BEVPOOL_F32: launch<BEVPOOL_F32>(a, vec, flat, stream); break;
        case BEVPOOL_BF16: launch<BEVPOOL_BF16>(a, vec, flat, stream); break;
        default: launch<BEVPOOL_F16>(a, vec, flat, stream); break;
    }
    BEVPOOL_HIP(hipGetLastError());
    return BEVPOOL_OK;
}
