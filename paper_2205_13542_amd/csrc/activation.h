// Activations of the map operators and their slopes (norm.hip, gated.hip).
#pragma once

#include <hip/hip_runtime.h>

#include "bevmap.h"

namespace bevmap {
namespace {

// exp(-z^2 / 2), and the share of a normal distribution below z, which the lower tail is as
// exact in as the rest (as (1 + erf) / 2 it is off by 4% at -5, and 0 below -6):
//   share(-|z|) = exp(-z^2 / 2) f(|z|),  share(|z|) = 1 - share(-|z|).
// f falls from 1/2 like 1 / |z|: a polynomial of nine terms in r = 1 / (1 + 0.34375 |z|), fitted
// over |z| up to 14.5 for the least relative error, 2.6e-8 (3e-7 as it is evaluated). The
// exponential's argument is rounded, which is off by z^2 2^-23 of the share at most.
struct Normal {
    float bell, share;
};
__device__ __forceinline__ Normal normal_of(float z) {
    Normal n;
    n.bell = __expf(-0.5f * z * z);
    const float r = __builtin_amdgcn_rcpf(fmaf(0.34375f, fabsf(z), 1.0f));
    float f = -0x1.c3e8bcp-6f;
    f = fmaf(f, r, 0x1.2476bcp-3f);
    f = fmaf(f, r, -0x1.142772p-2f);
    f = fmaf(f, r, 0x1.828c76p-3f);
    f = fmaf(f, r, -0x1.368beep-5f);
    f = fmaf(f, r, 0x1.cb315ap-4f);
    f = fmaf(f, r, 0x1.deb29cp-4f);
    f = fmaf(f, r, 0x1.19a724p-3f);
    f = fmaf(f, r, 0x1.18d2a8p-3f);
    const float tail = f * r * n.bell;
    n.share = z > 0.0f ? 1.0f - tail : tail;
    return n;
}

template <int ACT>
__device__ __forceinline__ float activate(float z) {
    if constexpr (ACT == BEVMAP_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if constexpr (ACT == BEVMAP_ACT_SILU) return z * __builtin_amdgcn_rcpf(1.0f + __expf(-z));
    if constexpr (ACT == BEVMAP_ACT_GELU) return z * normal_of(z).share;
    return z;
}

template <int ACT>
__device__ __forceinline__ float slope(float z) {
    if constexpr (ACT == BEVMAP_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if constexpr (ACT == BEVMAP_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.0f + __expf(-z));
        return s * (1.0f + z * (1.0f - s));
    }
    if constexpr (ACT == BEVMAP_ACT_GELU) {
        const Normal n = normal_of(z);
        return fmaf(z * n.bell, 0.39894228f, n.share);
    }
    return 1.0f;
}

// body(constant) with the activation as a constant: one uniform branch for a batch
// of rows instead of one for an element.
template <int V>
struct Constant {
    static constexpr int value = V;
};
template <class F>
__device__ __forceinline__ void with_act(int act, F body) {
    switch (act) {
        case BEVMAP_ACT_RELU: body(Constant<BEVMAP_ACT_RELU>()); break;
        case BEVMAP_ACT_SILU: body(Constant<BEVMAP_ACT_SILU>()); break;
        case BEVMAP_ACT_GELU: body(Constant<BEVMAP_ACT_GELU>()); break;
        default: body(Constant<BEVMAP_ACT_NONE>()); break;
    }
}

}  // namespace
}  // namespace bevmap
