// Activations of the map operators and their slopes (norm.hip, gated.hip).
#pragma once

#include <hip/hip_runtime.h>

#include "bevmap.h"

namespace bevmap {
namespace {

template <int ACT>
__device__ __forceinline__ float activate(float z) {
    if constexpr (ACT == BEVMAP_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if constexpr (ACT == BEVMAP_ACT_SILU) return z * __builtin_amdgcn_rcpf(1.0f + __expf(-z));
    if constexpr (ACT == BEVMAP_ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678f));
    return z;
}

template <int ACT>
__device__ __forceinline__ float slope(float z) {
    if constexpr (ACT == BEVMAP_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if constexpr (ACT == BEVMAP_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.0f + __expf(-z));
        return s * (1.0f + z * (1.0f - s));
    }
    if constexpr (ACT == BEVMAP_ACT_GELU)
        return 0.5f * (1.0f + erff(z * 0.70710678f)) + z * __expf(-0.5f * z * z) * 0.39894228f;
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
