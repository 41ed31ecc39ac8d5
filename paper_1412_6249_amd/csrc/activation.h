// Activations of the block operators and their slopes, in fp32.
#pragma once
#include <hip/hip_runtime.h>

#include "purine_block.h"

namespace purine {
namespace {

constexpr float kTanhIn = 0.7978845608028654f, kTanhCube = 0.044715f;     // sqrt(2 / pi)

// 1 / (1 + exp(-z)): exp saturates to 0 or infinity, the quotient to 1 or 0
__device__ __forceinline__ float sigmoid(float z) { return 1.0f / (1.0f + __expf(-z)); }

template <int ACT>
__device__ __forceinline__ float act_of(float z) {
    if constexpr (ACT == PURINE_ACT_RELU) return z > 0.0f ? z : (z == z ? 0.0f : z);
    if constexpr (ACT == PURINE_ACT_SILU) return z > -3.0e38f ? z * sigmoid(z) : (z == z ? 0.0f : z);
    if constexpr (ACT == PURINE_ACT_GELU) return z > -3.0e38f ? 0.5f * z * erfcf(z * -0.70710678118654752f) : (z == z ? 0.0f : z);
    if constexpr (ACT == PURINE_ACT_GELU_TANH) {
        // 0.5 (1 + tanh u) = sigmoid(2 u)
        return z > -3.0e38f ? z * sigmoid(2.0f * kTanhIn * (z + kTanhCube * z * z * z)) : (z == z ? 0.0f : z);
    }
    return z;
}

// d act / dz; of ReLU 0 at z = 0
template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
    if constexpr (ACT == PURINE_ACT_RELU) return z > 0.0f ? 1.0f : (z == z ? 0.0f : z);
    if constexpr (ACT == PURINE_ACT_SILU) {
        if (z < -100.0f) return 0.0f;                  // (s is 0 there, and z (1 - s) may be -infinity)
        const float s = sigmoid(z), t = 1.0f - s;
        return s * (1.0f + (t > 0.0f ? z * t : t));
    }
    if constexpr (ACT == PURINE_ACT_GELU)
        return 0.5f * erfcf(z * -0.70710678118654752f) + (fabsf(z) < 1.0e18f ? z * __expf(-0.5f * z * z) * 0.3989422804014327f : (z == z ? 0.0f : z));
    if constexpr (ACT == PURINE_ACT_GELU_TANH) {
        if (!(fabsf(z) < 1.0e9f)) return z > 0.0f ? 1.0f : (z == z ? 0.0f : z);
        const float s = sigmoid(2.0f * kTanhIn * (z + kTanhCube * z * z * z));
        return s + 2.0f * z * s * (1.0f - s) * kTanhIn * (1.0f + 3.0f * kTanhCube * z * z);
    }
    return 1.0f;
}

}  // namespace
}  // namespace purine
