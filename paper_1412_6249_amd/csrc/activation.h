// Activations of the block operators and their slopes, in fp32.
#pragma once
#include <hip/hip_runtime.h>

#include "purine_block.h"

namespace purine {
namespace {

constexpr float kTanhIn = 0.7978845608028654f, kTanhCube = 0.044715f;     // sqrt(2 / pi)

// 1 / (1 + exp(-z)): exp saturates to 0 or infinity, the quotient to 1 or 0. (The hardware's reciprocal, to one unit in the last place.)
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }

// The normal distribution's integral up to z, and exp(-z^2 / 2). Abramowitz and Stegun 7.1.26: erfc(x) = P(t) exp(-x^2) with
// t = 1 / (1 + 0.3275911 x), off by 1.5e-7 at most.
__device__ __forceinline__ float normal_integral(float z, float& e) {
    const float x = fabsf(z) * 0.70710678118654752f, t = __builtin_amdgcn_rcpf(1.0f + 0.3275911f * x);
    e = __expf(-x * x);
    const float half = 0.5f * e * t * (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
    return z > 0.0f ? 1.0f - half : half;
}

// (where z is -infinity, or nearly, its product with a factor that is 0 there is the limit 0)
template <int ACT>
__device__ __forceinline__ float act_of(float z) {
    if constexpr (ACT == PURINE_ACT_NONE) return z;
    if constexpr (ACT == PURINE_ACT_RELU) return z > 0.0f ? z : (z == z ? 0.0f : z);
    float f, e;
    if constexpr (ACT == PURINE_ACT_SILU) f = sigmoid(z);
    if constexpr (ACT == PURINE_ACT_GELU) f = normal_integral(z, e);
    if constexpr (ACT == PURINE_ACT_GELU_TANH) f = sigmoid(2.0f * kTanhIn * (z + kTanhCube * z * z * z));     // 0.5 (1 + tanh u) = sigmoid(2 u)
    return (z < -3.0e38f ? 0.0f : z) * f;
}

// d act / dz; of ReLU 0 at z = 0
template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
    if constexpr (ACT == PURINE_ACT_NONE) return 1.0f;
    if constexpr (ACT == PURINE_ACT_RELU) return z > 0.0f ? 1.0f : (z == z ? 0.0f : z);
    const float c = fminf(fmaxf(z, -100.0f), 100.0f), keep = z == z ? c : z;      // (the slopes are 0 or 1 past that; NaN stays)
    if constexpr (ACT == PURINE_ACT_SILU) {
        const float s = sigmoid(keep);
        return s + keep * s * (1.0f - s);
    }
    if constexpr (ACT == PURINE_ACT_GELU) {
        float e;
        const float n = normal_integral(keep, e);
        return n + keep * e * 0.3989422804014327f;
    }
    if constexpr (ACT == PURINE_ACT_GELU_TANH) {
        const float s = sigmoid(2.0f * kTanhIn * (keep + kTanhCube * keep * keep * keep));
        return s + 2.0f * keep * s * (1.0f - s) * kTanhIn * (1.0f + 3.0f * kTanhCube * keep * keep);
    }
}

__device__ __forceinline__ float act_any(int act, float z) {
    switch (act) {
        case PURINE_ACT_RELU: return act_of<PURINE_ACT_RELU>(z);
        case PURINE_ACT_SILU: return act_of<PURINE_ACT_SILU>(z);
        case PURINE_ACT_GELU: return act_of<PURINE_ACT_GELU>(z);
        case PURINE_ACT_GELU_TANH: return act_of<PURINE_ACT_GELU_TANH>(z);
        default: return z;
    }
}
__device__ __forceinline__ float slope_any(int act, float z) {
    switch (act) {
        case PURINE_ACT_RELU: return act_slope<PURINE_ACT_RELU>(z);
        case PURINE_ACT_SILU: return act_slope<PURINE_ACT_SILU>(z);
        case PURINE_ACT_GELU: return act_slope<PURINE_ACT_GELU>(z);
        case PURINE_ACT_GELU_TANH: return act_slope<PURINE_ACT_GELU_TANH>(z);
        default: return 1.0f;
    }
}

}  // namespace
}  // namespace purine
