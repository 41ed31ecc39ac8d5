// Activations of the block operators and their slopes, in fp32.
#pragma once
#include <hip/hip_runtime.h>

#include "purine_block.h"

namespace purine {
namespace {

constexpr float kTanhIn = 0.7978845608028654f, kTanhCube = 0.044715f;     // sqrt(2 / pi)

constexpr float kLog2e = 1.4426950408889634f;

// 1 / (1 + 2^u): the power saturates to 0 or infinity, the quotient to 1 or 0. (The hardware's power and reciprocal, to one unit in the last
// place each.)
__device__ __forceinline__ float inverse_of_1_plus_pow2(float u) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u)); }
__device__ __forceinline__ float sigmoid(float z) { return inverse_of_1_plus_pow2(-kLog2e * z); }
// 0.5 (1 + tanh u) = sigmoid(2 u), u = sqrt(2 / pi) (z + 0.044715 z^3)
constexpr float kGate1 = -2.0f * kLog2e * kTanhIn, kGate3 = kGate1 * kTanhCube;
__device__ __forceinline__ float tanh_gate(float z) { return inverse_of_1_plus_pow2(z * (kGate1 + kGate3 * (z * z))); }

// The normal distribution's integral up to z, and exp(-z^2 / 2). Abramowitz and Stegun 7.1.26: erfc(x) = P(t) exp(-x^2) with
// t = 1 / (1 + 0.3275911 x), off by 1.5e-7 at most.
__device__ __forceinline__ float normal_integral(float z, float& e) {
    const float t = __builtin_amdgcn_rcpf(1.0f + 0.3275911f * 0.70710678118654752f * fabsf(z));
    e = __builtin_amdgcn_exp2f(-0.5f * kLog2e * z * z);
    const float half = 0.5f * e * t * (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
    return z > 0.0f ? 1.0f - half : half;
}

// (where z is -infinity its product with a factor that is 0 there is the limit 0)
template <int ACT>
__device__ __forceinline__ float act_of(float z) {
    if constexpr (ACT == PURINE_ACT_NONE) return z;
    if constexpr (ACT == PURINE_ACT_RELU) return z > 0.0f ? z : (z == z ? 0.0f : z);
    float f = 0.0f, e;
    if constexpr (ACT == PURINE_ACT_SILU) f = sigmoid(z);
    if constexpr (ACT == PURINE_ACT_GELU) f = normal_integral(z, e);
    if constexpr (ACT == PURINE_ACT_GELU_TANH) f = tanh_gate(z);
    return fmaxf(z, -3.0e38f) * f;                  // (a NaN is in f)
}

// d act / dz; of ReLU 0 at z = 0. Past +-100 the slopes are 0 or 1: z counts as that where it would make 0 times infinity (a NaN is in the
// other factor).
template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
    if constexpr (ACT == PURINE_ACT_NONE) return 1.0f;
    if constexpr (ACT == PURINE_ACT_RELU) return z > 0.0f ? 1.0f : (z == z ? 0.0f : z);
    const float c = __builtin_amdgcn_fmed3f(z, -100.0f, 100.0f);
    if constexpr (ACT == PURINE_ACT_SILU) {
        const float s = sigmoid(z);
        return s + (c - c * s) * s;
    }
    if constexpr (ACT == PURINE_ACT_GELU) {
        float e;
        const float n = normal_integral(z, e);
        return n + c * (e * 0.3989422804014327f);
    }
    if constexpr (ACT == PURINE_ACT_GELU_TANH) {
        const float u = c * c, s = inverse_of_1_plus_pow2(z * (kGate1 + kGate3 * u));
        return s + s * ((c - c * s) * (2.0f * kTanhIn + 6.0f * kTanhIn * kTanhCube * u));
    }
    return 1.0f;
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
