// Activations of the block operators and their slopes, in fp32. FULL: for results of 32 bits, to a few units in their last place. Otherwise, for results that
// are rounded to bf16 (2e-3 of them): the hardware's power as it is, whose error grows with the exponent to some 1e-6 of the result.
#pragma once
#include <hip/hip_runtime.h>

#include "purine_block.h"

namespace purine {
namespace {

constexpr float kTanhIn = 0.7978845608028654f, kTanhCube = 0.044715f;     // sqrt(2 / pi)

constexpr float kLog2e = 1.4426950408889634f, kLog2eRest = 1.9259630335e-8f, kLn2 = 0.6931471805599453f;

// e^(x + rest) to two units in the last place: what the product with log2 e loses is put back behind the power. (Infinities and NaNs are the power's; what is
// lost is bounded so that it does not make NaNs of its own.) us, 64 x 12544 x 64 fp32 in both directions of a normalization: GELU 349, SiLU 342, by the power alone 344 and
// 342, by the library's exponential and a rounded quotient 364 and 348.
__device__ __forceinline__ float exp_full(float x, float rest = 0.0f) {
    const float t = x * kLog2e;
    const float lost = fmaf(rest, kLog2e, fmaf(x, kLog2eRest, fmaf(x, kLog2e, -t)));
    return __builtin_amdgcn_exp2f(t) * fmaf(kLn2, __builtin_amdgcn_fmed3f(lost, -1.0e-3f, 1.0e-3f), 1.0f);
}

// 1 / (1 + 2^u): the power saturates to 0 or infinity, the quotient to 1 or 0. (The hardware's power and reciprocal are to one unit in the last
// place each.)
__device__ __forceinline__ float inverse_of_1_plus_pow2(float u) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u)); }
template <bool FULL>
__device__ __forceinline__ float sigmoid(float z) {
    if constexpr (FULL) return __builtin_amdgcn_rcpf(1.0f + exp_full(-z));
    return inverse_of_1_plus_pow2(-kLog2e * z);
}
// 1 / (1 + e^-u) and one less that, neither by a difference.
__device__ __forceinline__ void sigmoids(float u, float& s, float& rest) {
    const float t = exp_full(-fabsf(u)), most = __builtin_amdgcn_rcpf(1.0f + t), least = t * most;
    s = u > 0.0f ? most : least;
    rest = u > 0.0f ? least : most;
}
// 0.5 (1 + tanh u) = sigmoid(2 u), u = sqrt(2 / pi) (z + 0.044715 z^3)
constexpr float kGate1 = -2.0f * kLog2e * kTanhIn, kGate3 = kGate1 * kTanhCube;
template <bool FULL>
__device__ __forceinline__ float tanh_gate(float z, float z2) {
    if constexpr (FULL) return __builtin_amdgcn_rcpf(1.0f + exp_full(z * (-2.0f * kTanhIn - 2.0f * kTanhIn * kTanhCube * z2)));
    return inverse_of_1_plus_pow2(z * (kGate1 + kGate3 * z2));
}

// The normal distribution's integral up to z, and e = exp(-z^2 / 2). Below 0 it is t Q(t) e with t = 1 / (1 + 0.35 |z|), Q of degree 8 fitted to least
// largest relative error (3.3e-8 down to z = -15, so that the tail keeps its digits), above 0 one less that.
template <bool FULL>
__device__ __forceinline__ float normal_integral(float z, float& e) {
    if constexpr (FULL) {
        const float u = z * z;
        e = exp_full(-0.5f * u, -0.5f * fmaf(z, z, -u));        // (with what the square lost)
    } else {
        e = __builtin_amdgcn_exp2f(-0.5f * kLog2e * z * z);
    }
    const float t = __builtin_amdgcn_rcpf(1.0f + 0.35f * fabsf(z));
    float q = -0.029162863f;
    q = fmaf(q, t, 0.144056131f);
    q = fmaf(q, t, -0.255893188f);
    q = fmaf(q, t, 0.159384042f);
    q = fmaf(q, t, -0.0232583893f);
    q = fmaf(q, t, 0.105572751f);
    q = fmaf(q, t, 0.119815959f);
    q = fmaf(q, t, 0.13986428f);
    q = fmaf(q, t, 0.139621261f);
    const float below = e * (t * q);
    return z > 0.0f ? 1.0f - below : below;
}

// (where z is -infinity its product with a factor that is 0 there is the limit 0)
template <int ACT, bool FULL>
__device__ __forceinline__ float act_of(float z) {
    if constexpr (ACT == PURINE_ACT_NONE) return z;
    if constexpr (ACT == PURINE_ACT_RELU) return z > 0.0f ? z : (z == z ? 0.0f : z);
    float f = 0.0f, e;
    if constexpr (ACT == PURINE_ACT_SILU) f = sigmoid<FULL>(z);
    if constexpr (ACT == PURINE_ACT_GELU) f = normal_integral<FULL>(z, e);
    if constexpr (ACT == PURINE_ACT_GELU_TANH) f = tanh_gate<FULL>(z, z * z);
    return fmaxf(z, -3.0e38f) * f;                  // (a NaN is in f)
}

// d act / dz; of ReLU 0 at z = 0. Past +-100 the slopes are 0 or 1: z counts as that where it would make 0 times infinity (a NaN is in the
// other factor).
template <int ACT, bool FULL>
__device__ __forceinline__ float act_slope(float z) {
    if constexpr (ACT == PURINE_ACT_NONE) return 1.0f;
    if constexpr (ACT == PURINE_ACT_RELU) return z > 0.0f ? 1.0f : (z == z ? 0.0f : z);
    const float c = __builtin_amdgcn_fmed3f(z, -100.0f, 100.0f);
    if constexpr (ACT == PURINE_ACT_SILU) {
        if constexpr (FULL) {
            float s, rest;
            sigmoids(z, s, rest);
            return s + c * (s * rest);
        }
        const float s = sigmoid<FULL>(z);
        return s + (c - c * s) * s;
    }
    if constexpr (ACT == PURINE_ACT_GELU) {
        float e;
        const float n = normal_integral<FULL>(z, e);
        return n + c * (e * 0.3989422804014327f);
    }
    if constexpr (ACT == PURINE_ACT_GELU_TANH) {
        const float u = c * c;
        if constexpr (FULL) {
            float s, rest;
            sigmoids(z * (2.0f * kTanhIn + 2.0f * kTanhIn * kTanhCube * u), s, rest);
            return s + c * (s * rest) * (2.0f * kTanhIn + 6.0f * kTanhIn * kTanhCube * u);
        }
        const float s = tanh_gate<FULL>(z, u);
        return s + s * ((c - c * s) * (2.0f * kTanhIn + 6.0f * kTanhIn * kTanhCube * u));
    }
    return 1.0f;
}

template <bool FULL>
__device__ __forceinline__ float act_any(int act, float z) {
    switch (act) {
        case PURINE_ACT_RELU: return act_of<PURINE_ACT_RELU, FULL>(z);
        case PURINE_ACT_SILU: return act_of<PURINE_ACT_SILU, FULL>(z);
        case PURINE_ACT_GELU: return act_of<PURINE_ACT_GELU, FULL>(z);
        case PURINE_ACT_GELU_TANH: return act_of<PURINE_ACT_GELU_TANH, FULL>(z);
        default: return z;
    }
}
template <bool FULL>
__device__ __forceinline__ float slope_any(int act, float z) {
    switch (act) {
        case PURINE_ACT_RELU: return act_slope<PURINE_ACT_RELU, FULL>(z);
        case PURINE_ACT_SILU: return act_slope<PURINE_ACT_SILU, FULL>(z);
        case PURINE_ACT_GELU: return act_slope<PURINE_ACT_GELU, FULL>(z);
        case PURINE_ACT_GELU_TANH: return act_slope<PURINE_ACT_GELU_TANH, FULL>(z);
        default: return 1.0f;
    }
}

}  // namespace
}  // namespace purine
