// AdamW step over many parameter tensors (purine_adamw_step), states in fp32 or as e4m3 codes with a power of two per 256 elements.
//
//     g = grad_scale dw;  m = beta1 m + (1 - beta1) g;  v = beta2 v + (1 - beta2) g^2
//     w = w (1 - lr weight_decay) - lr / (1 - beta1^t) m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
//
// Bound: HBM, every tensor read once and written once: 62 M parameters (AlexNet) with fp32 states 342 us (28 bytes a parameter, 5.1 TB/s), with bf16 gradients, a
// bf16 copy and 8-bit states 195 us (16 bytes, 5.1 TB/s); 12 tensors of 164 k parameters in all 4.8 us, a launch. The table of tensors travels in the kernel arguments, 40 tensors a launch,
// so that a step needs no memory of its own; a workgroup takes 2048 consecutive elements of one tensor, found from the tensors' first
// workgroups in the table.
#include <math.h>

#include "bf16.h"
#include "block.h"

namespace purine {
namespace {

constexpr int NT = 256, PER = 8, CHUNK = NT * PER, TABLE = 40;
constexpr unsigned MOST = 1u << 22;        // workgroups of a launch, the last tensor's (2^20 at most) aside: a launch ends at 2^32 threads
static_assert(PURINE_ADAMW_BLOCK == 32 * PER, "a block's elements lie in half a wavefront");

struct AdamwTensor {
    void* w; const void* dw; void* m; void* v;
    float* ms; float* vs;
    uint16_t* copy;
    unsigned n;
};
struct AdamwParams {
    AdamwTensor t[TABLE];
    unsigned first[TABLE];     // tensors' first workgroups
    const int* done;           // steps done before, or null: `step` is this one
    float decay, lr, beta1, beta1c, beta2, beta2c, eps, grad_scale;
    float log1, log2;          // log beta
    float step_size, v_scale;  // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t) of a step given by the host
    unsigned step, seed, ordinal;      // ordinal: of the table's first tensor in the call
    int count, dither;
};
static_assert(sizeof(AdamwParams) <= 4096, "kernel arguments");

// Two rounds of shift, exclusive or and an odd multiplier, as in published integer hashes (T. Mueller's has 0x45D9F3B twice); no other multipliers were tried. Over 2^20
// inputs a bit of the input changes each bit of the output with a probability of 0.489 to 0.511, and the bytes for neighbouring elements correlate by less than 1e-3.
__device__ __forceinline__ uint32_t mix(uint32_t h) {
    h = (h ^ (h >> 16)) * 0x45D9F3B3u;
    h = (h ^ (h >> 15)) * 0x2C1B3C6Du;
    return h ^ (h >> 16);
}

// Largest finite magnitude of the 32 lanes that hold a block.
__device__ __forceinline__ float block_max(const float (&x)[PER]) {
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const float a = fabsf(x[i]);
        most = fmaxf(most, a < INFINITY ? a : 0.0f);
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
    return most;
}
// The exponent of the block's scale: the smallest power of two, from 2^-100, that brings `most` to 448 = 1.75 * 2^8 or less.
__device__ __forceinline__ int scale_exponent(float most) {
    const uint32_t b = __float_as_uint(most);
    const int e = (int)(b >> 23) - 135 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < -100 ? -100 : e;
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// A magnitude up to 448 at a code: up where its place between two codes plus d reaches 1.
__device__ __forceinline__ float round_code(float z, float d) {
    const int e = max((int)(__float_as_uint(z) >> 23) - 127, -6);
    return floorf(z * pow2(3 - e) + d) * pow2(e - 3);
}
__device__ __forceinline__ void decode(const uint2 c, float s, float (&x)[PER]) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    const f2 a = __builtin_amdgcn_cvt_pk_f32_fp8(c.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(c.x, true);
    const f2 e = __builtin_amdgcn_cvt_pk_f32_fp8(c.y, false), f = __builtin_amdgcn_cvt_pk_f32_fp8(c.y, true);
    x[0] = a.x * s; x[1] = a.y * s; x[2] = b.x * s; x[3] = b.y * s;
    x[4] = e.x * s; x[5] = e.y * s; x[6] = f.x * s; x[7] = f.y * s;
}
// Codes of x (magnitudes up to 448 scales) and the block's scale. d: the elements' thresholds. FLOOR: what is above zero stays so.
template <bool FLOOR>
__device__ __forceinline__ uint2 encode(const float (&x)[PER], const float (&d)[PER], float& scale) {
    const float most = block_max(x);
    const int e = scale_exponent(most);
    const float inv = most > 0.0f ? pow2(-e) : 0.0f;
    scale = most > 0.0f ? pow2(e) : 0.0f;
    float q[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const float a = fabsf(x[i]);
        float r = round_code(a * inv, d[i]);
        if (FLOOR) r = a > 0.0f ? fmaxf(r, 0x1p-9f) : r;
        q[i] = a < INFINITY ? copysignf(r, x[i]) : __uint_as_float(0x7fc00000u);
    }
    uint2 c;
    int lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(q[4], q[5], 0, false);
    c.x = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], lo, true);
    c.y = __builtin_amdgcn_cvt_pk_fp8_f32(q[6], q[7], hi, true);
    return c;
}

// PER elements from at, `left` of them inside the tensor (PER or more: all, in whole vectors).
__device__ __forceinline__ void get(const float* p, int left, float (&x)[PER]) {
    if (left >= PER) {
        const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) x[i] = i < left ? p[i] : 0.0f;
    }
}
__device__ __forceinline__ void get(const uint16_t* p, int left, float (&x)[PER]) {
    if (left >= PER) {
        const uint4 a = *reinterpret_cast<const uint4*>(p);
        const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(u[i] << 16); x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) x[i] = i < left ? bf2f(p[i]) : 0.0f;
    }
}
__device__ __forceinline__ uint2 get_codes(const uint8_t* p, int left) {
    if (left >= PER) return *reinterpret_cast<const uint2*>(p);
    uint32_t c[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < PER; ++i) c[i >> 2] |= i < left ? (uint32_t)p[i] << (8 * (i & 3)) : 0u;
    return make_uint2(c[0], c[1]);
}
__device__ __forceinline__ void put(float* p, int left, const float (&x)[PER]) {
    if (left >= PER) {
        reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) if (i < left) p[i] = x[i];
    }
}
__device__ __forceinline__ void put(uint16_t* p, int left, const float (&x)[PER]) {
    if (left >= PER) {
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = (uint32_t)f2bf(x[2 * i]) | (uint32_t)f2bf(x[2 * i + 1]) << 16;
        *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) if (i < left) p[i] = f2bf(x[i]);
    }
}
__device__ __forceinline__ void put_codes(uint8_t* p, int left, uint2 c) {
    if (left >= PER) {
        *reinterpret_cast<uint2*>(p) = c;
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) if (i < left) p[i] = (uint8_t)((i < 4 ? c.x : c.y) >> (8 * (i & 3)));
    }
}

template <typename W, typename D, bool CODED>
__global__ __launch_bounds__(NT) void adamw_kernel(const AdamwParams p) {
    // the last tensor that begins at or before this workgroup: one load for the wavefront (a search by halves is six, one after the other)
    const int lane = threadIdx.x & 63;
    const bool before = lane < p.count && p.first[lane < TABLE ? lane : 0] <= blockIdx.x;
    const int k = __builtin_amdgcn_readfirstlane(__popcll(__ballot(before)) - 1);
    const AdamwTensor& t = p.t[k];
    const unsigned at = (blockIdx.x - p.first[k]) * CHUNK + threadIdx.x * PER;
    const int left = at < t.n ? (int)min(t.n - at, (unsigned)PER) : 0;
    float step_size = p.step_size, v_scale = p.v_scale;
    unsigned step = p.step;
    if (p.done) {
        step = (unsigned)*p.done + 1u;
        step_size = p.lr / -expm1f((float)step * p.log1);       // 1 - beta^t; log of 0 is -infinity
        v_scale = 1.0f / sqrtf(-expm1f((float)step * p.log2));
    }
    float w[PER], g[PER], m[PER], v[PER];
    get((const W*)t.w + at, left, w);
    get((const D*)t.dw + at, left, g);
    const unsigned block = at / PURINE_ADAMW_BLOCK;
    if constexpr (CODED) {
        const float ms = left ? t.ms[block] : 0.0f, vs = left ? t.vs[block] : 0.0f;
        decode(get_codes((const uint8_t*)t.m + at, left), ms, m);
        decode(get_codes((const uint8_t*)t.v + at, left), vs, v);
#pragma unroll
        for (int i = 0; i < PER; ++i) v[i] *= v[i];
    } else {
        get((const float*)t.m + at, left, m);
        get((const float*)t.v + at, left, v);
    }
    // Every product and sum of the states is rounded by itself (no fused multiply-add), so that the codes do not depend on how the
    // formula is evaluated: with bf16 gradients values often lie exactly between two codes.
    float u[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
#pragma clang fp contract(off)
        const float d = g[i] * p.grad_scale;
        m[i] = p.beta1 * m[i] + p.beta1c * d;
        v[i] = p.beta2 * v[i] + p.beta2c * (d * d);
        u[i] = sqrtf(v[i]);
        w[i] = w[i] * p.decay - step_size * (m[i] / (u[i] * v_scale + p.eps));
    }
    put((W*)t.w + at, left, w);
    if (t.copy) put(t.copy + at, left, w);
    if constexpr (CODED) {
        float dm[PER], dv[PER];
        if (p.dither) {
            const uint32_t salt = mix(mix(p.seed + 0x9E3779B9u * step) + 0x85EBCA6Bu * (p.ordinal + (unsigned)k + 1u));
#pragma unroll
            for (int i = 0; i < PER; i += 2) {
                const uint32_t h = mix(salt + ((at + i) >> 1));
                dm[i] = ((float)(h & 255u) + 0.5f) * 0x1p-8f;
                dv[i] = ((float)(h >> 8 & 255u) + 0.5f) * 0x1p-8f;
                dm[i + 1] = ((float)(h >> 16 & 255u) + 0.5f) * 0x1p-8f;
                dv[i + 1] = ((float)(h >> 24) + 0.5f) * 0x1p-8f;
            }
        } else {
#pragma unroll
            for (int i = 0; i < PER; ++i) dm[i] = dv[i] = 0.5f;
        }
        // (elements past the end are zeros: they take part in the maximum and are not stored)
        float ms, vs;
        const uint2 mc = encode<false>(m, dm, ms), vc = encode<true>(u, dv, vs);
        put_codes((uint8_t*)t.m + at, left, mc);
        put_codes((uint8_t*)t.v + at, left, vc);
        if (left && (threadIdx.x & 31) == 0) { t.ms[block] = ms; t.vs[block] = vs; }
    } else {
        put((float*)t.m + at, left, m);
        put((float*)t.v + at, left, v);
    }
}

__global__ void adamw_count_kernel(int* done) { if (threadIdx.x == 0) ++*done; }

template <typename W, typename D>
void launch(const AdamwParams& p, unsigned grid, bool coded, hipStream_t st) {
    if (coded) hipLaunchKernelGGL((adamw_kernel<W, D, true>), dim3(grid), dim3(NT), 0, st, p);
    else hipLaunchKernelGGL((adamw_kernel<W, D, false>), dim3(grid), dim3(NT), 0, st, p);
}

int64_t elements(const purine_tensor& t) {
    int64_t n = 1;
    for (int i = 0; i < t.ndim; ++i) n *= t.dim[i];
    return n;
}

}  // namespace

hipError_t launch_adamw(const purine_adamw_desc& d, const purine_adamw_param* params, int n, int* done, hipStream_t st) {
    if (n == 0 && !done) return hipSuccess;
    AdamwParams p{};
    p.done = done;
    const double b1 = d.beta1, b2 = d.beta2, t = d.step;
    p.lr = (float)d.lr;
    p.decay = (float)(1.0 - d.lr * d.weight_decay);
    p.beta1 = (float)b1; p.beta1c = (float)(1.0 - b1);      // (1 - the fp32 beta would be off by 1e-5 of itself at 0.999)
    p.beta2 = (float)b2; p.beta2c = (float)(1.0 - b2);
    p.eps = (float)d.eps; p.grad_scale = (float)d.grad_scale;
    p.log1 = (float)log(b1); p.log2 = (float)log(b2);
    if (!done) {
        p.step_size = (float)(d.lr / (1.0 - pow(b1, t)));
        p.v_scale = (float)(1.0 / sqrt(1.0 - pow(b2, t)));
    }
    p.step = (unsigned)d.step;
    p.seed = d.seed;
    p.dither = d.dither;
    (void)hipGetLastError();
    ProbeScope probe(st);
    for (int from = 0; from < n; from += p.count) {
        p.count = 0;
        p.ordinal = (unsigned)from;
        unsigned grid = 0;
        bool coded = false;
        for (; p.count < TABLE && from + p.count < n && grid < MOST; ++p.count) {
            const purine_adamw_param& q = params[from + p.count];
            AdamwTensor& o = p.t[p.count];
            o.w = q.w.data; o.dw = q.dw.data; o.m = q.m.data; o.v = q.v.data;
            o.copy = (uint16_t*)q.copy.data;
            coded = q.m.dtype == PURINE_F8;
            o.ms = coded ? (float*)q.m_scale.data : nullptr;
            o.vs = coded ? (float*)q.v_scale.data : nullptr;
            o.n = (unsigned)elements(q.w);
            p.first[p.count] = grid;
            grid += (o.n + CHUNK - 1) / CHUNK;
        }
        const bool w16 = params[from].w.dtype == PURINE_BF16, d16 = params[from].dw.dtype == PURINE_BF16;
        if (w16 && d16) launch<uint16_t, uint16_t>(p, grid, coded, st);
        else if (w16) launch<uint16_t, float>(p, grid, coded, st);
        else if (d16) launch<float, uint16_t>(p, grid, coded, st);
        else launch<float, float>(p, grid, coded, st);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (done) hipLaunchKernelGGL(adamw_count_kernel, dim3(1), dim3(1), 0, st, done);
    return hipGetLastError();
}

}  // namespace purine
