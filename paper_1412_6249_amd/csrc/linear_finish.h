// What the kernels of the matrix products share (linear.hip, linear_direct.hip): where an operand's elements are, what a sum goes through on its
// way to memory.
#pragma once
#include "activation.h"
#include "bf16.h"
#include "block.h"
#include "packets.h"

namespace purine {
namespace {

template <typename T> __device__ __forceinline__ float widen(T v);
template <> __device__ __forceinline__ float widen<float>(float v) { return v; }
template <> __device__ __forceinline__ float widen<uint16_t>(uint16_t v) { return bf2f(v); }
__device__ __forceinline__ void narrow(float v, float* p) { *p = v; }
__device__ __forceinline__ void narrow(float v, uint16_t* p) { *p = f2bf(v); }

// Element (i, k) of an operand at i * i_step + k * k_step.
struct Source { const void* p; int64_t i_step, k_step; };

// What the sum goes through on its way to memory (E: the operands' type).
struct Finish {
    const void* bias; const void* res; void* pre; const void* slope; void* out;
    int64_t res_ld, pre_ld, slope_ld, out_ld;
    int act, accumulate;
};
template <typename E, typename O>
__device__ __forceinline__ void finish(const Finish& f, int64_t i, int j, float z) {
    if (f.bias) z += widen<E>(((const E*)f.bias)[j]);
    if (f.pre) narrow(z, (E*)f.pre + i * f.pre_ld + j);
    if (f.slope) z *= slope_any<sizeof(E) == 4>(f.act, widen<E>(((const E*)f.slope)[i * f.slope_ld + j]));
    else z = act_any<sizeof(E) == 4>(f.act, z);
    if (f.res) z += widen<E>(((const E*)f.res)[i * f.res_ld + j]);
    O* o = (O*)f.out + i * f.out_ld + j;
    if (f.accumulate) z += widen<O>(*o);
    narrow(z, o);
}

// The sum of an fp32 product's parts, scaled back; where it is infinite or NaN the sum is computed again, in plain fp32.
__device__ __forceinline__ float joined(float z, const Source& a, const Source& b, int64_t i, int64_t j, int K) {
    z *= packets::JOIN_SCALE;
    if (z - z == 0.0f) return z;
    const float* x = (const float*)a.p + i * a.i_step;
    const float* y = (const float*)b.p + j * b.i_step;
    z = 0.0f;
    for (int k = 0; k < K && z == z; ++k) z = fmaf(x[k * a.k_step], y[k * b.k_step], z);
    return z;
}

Source source_of(const void* p, int64_t ld, bool in) { return {p, in ? ld : 1, in ? 1 : ld}; }
Finish finish_of(const LinearCall& c) { return {c.bias, c.res, c.pre, c.slope, c.out, c.res_ld, c.pre_ld, c.slope_ld, c.out_ld, c.act, c.accumulate}; }

}  // namespace

// Products in one launch (linear_direct.hip, linear_stream.hip): few rows, small matrices, many rows by a small matrix.
enum DirectForm { DIRECT_NONE = 0, DIRECT_ROW /* up to 4 rows, whole packets */, DIRECT_ROWS /* up to 16 */, DIRECT_SMALL, DIRECT_STREAM };      // (the first two: both reductions inner)
hipError_t launch_linear_direct(const LinearCall& c, DirectForm form, hipStream_t st);
// bf16, A's reduction inner, whole packets
bool stream_fits(int64_t cols, int64_t K);
double stream_us(int64_t rows, int64_t cols, int64_t K);
hipError_t launch_linear_stream(const LinearCall& c, hipStream_t st);

}  // namespace purine
