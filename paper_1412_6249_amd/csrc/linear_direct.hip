// Matrix products in one launch: few rows, whose time is reading the other operand, and small matrices, whose time is launches.
//
//     out[i][j] = epilogue(sum over k of A(i, k) B(j, k))
//
// Up to four rows (linear_row_kernel): a wavefront reads 1024 bytes of a row of B at a time, four such rows beside each other, multiplies them with the same
// part of the rows of A in fp32, and adds up its lanes; four wavefronts share the reduction. Bound: reading B (1 x 4096 x 4096 bf16: 33.6 MB in 7.2 us from memory,
// 4.6 from the caches).
//
// Else (linear_direct_kernel) a workgroup owns 16 TI x 16 TJ results. Its wavefronts take the steps of the reduction (32 elements) in turn, load their fragments straight from
// memory, a group of steps ahead, multiply them (bf16 as they are; fp32 as three exact bf16 parts, the five small products in an accumulator of
// their own) and add their sums through LDS in order. Nothing is laid out beforehand and there is no second launch.
//
// Bound: a chain of a few loads, and one launch (777 x 501 x 333 fp32: each pass 10 - 13 us; packed operands, product and join of linear.hip take 24 - 26).
#include "linear_gemm.h"
#include "linear_finish.h"
#include "packets.h"

namespace purine {
namespace {

using lin::bf16x8;
using lin::floatx4;
using lin::u32x4;

struct DirectParams {
    Source a, b;
    Finish f;
    unsigned a_bytes, b_bytes;
    int a_ld, b_ld;
    int rows, cols, K, tiles_j, steps;
};
constexpr unsigned NOWHERE = 0x80000000u;

// Eight reduction elements as memory has them. bf16 with the reduction inner: from the dword that holds the first, five of them.
template <typename E, bool IN> struct Raw { uint32_t w[sizeof(E) == 4 ? 8 : IN ? 5 : 8]; };

// ROW_OK rows and elements up to K exist; packets are whole (WHOLE: rows begin at 16 bytes) or begin at any element.
template <typename E, bool IN, bool WHOLE>
__device__ __forceinline__ void fetch(__amdgpu_buffer_rsrc_t r, unsigned row_at, bool ok, int k, int K, int ld, Raw<E, IN>& v) {
    if constexpr (IN) {
        const unsigned at = row_at + (unsigned)k * (unsigned)sizeof(E), o = ok && k < K ? (sizeof(E) == 2 && !WHOLE ? at & ~3u : at) : NOWHERE;
        const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(r, o, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) v.w[e] = x[e];
        if constexpr (sizeof(E) == 4) {
            const u32x4 y = __builtin_amdgcn_raw_buffer_load_b128(r, o == NOWHERE ? o : o + 16, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) v.w[4 + e] = y[e];
        } else {
            v.w[4] = WHOLE ? 0u : __builtin_amdgcn_raw_buffer_load_b32(r, o == NOWHERE ? o : o + 16, 0, 0);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const unsigned o = ok && k + e < K ? row_at + (unsigned)(k + e) * (unsigned)ld * (unsigned)sizeof(E) : NOWHERE;
            if constexpr (sizeof(E) == 4) v.w[e] = __builtin_amdgcn_raw_buffer_load_b32(r, o, 0, 0);
            else v.w[e] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(r, o, 0, 0);
        }
    }
}

// The parts of a fragment: one, or three of fp32. Elements past the reduction's end (a row's next, or the range check's zeros) become zeros.
template <typename E, bool IN, bool WHOLE>
__device__ __forceinline__ void parts_of(const Raw<E, IN>& v, unsigned row_at, int k, int K, bf16x8 (&p)[sizeof(E) == 4 ? 3 : 1]) {
    if constexpr (sizeof(E) == 2) {
        u32x4 w;
        if constexpr (IN) {
            const unsigned sh = !WHOLE && (row_at & 2u) != ((unsigned)k * 2u & 2u) ? 16u : 0u;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = WHOLE ? v.w[e] : __builtin_amdgcn_alignbit(v.w[e + 1], v.w[e], sh);
            if (k + 8 > K) {
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] &= (k + 2 * e < K ? 0xffffu : 0u) | (k + 2 * e + 1 < K ? 0xffff0000u : 0u);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = v.w[2 * e] | v.w[2 * e + 1] << 16;
        }
        p[0] = __builtin_bit_cast(bf16x8, w);
    } else {
        u32x4 w[3];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float x = __uint_as_float(v.w[2 * e]), y = __uint_as_float(v.w[2 * e + 1]);
            if (IN) { x = k + 2 * e < K ? x : 0.0f; y = k + 2 * e + 1 < K ? y : 0.0f; }
            uint32_t part[3];
            packets::split_pair(x, y, part);
#pragma unroll
            for (int l = 0; l < 3; ++l) w[l][e] = part[l];
        }
#pragma unroll
        for (int l = 0; l < 3; ++l) p[l] = __builtin_bit_cast(bf16x8, w[l]);
    }
}

template <typename E, typename O, int TI, int TJ, int WAVES, bool AIN, bool BIN, bool WHOLE>
__global__ __launch_bounds__(WAVES * 64) void linear_direct_kernel(const DirectParams p) {
    constexpr bool F32 = sizeof(E) == 4;
    constexpr int DEPTH = TI * TJ == 1 ? 4 : F32 || !AIN || !BIN ? 1 : 2, P = F32 ? 3 : 1, SETS = F32 ? 2 : 1;
    __shared__ floatx4 sums[WAVES][TI * TJ][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ti = blockIdx.x / p.tiles_j, i0 = ti * 16 * TI, j0 = (int)(blockIdx.x - (unsigned)ti * p.tiles_j) * 16 * TJ;
    const int r = lane & 15, k8 = (lane >> 4) * 8;
    const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p.a.p), (short)0, (int)p.a_bytes, 0x00020000);
    const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p.b.p), (short)0, (int)p.b_bytes, 0x00020000);
    unsigned a_at[TI], b_at[TJ];
#pragma unroll
    for (int i = 0; i < TI; ++i) a_at[i] = (unsigned)(min(i0 + i * 16 + r, p.rows - 1) * (AIN ? p.a_ld : 1)) * (unsigned)sizeof(E);      // (rows past the last read it again)
#pragma unroll
    for (int j = 0; j < TJ; ++j) b_at[j] = (unsigned)(min(j0 + j * 16 + r, p.cols - 1) * (BIN ? p.b_ld : 1)) * (unsigned)sizeof(E);
    struct Group { Raw<E, AIN> a[DEPTH][TI]; Raw<E, BIN> b[DEPTH][TJ]; };
    auto load = [&](int s, Group& g) {          // this wavefront's steps s, s + WAVES, ...
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            const int k = (s + d * WAVES) * 32 + k8;
#pragma unroll
            for (int j = 0; j < TJ; ++j) fetch<E, BIN, WHOLE>(rb, b_at[j], true, k, p.K, p.b_ld, g.b[d][j]);
#pragma unroll
            for (int i = 0; i < TI; ++i) fetch<E, AIN, WHOLE>(ra, a_at[i], true, k, p.K, p.a_ld, g.a[d][i]);
        }
    };
    floatx4 acc[SETS][TI][TJ];
#pragma unroll
    for (int q = 0; q < SETS; ++q)
#pragma unroll
        for (int i = 0; i < TI; ++i)
#pragma unroll
            for (int j = 0; j < TJ; ++j) acc[q][i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    auto multiply = [&](int s, const Group& g) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            const int k = (s + d * WAVES) * 32 + k8;
            bf16x8 a[TI][P], b[TJ][P];
#pragma unroll
            for (int i = 0; i < TI; ++i) parts_of<E, AIN, WHOLE>(g.a[d][i], a_at[i], k, p.K, a[i]);
#pragma unroll
            for (int j = 0; j < TJ; ++j) parts_of<E, BIN, WHOLE>(g.b[d][j], b_at[j], k, p.K, b[j]);
#pragma unroll
            for (int i = 0; i < TI; ++i)
#pragma unroll
                for (int j = 0; j < TJ; ++j) {
                    acc[0][i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j][0], a[i][0], acc[0][i][j], 0, 0, 0);
                    if constexpr (F32) {
                        floatx4& c = acc[1][i][j];
                        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j][1], a[i][1], c, 0, 0, 0);
                        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j][2], a[i][0], c, 0, 0, 0);
                        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j][0], a[i][2], c, 0, 0, 0);
                        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j][1], a[i][0], c, 0, 0, 0);
                        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j][0], a[i][1], c, 0, 0, 0);
                    }
                }
        }
    };
    // (steps past the last one read zeros: two groups a turn, in registers of their own)
    Group g0, g1;
    load(wave, g0);
    for (int s = wave; s < p.steps; s += 2 * DEPTH * WAVES) {
        load(s + DEPTH * WAVES, g1);
        multiply(s, g0);
        load(s + 2 * DEPTH * WAVES, g0);
        multiply(s + DEPTH * WAVES, g1);
    }
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
            floatx4 v = acc[0][i][j];
            if constexpr (F32) v += acc[1][i][j];
            sums[wave][i * TJ + j][lane] = v;
        }
    __syncthreads();
    // a lane has four neighbouring columns of a row
    for (int t = wave; t < TI * TJ; t += WAVES) {
        floatx4 v = sums[0][t][lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += sums[w][t][lane];
        const int i = i0 + t / TJ * 16 + r, j = j0 + t % TJ * 16 + (lane >> 4) * 4;
        if (i >= p.rows) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (j + e >= p.cols) break;
            float z = v[e];
            if constexpr (F32) z = joined(z, p.a, p.b, i, j + e, p.K);
            finish<E, O>(p.f, i, j + e, z);
        }
    }
}

// Four rows of B, `rows` (M at most) of A.
constexpr int RJ = 4, RWAVES = 4, RAHEAD = 2;
template <typename E, typename O, int M>
__global__ __launch_bounds__(RWAVES * 64) void linear_row_kernel(const DirectParams p) {
    constexpr int PER = 16 / (int)sizeof(E), VALUES = M * RJ;
    __shared__ float sums[RWAVES][VALUES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j0 = blockIdx.x * RJ;
    const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p.a.p), (short)0, (int)p.a_bytes, 0x00020000);
    const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p.b.p), (short)0, (int)p.b_bytes, 0x00020000);
    float v[VALUES];
#pragma unroll
    for (int e = 0; e < VALUES; ++e) v[e] = 0.0f;
    auto numbers = [](const u32x4& k, float (&x)[PER]) {
        if constexpr (PER == 8) lin::widen8(k, x);
        else
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(k[e]);
    };
    for (int k0 = wave * 64 * PER; k0 < p.K; k0 += RAHEAD * RWAVES * 64 * PER) {
        u32x4 a[RAHEAD][M], b[RAHEAD][RJ];
#pragma unroll
        for (int u = 0; u < RAHEAD; ++u) {
            const int k = k0 + u * RWAVES * 64 * PER + lane * PER;      // (K is a whole number of packets)
            const unsigned at = k < p.K ? (unsigned)k * (unsigned)sizeof(E) : NOWHERE;
#pragma unroll
            for (int j = 0; j < RJ; ++j) b[u][j] = __builtin_amdgcn_raw_buffer_load_b128(rb, at, min(j0 + j, p.cols - 1) * p.b_ld * (int)sizeof(E), 0);
#pragma unroll
            for (int i = 0; i < M; ++i) a[u][i] = __builtin_amdgcn_raw_buffer_load_b128(ra, at, min(i, p.rows - 1) * p.a_ld * (int)sizeof(E), 0);
        }
#pragma unroll
        for (int u = 0; u < RAHEAD; ++u) {
            float x[M][PER];
#pragma unroll
            for (int i = 0; i < M; ++i) numbers(a[u][i], x[i]);
#pragma unroll
            for (int j = 0; j < RJ; ++j) {
                float w[PER];
                numbers(b[u][j], w);
#pragma unroll
                for (int i = 0; i < M; ++i)
#pragma unroll
                    for (int e = 0; e < PER; ++e) v[i * RJ + j] = fmaf(x[i][e], w[e], v[i * RJ + j]);
            }
        }
    }
    // sums over the lanes: halves of the values go to halves of the lanes until each has one, whose lanes then add theirs
    int index = 0, far = 32;
#pragma unroll
    for (int n = VALUES / 2; n; n /= 2, far /= 2) {
        const bool upper = lane & far;
#pragma unroll
        for (int e = 0; e < n; ++e) {
            const float keep = upper ? v[n + e] : v[e], give = upper ? v[e] : v[n + e];
            v[e] = keep + __shfl_xor(give, far);
        }
        index = 2 * index + (upper ? 1 : 0);
    }
    for (; far; far /= 2) v[0] += __shfl_xor(v[0], far);
    if ((lane & (64 / VALUES - 1)) == 0) sums[wave][index] = v[0];
    __syncthreads();
    if (threadIdx.x >= VALUES) return;
    float z = sums[0][threadIdx.x];
#pragma unroll
    for (int w = 1; w < RWAVES; ++w) z += sums[w][threadIdx.x];
    const int i = threadIdx.x / RJ, j = j0 + threadIdx.x % RJ;
    if (i < p.rows && j < p.cols) finish<E, O>(p.f, i, j, z);
}
template <typename E, typename O>
hipError_t launch_row(const DirectParams& p, hipStream_t st) {
    const unsigned grid = (unsigned)((p.cols + RJ - 1) / RJ);
    ProbeScope probe(st);
    if (p.rows == 1) hipLaunchKernelGGL((linear_row_kernel<E, O, 1>), dim3(grid), dim3(RWAVES * 64), 0, st, p);
    else if (p.rows == 2) hipLaunchKernelGGL((linear_row_kernel<E, O, 2>), dim3(grid), dim3(RWAVES * 64), 0, st, p);
    else hipLaunchKernelGGL((linear_row_kernel<E, O, 4>), dim3(grid), dim3(RWAVES * 64), 0, st, p);
    return hipGetLastError();
}

template <typename E, typename O, int TI, int TJ, int WAVES, bool AIN, bool BIN>
hipError_t launch(const DirectParams& q, bool whole, hipStream_t st) {
    DirectParams p = q;
    p.tiles_j = (p.cols + 16 * TJ - 1) / (16 * TJ);
    const int64_t grid = (int64_t)((p.rows + 16 * TI - 1) / (16 * TI)) * p.tiles_j;
    ProbeScope probe(st);
    if constexpr (sizeof(E) == 2 && (AIN || BIN))
        if (!whole) {
            hipLaunchKernelGGL((linear_direct_kernel<E, O, TI, TJ, WAVES, AIN, BIN, false>), dim3((unsigned)grid), dim3(WAVES * 64), 0, st, p);
            return hipGetLastError();
        }
    hipLaunchKernelGGL((linear_direct_kernel<E, O, TI, TJ, WAVES, AIN, BIN, true>), dim3((unsigned)grid), dim3(WAVES * 64), 0, st, p);
    return hipGetLastError();
}
template <typename E, typename O, int TI, int TJ, int WAVES>
hipError_t by_sides(const DirectParams& p, bool a_in, bool b_in, bool whole, hipStream_t st) {
    if (a_in && b_in) return launch<E, O, TI, TJ, WAVES, true, true>(p, whole, st);
    if (a_in) return launch<E, O, TI, TJ, WAVES, true, false>(p, whole, st);
    return launch<E, O, TI, TJ, WAVES, false, false>(p, whole, st);
}
template <typename E, typename O>
hipError_t by_form(const DirectParams& p, DirectForm form, bool a_in, bool b_in, bool whole, hipStream_t st) {
    if (form == DIRECT_ROW) return launch_row<E, O>(p, st);
    if (form == DIRECT_ROWS) return launch<E, O, 1, 1, 8, true, true>(p, whole, st);
    return by_sides<E, O, 2, 2, 4>(p, a_in, b_in, whole, st);
}

}  // namespace

hipError_t launch_linear_direct(const LinearCall& c, DirectForm form, hipStream_t st) {
    const int es = c.dtype == PURINE_F32 ? 4 : 2;
    DirectParams p{};
    p.a = source_of(c.a, c.a_ld, c.a_in);
    p.b = source_of(c.b, c.b_ld, c.b_in);
    p.f = finish_of(c);
    p.rows = (int)c.rows; p.cols = (int)c.cols; p.K = (int)c.K;
    p.steps = (int)((c.K + 31) / 32);
    p.a_ld = (int)c.a_ld; p.b_ld = (int)c.b_ld;
    const int64_t a_size = (((c.a_in ? c.rows : c.K) - 1) * c.a_ld + (c.a_in ? c.K : c.rows)) * es, b_size = (((c.b_in ? c.cols : c.K) - 1) * c.b_ld + (c.b_in ? c.K : c.cols)) * es;
    if (a_size >= 0x7fffffff || b_size >= 0x7fffffff) return hipErrorInvalidValue;
    // (the range check works by the dword: a last odd element of bf16 would be cut off with its dword)
    p.a_bytes = (unsigned)((a_size + 3) & ~(int64_t)3);
    p.b_bytes = (unsigned)((b_size + 3) & ~(int64_t)3);
    const bool whole = (!c.a_in || (c.a_ld % 8 == 0)) && (!c.b_in || (c.b_ld % 8 == 0));
    if (c.dtype == PURINE_F32) return by_form<float, float>(p, form, c.a_in, c.b_in, true, st);
    if (c.out_dtype == PURINE_F32) return by_form<uint16_t, float>(p, form, c.a_in, c.b_in, whole, st);
    return by_form<uint16_t, uint16_t>(p, form, c.a_in, c.b_in, whole, st);
}

}  // namespace purine
