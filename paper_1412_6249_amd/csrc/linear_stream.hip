// Matrix products of many rows with a small matrix (bf16): 1x1 layers over the pixels of a batch.
//
//     out[i][j] = epilogue(sum over k of A(i, k) B(j, k)),  A's reduction inner
//
// Bound: HBM, A read once and the results written once. B stays in LDS as the fragments that the MFMAs (16x16x32) read, 16 bytes a lane, laid out by every
// workgroup for itself; then a wavefront goes through its share of the rows by itself, 16 at a time: A's fragments straight from memory into
// registers, a tile ahead of their use, then 32 columns after the other. No barrier after the first. Columns are dealt to a pair of tiles so that a lane has
// eight neighbours of one row, 16 bytes, as in linear_gemm.h.
//
// us, with the tiles of linear_gemm.h / here, 100352 rows: 96 x 96 forward 16.9 / 9.8, with an activation and what it was taken of 22.7 / 14.1, data gradient
// 15.6 / 9.5; 192 -> 96 forward 25.4 / 20.8, its data gradient 23.1 / 16.7 (its 58 MB at the rate of a copy: 11). Tiles of 64 and 128 spend a third of
// their work on columns that do not exist there; where columns fill them they stay the faster ones (50000 x 128 x 128: 9.7 / 10.7). Two tiles of rows
// at a time, with branch-free stores, measured slower (11.1, 22.2).
#include "linear_finish.h"
#include "linear_gemm.h"

namespace purine {
namespace {

using lin::bf16x8;
using lin::floatx4;
using lin::u32x4;

struct StreamParams {
    const uint16_t* a; const uint16_t* b; const uint16_t* bias; const uint16_t* other; uint16_t* pre; uint16_t* out;
    int64_t a_ld, b_ld, other_ld, pre_ld, out_ld;
    int rows, cols, K, tiles, pairs, accumulate;       // tiles of 16 rows, pairs of tiles of 16 columns
};
constexpr int SWAVES = 8, AT_ONCE = 2;     // wavefronts; pairs whose other operands are asked for together
constexpr int MOST = 256 * 2 * SWAVES;      // wavefronts that the card holds, two workgroups on a compute unit

// Where column c (of a pair's 32) lies: its tile, its row among the fragment's 16.
__device__ __forceinline__ int place_of(int c) { return (c >> 2 & 1) * 16 + (c >> 3) * 4 + (c & 3); }

template <int KS, bool BIN, int ACT>
__global__ __launch_bounds__(SWAVES * 64, 4) void linear_stream_kernel(const StreamParams p) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q = lane >> 4;
    u32x4* const frag = reinterpret_cast<u32x4*>(smem);                 // [pair][tile][step][lane]
    float* const bias = reinterpret_cast<float*>(smem + (size_t)p.pairs * 2 * KS * 1024);
    const int waves = (int)gridDim.x * SWAVES;
    int tile = (int)blockIdx.x * SWAVES + wave;
    u32x4 next[KS];
    auto load = [&](int t) {               // (rows past the last read it, and so do tiles)
        const uint16_t* a = p.a + (int64_t)min(t * 16 + r, p.rows - 1) * p.a_ld;
#pragma unroll
        for (int s = 0; s < KS; ++s) next[s] = *reinterpret_cast<const u32x4*>(a + min(s * 32 + q * 8, p.K - 8));
    };
    load(min(tile, p.tiles - 1));
    // B's fragments, eight loads before the first is used
    constexpr int BATCH = 8, THREADS = SWAVES * 64;
    if constexpr (BIN) {
        const int all = p.pairs * 2 * KS * 64;
        for (int t0 = threadIdx.x; t0 < all; t0 += BATCH * THREADS) {
            u32x4 v[BATCH];
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                const int t = min(t0 + u * THREADS, all - 1), l = t & 63, s = (t >> 6) % KS, h = (t >> 6) / KS, m = l & 15;
                const int j = (h >> 1) * 32 + (m >> 2) * 8 + (h & 1) * 4 + (m & 3), k = s * 32 + (l >> 4) * 8;
                v[u] = *reinterpret_cast<const u32x4*>(p.b + min(j, p.cols - 1) * p.b_ld + min(k, p.K - 8));
                if (j >= p.cols || k >= p.K) v[u] = u32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int u = 0; u < BATCH; ++u) if (t0 + u * THREADS < all) frag[t0 + u * THREADS] = v[u];
        }
        for (int j = threadIdx.x; j < p.pairs * 32; j += THREADS) bias[j] = p.bias && j < p.cols ? bf2f(p.bias[j]) : 0.0f;
    } else {
        uint16_t* const cell = reinterpret_cast<uint16_t*>(smem);
        const int all = p.pairs * 4 * KS * 32;
        for (int t0 = threadIdx.x; t0 < all; t0 += BATCH * THREADS) {
            u32x4 v[BATCH];
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                const int t = min(t0 + u * THREADS, all - 1), k = t / (p.pairs * 4), c = (t - k * (p.pairs * 4)) * 8;
                v[u] = *reinterpret_cast<const u32x4*>(p.b + min(k, p.K - 1) * p.b_ld + min(c, p.cols - 8));
                if (c >= p.cols || k >= p.K) v[u] = u32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                const int t = t0 + u * THREADS, k = t / (p.pairs * 4), c8 = t - k * (p.pairs * 4);
                if (t >= all) break;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int at = place_of((c8 & 3) * 8 + e), h = (c8 >> 2) * 2 + (at >> 4);
                    cell[((h * KS + (k >> 5)) * 64 + (k >> 3 & 3) * 16 + (at & 15)) * 8 + (k & 7)] = (uint16_t)(v[u][e >> 1] >> (e & 1) * 16);
                }
            }
        }
    }
    __syncthreads();
    const bool reads = BIN ? p.other != nullptr : ACT != PURINE_ACT_NONE;
    while (tile < p.tiles) {
        bf16x8 a[KS];
#pragma unroll
        for (int s = 0; s < KS; ++s) {     // (what lies past the reduction's end may be anything)
            u32x4 v = next[s];
            if (s * 32 + q * 8 >= p.K) v = u32x4{0, 0, 0, 0};
            a[s] = __builtin_bit_cast(bf16x8, v);
        }
        const int row = tile * 16 + r, row_in = min(row, p.rows - 1);
        tile += waves;
        load(min(tile, p.tiles - 1));
        for (int p0 = 0; p0 < p.pairs; p0 += AT_ONCE) {
            u32x4 t[AT_ONCE], o[AT_ONCE];
            if (reads)
#pragma unroll
                for (int u = 0; u < AT_ONCE; ++u) t[u] = *reinterpret_cast<const u32x4*>(p.other + row_in * p.other_ld + min((p0 + u) * 32 + q * 8, p.cols - 8));
            if (p.accumulate)
#pragma unroll
                for (int u = 0; u < AT_ONCE; ++u) o[u] = *reinterpret_cast<const u32x4*>(p.out + row_in * p.out_ld + min((p0 + u) * 32 + q * 8, p.cols - 8));
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                if (p0 + u >= p.pairs) break;
                const u32x4* f = frag + (size_t)(p0 + u) * 2 * KS * 64 + lane;
                floatx4 x{0.0f, 0.0f, 0.0f, 0.0f}, y{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f[s * 64]), a[s], x, 0, 0, 0);
                    y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f[(KS + s) * 64]), a[s], y, 0, 0, 0);
                }
                const int j = (p0 + u) * 32 + q * 8;
                float v[8], w[8], pre[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) { v[e] = x[e]; v[4 + e] = y[e]; }
                if (reads) lin::widen8(t[u], w);
                if constexpr (BIN) {
                    const floatx4 b0 = *reinterpret_cast<const floatx4*>(bias + j), b1 = *reinterpret_cast<const floatx4*>(bias + j + 4);
#pragma unroll
                    for (int e = 0; e < 8; ++e) { pre[e] = v[e] + (e < 4 ? b0[e & 3] : b1[e & 3]); v[e] = act_of<ACT, false>(pre[e]); }
                    if (reads)
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] += w[e];
                } else if constexpr (ACT != PURINE_ACT_NONE) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] *= act_slope<ACT, false>(w[e]);
                }
                if (p.accumulate) {
                    lin::widen8(o[u], w);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] += w[e];
                }
                if (row < p.rows && j < p.cols) {
                    if (BIN && p.pre) lin::put8(p.pre + row * p.pre_ld + j, true, 8, pre);
                    lin::put8(p.out + row * p.out_ld + j, true, 8, v);
                }
            }
        }
    }
}

size_t stream_lds(int64_t cols, int64_t KS) { return (size_t)((cols + 31) / 32) * (2 * KS * 1024 + 32 * 4); }
int stream_steps(int64_t K) { const int s = (int)((K + 31) / 32); return s <= 2 ? 2 : s <= 4 ? s : 6; }

template <int KS, bool BIN, int ACT>
hipError_t launch(const StreamParams& p, hipStream_t st) {
    const size_t lds = stream_lds(p.cols, KS);
    const auto kernel = &linear_stream_kernel<KS, BIN, ACT>;
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    // the tiles in equal shares, no more wavefronts than run at once
    const int each = (p.tiles + MOST - 1) / MOST;
    const unsigned grid = (unsigned)(((p.tiles + each - 1) / each + SWAVES - 1) / SWAVES);
    ProbeScope probe(st);
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(SWAVES * 64), lds, st, p);
    return hipGetLastError();
}
template <int KS, bool BIN>
hipError_t by_act(const StreamParams& p, int act, hipStream_t st) {
    switch (act) {
        case PURINE_ACT_NONE: return launch<KS, BIN, PURINE_ACT_NONE>(p, st);
        case PURINE_ACT_RELU: return launch<KS, BIN, PURINE_ACT_RELU>(p, st);
        case PURINE_ACT_SILU: return launch<KS, BIN, PURINE_ACT_SILU>(p, st);
        case PURINE_ACT_GELU: return launch<KS, BIN, PURINE_ACT_GELU>(p, st);
        case PURINE_ACT_GELU_TANH: return launch<KS, BIN, PURINE_ACT_GELU_TANH>(p, st);
    }
    return hipErrorInvalidValue;
}
template <bool BIN>
hipError_t by_steps(const StreamParams& p, int act, hipStream_t st) {
    switch (stream_steps(p.K)) {
        case 2: return by_act<2, BIN>(p, act, st);
        case 3: return by_act<3, BIN>(p, act, st);
        case 4: return by_act<4, BIN>(p, act, st);
        default: return by_act<6, BIN>(p, act, st);
    }
}

}  // namespace

// (longer reductions do not leave the registers for a tile ahead)
bool stream_fits(int64_t cols, int64_t K) { return K % 8 == 0 && cols % 8 == 0 && K <= 192 && stream_lds(cols, stream_steps(K)) <= 80 * 1024; }
// Expected time (us): a launch, B's way into LDS, and the rows at memory's rate, or the chain of a wavefront's pairs of columns.
double stream_us(int64_t rows, int64_t cols, int64_t K) {
    const double chain = 0.36 * (double)((rows + 16 * MOST - 1) / (16 * MOST)) * (double)((cols + 31) / 32);
    return 3.0 + 2.0 * (double)K * (double)cols / 14e3 + fmax(chain, 2.0 * (double)rows * (double)(K + cols) / 5.2e6);
}

hipError_t launch_linear_stream(const LinearCall& c, hipStream_t st) {
    if (!c.a_in || c.dtype != PURINE_BF16 || c.out_dtype != PURINE_BF16 || !stream_fits(c.cols, c.K)) return hipErrorInvalidValue;
    StreamParams p{};
    p.a = (const uint16_t*)c.a; p.b = (const uint16_t*)c.b; p.bias = (const uint16_t*)c.bias;
    p.other = (const uint16_t*)(c.b_in ? c.res : c.slope);
    p.pre = (uint16_t*)c.pre; p.out = (uint16_t*)c.out;
    p.a_ld = c.a_ld; p.b_ld = c.b_ld; p.other_ld = c.b_in ? c.res_ld : c.slope_ld; p.pre_ld = c.pre_ld; p.out_ld = c.out_ld;
    p.rows = (int)c.rows; p.cols = (int)c.cols; p.K = (int)c.K;
    p.tiles = (int)((c.rows + 15) / 16);
    p.pairs = (int)((c.cols + 31) / 32);
    p.accumulate = c.accumulate;
    return c.b_in ? by_steps<true>(p, c.act, st) : by_steps<false>(p, c.slope ? c.act : PURINE_ACT_NONE, st);
}

}  // namespace purine
