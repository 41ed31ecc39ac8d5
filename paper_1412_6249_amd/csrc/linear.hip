// Matrix product with bias, activation and residual in its epilogue, its gradients (purine_linear_*), and the gradient of an
// activation by itself (purine_act_bwd).
#include "activation.h"
#include "bf16.h"
#include "block.h"

namespace purine {
namespace {

template <typename T> __device__ __forceinline__ float widen(T v);
template <> __device__ __forceinline__ float widen<float>(float v) { return v; }
template <> __device__ __forceinline__ float widen<uint16_t>(uint16_t v) { return bf2f(v); }
__device__ __forceinline__ void narrow(float v, float* p) { *p = v; }
__device__ __forceinline__ void narrow(float v, uint16_t* p) { *p = f2bf(v); }

struct LinearParams {
    const void* a; const void* b; void* out;
    const void* bias; const void* res; void* pre; const void* slope;
    int64_t a_i, a_k, b_i, b_k, out_ld, res_ld, pre_ld, slope_ld;
    int rows, cols, K, tiles_j;
    int act, accumulate;
};

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

// The plain kernel: 64 x 64 results per workgroup, 16 per thread, fp32 products.
constexpr int TS = 64, KS = 16;
template <typename T, typename O>
__global__ __launch_bounds__(256) void linear_kernel(const LinearParams p) {
    __shared__ float as[KS][TS + 1], bs[KS][TS + 1];
    const int i0 = (int)(blockIdx.x / p.tiles_j) * TS, j0 = (int)(blockIdx.x % p.tiles_j) * TS;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const T* a = (const T*)p.a;
    const T* b = (const T*)p.b;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < p.K; k0 += KS) {
        for (int e = threadIdx.x; e < KS * TS; e += 256) {
            const int k = e / TS, i = e % TS;
            as[k][i] = k0 + k < p.K && i0 + i < p.rows ? widen<T>(a[(i0 + i) * p.a_i + (k0 + k) * p.a_k]) : 0.0f;
            bs[k][i] = k0 + k < p.K && j0 + i < p.cols ? widen<T>(b[(j0 + i) * p.b_i + (k0 + k) * p.b_k]) : 0.0f;
        }
        __syncthreads();
        for (int k = 0; k < KS; ++k)
            for (int u = 0; u < 4; ++u)
                for (int v = 0; v < 4; ++v) acc[u][v] += as[k][ty * 4 + u] * bs[k][tx * 4 + v];
        __syncthreads();
    }
    for (int u = 0; u < 4; ++u)
        for (int v = 0; v < 4; ++v) {
            const int64_t i = i0 + ty * 4 + u;
            const int j = j0 + tx * 4 + v;
            if (i >= p.rows || j >= p.cols) continue;
            float z = acc[u][v];
            if (p.bias) z += widen<T>(((const T*)p.bias)[j]);
            if (p.pre) narrow(z, (T*)p.pre + i * p.pre_ld + j);
            if (p.slope) z *= slope_any(p.act, widen<T>(((const T*)p.slope)[i * p.slope_ld + j]));
            else z = act_any(p.act, z);
            if (p.res) z += widen<T>(((const T*)p.res)[i * p.res_ld + j]);
            O* o = (O*)p.out + i * p.out_ld + j;
            if (p.accumulate) z += widen<O>(*o);
            narrow(z, o);
        }
}

// g = dy act'(pre), and the sums of its columns over a slice of the rows: a thread per column, rows in order.
struct ActParams {
    const void* pre; const void* dy; void* g; float* part;
    int64_t pre_ld, dy_ld, g_ld;
    int N, K, rows, act;
};
template <typename T>
__global__ __launch_bounds__(256) void act_bwd_kernel(const ActParams p) {
    const int tiles = (p.K + 255) / 256, slice = blockIdx.x / tiles, j = (int)(blockIdx.x % tiles) * 256 + threadIdx.x;
    if (j >= p.K) return;
    float sum = 0.0f;
    for (int64_t i = (int64_t)slice * p.rows; i < min((int64_t)(slice + 1) * p.rows, (int64_t)p.N); ++i) {
        float v = widen<T>(((const T*)p.dy)[i * p.dy_ld + j]);
        if (p.pre) v *= slope_any(p.act, widen<T>(((const T*)p.pre)[i * p.pre_ld + j]));
        if (p.g) narrow(v, (T*)p.g + i * p.g_ld + j);
        sum += v;
    }
    if (p.part) p.part[(size_t)slice * p.K + j] = sum;
}
template <typename O>
__global__ __launch_bounds__(256) void column_sums_kernel(const float* part, O* db, int slices, int K, int accumulate) {
    const int j = blockIdx.x * 256 + threadIdx.x;
    if (j >= K) return;
    float sum = 0.0f;
    for (int s = 0; s < slices; ++s) sum += part[(size_t)s * K + j];
    if (accumulate) sum += widen<O>(db[j]);
    narrow(sum, db + j);
}
int act_rows(int64_t N, int64_t K) {
    int64_t tiles = (K + 255) / 256, slices = 1024 / tiles;
    if (slices < 1) slices = 1;
    int64_t rows = (N + slices - 1) / slices;
    return (int)(rows < 16 ? 16 : rows);
}

}  // namespace

size_t linear_ws_bytes(int64_t, int64_t, int64_t, bool, bool, int) { return 0; }

hipError_t launch_linear(const LinearCall& c, void*, hipStream_t st) {
    LinearParams p{};
    p.a = c.a; p.b = c.b; p.out = c.out; p.bias = c.bias; p.res = c.res; p.pre = c.pre; p.slope = c.slope;
    p.a_i = c.a_in ? c.a_ld : 1; p.a_k = c.a_in ? 1 : c.a_ld;
    p.b_i = c.b_in ? c.b_ld : 1; p.b_k = c.b_in ? 1 : c.b_ld;
    p.out_ld = c.out_ld; p.res_ld = c.res_ld; p.pre_ld = c.pre_ld; p.slope_ld = c.slope_ld;
    p.rows = (int)c.rows; p.cols = (int)c.cols; p.K = (int)c.K;
    p.act = c.act; p.accumulate = c.accumulate;
    p.tiles_j = (int)((c.cols + TS - 1) / TS);
    const unsigned grid = (unsigned)((c.rows + TS - 1) / TS * p.tiles_j);
    ProbeScope probe(st);
    (void)hipGetLastError();
    if (c.dtype == PURINE_F32) hipLaunchKernelGGL((linear_kernel<float, float>), dim3(grid), dim3(256), 0, st, p);
    else if (c.out_dtype == PURINE_F32) hipLaunchKernelGGL((linear_kernel<uint16_t, float>), dim3(grid), dim3(256), 0, st, p);
    else hipLaunchKernelGGL((linear_kernel<uint16_t, uint16_t>), dim3(grid), dim3(256), 0, st, p);
    return hipGetLastError();
}

size_t act_bwd_ws_bytes(int64_t N, int64_t K) {
    const int64_t rows = act_rows(N, K), slices = (N + rows - 1) / rows;
    return (size_t)slices * K * 4;
}

hipError_t launch_act_bwd(int dtype, const void* pre, int64_t pre_ld, const void* dy, int64_t dy_ld, void* g, int64_t g_ld, void* db, int db_dtype,
                          bool accumulate, int64_t N, int64_t K, int act, void* ws, hipStream_t st) {
    ActParams p{pre, dy, g, db ? (float*)ws : nullptr, pre_ld, dy_ld, g_ld, (int)N, (int)K, act_rows(N, K), act};
    const int slices = (int)((N + p.rows - 1) / p.rows), tiles = (int)((K + 255) / 256);
    (void)hipGetLastError();
    {
        ProbeScope probe(st);
        if (dtype == PURINE_F32) hipLaunchKernelGGL((act_bwd_kernel<float>), dim3((unsigned)(slices * (int64_t)tiles)), dim3(256), 0, st, p);
        else hipLaunchKernelGGL((act_bwd_kernel<uint16_t>), dim3((unsigned)(slices * (int64_t)tiles)), dim3(256), 0, st, p);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !db) return e;
    if (db_dtype == PURINE_F32) hipLaunchKernelGGL((column_sums_kernel<float>), dim3(tiles), dim3(256), 0, st, p.part, (float*)db, slices, (int)K, accumulate);
    else hipLaunchKernelGGL((column_sums_kernel<uint16_t>), dim3(tiles), dim3(256), 0, st, p.part, (uint16_t*)db, slices, (int)K, accumulate);
    return hipGetLastError();
}

}  // namespace purine
