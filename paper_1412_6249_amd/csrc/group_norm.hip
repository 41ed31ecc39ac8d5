// Group normalization with an activation on channels-last tensors, and its gradient (purine_group_norm_fwd / _bwd).
//
//     xhat = (x - mean) rstd,  z = xhat scale[c] + shift[c],  y = act(z)            mean, var: over a group's channels and all positions
//     dz = dy act'(z),  h = dz scale,  dx = rstd (h - avg(h) - xhat avg(h xhat)),  dshift = sum dz,  dscale = sum dz xhat
//
// Bound: HBM. A thread owns V neighbouring channels (16 bytes where the row allows it) and walks down the positions, so that
// loads are whole rows and the affine parameters stay in registers. Sums are kept per channel, which serves any number of
// channels per group: for the statistics s = sum (x - k), q = sum (x - k)^2 about the channel's value k at the image's first
// position (a large mean costs no digits), for the gradient sum dz and sum dz xhat. One kernel sums over slices of the
// positions, one joins slices and channels in a fixed order, one writes the results.
#include "activation.h"
#include "bf16.h"
#include "block.h"

namespace purine {
namespace {

constexpr int NT = 256;

template <typename T, int V>
__device__ __forceinline__ void load_v(const T* p, float (&v)[V]) {
    struct alignas(sizeof(T) * V) Pack { T e[V]; };
    const Pack k = *reinterpret_cast<const Pack*>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if constexpr (sizeof(T) == 2) v[i] = bf2f(k.e[i]);
        else v[i] = k.e[i];
    }
}
template <typename T, int V>
__device__ __forceinline__ void store_v(T* p, const float (&v)[V]) {
    struct alignas(sizeof(T) * V) Pack { T e[V]; };
    Pack k;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if constexpr (sizeof(T) == 2) k.e[i] = f2bf(v[i]);
        else k.e[i] = v[i];
    }
    *reinterpret_cast<Pack*>(p) = k;
}

struct NormParams {
    const void* x; const void* dy; void* out;
    int64_t x_ns, dy_ns, out_ns;
    const float* scale; const float* shift;     // or null
    float2* part;              // per image, slice and channel: the two sums
    float2* stat;              // per image and group: mean, rstd; of the gradient avg(h), avg(h xhat)
    const float* mean; const float* rstd;       // gradient: as saved
    float* mean_out; float* rstd_out;           // or null
    float* dscale; float* dshift;
    int N, S, C, G, per;       // channels per group
    int slices, rows;          // slices of the positions, positions per slice
    int tiles;                 // of NT vectors of channels
    float eps;
    int accumulate;
};

// What a workgroup works on (image, slice of the positions, tile of the channels), the channels of this thread, its place among the
// threads that share them, and their number.
template <int V>
struct Place {
    int n, slice, s0, s1, c, r, R, tile;
    bool on;
    __device__ explicit Place(const NormParams& p) {
        const int b = blockIdx.x / p.tiles, cv = p.C / V, first = (int)(blockIdx.x - b * p.tiles) * NT;
        n = b / p.slices;
        slice = b - n * p.slices;
        s0 = slice * p.rows;
        s1 = min(s0 + p.rows, p.S);
        tile = min(NT, cv - first);
        R = NT / tile;
        r = threadIdx.x / tile;
        on = r < R;
        c = (first + (int)threadIdx.x % tile) * V;
    }
};

// Adds the R threads' sums of every channel of the tile and hands them to the first of each.
template <int V>
__device__ __forceinline__ bool join_rows(const Place<V>& at, float (&s)[V], float (&q)[V]) {
    __shared__ float sums[NT * V * 2];
    float* mine = sums + threadIdx.x * (2 * V);
    if (at.on)
#pragma unroll
        for (int i = 0; i < V; ++i) { mine[i] = s[i]; mine[V + i] = q[i]; }
    __syncthreads();
    if (at.r != 0) return false;
    for (int r = 1; r < at.R; ++r) {
        const float* o = sums + (threadIdx.x + r * at.tile) * (2 * V);
#pragma unroll
        for (int i = 0; i < V; ++i) { s[i] += o[i]; q[i] += o[V + i]; }
    }
    return true;
}

template <typename T, int V>
__global__ __launch_bounds__(NT) void norm_sums_kernel(const NormParams p) {
    const Place<V> at(p);
    const int n = at.n, s0 = at.s0, s1 = at.s1;
    const T* x = (const T*)p.x + n * p.x_ns + at.c;
    float k[V], s[V], q[V];
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = q[i] = k[i] = 0.0f;
    if (at.on) {
        load_v<T, V>(x, k);
        for (int t = s0 + at.r; t < s1; t += at.R) {
            float v[V];
            load_v<T, V>(x + (int64_t)t * p.C, v);
#pragma unroll
            for (int i = 0; i < V; ++i) { const float d = v[i] - k[i]; s[i] += d; q[i] += d * d; }
        }
    }
    if (!join_rows<V>(at, s, q)) return;
    float2* o = p.part + ((int64_t)n * p.slices + at.slice) * p.C + at.c;
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = make_float2(s[i], q[i]);
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// One wavefront per group: channels' means and squares about them, then the group's.
template <typename T>
__global__ __launch_bounds__(64) void norm_stats_kernel(const NormParams p) {
    const int n = blockIdx.x / p.G, g = blockIdx.x - n * p.G, lane = threadIdx.x;
    const T* x = (const T*)p.x + n * p.x_ns;
    const float2* part = p.part + (int64_t)n * p.slices * p.C;
    auto channel = [&](int c, float& mean, float& m2) {
        float s = 0.0f, q = 0.0f;
        for (int k = 0; k < p.slices; ++k) { const float2 o = part[(int64_t)k * p.C + c]; s += o.x; q += o.y; }
        float v[1];
        load_v<T, 1>(x + c, v);
        mean = v[0] + s / (float)p.S;
        m2 = fmaxf(q - s * (s / (float)p.S), 0.0f) + 0.0f * q;      // (not below zero; infinities stay NaN)
    };
    float sum = 0.0f, mean, m2;
    for (int c = g * p.per + lane; c < (g + 1) * p.per; c += 64) { channel(c, mean, m2); sum += mean; }
    const float mu = wave_sum(sum) / (float)p.per;
    float var = 0.0f;
    for (int c = g * p.per + lane; c < (g + 1) * p.per; c += 64) {
        channel(c, mean, m2);
        var += m2 / (float)p.S + (mean - mu) * (mean - mu);
    }
    var = wave_sum(var) / (float)p.per;
    if (lane) return;
    const float rstd = 1.0f / sqrtf(var + p.eps);
    p.stat[n * p.G + g] = make_float2(mu, rstd);
    if (p.mean_out) { p.mean_out[n * p.G + g] = mu; p.rstd_out[n * p.G + g] = rstd; }
}

// The affine parameters and the group statistics of a thread's channels.
template <int V>
struct Affine {
    float mu[V], rstd[V], scale[V], shift[V];
    __device__ Affine(const NormParams& p, int n, int c, const float2* stat) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int g = n * p.G + (c + i) / p.per;
            if (stat) { const float2 o = stat[g]; mu[i] = o.x; rstd[i] = o.y; }
            else { mu[i] = p.mean[g]; rstd[i] = p.rstd[g]; }
            scale[i] = p.scale ? p.scale[c + i] : 1.0f;
            shift[i] = p.shift ? p.shift[c + i] : 0.0f;
        }
    }
};

template <typename T, int V, int ACT>
__global__ __launch_bounds__(NT) void norm_apply_kernel(const NormParams p) {
    const Place<V> at(p);
    if (!at.on) return;
    const int n = at.n, s0 = at.s0, s1 = at.s1;
    const Affine<V> a(p, n, at.c, p.stat);
    const T* x = (const T*)p.x + n * p.x_ns + at.c;
    T* y = (T*)p.out + n * p.out_ns + at.c;
    for (int t = s0 + at.r; t < s1; t += at.R) {
        float v[V];
        load_v<T, V>(x + (int64_t)t * p.C, v);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = act_of<ACT>((v[i] - a.mu[i]) * a.rstd[i] * a.scale[i] + a.shift[i]);
        store_v<T, V>(y + (int64_t)t * p.C, v);
    }
}

template <typename T, int V, int ACT>
__global__ __launch_bounds__(NT) void norm_grad_sums_kernel(const NormParams p) {
    const Place<V> at(p);
    const int n = at.n, s0 = at.s0, s1 = at.s1;
    float s[V], q[V];
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = q[i] = 0.0f;
    if (at.on) {
        const Affine<V> a(p, n, at.c, nullptr);
        const T* x = (const T*)p.x + n * p.x_ns + at.c;
        const T* dy = (const T*)p.dy + n * p.dy_ns + at.c;
        for (int t = s0 + at.r; t < s1; t += at.R) {
            float v[V], d[V];
            load_v<T, V>(x + (int64_t)t * p.C, v);
            load_v<T, V>(dy + (int64_t)t * p.C, d);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float xhat = (v[i] - a.mu[i]) * a.rstd[i], dz = d[i] * act_slope<ACT>(xhat * a.scale[i] + a.shift[i]);
                s[i] += dz;
                q[i] += dz * xhat;
            }
        }
    }
    if (!join_rows<V>(at, s, q)) return;
    float2* o = p.part + ((int64_t)n * p.slices + at.slice) * p.C + at.c;
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = make_float2(s[i], q[i]);
}

__global__ __launch_bounds__(64) void norm_grad_stats_kernel(const NormParams p) {
    const int n = blockIdx.x / p.G, g = blockIdx.x - n * p.G, lane = threadIdx.x;
    const float2* part = p.part + (int64_t)n * p.slices * p.C;
    float a = 0.0f, b = 0.0f;
    for (int c = g * p.per + lane; c < (g + 1) * p.per; c += 64) {
        float s = 0.0f, q = 0.0f;
        for (int k = 0; k < p.slices; ++k) { const float2 o = part[(int64_t)k * p.C + c]; s += o.x; q += o.y; }
        const float w = p.scale ? p.scale[c] : 1.0f;
        a += s * w;
        b += q * w;
    }
    a = wave_sum(a);
    b = wave_sum(b);
    const float count = (float)p.per * (float)p.S;
    if (lane == 0) p.stat[n * p.G + g] = make_float2(a / count, b / count);
}

// dscale, dshift: a wavefront per 64 channels' worth of sums would leave the chip idle; 256 threads per 16 channels share the
// images and slices, and join in LDS.
__global__ __launch_bounds__(NT) void norm_grad_params_kernel(const NormParams p) {
    __shared__ float2 sums[16][17];
    const int l = threadIdx.x & 15, r = threadIdx.x >> 4, c = blockIdx.x * 16 + l;
    const int64_t rows = (int64_t)p.N * p.slices;
    float s = 0.0f, q = 0.0f;
    if (c < p.C)
        for (int64_t k = r; k < rows; k += 16) { const float2 o = p.part[k * p.C + c]; s += o.x; q += o.y; }
    sums[r][l] = make_float2(s, q);
    __syncthreads();
    if (r || c >= p.C) return;
    for (int k = 1; k < 16; ++k) { s += sums[k][l].x; q += sums[k][l].y; }
    p.dshift[c] = s;
    p.dscale[c] = q;
}

template <typename T, int V, int ACT>
__global__ __launch_bounds__(NT) void norm_grad_apply_kernel(const NormParams p) {
    const Place<V> at(p);
    if (!at.on) return;
    const int n = at.n, s0 = at.s0, s1 = at.s1;
    const Affine<V> a(p, n, at.c, nullptr);
    float ah[V], ahx[V];
#pragma unroll
    for (int i = 0; i < V; ++i) { const float2 o = p.stat[n * p.G + (at.c + i) / p.per]; ah[i] = o.x; ahx[i] = o.y; }
    const T* x = (const T*)p.x + n * p.x_ns + at.c;
    const T* dy = (const T*)p.dy + n * p.dy_ns + at.c;
    T* dx = (T*)p.out + n * p.out_ns + at.c;
    for (int t = s0 + at.r; t < s1; t += at.R) {
        float v[V], d[V], old[V];
        load_v<T, V>(x + (int64_t)t * p.C, v);
        load_v<T, V>(dy + (int64_t)t * p.C, d);
        if (p.accumulate) load_v<T, V>(dx + (int64_t)t * p.C, old);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float xhat = (v[i] - a.mu[i]) * a.rstd[i], h = d[i] * act_slope<ACT>(xhat * a.scale[i] + a.shift[i]) * a.scale[i];
            v[i] = a.rstd[i] * (h - ah[i] - xhat * ahx[i]);
            if (p.accumulate) v[i] += old[i];
        }
        store_v<T, V>(dx + (int64_t)t * p.C, v);
    }
}

// Slices of the positions: some 1024 workgroups, 64 positions each at least.
int slices_of(int64_t N, int64_t S, int64_t C) {
    int64_t want = 1024 / (N < 1024 ? N : 1024), most = (S + 63) / 64;
    want = want < most ? want : most;
    return (int)(want < 1 ? 1 : want);
}

// Channels per thread: a divisor of C that keeps loads of 16 bytes or less aligned in every row.
int vector_of(int64_t C, int dtype) {
    for (int v = dtype == PURINE_BF16 ? 8 : 4; v > 1; v >>= 1)
        if (C % v == 0) return v;
    return 1;
}

template <typename F>
hipError_t by_act(int act, F&& f) {
    switch (act) {
        case PURINE_ACT_NONE: return f(std::integral_constant<int, PURINE_ACT_NONE>());
        case PURINE_ACT_RELU: return f(std::integral_constant<int, PURINE_ACT_RELU>());
        case PURINE_ACT_SILU: return f(std::integral_constant<int, PURINE_ACT_SILU>());
        case PURINE_ACT_GELU: return f(std::integral_constant<int, PURINE_ACT_GELU>());
        case PURINE_ACT_GELU_TANH: return f(std::integral_constant<int, PURINE_ACT_GELU_TANH>());
        default: return hipErrorInvalidValue;
    }
}
template <typename F>
hipError_t by_vector(int dtype, int v, F&& f) {
    if (dtype == PURINE_BF16) {
        switch (v) {
            case 8: return f(uint16_t(), std::integral_constant<int, 8>());
            case 4: return f(uint16_t(), std::integral_constant<int, 4>());
            case 2: return f(uint16_t(), std::integral_constant<int, 2>());
            default: return f(uint16_t(), std::integral_constant<int, 1>());
        }
    }
    switch (v) {
        case 4: return f(float(), std::integral_constant<int, 4>());
        case 2: return f(float(), std::integral_constant<int, 2>());
        default: return f(float(), std::integral_constant<int, 1>());
    }
}

NormParams params_of(const NormShape& s, void* ws) {
    NormParams p{};
    p.N = s.N; p.S = s.S; p.C = s.C; p.G = s.G; p.per = s.C / s.G;
    p.eps = s.eps;
    p.x_ns = s.x_ns; p.dy_ns = s.dy_ns;
    p.slices = slices_of(s.N, s.S, s.C);
    p.rows = (s.S + p.slices - 1) / p.slices;
    p.slices = (s.S + p.rows - 1) / p.rows;
    p.stat = (float2*)ws;
    p.part = p.stat + (size_t)s.N * s.G;
    return p;
}

// Workgroups of the kernels that walk over positions (fewer than elements / 64, so fewer than 2^31).
unsigned grid_of(NormParams& p, int v) {
    p.tiles = (p.C / v + NT - 1) / NT;
    return (unsigned)((int64_t)p.N * p.slices * p.tiles);
}

}  // namespace

size_t group_norm_ws_bytes(bool, int64_t N, int64_t S, int64_t C, int64_t G, int) {
    const int64_t slices = slices_of(N, S, C);
    return (size_t)(N * G + N * slices * C) * sizeof(float2);
}

hipError_t launch_group_norm_fwd(int dtype, const NormShape& s, const void* x, const float* scale, const float* shift, void* y, float* mean,
                                 float* rstd, void* ws, hipStream_t st) {
    NormParams p = params_of(s, ws);
    p.x = x; p.scale = scale; p.shift = shift; p.out = y; p.out_ns = s.y_ns;
    p.mean_out = mean; p.rstd_out = rstd;
    const int v = vector_of(s.C, dtype);
    const unsigned grid = grid_of(p, v);
    (void)hipGetLastError();
    return by_vector(dtype, v, [&](auto t, auto V) {
        typedef decltype(t) T;
        hipLaunchKernelGGL((norm_sums_kernel<T, V.value>), dim3(grid), dim3(NT), 0, st, p);
        hipLaunchKernelGGL((norm_stats_kernel<T>), dim3(p.N * p.G), dim3(64), 0, st, p);
        return by_act(s.act, [&](auto A) {
            ProbeScope probe(st);
            hipLaunchKernelGGL((norm_apply_kernel<T, V.value, A.value>), dim3(grid), dim3(NT), 0, st, p);
            return hipGetLastError();
        });
    });
}

hipError_t launch_group_norm_bwd(int dtype, const NormShape& s, const void* x, const float* scale, const float* shift, const float* mean,
                                 const float* rstd, const void* dy, void* dx, float* dscale, float* dshift, float beta, void* ws, hipStream_t st) {
    NormParams p = params_of(s, ws);
    p.x = x; p.scale = scale; p.shift = shift; p.mean = mean; p.rstd = rstd; p.dy = dy;
    p.out = dx; p.out_ns = s.dx_ns; p.dscale = dscale; p.dshift = dshift;
    p.accumulate = beta != 0.0f;
    const int v = vector_of(s.C, dtype);
    const unsigned grid = grid_of(p, v);
    (void)hipGetLastError();
    return by_vector(dtype, v, [&](auto t, auto V) {
        typedef decltype(t) T;
        return by_act(s.act, [&](auto A) {
            hipLaunchKernelGGL((norm_grad_sums_kernel<T, V.value, A.value>), dim3(grid), dim3(NT), 0, st, p);
            hipLaunchKernelGGL(norm_grad_stats_kernel, dim3(p.N * p.G), dim3(64), 0, st, p);
            if (dscale) hipLaunchKernelGGL(norm_grad_params_kernel, dim3((p.C + 15) / 16), dim3(NT), 0, st, p);
            ProbeScope probe(st);
            hipLaunchKernelGGL((norm_grad_apply_kernel<T, V.value, A.value>), dim3(grid), dim3(NT), 0, st, p);
            return hipGetLastError();
        });
    });
}

}  // namespace purine
