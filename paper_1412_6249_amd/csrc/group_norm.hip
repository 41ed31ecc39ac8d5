// Group normalization with an activation on channels-last tensors, and its gradient (purine_group_norm_fwd / _bwd).
//
//     xhat = (x - mean) rstd,  z = xhat scale[c] + shift[c],  y = act(z)            mean, var: over a group's channels and all positions
//     dz = dy act'(z),  h = dz scale,  dx = rstd (h - avg(h) - xhat avg(h xhat)),  dshift = sum dz,  dscale = sum dz xhat
//
// A thread owns V neighbouring channels (16 bytes where the row allows it) and walks down the positions, so that loads are whole pieces of
// rows and the affine parameters stay in registers. Sums are kept per channel, which serves any number of channels per group. For the statistics they are
// means and sums of squares about these means: of a few positions of a thread about one of them, then of more and more of them by
//     n = a + b,  mean = (a mean_a + b mean_b) / n,  M = M_a + a (mean_a - mean)^2 + M_b + b (mean_b - mean)^2,
// so that no difference of large sums is taken, whatever values come first (means are kept relative to the channel's value k at the image's first position:
// of a large common mean no digits are lost). For the gradient they are sum dz and sum dz xhat. Everything is joined in a fixed order.
//
// Bound: HBM, and with an activation the vector units nearly as much (about 30 instructions a gradient element). us, bf16: 128 x 784 x 192 in 32 groups, SiLU, held:
// forward 21 (77 MB; 15 at the rate of a copy), gradient 34 (115 MB; 23); 64 x 12544 x 64 in 32 groups, GELU by tanh, sliced: sums 21 and result 38 (103 and 206 MB;
// 20 and 40), gradient sums 45 and result 57 (206 and 308 MB; 40 and 60).
//
// Where an image's share of a few whole groups fits a workgroup's registers (norm_held_kernel, norm_grad_held_kernel), one workgroup reads it once and
// writes the results: every tensor moves once. Otherwise (norm_sums / norm_apply) one kernel sums over slices of the positions and a second
// one joins the slices for itself, or finds them joined by norm_join, and reads its tensors again, if they are not too large from the last-level cache.
#include "activation.h"
#include "bf16.h"
#include "block.h"

namespace purine {
namespace {

constexpr int NT = 256;

template <typename T, int V> struct alignas(sizeof(T) * V) Pack { T e[V]; };
template <typename T, int V>
__device__ __forceinline__ void widen_v(const Pack<T, V>& k, float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if constexpr (sizeof(T) == 2) v[i] = bf2f(k.e[i]);
        else v[i] = k.e[i];
    }
}
template <typename T, int V>
__device__ __forceinline__ void load_v(const T* p, float (&v)[V]) { widen_v<T, V>(*reinterpret_cast<const Pack<T, V>*>(p), v); }
template <typename T, int V>
__device__ __forceinline__ void store_v(T* p, const float (&v)[V]) {
    if constexpr (sizeof(T) == 2 && V > 1) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        typedef float floatx2 __attribute__((ext_vector_type(2)));
        Pack<uint32_t, V / 2> k;
#pragma unroll
        for (int i = 0; i < V / 2; ++i) { const floatx2 f = {v[2 * i], v[2 * i + 1]}; k.e[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2)); }
        *reinterpret_cast<Pack<uint32_t, V / 2>*>(p) = k;
    } else {
        Pack<T, V> k;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if constexpr (sizeof(T) == 2) k.e[i] = f2bf(v[i]);
            else k.e[i] = v[i];
        }
        *reinterpret_cast<Pack<T, V>*>(p) = k;
    }
}

// Makes the compiler forget what it computed from the pieces: it would keep the numbers of one pass over them for the next, in four times the
// registers.
template <typename T, int V, int N>
__device__ __forceinline__ void forget(Pack<T, V> (&k)[N]) {
    if constexpr (sizeof(T) * V >= 4) {
#pragma unroll
        for (int u = 0; u < N; ++u) {
            uint32_t w[sizeof(T) * V / 4];
            __builtin_memcpy(w, &k[u], sizeof(w));
#pragma unroll
            for (unsigned i = 0; i < sizeof(w) / 4; ++i) asm volatile("" : "+v"(w[i]));
            __builtin_memcpy(&k[u], w, sizeof(w));
        }
    }
}

struct NormParams {
    const void* x; const void* dy; void* out;
    int64_t x_ns, dy_ns, out_ns;
    const float* scale; const float* shift;     // or null
    float2* part;              // per image, slice and channel: mean and sum of squares about it, or the gradient's two sums
    float* about;              // per image and channel: the value that the means are relative to
    float2* stat;              // per image and group: mean and rstd, or the gradient's averages, where a kernel of their own joins them; else null
    float4* chunk;             // of that kernel: what its workgroups make of their part of a group
    const float* mean; const float* rstd;       // gradient: as saved
    float* mean_out; float* rstd_out;           // or null
    float* dscale; float* dshift;               // or null
    int N, S, C, G, per;       // channels per group
    int slices, rows;          // slices of the positions, positions per slice
    int chunks;                // workgroups that join a group's sums
    int tiles;                 // of NT vectors of channels
    int width;                 // held kernels: channels of a workgroup
    float eps;
    int accumulate;
};

// f(group, lane, lanes, sum over the lanes): a few lanes (a power of two) for each of the groups first .. first + count - 1; all threads of
// the workgroup (THREADS) take part.
template <int THREADS, typename F>
__device__ __forceinline__ void for_groups(int count, int per, F&& f) {
    int lanes = 1;
    while (lanes < 64 && lanes < per) lanes *= 2;
    auto sum = [lanes](float v) {
        for (int d = lanes >> 1; d; d >>= 1) v += __shfl_xor(v, d);
        return v;
    };
    for (int g = threadIdx.x / lanes; g < count; g += THREADS / lanes) f(g, (int)threadIdx.x & (lanes - 1), lanes, sum);
}

// Joins the means of `width` channels, and the sums of squares about them, over R rows of threads: sums[r * width + c] is of the positions r, r + R, ... of
// `total`. All threads take part; the result is in the first row. Sixteen rows at a time, so that a few rounds do and the loads of a round wait together;
// about the first one's mean, which loses sixteen times the last place at most, whatever it is.
template <int THREADS>
__device__ __forceinline__ void join_moments(float2* sums, int width, int R, int total) {
    constexpr int STEP = 16, AT_ONCE = 8;                           // (all sixteen at once would take the registers of a wavefront)
    const int columns = min(width, THREADS), lanes = THREADS / columns, c0 = threadIdx.x % columns, l = threadIdx.x / columns;
    R = min(R, total);                                              // (no positions in rows past that)
    const int base = total / R;                                     // positions of a row: base, or one more in the first `more`
    const float each = (float)base, more = (float)(total - base * R), most = (float)R;
    __syncthreads();
    for (int rows = R, span = 1; rows > 1; rows = (rows + STEP - 1) / STEP, span *= STEP) {
        const int next = (rows + STEP - 1) / STEP;
        const float wide = (float)span;
        for (int c1 = 0; c1 < width; c1 += columns)
            for (int j1 = 0; j1 < next; j1 += lanes) {
                const int c = c1 + c0, j = j1 + l, first = j * STEP, end = min(first + STEP, rows);
                const bool mine = c < width && j < next && l < lanes;
                float2 o = make_float2(0.0f, 0.0f);
                if (mine) {
                    const float about = sums[first * width + c].x;
                    float a = 0.0f, b = 0.0f, n = 0.0f, row = (float)first * wide;
#pragma unroll 1
                    for (int u0 = first; u0 < end; u0 += AT_ONCE) {
                        float2 v[AT_ONCE];
#pragma unroll
                        for (int u = 0; u < AT_ONCE; ++u) v[u] = sums[min(u0 + u, rows - 1) * width + c];
#pragma unroll
                        for (int u = 0; u < AT_ONCE; ++u, row += wide) {
                            const float w = fmaxf(each * fminf(wide, most - row) + __builtin_amdgcn_fmed3f(more - row, 0.0f, wide), 0.0f), d = v[u].x - about;
                            n += w;
                            a += w * d;
                            b += w * (d * d) + (u0 + u < rows ? v[u].y : 0.0f);
                        }
                    }
                    const float d = a * __builtin_amdgcn_rcpf(fmaxf(n, 1.0f));
                    o = make_float2(about + d, b - a * d);
                }
                __syncthreads();                   // (rows that others read: what is written lies before what is still to be read)
                if (mine) sums[j * width + c] = o;
            }
        __syncthreads();
    }
}

// Mean and rstd of a group: mean(c) gives its c-th channel's mean, squares(c, mu) that channel's sum of squares about mu.
template <typename Sum, typename Mean, typename Squares>
__device__ __forceinline__ float2 group_stats(const NormParams& p, int lane, int lanes, Sum&& sum, Mean&& mean, Squares&& squares) {
    float all = 0.0f, var = 0.0f;
    for (unsigned c = lane; c < (unsigned)p.per; c += lanes) all += mean(c);
    const float mu = sum(all) / (float)p.per;
    for (unsigned c = lane; c < (unsigned)p.per; c += lanes) var += squares(c, mu) / (float)p.S;
    var = sum(var) / (float)p.per;
    return make_float2(mu, 1.0f / sqrtf(var + p.eps));
}

// What a workgroup of the kernels over slices works on (image, slice of the positions, tile of the channels), the channels of this thread, its
// place among the threads that share them, and their number. Positions count from the slice's first, so that the sums of them below stay far from 2^31.
template <int V>
struct Place {
    int n, slice, len, c, r, R, tile, c0, c1;           // len: positions; c0 .. c1 - 1: the tile's channels
    int64_t at;                                         // elements from the image's first to the slice's first of these channels
    bool on;
    __device__ __forceinline__ explicit Place(const NormParams& p) {
        const int b = blockIdx.x / p.tiles, cv = p.C / V, first = (int)(blockIdx.x - b * p.tiles) * NT;
        n = b / p.slices;
        slice = b - n * p.slices;
        const int s0 = slice * p.rows;
        len = min(p.rows, p.S - s0);
        tile = min(NT, cv - first);
        R = NT / tile;
        r = threadIdx.x / tile;
        on = r < R;
        c = (first + (int)threadIdx.x % tile) * V;
        c0 = first * V;
        c1 = c0 + tile * V;
        at = (int64_t)s0 * p.C + c;
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

constexpr int AHEAD = 4;                       // positions that a thread loads before it uses the first

template <typename T, int V>
__global__ __launch_bounds__(NT) void norm_sums_kernel(const NormParams p) {
    __shared__ float2 sums[NT * V];
    const Place<V> at(p);
    const T* x = (const T*)p.x + at.n * p.x_ns + at.at;
    float k[V], mean[V], m2[V];
#pragma unroll
    for (int i = 0; i < V; ++i) mean[i] = m2[i] = k[i] = 0.0f;
    if (at.on) {
        load_v<T, V>((const T*)p.x + at.n * p.x_ns + at.c, k);
        Pack<T, V> in[AHEAD], next[AHEAD];
        auto load = [&](int t) {
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) next[u] = *reinterpret_cast<const Pack<T, V>*>(x + (int64_t)min(t + u * at.R, at.len - 1) * p.C);
        };
        float before = 0.0f;
        load(at.r);
        for (int t = at.r; t < at.len; t += AHEAD * at.R) {
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) in[u] = next[u];
            load(t + AHEAD * at.R);
            float first[V], s[V], q[V], count = 1.0f;
            widen_v<T, V>(in[0], first);
#pragma unroll
            for (int i = 0; i < V; ++i) s[i] = q[i] = 0.0f;
#pragma unroll
            for (int u = 1; u < AHEAD; ++u) {
                if (t + u * at.R >= at.len) break;
                float v[V];
                widen_v<T, V>(in[u], v);
#pragma unroll
                for (int i = 0; i < V; ++i) { const float d = v[i] - first[i]; s[i] += d; q[i] += d * d; }
                count += 1.0f;
            }
            const float inv = __builtin_amdgcn_rcpf(count), share = count * __builtin_amdgcn_rcpf(before + count), cross = before * share;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = s[i] * inv, off = (first[i] - k[i]) + d - mean[i];
                mean[i] += off * share;
                m2[i] += (q[i] - s[i] * d) + cross * (off * off);
            }
            before += count;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) sums[threadIdx.x * V + i] = make_float2(mean[i], m2[i]);
    }
    join_moments<NT>(sums, at.tile * V, at.R, at.len);
    if (at.r != 0) return;
    float2* o = p.part + ((int64_t)at.n * p.slices + at.slice) * p.C + at.c;
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = sums[threadIdx.x * V + i];
    if (at.slice == 0)
#pragma unroll
        for (int i = 0; i < V; ++i) p.about[(int64_t)at.n * p.C + at.c + i] = k[i];
}

// f(0) + ... + f(n - 1) as eight sums: a thousand terms one after the other would lose ten times the last place.
template <typename F>
__device__ __forceinline__ float sum_of(int n, F&& f) {
    float s[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) s[u] = 0.0f;
    int k = 0;
    for (; k + 8 <= n; k += 8)
#pragma unroll
        for (int u = 0; u < 8; ++u) s[u] += f(k + u);
    if (k < n) {
        float v[7];
#pragma unroll
        for (int u = 0; u < 7; ++u) v[u] = f(min(k + u, n - 1));
#pragma unroll
        for (int u = 0; u < 7; ++u) s[u] += k + u < n ? v[u] : 0.0f;
    }
    return ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
}
// The sums of a channel over the slices, in order.
__device__ __forceinline__ float2 over_slices(const NormParams& p, int n, int c) {
    const float2* part = p.part + (int64_t)n * p.slices * p.C + c;
    float s = 0.0f, q = 0.0f;
#pragma unroll 8
    for (int k = 0; k < p.slices; ++k) { const float2 o = part[(int64_t)k * p.C]; s += o.x; q += o.y; }
    return make_float2(s, q);
}

// A channel's affine parameters.
__device__ __forceinline__ float scale_of(const NormParams& p, int c) { return p.scale ? p.scale[c] : 1.0f; }
__device__ __forceinline__ float shift_of(const NormParams& p, int c) { return p.shift ? p.shift[c] : 0.0f; }

// (y may be x: a workgroup reads no element of x but those that it replaces, the values that the sums are about come from the scratch)
template <typename T, int V, int ACT>
__global__ __launch_bounds__(NT) void norm_apply_kernel(const NormParams p) {
    __shared__ float2 stat[NT * V + 1];
    const Place<V> at(p);
    const int g0 = at.c0 / p.per, g1 = (at.c1 - 1) / p.per;
    if (p.stat) for (int g = threadIdx.x; g <= g1 - g0; g += NT) stat[g] = p.stat[at.n * p.G + g0 + g];
    else for_groups<NT>(g1 - g0 + 1, p.per, [&](int g, int lane, int lanes, auto&& sum) {
        const int first = (g0 + g) * p.per;
        const float* about = p.about + (int64_t)at.n * p.C + first;
        const float2* part = p.part + (int64_t)at.n * p.slices * p.C + first;
        const int last = p.slices - 1;
        const float n = (float)p.rows, n_last = (float)(p.S - last * p.rows);
        const float2 o = group_stats(
            p, lane, lanes, sum,
            [&](int c) {
                const float s = sum_of(last, [&](int s) { return part[(int64_t)s * p.C + c].x; });
                return about[c] + (n * s + n_last * part[(int64_t)last * p.C + c].x) / (float)p.S;
            },
            [&](int c, float mu) {
                const float k = about[c] - mu;
                auto squares = [k](float2 o, float n) { return o.y + n * ((k + o.x) * (k + o.x)); };
                return sum_of(last, [&](int s) { return squares(part[(int64_t)s * p.C + c], n); }) + squares(part[(int64_t)last * p.C + c], n_last);
            });
        if (lane == 0) {
            stat[g] = o;
            if (at.slice == 0 && p.mean_out) { p.mean_out[at.n * p.G + g0 + g] = o.x; p.rstd_out[at.n * p.G + g0 + g] = o.y; }
        }
    });
    __syncthreads();
    if (!at.on) return;
    float mu[V], a[V], b[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float2 o = stat[(at.c + i) / p.per - g0];
        mu[i] = o.x; a[i] = o.y * scale_of(p, at.c + i); b[i] = shift_of(p, at.c + i);
    }
    const T* x = (const T*)p.x + at.n * p.x_ns + at.at;
    T* y = (T*)p.out + at.n * p.out_ns + at.at;
    for (int t = at.r; t < at.len; t += AHEAD * at.R) {
        Pack<T, V> in[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) in[u] = *reinterpret_cast<const Pack<T, V>*>(x + (int64_t)min(t + u * at.R, at.len - 1) * p.C);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (t + u * at.R >= at.len) break;
            float v[V];
            widen_v<T, V>(in[u], v);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = act_of<ACT, sizeof(T) == 4>((v[i] - mu[i]) * a[i] + b[i]);
            store_v<T, V>(y + (int64_t)(t + u * at.R) * p.C, v);
        }
    }
}

// x's place in its distribution and the gradient before the activation, of one element.
template <int ACT, bool FULL>
__device__ __forceinline__ void grad_of(float x, float dy, float mu, float rstd, float scale, float shift, float& xhat, float& dz) {
    xhat = (x - mu) * rstd;
    dz = dy * act_slope<ACT, FULL>(xhat * scale + shift);
}

template <typename T, int V, int ACT>
__global__ __launch_bounds__(NT, 4) void norm_grad_sums_kernel(const NormParams p) {
    constexpr int BATCH = V == 8 && ACT == PURINE_ACT_GELU ? 3 : AHEAD;        // (of what 128 registers hold)
    const Place<V> at(p);
    float s[V], q[V];
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = q[i] = 0.0f;
    if (at.on) {
        float mu[V], rstd[V], sc[V], sh[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int g = at.n * p.G + (at.c + i) / p.per;
            mu[i] = p.mean[g]; rstd[i] = p.rstd[g]; sc[i] = scale_of(p, at.c + i); sh[i] = shift_of(p, at.c + i);
        }
        const T* x = (const T*)p.x + at.n * p.x_ns + at.at;
        const T* dy = (const T*)p.dy + at.n * p.dy_ns + at.at;
        // (a batch of positions ahead of its use: 64 x 12544 x 64 in bf16 43.8 us, without 53.6; its 206 MB at the rate of a copy 40)
        Pack<T, V> in[BATCH], gr[BATCH], in_next[BATCH], gr_next[BATCH];
        auto load = [&](int t) {
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                const int64_t row = (int64_t)min(t + u * at.R, at.len - 1) * p.C;
                in_next[u] = *reinterpret_cast<const Pack<T, V>*>(x + row);
                gr_next[u] = *reinterpret_cast<const Pack<T, V>*>(dy + row);
            }
        };
        load(at.r);
        for (int t = at.r; t < at.len; t += BATCH * at.R) {
#pragma unroll
            for (int u = 0; u < BATCH; ++u) { in[u] = in_next[u]; gr[u] = gr_next[u]; }
            load(t + BATCH * at.R);
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                if (t + u * at.R >= at.len) break;
                float v[V], d[V];
                widen_v<T, V>(in[u], v);
                widen_v<T, V>(gr[u], d);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float xhat, dz;
                    grad_of<ACT, sizeof(T) == 4>(v[i], d[i], mu[i], rstd[i], sc[i], sh[i], xhat, dz);
                    s[i] += dz;
                    q[i] += dz * xhat;
                }
            }
        }
    }
    if (!join_rows<V>(at, s, q)) return;
    float2* o = p.part + ((int64_t)at.n * p.slices + at.slice) * p.C + at.c;
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = make_float2(s[i], q[i]);
}

// avg(h), avg(h xhat) of a group from its channels' sums.
template <typename Sum, typename Channel>
__device__ __forceinline__ float2 group_averages(const NormParams& p, int lane, int lanes, Sum&& sum, Channel&& channel) {
    float a = 0.0f, b = 0.0f;
    for (unsigned c = lane; c < (unsigned)p.per; c += lanes) {
        float w;
        const float2 o = channel(c, w);
        a += o.x * w;
        b += o.y * w;
    }
    const float count = (float)p.per * (float)p.S;
    return make_float2(sum(a) / count, sum(b) / count);
}

// dscale and dshift of 16 channels: 16 threads each share the images and slices, and join in LDS. They lie `stride` rows apart, `count` of them. Where there
// are many, workgroups take PER of them each and leave their sums in the first (nobody else reads it), for a next launch.
constexpr int PER = 1024;
template <bool LAST>
__global__ __launch_bounds__(NT) void norm_grad_params_kernel(const NormParams p, int from, int blocks, int64_t stride, int64_t count) {
    __shared__ float2 sums[16][17];
    const int piece = LAST ? 0 : (int)(blockIdx.x / blocks), l = threadIdx.x & 15, r = threadIdx.x >> 4;
    const unsigned c = (unsigned)from + (blockIdx.x - (unsigned)piece * blocks) * 16 + l;
    const int64_t first = (int64_t)piece * PER, end = LAST || count - first < PER ? count : first + PER;
    float s = 0.0f, q = 0.0f;
    if (c < (unsigned)p.C)
#pragma unroll 8
        for (int64_t k = first + r; k < end; k += 16) { const float2 o = p.part[k * stride * p.C + c]; s += o.x; q += o.y; }
    sums[r][l] = make_float2(s, q);
    __syncthreads();
    if (r || c >= (unsigned)p.C) return;
    for (int k = 1; k < 16; ++k) { s += sums[k][l].x; q += sums[k][l].y; }
    if (LAST) { p.dshift[c] = s; p.dscale[c] = q; }
    else p.part[first * stride * p.C + c] = make_float2(s, q);
}

template <typename T, int V, int ACT>
__global__ __launch_bounds__(NT) void norm_grad_apply_kernel(const NormParams p) {
    __shared__ float2 stat[NT * V + 1];
    const Place<V> at(p);
    const int g0 = at.c0 / p.per, g1 = (at.c1 - 1) / p.per;
    if (p.stat) for (int g = threadIdx.x; g <= g1 - g0; g += NT) stat[g] = p.stat[at.n * p.G + g0 + g];
    else for_groups<NT>(g1 - g0 + 1, p.per, [&](int g, int lane, int lanes, auto&& sum) {
        const int first = (g0 + g) * p.per;
        const float2 o = group_averages(p, lane, lanes, sum, [&](int c, float& w) { w = scale_of(p, first + c); return over_slices(p, at.n, first + c); });
        if (lane == 0) stat[g] = o;
    });
    __syncthreads();
    if (!at.on) return;
    float mu[V], rstd[V], sc[V], sh[V], c1[V], c2[V], rs[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int gi = (at.c + i) / p.per, g = at.n * p.G + gi;
        const float2 o = stat[gi - g0];
        mu[i] = p.mean[g]; rstd[i] = p.rstd[g]; sc[i] = scale_of(p, at.c + i); sh[i] = shift_of(p, at.c + i);
        c1[i] = rstd[i] * o.x; c2[i] = rstd[i] * o.y; rs[i] = rstd[i] * sc[i];
    }
    const T* x = (const T*)p.x + at.n * p.x_ns + at.at;
    const T* dy = (const T*)p.dy + at.n * p.dy_ns + at.at;
    T* dx = (T*)p.out + at.n * p.out_ns + at.at;
    for (int t = at.r; t < at.len; t += AHEAD * at.R) {
        Pack<T, V> in[AHEAD], gr[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int64_t row = (int64_t)min(t + u * at.R, at.len - 1) * p.C;
            in[u] = *reinterpret_cast<const Pack<T, V>*>(x + row);
            gr[u] = *reinterpret_cast<const Pack<T, V>*>(dy + row);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (t + u * at.R >= at.len) break;
            T* o = dx + (int64_t)(t + u * at.R) * p.C;
            float v[V], d[V], old[V];
            widen_v<T, V>(in[u], v);
            widen_v<T, V>(gr[u], d);
            if (p.accumulate) load_v<T, V>(o, old);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float xhat, dz;
                grad_of<ACT, sizeof(T) == 4>(v[i], d[i], mu[i], rstd[i], sc[i], sh[i], xhat, dz);
                v[i] = dz * rs[i] - (xhat * c2[i] + c1[i]);
                if (p.accumulate) v[i] += old[i];
            }
            store_v<T, V>(o, v);
        }
    }
}

// ---- the sums of long groups, joined once
constexpr int CHUNK = NT * 64;                 // pairs of sums of a workgroup at most

// The sum over the workgroup's threads, in a fixed order, in every thread.
__device__ __forceinline__ float sum_over_block(float v, float* sums) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = v;
    __syncthreads();
    v = sums[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) v += sums[w];
    return v;
}
// Number, mean and sum of squares about it of `count` members: member(i, n, mean about the first member's, squares).
template <typename Member>
__device__ __forceinline__ float3 join_members(unsigned count, float* sums, Member&& member) {
    float n, m, q, all = 0.0f, s = 0.0f;
#pragma unroll 8
    for (unsigned i = threadIdx.x; i < count; i += NT) { member(i, n, m, q); all += n; s += n * m; }
    all = sum_over_block(all, sums);
    const float mean = sum_over_block(s, sums) / all;
    s = 0.0f;
#pragma unroll 8
    for (unsigned i = threadIdx.x; i < count; i += NT) { member(i, n, m, q); s += q + n * ((m - mean) * (m - mean)); }
    return make_float3(all, mean, sum_over_block(s, sums));
}
__device__ __forceinline__ void put_stats(const NormParams& p, unsigned group, float mean, float var) {
    if (threadIdx.x) return;
    const float2 o = make_float2(mean, 1.0f / sqrtf(var + p.eps));
    p.stat[group] = o;
    if (p.mean_out) { p.mean_out[group] = o.x; p.rstd_out[group] = o.y; }
}
// A workgroup per CHUNK of a group's slices x channels, whose results are those of the group if there is one.
template <bool GRAD>
__global__ __launch_bounds__(NT) void norm_join_kernel(const NormParams p) {
    __shared__ float sums[NT / 64];
    const unsigned group = blockIdx.x / p.chunks, first = (blockIdx.x - group * p.chunks) * CHUNK, per = p.per;
    const unsigned n = group / p.G, c0 = (group - n * p.G) * per, count = min((unsigned)CHUNK, p.slices * per - first);
    const float2* part = p.part + (int64_t)n * p.slices * p.C + c0;
    auto place = [=](unsigned i, unsigned& slice, unsigned& c) { slice = (first + i) / per; c = first + i - slice * per; };
    if constexpr (GRAD) {
        float a = 0.0f, b = 0.0f;
#pragma unroll 8
        for (unsigned i = threadIdx.x; i < count; i += NT) {
            unsigned s, c;
            place(i, s, c);
            const float2 o = part[(int64_t)s * p.C + c];
            const float w = scale_of(p, (int)(c0 + c));
            a += o.x * w;
            b += o.y * w;
        }
        a = sum_over_block(a, sums);
        b = sum_over_block(b, sums);
        const float all = (float)per * (float)p.S;
        if (threadIdx.x) return;
        if (p.chunks == 1) p.stat[group] = make_float2(a / all, b / all);
        else p.chunk[blockIdx.x] = make_float4(a, b, 0.0f, 0.0f);
    } else {
        const float* about = p.about + (int64_t)n * p.C + c0;
        unsigned s, c;
        place(0, s, c);
        const float zero = about[c] + part[(int64_t)s * p.C + c].x, rows = (float)p.rows, rest = (float)(p.S - (p.slices - 1) * p.rows);
        const float3 o = join_members(count, sums, [&](unsigned i, float& k, float& m, float& q) {
            unsigned s, c;
            place(i, s, c);
            const float2 v = part[(int64_t)s * p.C + c];
            k = (int)s == p.slices - 1 ? rest : rows;
            m = (about[c] - zero) + v.x;
            q = v.y;
        });
        if (p.chunks == 1) put_stats(p, group, zero + o.y, o.z / o.x);
        else if (threadIdx.x == 0) p.chunk[blockIdx.x] = make_float4(o.x, zero + o.y, o.z, 0.0f);
    }
}
// The same of a group's chunks.
template <bool GRAD>
__global__ __launch_bounds__(NT) void norm_join_chunks_kernel(const NormParams p) {
    __shared__ float sums[NT / 64];
    const float4* chunk = p.chunk + (int64_t)blockIdx.x * p.chunks;
    if constexpr (GRAD) {
        float a = 0.0f, b = 0.0f;
        for (int i = threadIdx.x; i < p.chunks; i += NT) { a += chunk[i].x; b += chunk[i].y; }
        a = sum_over_block(a, sums);
        b = sum_over_block(b, sums);
        const float all = (float)p.per * (float)p.S;
        if (threadIdx.x == 0) p.stat[blockIdx.x] = make_float2(a / all, b / all);
    } else {
        const float zero = chunk[0].y;
        const float3 o = join_members(p.chunks, sums, [&](unsigned i, float& n, float& m, float& q) { const float4 v = chunk[i]; n = v.x; m = v.y - zero; q = v.z; });
        put_stats(p, blockIdx.x, zero + o.y, o.z / o.x);
    }
}

// ---- an image's share of a few whole groups, in registers
constexpr int HT = 512, HELD = 16, HELD_GRAD = 10;      // threads; pieces of a thread at most, and of eight bf16 numbers in the gradient (120 registers)

// Consecutive workgroups go to the eight dies in turn; those of one image share lines of memory, so a die takes consecutive ones.
__device__ __forceinline__ int held_block() {
    const int total = gridDim.x, per = total >> 3, b = blockIdx.x;
    return per > 0 && b < per * 8 ? (b & 7) * per + (b >> 3) : b;
}
// Sums of every channel of the workgroup, from each thread's: left in `chan` (width of them).
template <int V, int THREADS>
__device__ __forceinline__ void join_held(const float (&s)[V], const float (&q)[V], float2* sums, float2* chan, int width, int R, bool on) {
    if (on)
#pragma unroll
        for (int i = 0; i < V; ++i) sums[threadIdx.x * V + i] = make_float2(s[i], q[i]);        // [r][channel]
    __syncthreads();
    // width channels over THREADS / width threads each, then over one
    const int lanes = THREADS / width, c = threadIdx.x % width, l = threadIdx.x / width;
    float2 t = make_float2(0.0f, 0.0f);
    if (l < lanes)
        for (int r = l; r < R; r += lanes) { const float2 o = sums[r * width + c]; t.x += o.x; t.y += o.y; }
    __syncthreads();
    if (l < lanes) sums[l * width + c] = t;
    __syncthreads();
    if (threadIdx.x < width) {
        for (int k = 1; k < min(lanes, R); ++k) { const float2 o = sums[k * width + c]; t.x += o.x; t.y += o.y; }
        chan[c] = t;
    }
    __syncthreads();
}

template <typename T, int V, int ACT, int NV, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_held_kernel(const NormParams p) {
    __shared__ float2 sums[THREADS * V], stat[THREADS];
    __shared__ float about[THREADS];           // the channels' values that the means are relative to
    const int b = held_block(), n = b / p.tiles, c0 = (b - n * p.tiles) * p.width, cv = p.width / V, R = THREADS / cv;
    const int r = threadIdx.x / cv, c = c0 + (int)threadIdx.x % cv * V;
    const bool on = r < R;
    const T* x = (const T*)p.x + n * p.x_ns + c;
    Pack<T, V> in[NV];
    float k[V], mean[V], q[V];
#pragma unroll
    for (int i = 0; i < V; ++i) mean[i] = q[i] = k[i] = 0.0f;
    if (on) {
        load_v<T, V>(x, k);
#pragma unroll
        for (int u = 0; u < NV; ++u) in[u] = *reinterpret_cast<const Pack<T, V>*>(x + (int64_t)min(r + u * R, p.S - 1) * p.C);
        float s[V], first[V], count = 1.0f;
        widen_v<T, V>(in[0], first);
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = 0.0f;
#pragma unroll
        for (int u = 1; u < NV; ++u) {
            if (r + u * R >= p.S) break;
            float v[V];
            widen_v<T, V>(in[u], v);
#pragma unroll
            for (int i = 0; i < V; ++i) { const float d = v[i] - first[i]; s[i] += d; q[i] += d * d; }
            count += 1.0f;
        }
        const float inv = __builtin_amdgcn_rcpf(count);
#pragma unroll
        for (int i = 0; i < V; ++i) { const float d = s[i] * inv; mean[i] = (first[i] - k[i]) + d; q[i] -= s[i] * d; }
    }
    if (r == 0)
#pragma unroll
        for (int i = 0; i < V; ++i) about[c - c0 + i] = k[i];
    if (on)
#pragma unroll
        for (int i = 0; i < V; ++i) sums[threadIdx.x * V + i] = make_float2(mean[i], q[i]);
    join_moments<THREADS>(sums, p.width, R, p.S);
    for_groups<THREADS>(p.width / p.per, p.per, [&](int g, int lane, int lanes, auto&& sum) {
        const float2 o = group_stats(
            p, lane, lanes, sum, [&](int i) { return about[g * p.per + i] + sums[g * p.per + i].x; },
            [&](int i, float mu) {
                const float2 w = sums[g * p.per + i];
                const float off = about[g * p.per + i] - mu + w.x;
                return w.y + (float)p.S * (off * off);
            });
        if (lane == 0) {
            stat[g] = o;
            const int at = n * p.G + c0 / p.per + g;
            if (p.mean_out) { p.mean_out[at] = o.x; p.rstd_out[at] = o.y; }
        }
    });
    __syncthreads();
    if (!on) return;
    float mu[V], a[V], sh[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float2 o = stat[(c + i - c0) / p.per];
        mu[i] = o.x; a[i] = o.y * scale_of(p, c + i); sh[i] = shift_of(p, c + i);
    }
    T* y = (T*)p.out + n * p.out_ns + c;
    forget(in);
#pragma unroll
    for (int u = 0; u < NV; ++u) {
        if (r + u * R >= p.S) break;
        float v[V];
        widen_v<T, V>(in[u], v);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = act_of<ACT, sizeof(T) == 4>((v[i] - mu[i]) * a[i] + sh[i]);
        store_v<T, V>(y + (int64_t)(r + u * R) * p.C, v);
    }
}

// (dz stays in fp32 between the passes: with x and dy held and the slope computed again, 128 x 784 x 192 in bf16 took 46 us)
template <typename T, int V, int ACT, int NV, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_grad_held_kernel(const NormParams p) {
    __shared__ float2 sums[THREADS * V], chan[THREADS], stat[THREADS];
    const int b = held_block(), n = b / p.tiles, c0 = (b - n * p.tiles) * p.width, cv = p.width / V, R = THREADS / cv;
    const int r = threadIdx.x / cv, c = c0 + (int)threadIdx.x % cv * V;
    const bool on = r < R;
    const T* x = (const T*)p.x + n * p.x_ns + c;
    const T* dy = (const T*)p.dy + n * p.dy_ns + c;
    Pack<T, V> in[NV];
    float dz[NV][V], mu[V], rstd[V], s[V], q[V];
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = q[i] = mu[i] = rstd[i] = 0.0f;
    if (on) {
        Pack<T, V> gr[NV];
        float sc[V], sh[V];
        // (first: loads arrive in order, and every piece needs these)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int g = n * p.G + (c + i) / p.per;
            mu[i] = p.mean[g]; rstd[i] = p.rstd[g]; sc[i] = scale_of(p, c + i); sh[i] = shift_of(p, c + i);
        }
        asm volatile("" ::: "memory");
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            const int64_t row = (int64_t)min(r + u * R, p.S - 1) * p.C;
            in[u] = *reinterpret_cast<const Pack<T, V>*>(x + row);
            gr[u] = *reinterpret_cast<const Pack<T, V>*>(dy + row);
        }
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            if (r + u * R >= p.S) break;
            float v[V], d[V];
            widen_v<T, V>(in[u], v);
            widen_v<T, V>(gr[u], d);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float xhat;
                grad_of<ACT, sizeof(T) == 4>(v[i], d[i], mu[i], rstd[i], sc[i], sh[i], xhat, dz[u][i]);
                s[i] += dz[u][i];
                q[i] += dz[u][i] * xhat;
            }
        }
    }
    join_held<V, THREADS>(s, q, sums, chan, p.width, R, on);
    if (p.dscale && threadIdx.x < p.width) p.part[(int64_t)n * p.C + c0 + threadIdx.x] = chan[threadIdx.x];
    for_groups<THREADS>(p.width / p.per, p.per, [&](int g, int lane, int lanes, auto&& sum) {
        const float2 o = group_averages(p, lane, lanes, sum, [&](int i, float& w) { w = scale_of(p, c0 + g * p.per + i); return chan[g * p.per + i]; });
        if (lane == 0) stat[g] = o;
    });
    __syncthreads();
    if (!on) return;
    float c1[V], c2[V], rs[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float2 o = stat[(c + i - c0) / p.per];
        c1[i] = rstd[i] * o.x; c2[i] = rstd[i] * o.y; rs[i] = rstd[i] * scale_of(p, c + i);
    }
    T* dx = (T*)p.out + n * p.out_ns + c;
    forget(in);
#pragma unroll
    for (int u = 0; u < NV; ++u) {
        if (r + u * R >= p.S) break;
        T* o = dx + (int64_t)(r + u * R) * p.C;
        float v[V], old[V];
        widen_v<T, V>(in[u], v);
        if (p.accumulate) load_v<T, V>(o, old);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            v[i] = dz[u][i] * rs[i] - ((v[i] - mu[i]) * rstd[i] * c2[i] + c1[i]);
            if (p.accumulate) v[i] += old[i];
        }
        store_v<T, V>(o, v);
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

// Channels of a workgroup that holds its share of an image in registers, its pieces per thread and its threads; no width where that does not apply.
// Whole groups and whole pieces; as wide as fits up to a line of memory (128 bytes), unless that leaves fewer than 512 workgroups. Workgroups of
// 256 threads where they hold 48 bytes of a row or more, else of 512: the more workgroups a compute unit has, the more their loads, sums and
// stores overlap (us, bf16: 256 x 196 x 256 in 128 bytes by 256 threads forward 16.9 and gradient 26.7, by 512 22.0 and 26.8; 128 x 784 x 192 in 48 by 256 21.1 and
// 34.5, in 96 by 512 22.6 and 36.6; gradients of fp32 lose as much).
struct HeldPlan { int width, pieces, threads; };
HeldPlan held_plan(int64_t N, int64_t S, int64_t C, int64_t G, int dtype, int v, bool backward) {
    const int64_t per = C / G, bytes = dtype == PURINE_BF16 ? 2 : 4;
    int64_t unit = per;
    while (unit % v) unit += per;
    if (unit > C || C % unit) return HeldPlan{0, 0, 0};
    auto widest = [&](bool few) {
        HeldPlan best{0, 0, 0};
        for (int64_t m = 1; unit * m <= C; ++m) {
            const int64_t w = unit * m, cv = w / v;
            if (C % w) continue;
            if (w > 256 || cv > 256) break;
            if (C / w > 1 << 21) continue;         // (workgroups of one image: below 2^31 threads)
            if (best.width && (w * bytes > 128 && best.width * bytes >= 64)) break;
            if (best.width && N * (C / w) < 512) break;
            const int threads = few || S * cv <= 256 * 4 ? 256 : HT;
            const int64_t R = threads / cv, pieces = (S + R - 1) / R;
            if (pieces > (few || (backward && v == 8) ? HELD_GRAD : HELD)) break;
            best = HeldPlan{(int)w, (int)pieces, threads};
        }
        return best;
    };
    if (!backward || dtype == PURINE_BF16) {
        const HeldPlan few = widest(true);
        if (few.width * bytes >= 48) return few;
    }
    return widest(false);
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
// f(pieces as a constant, threads as a constant)
template <int MOST, typename F>
hipError_t by_pieces(const HeldPlan& h, F&& f) {
    if (h.threads == 256 && h.pieces <= 4) return f(std::integral_constant<int, 4>(), std::integral_constant<int, 256>());
    if (h.threads == 256) return f(std::integral_constant<int, HELD_GRAD>(), std::integral_constant<int, 256>());
    if (h.pieces <= 4) return f(std::integral_constant<int, 4>(), std::integral_constant<int, HT>());
    if (h.pieces <= HELD_GRAD) return f(std::integral_constant<int, HELD_GRAD>(), std::integral_constant<int, HT>());
    if constexpr (MOST > HELD_GRAD) return f(std::integral_constant<int, MOST>(), std::integral_constant<int, HT>());
    return hipErrorInvalidValue;
}

// Slices, and where the scratch has what. The kernels that use a group's sums join them for themselves, which saves a launch, unless a thread would go
// through more than LONG slices for it. us, bf16, both directions, for themselves / by kernels of their own: 64 in turn 16 x 12544 x 64 in one group 68 / 75; 128
// 16 x 4096 x 320 in 32 groups 123 / 93, 8 x 12544 x 64 62 / 53; 2048 2 x 65536 x 2048 in 32 groups 2220 / 920.
constexpr int64_t LONG = 64;
struct SlicedPlan { int rows, slices, chunks; size_t about, stat, chunk, bytes; };
SlicedPlan sliced_plan(int64_t N, int64_t S, int64_t C, int64_t G) {
    SlicedPlan o{};
    o.rows = (int)((S - 1) / slices_of(N, S, C) + 1);
    o.slices = (int)((S - 1) / o.rows + 1);
    const int64_t per = C / G, pairs = o.slices * per;
    int64_t lanes = 1;
    while (lanes < 64 && lanes < per) lanes *= 2;
    const int64_t groups = per < 1024 ? (C < 1024 ? C : 1024) / per : 1;       // of a tile of channels
    if (o.slices * ((per + lanes - 1) / lanes) * ((groups * lanes + NT - 1) / NT) > LONG) o.chunks = (int)((pairs + CHUNK - 1) / CHUNK);
    auto whole = [](size_t n) { return (n + 15) / 16 * 16; };
    o.about = whole((size_t)(N * o.slices * C) * sizeof(float2));
    o.stat = o.about + whole((size_t)(N * C) * sizeof(float));
    o.chunk = o.stat + (o.chunks ? whole((size_t)(N * G) * sizeof(float2)) : 0);
    o.bytes = o.chunk + (o.chunks > 1 ? (size_t)(N * G * o.chunks) * sizeof(float4) : 0);
    return o;
}

NormParams params_of(const NormShape& s, void* ws) {
    NormParams p{};
    p.N = s.N; p.S = s.S; p.C = s.C; p.G = s.G; p.per = s.C / s.G;
    p.eps = s.eps;
    p.x_ns = s.x_ns; p.dy_ns = s.dy_ns;
    const SlicedPlan plan = sliced_plan(s.N, s.S, s.C, s.G);
    p.rows = plan.rows;
    p.slices = plan.slices;
    p.chunks = plan.chunks;
    char* const scratch = (char*)ws;
    p.part = (float2*)scratch;
    p.about = (float*)(scratch + plan.about);
    p.stat = plan.chunks ? (float2*)(scratch + plan.stat) : nullptr;
    p.chunk = (float4*)(scratch + plan.chunk);
    return p;
}
// Joins the groups' sums of the images of a call.
template <bool GRAD>
void join_groups(const NormParams& p, hipStream_t st) {
    if (!p.stat) return;
    const unsigned groups = (unsigned)p.N * (unsigned)p.G;
    hipLaunchKernelGGL((norm_join_kernel<GRAD>), dim3(groups * (unsigned)p.chunks), dim3(NT), 0, st, p);
    if (p.chunks > 1) hipLaunchKernelGGL((norm_join_chunks_kernel<GRAD>), dim3(groups), dim3(NT), 0, st, p);
}

// Workgroups of an image in the kernels that walk over positions, and in the held ones.
int64_t blocks_of(NormParams& p, int v) {
    p.tiles = (p.C / v - 1) / NT + 1;
    return (int64_t)p.slices * p.tiles;
}
int64_t held_blocks(NormParams& p, const HeldPlan& h) {
    p.width = h.width;
    p.tiles = p.C / h.width;
    p.slices = 1;
    return p.tiles;
}
// launch(parameters, workgroups) for all images, in as many calls as keep each below 2^31 threads (a launch ends at 2^32 of them: 2^24 images of a
// workgroup each; one image has fewer in every form).
template <typename T, typename F>
hipError_t over_images(const NormParams& p, int64_t blocks, int threads, F&& launch) {
    const int64_t most = (((int64_t)1 << 31) / threads) / blocks, images = most < 1 ? 1 : most;
    for (int64_t n = 0; n < p.N; n += images) {
        NormParams q = p;
        const int64_t groups = n * p.G;
        q.N = (int)(p.N - n < images ? p.N - n : images);
        q.x = (const T*)p.x + n * p.x_ns;
        q.out = (T*)p.out + n * p.out_ns;
        if (p.dy) q.dy = (const T*)p.dy + n * p.dy_ns;
        if (p.mean) { q.mean += groups; q.rstd += groups; }
        if (p.mean_out) { q.mean_out += groups; q.rstd_out += groups; }
        q.part += n * p.slices * p.C;
        q.about += n * p.C;
        if (p.stat) q.stat += groups;
        const hipError_t e = launch(q, dim3((unsigned)(q.N * blocks)));
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

// Rows of sums that one launch adds up for the parameters (us, bf16, both directions, N x 16 x 64 in 8 groups, in one launch / in two: 1500 images 34.0 / 33.4, 3000 59.2 / 55.8,
// 12000 206 / 176; in one a thread goes through a chain of N / 128 batches of loads).
constexpr int64_t MANY = 2048;
// What the sliced kernels take, whichever a call gets (the held ones need a slice's at most).
size_t group_norm_ws_bytes(int64_t N, int64_t S, int64_t C, int64_t G) { return sliced_plan(N, S, C, G).bytes; }

hipError_t launch_group_norm_fwd(int dtype, const NormShape& s, const void* x, const float* scale, const float* shift, void* y, float* mean,
                                 float* rstd, void* ws, hipStream_t st) {
    NormParams p = params_of(s, ws);
    p.x = x; p.scale = scale; p.shift = shift; p.out = y; p.out_ns = s.y_ns;
    p.mean_out = mean; p.rstd_out = rstd;
    const int v = vector_of(s.C, dtype);
    const HeldPlan h = held_plan(s.N, s.S, s.C, s.G, dtype, v, false);
    (void)hipGetLastError();
    return by_vector(dtype, v, [&](auto t, auto V) {
        typedef decltype(t) T;
        return by_act(s.act, [&](auto A) {
            if (h.width) {
                const int64_t blocks = held_blocks(p, h);
                ProbeScope probe(st);
                return by_pieces<HELD>(h, [&](auto P, auto H) {
                    return over_images<T>(p, blocks, H.value, [&](const NormParams& q, dim3 grid) {
                        hipLaunchKernelGGL((norm_held_kernel<T, V.value, A.value, P.value, H.value>), grid, dim3(H.value), 0, st, q);
                        return hipGetLastError();
                    });
                });
            }
            return over_images<T>(p, blocks_of(p, v), NT, [&](const NormParams& q, dim3 grid) {
                hipLaunchKernelGGL((norm_sums_kernel<T, V.value>), grid, dim3(NT), 0, st, q);
                join_groups<false>(q, st);
                ProbeScope probe(st);
                hipLaunchKernelGGL((norm_apply_kernel<T, V.value, A.value>), grid, dim3(NT), 0, st, q);
                return hipGetLastError();
            });
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
    const HeldPlan h = held_plan(s.N, s.S, s.C, s.G, dtype, v, true);
    (void)hipGetLastError();
    const hipError_t e = by_vector(dtype, v, [&](auto t, auto V) {
        typedef decltype(t) T;
        return by_act(s.act, [&](auto A) {
            if (h.width) {
                const int64_t blocks = held_blocks(p, h);
                ProbeScope probe(st);
                return by_pieces<V.value == 8 ? HELD_GRAD : HELD>(h, [&](auto P, auto H) {
                    return over_images<T>(p, blocks, H.value, [&](const NormParams& q, dim3 grid) {
                        hipLaunchKernelGGL((norm_grad_held_kernel<T, V.value, A.value, P.value, H.value>), grid, dim3(H.value), 0, st, q);
                        return hipGetLastError();
                    });
                });
            }
            return over_images<T>(p, blocks_of(p, v), NT, [&](const NormParams& q, dim3 grid) {
                hipLaunchKernelGGL((norm_grad_sums_kernel<T, V.value, A.value>), grid, dim3(NT), 0, st, q);
                join_groups<true>(q, st);
                ProbeScope probe(st);
                hipLaunchKernelGGL((norm_grad_apply_kernel<T, V.value, A.value>), grid, dim3(NT), 0, st, q);
                return hipGetLastError();
            });
        });
    });
    if (e != hipSuccess || !dscale) return e;
    constexpr int64_t MOST = 16 << 23;             // channels of a launch: below 2^32 threads (where there are more, images are few)
    for (int64_t from = 0; from < p.C; from += MOST) {
        const int blocks = (int)(((p.C - from < MOST ? p.C - from : MOST) + 15) / 16);
        int64_t stride = 1, count = (int64_t)p.N * p.slices;
        for (; count > MANY; count = (count + PER - 1) / PER, stride *= PER) {
            const int64_t pieces = (count + PER - 1) / PER;
            hipLaunchKernelGGL((norm_grad_params_kernel<false>), dim3((unsigned)(blocks * pieces)), dim3(NT), 0, st, p, (int)from, blocks, stride, count);
        }
        hipLaunchKernelGGL((norm_grad_params_kernel<true>), dim3((unsigned)blocks), dim3(NT), 0, st, p, (int)from, blocks, stride, count);
    }
    return hipGetLastError();
}

}  // namespace purine
