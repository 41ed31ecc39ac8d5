// Matrix product with bias, activation and residual in its epilogue, its gradients (purine_linear_*), and the gradient of an
// activation by itself (purine_act_bwd).
#include "linear_finish.h"
#include "linear_gemm.h"
#include "packets.h"

namespace purine {
namespace {

// Operands whose rows lie 2^24 elements apart or more, past the 32-bit offsets of the kernels on the matrix cores: 64 x 64 results per
// workgroup, 16 per thread, fp32 products. Where the rows themselves are that long, results are few (128 x 128 at most) and the reduction is split over some thousand
// workgroups, whose sums the join adds (2 x 2^29 by 3 bf16 105 ms; one workgroup would need a thousand times that).
struct FarParams { Source a, b; Finish f; int rows, cols, K, tiles_j, tiles; float* part; unsigned per; int part_ld; };    // part: of splits of `per`, or null
constexpr int TS = 64, KS = 16;
template <typename T, typename O>
__global__ __launch_bounds__(256) void linear_far_kernel(const FarParams p) {
    __shared__ float as[KS][TS + 1], bs[KS][TS + 1];
    const int split = blockIdx.x / p.tiles, tile = (int)blockIdx.x - split * p.tiles, i0 = tile / p.tiles_j * TS, j0 = tile % p.tiles_j * TS;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const T* a = (const T*)p.a.p;
    const T* b = (const T*)p.b.p;
    float acc[4][4] = {};
    const unsigned first = split * p.per, K = min((unsigned)p.K, first + p.per);            // (k0 + k passes 2^31 where K is near it)
    for (unsigned k0 = first; k0 < K; k0 += KS) {
        for (int e = threadIdx.x; e < KS * TS; e += 256) {
            const unsigned k = e / TS;
            const int i = e % TS;
            as[k][i] = k0 + k < K && i0 + i < p.rows ? widen<T>(a[(i0 + i) * p.a.i_step + (k0 + k) * p.a.k_step]) : 0.0f;
            bs[k][i] = k0 + k < K && j0 + i < p.cols ? widen<T>(b[(j0 + i) * p.b.i_step + (k0 + k) * p.b.k_step]) : 0.0f;
        }
        __syncthreads();
        for (int k = 0; k < KS; ++k)
            for (int u = 0; u < 4; ++u)
                for (int v = 0; v < 4; ++v) acc[u][v] += as[k][ty * 4 + u] * bs[k][tx * 4 + v];
        __syncthreads();
    }
    for (int u = 0; u < 4; ++u)
        for (int v = 0; v < 4; ++v) {
            const int i = i0 + ty * 4 + u, j = j0 + tx * 4 + v;
            if (i >= p.rows || j >= p.cols) continue;
            if (p.part) p.part[((int64_t)split * p.rows + i) * p.part_ld + j] = acc[u][v];
            else finish<T, O>(p.f, i, j, acc[u][v]);
        }
}

// Lays an operand out in rows of whole 16-byte packets, zeros behind a row's end: bf16 rows that are not, and fp32 ones in three exact bf16
// parts, a plane each. A thread per packet.
template <typename T>
__global__ __launch_bounds__(256) void linear_pack_kernel(const T* __restrict__ src, int64_t ld, uint16_t* __restrict__ dst, int rows, int len, int packets,
                                                          int64_t plane) {
    const int64_t total = (int64_t)rows * packets;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
        const int row = (int)(t / packets), at = (int)(t - (int64_t)row * packets) * 8, n = len - at;
        const T* s = src + row * ld + at;
        uint16_t* d = dst + t * 8;
        if constexpr (sizeof(T) == 2) {
            uint32_t k[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) k[e] = (uint32_t)(2 * e < n ? s[2 * e] : 0) | (uint32_t)(2 * e + 1 < n ? s[2 * e + 1] : 0) << 16;
            *reinterpret_cast<uint4*>(d) = make_uint4(k[0], k[1], k[2], k[3]);
        } else {
            float v[8];
            lin::get8(s, n >= 8 && ld % 4 == 0, n, v);
            packets::store_split8(v, (unsigned char*)d, (size_t)plane);
        }
    }
}

// Adds the partial sums of the splits in order and finishes the results. A thread has four neighbouring columns of a row of the sums, which are padded to whole
// 16-byte packets, and `lanes` threads share the splits of one (few results of many splits: dw of a narrow layer over many positions). SPLIT3: sums of an
// fp32 product's parts. Bound: memory (14173 x 4771 fp32, 541 MB: 147 us, rows that are no whole packets are stored element by element; with sums in such rows, one result a
// thread, 252, and the product before it 305 for 169).
struct JoinParams { const float* part; Finish f; Source a, b; int rows, cols, K, splits, lanes; };
template <typename E, typename O, bool SPLIT3>
__global__ __launch_bounds__(256) void linear_join_kernel(const JoinParams p) {
    __shared__ float sums[256][5];
    const int lanes = p.lanes, per = 256 / lanes, lane = threadIdx.x / per, mine = threadIdx.x % per;
    const unsigned chunks = (unsigned)(p.cols + 3) / 4, total = (unsigned)p.rows * chunks, t = blockIdx.x * (unsigned)per + mine;     // (below 2^31)
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (t < total) {
        const int each = (p.splits + lanes - 1) / lanes, last = min(p.splits, (lane + 1) * each);
        const float4* src = reinterpret_cast<const float4*>(p.part) + t;
#pragma unroll 4
        for (int s = lane * each; s < last; ++s) {
            const float4 x = src[(int64_t)s * total];
            v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
        }
    }
    if (lanes > 1) {
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[threadIdx.x][e] = v[e];
        __syncthreads();
        if (lane) return;
        for (int l = 1; l < lanes; ++l)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += sums[threadIdx.x + l * per][e];
    }
    if (t >= total) return;
    const int i = (int)(t / chunks), j = (int)(t - i * chunks) * 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (j + e >= p.cols) break;
        float z = v[e];
        if constexpr (SPLIT3) z = joined(z, p.a, p.b, i, j + e, p.K);
        finish<E, O>(p.f, i, j + e, z);
    }
}

// How a product is computed: the same answer for the workspace query and for the launch.
struct GemmPlan {
    int tile, bufs, tiles_i, tiles_j, steps, splits, per_split;
    double us;
};

// The forms of the kernel on the matrix cores, and what a compute unit takes with them (us, measured at 1024 and 8192 on a side over 64 to 4096):
// workgroups that it holds; a round of them apart from its steps (first loads, results); a step of 64 with all of them, and with one.
struct Form { int tile, bufs, resident; double round, step, alone; };
constexpr Form kForms[] = {{256, 2, 1, 13.0, 1.30, 1.05}, {128, 2, 2, 5.5, 0.79, 0.50}, {128, 4, 1, 5.0, 0.50, 0.50}, {64, 2, 4, 3.5, 0.68, 0.30}, {64, 4, 2, 3.0, 0.38, 0.21}};

// The form and the split of the reduction (where tiles alone leave compute units idle) with the least expected time. The compute units with the most
// workgroups count; smaller tiles fetch an operand more often (a microsecond per 40 MB). us, weights from memory: 128 x 9216 x 4096 in tiles of 64 and 3 parts
// of the reduction 38, 2 parts 33, in tiles of 128 and 8 parts 29.5; 256 x 4096 x 4096 in tiles of 64 23, of 128 and 4 parts 26.
GemmPlan plan_gemm(int64_t rows, int64_t cols, int64_t K, int planes) {
    GemmPlan best{};
    best.us = 1e30;
    const int64_t steps = (K + lin::BK - 1) / lin::BK;
    const double products = planes == 3 ? 6.0 : 1.0;
    for (const Form& f : kForms) {
        const int64_t ti = (rows + f.tile - 1) / f.tile, tj = (cols + f.tile - 1) / f.tile, tiles = ti * tj;
        int64_t last = 0;
        for (int64_t want = 1; want <= 1024; want += want < 4 ? 1 : want / 4) {
            const int64_t per = (steps + want - 1) / want, splits = (steps + per - 1) / per;
            if (splits == last) continue;
            last = splits;
            const double part = (splits > 1 || planes > 1) ? 4.0 * splits * rows * cols : 0.0;
            if (tiles * splits > 0x7fffffff || (splits > 1 && (part > 256e6 || tiles * splits > 4096))) break;
            const double load = (double)tiles * splits / 256.0, rounds = ceil(load / f.resident);
            double step = f.step;
            if (load <= 1.0) step = f.alone;
            else if (load < f.resident) step = f.alone + (f.step - f.alone) * (ceil(load) - 1.0) / (f.resident - 1.0);
            const double read = 2.0 * products * (double)K * ((double)rows * (double)tj + (double)cols * (double)ti);
            const double work = rounds * f.round + (rounds > 1.0 ? load / f.resident * 0.5 + rounds * 0.5 : 1.0) * step * (double)per * products;
            const double us = work + read / 40e6 + (part > 0.0 ? 4.0 + 2.0 * part / 5e6 : 0.0);
            if (us < best.us) best = GemmPlan{f.tile, f.bufs, (int)ti, (int)tj, (int)steps, (int)splits, (int)per, us};
        }
    }
    return best;
}

// Products that one launch without scratch computes faster than the kernels above, by the measured times of both (us): a launch, steps of 32 in
// each of the workgroup's wavefronts, alone on a compute unit or beside `load` others.
DirectForm direct_form(int64_t rows, int64_t cols, int64_t K, bool a_in, bool b_in, int dtype) {
    const bool f32 = dtype == PURINE_F32;
    const int64_t steps = (K + 31) / 32;
    double best = 1e30;
    DirectForm form = DIRECT_NONE;
    auto offer = [&](DirectForm f, double us) { if (us < best) { best = us; form = f; } };
    // (a wavefront works on two groups of `depth` steps in turn, whether they exist or not)
    auto chain = [&](int64_t groups, int64_t waves, int64_t depth, double alone, double full) {
        const double load = (double)groups / 256.0;
        const int64_t each = ((steps + waves - 1) / waves + 2 * depth - 1) / (2 * depth) * (2 * depth);
        return 3.8 + (double)each * fmax(alone, full * load) + 0.4 * load;
    };
    if (a_in && b_in) {
        if (rows <= 4 && K % (f32 ? 4 : 8) == 0) {
            // reading B, or what a column costs however short it is (2^20 columns of 64: bf16 284, 549 and 1451 us with 1, 2 and 4 rows, fp32 157, 323 and 1354)
            const double read = (double)K * (f32 ? 4.0 : 2.0) / (rows > 2 && !f32 ? 3.6e6 : 5.0e6);
            const double column = rows > 2 ? 1.35e-3 : (f32 ? 0.15e-3 : 0.27e-3) * (double)rows;
            offer(DIRECT_ROW, 4.0 + (double)cols * fmax(read, column));
        }
        if (rows <= 16) offer(DIRECT_ROWS, chain((cols + 15) / 16, 8, 4, f32 ? 0.75 : 0.29, f32 ? 1.08 : 0.47));
    }
    const int64_t groups = ((rows + 31) / 32) * ((cols + 31) / 32);
    if (groups <= 0x7fffffff)
        offer(DIRECT_SMALL, f32 ? chain(groups, 4, 1, 0.85, 0.95) : a_in && b_in ? chain(groups, 4, 2, 0.36, 0.36) : a_in ? chain(groups, 4, 1, 0.44, 0.55) :
                            chain(groups, 4, 1, 0.60, 0.62));
    if (!f32 && a_in && rows >= 4096 && stream_fits(cols, K)) offer(DIRECT_STREAM, stream_us(rows, cols, K));
    if (best < 6.0) return form;                   // (as short as any launch)
    // the kernels above, with the launches that lay operands out and that join sums
    auto laid = [&](int64_t n, bool in) { return f32 || (in ? K : n) % 8 ? 3.0 + (double)n * (double)K * (f32 ? 10.0 : 4.0) / 4.5e6 : 0.0; };
    if (plan_gemm(rows, cols, K, f32 ? 3 : 1).us + 2.0 + laid(rows, a_in) + laid(cols, b_in) <= best) return DIRECT_NONE;
    return form;
}

// rows of partial sums: whole 16-byte packets
int64_t part_ld(int64_t cols) { return (cols + 3) / 4 * 4; }
int64_t packed_ld(int64_t len) { return (len + 7) / 8 * 8; }
size_t whole(size_t n) { return (n + 255) / 256 * 256; }
// bytes of an operand's copy: reduction inner (rows x K) or outer (K x rows)
size_t packed_bytes(int64_t rows, int64_t K, bool in, int planes) { return whole((size_t)(in ? rows * packed_ld(K) : K * packed_ld(rows)) * 2 * planes); }
bool whole_packets(int64_t rows, int64_t K, bool in) { return (in ? K : rows) % 8 == 0; }

// g = dy act'(pre), and the sums of its columns over a slice of the rows. (g is rounded to the type that the products read, the sums are taken before: fp32 g
// would be 4 bytes for 2 here and in two products, and three bf16 parts in them.) Bound: HBM (us: 8192 x 8192 bf16 85, 403 MB at 4.7 TB/s; 100352 x 96 12.3,
// 58 MB at 4.7; 777 x 333 fp32 in single elements 4.4), then a launch of 4 - 5 for the slices' sums. A thread owns V neighbouring columns (16 bytes where
// rows are whole packets) and walks down the slice, four rows at a time; the threads of a column join in LDS, the slices in a
// second kernel, both in order.
struct ActParams {
    const void* pre; const void* dy; void* g; float* part;
    int64_t pre_ld, dy_ld, g_ld;
    int N, K, rows, slices, tiles;
};
constexpr int ANT = 256;
template <typename T, int V, int ACT>
__global__ __launch_bounds__(ANT) void act_bwd_kernel(const ActParams p) {
    __shared__ float sums[ANT * V];
    const int slice = blockIdx.x / p.tiles, first = (int)(blockIdx.x - (unsigned)slice * p.tiles) * ANT;
    const int tile = min(ANT, p.K / V - first), R = ANT / tile, r = threadIdx.x / tile, j = (first + (int)threadIdx.x % tile) * V;
    const int i0 = slice * p.rows, n = min(p.rows, p.N - i0);         // rows from i0 on (counted from there: sums stay far from 2^31)
    float sum[V];
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] = 0.0f;
    if (r < R) {
        const T* dy = (const T*)p.dy + i0 * p.dy_ld + j;
        const T* pre = (const T*)p.pre + i0 * p.pre_ld + j;
        T* g = (T*)p.g + i0 * p.g_ld + j;
        constexpr int AHEAD = 4;
        for (int i = r; i < n; i += R * AHEAD) {
            float v[AHEAD][V], z[AHEAD][V];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int64_t row = min(i + u * R, n - 1);
                lin::get_v(dy + row * p.dy_ld, v[u]);
                if (ACT != PURINE_ACT_NONE) lin::get_v(pre + row * p.pre_ld, z[u]);
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int64_t row = i + u * R;
                if (row >= n) break;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    if (ACT != PURINE_ACT_NONE) v[u][e] *= act_slope<ACT, sizeof(T) == 4>(z[u][e]);
                    sum[e] += v[u][e];
                }
                if (p.g) lin::put_v(g + row * p.g_ld, v[u]);
            }
        }
    }
    if (!p.part) return;
#pragma unroll
    for (int e = 0; e < V; ++e) sums[threadIdx.x * V + e] = sum[e];
    __syncthreads();
    if (r) return;
    for (int k = 1; k < R; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) sum[e] += sums[(threadIdx.x + k * tile) * V + e];
    float* o = p.part + (size_t)slice * p.K + j;
#pragma unroll
    for (int e = 0; e < V; ++e) o[e] = sum[e];
}
// CS columns per workgroup, the slices over 256 / CS threads each. first: the launch's first workgroup.
template <typename O, int CS>
__global__ __launch_bounds__(256) void column_sums_kernel(const float* part, O* db, int slices, int K, int accumulate, unsigned first) {
    __shared__ float sums[256 / CS][CS + 1];
    const int l = threadIdx.x % CS, r = threadIdx.x / CS;
    const unsigned j = (first + blockIdx.x) * CS + l;
    float sum = 0.0f;
    if (j < (unsigned)K) {
#pragma unroll 8
        for (int s = r; s < slices; s += 256 / CS) sum += part[(size_t)s * K + j];
    }
    sums[r][l] = sum;
    __syncthreads();
    for (int half = 128 / CS; half; half /= 2) {
        if (r < half) sums[r][l] += sums[r + half][l];
        __syncthreads();
    }
    if (r || j >= (unsigned)K) return;
    sum = sums[0][l];
    if (accumulate) sum += widen<O>(db[j]);
    narrow(sum, db + j);
}
// Four columns a workgroup while they are too few to fill the card (1024 slices of 96: 4.6 us), else a line of memory's 32, of which four would fetch
// the line eight times (256 slices of 8192: 12.9 us by four, 5.0 by 32).
template <typename O>
hipError_t column_sums(const float* part, O* db, int slices, int K, int accumulate, hipStream_t st) {
    if (K < 4096) hipLaunchKernelGGL((column_sums_kernel<O, 4>), dim3((unsigned)((K + 3) / 4)), dim3(256), 0, st, part, db, slices, K, accumulate, 0u);
    else {
        // (below 2^32 threads a launch)
        const unsigned groups = ((unsigned)K + 31) / 32, most = 1u << 23;
        for (unsigned from = 0; from < groups; from += most)
            hipLaunchKernelGGL((column_sums_kernel<O, 32>), dim3(groups - from < most ? groups - from : most), dim3(256), 0, st, part, db, slices, K, accumulate, from);
    }
    return hipGetLastError();
}
// Rows of a slice where threads own V columns: some 1024 workgroups, and one batch of loads per thread at least.
int act_rows(int64_t N, int64_t K, int V) {
    const int64_t vectors = (K + V - 1) / V, tiles = (vectors + ANT - 1) / ANT, R = vectors < ANT ? ANT / vectors : 1;
    int64_t slices = 1024 / tiles;
    if (slices < 1) slices = 1;
    int64_t rows = (N + slices - 1) / slices;
    if (rows < 4 * R) rows = 4 * R;
    return (int)(rows < N ? rows : N);
}

}  // namespace

namespace {

// Parts of the reduction in the kernel for far rows, where they are long themselves.
constexpr int64_t FAR = (int64_t)1 << 24;
int64_t far_splits(int64_t rows, int64_t cols, int64_t K) {
    const int64_t tiles = ((rows + TS - 1) / TS) * ((cols + TS - 1) / TS);
    return K >= FAR && tiles < 1024 ? 1024 / tiles : 1;
}
size_t far_ws_bytes(int64_t rows, int64_t cols, int64_t K) {
    const int64_t splits = far_splits(rows, cols, K);
    return splits > 1 ? (size_t)(splits * rows * part_ld(cols)) * 4 : 0;
}
size_t near_ws_bytes(int64_t rows, int64_t cols, int64_t K, bool a_in, bool b_in, int dtype) {
    if (direct_form(rows, cols, K, a_in, b_in, dtype) != DIRECT_NONE) return 0;
    const int planes = dtype == PURINE_F32 ? 3 : 1;
    const GemmPlan g = plan_gemm(rows, cols, K, planes);
    size_t n = 0;
    if (planes == 3 || !whole_packets(rows, K, a_in)) n += packed_bytes(rows, K, a_in, planes);
    if (planes == 3 || !whole_packets(cols, K, b_in)) n += packed_bytes(cols, K, b_in, planes);
    if (planes == 3 || g.splits > 1) n += (size_t)g.splits * rows * part_ld(cols) * 4;
    return n;
}
size_t piece_ws_bytes(int64_t rows, int64_t cols, int64_t K, bool a_in, bool b_in, int dtype) {
    const size_t near = near_ws_bytes(rows, cols, K, a_in, b_in, dtype), far = a_in || b_in ? far_ws_bytes(rows, cols, K) : 0;
    return near > far ? near : far;
}

// Rows and columns of a launch at most: a launch ends at 2^32 threads, and the single row's kernel has 64 for a column.
constexpr int64_t MOST = (int64_t)1 << 25;
// The rows and columns [i, i + rows) x [j, j + cols) of a product.
LinearCall part_of(const LinearCall& c, int64_t i, int64_t rows, int64_t j, int64_t cols) {
    const int64_t es = c.dtype == PURINE_F32 ? 4 : 2, os = c.out_dtype == PURINE_F32 ? 4 : 2;
    auto at = [](auto* p, int64_t bytes) { return p ? (decltype(p))((const char*)p + bytes) : p; };
    LinearCall q = c;
    q.rows = rows; q.cols = cols;
    q.a = at(c.a, i * (c.a_in ? c.a_ld : 1) * es);
    q.b = at(c.b, j * (c.b_in ? c.b_ld : 1) * es);
    q.bias = at(c.bias, j * es);
    q.res = at(c.res, (i * c.res_ld + j) * es);
    q.pre = at(c.pre, (i * c.pre_ld + j) * es);
    q.slope = at(c.slope, (i * c.slope_ld + j) * es);
    q.out = at(c.out, (i * c.out_ld + j) * os);
    return q;
}
// f(part) for all parts of at most `rows` x `cols`
template <typename F>
hipError_t by_parts(const LinearCall& c, int64_t rows, int64_t cols, F&& f) {
    for (int64_t i = 0; i < c.rows; i += rows)
        for (int64_t j = 0; j < c.cols; j += cols) {
            const hipError_t e = f(part_of(c, i, c.rows - i < rows ? c.rows - i : rows, j, c.cols - j < cols ? c.cols - j : cols));
            if (e != hipSuccess) return e;
        }
    return hipSuccess;
}

template <typename E, typename O, bool SPLIT3 = sizeof(E) == 4>
hipError_t join(const JoinParams& q, hipStream_t st) {
    JoinParams p = q;
    const int64_t threads = (int64_t)p.rows * part_ld(p.cols) / 4;
    p.lanes = 1;
    while (p.lanes < 32 && p.lanes * 4 <= p.splits && threads * p.lanes < 256 * 512) p.lanes *= 2;
    const int64_t per = 256 / p.lanes, grid = (threads + per - 1) / per;
    hipLaunchKernelGGL((linear_join_kernel<E, O, SPLIT3>), dim3((unsigned)grid), dim3(256), 0, st, p);
    return hipGetLastError();
}

template <typename T>
void pack(const void* src, int64_t ld, void* dst, int64_t rows, int64_t K, bool in, hipStream_t st) {
    const int64_t r = in ? rows : K, len = in ? K : rows, packets = packed_ld(len) / 8, total = r * packets;
    const unsigned grid = (unsigned)((total + 255) / 256 < 65536 ? (total + 255) / 256 : 65536);
    hipLaunchKernelGGL((linear_pack_kernel<T>), dim3(grid), dim3(256), 0, st, (const T*)src, ld, (uint16_t*)dst, (int)r, (int)len, (int)packets, r * packets * 16);
}

hipError_t launch_piece(const LinearCall& c, void* ws, hipStream_t st) {
    const bool f32 = c.dtype == PURINE_F32;
    const int planes = f32 ? 3 : 1;
    const Finish f = finish_of(c);
    const Source a = source_of(c.a, c.a_ld, c.a_in), b = source_of(c.b, c.b_ld, c.b_in);
    (void)hipGetLastError();
    const DirectForm direct = direct_form(c.rows, c.cols, c.K, c.a_in, c.b_in, c.dtype);
    const int64_t far = FAR, es = f32 ? 4 : 2;
    const int64_t span = ((c.a_in ? c.rows : c.K) * c.a_ld > (c.b_in ? c.cols : c.K) * c.b_ld ? (c.a_in ? c.rows : c.K) * c.a_ld : (c.b_in ? c.cols : c.K) * c.b_ld) * es;
    if (direct == DIRECT_STREAM) return launch_linear_stream(c, st);
    if (direct != DIRECT_NONE && span < 0x7fffffff) return launch_linear_direct(c, direct, st);
    if (direct != DIRECT_NONE && c.a_in && c.b_in && c.a_ld < far && c.b_ld < far) {
        // as many rows of either operand as 32-bit offsets reach, in eights, whose results begin at 16 bytes (24 at least)
        const int64_t rows = 0x7ffffff0 / (c.a_ld * es) / 8 * 8, cols = 0x7ffffff0 / (c.b_ld * es) / 8 * 8;
        return by_parts(c, rows, cols, [&](const LinearCall& q) { return launch_linear_direct(q, direct, st); });
    }
    if (direct != DIRECT_NONE || c.a_ld >= far || c.b_ld >= far) {
        const int64_t splits = c.a_in || c.b_in ? far_splits(c.rows, c.cols, c.K) : 1, per = (c.K + splits - 1) / splits;
        FarParams p{a, b, f, (int)c.rows, (int)c.cols, (int)c.K, (int)((c.cols + TS - 1) / TS), 0, splits > 1 ? (float*)ws : nullptr, (unsigned)per, (int)part_ld(c.cols)};
        p.tiles = (int)((c.rows + TS - 1) / TS) * p.tiles_j;
        const unsigned grid = (unsigned)(p.tiles * splits);
        {
            ProbeScope probe(st);
            if (f32) hipLaunchKernelGGL((linear_far_kernel<float, float>), dim3(grid), dim3(256), 0, st, p);
            else if (c.out_dtype == PURINE_F32) hipLaunchKernelGGL((linear_far_kernel<uint16_t, float>), dim3(grid), dim3(256), 0, st, p);
            else hipLaunchKernelGGL((linear_far_kernel<uint16_t, uint16_t>), dim3(grid), dim3(256), 0, st, p);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || splits == 1) return e;
        const JoinParams q{p.part, f, a, b, p.rows, p.cols, p.K, (int)splits, 1};
        if (f32) return join<float, float, false>(q, st);
        return c.out_dtype == PURINE_F32 ? join<uint16_t, float>(q, st) : join<uint16_t, uint16_t>(q, st);
    }
    GemmPlan g = plan_gemm(c.rows, c.cols, c.K, planes);
    if (c.a_ld >= far / 4 || c.b_ld >= far / 4) {          // (a tile of 256 rows would span 2^31 bytes)
        g.tile = 64;
        g.bufs = 4;
        g.tiles_i = (int)((c.rows + 63) / 64);
        g.tiles_j = (int)((c.cols + 63) / 64);
    }
    lin::GemmParams p{};
    char* scratch = (char*)ws;
    struct Laid { const char* p; int64_t ld, size, plane; };
    auto lay = [&](const void* src, int64_t ld, int64_t rows, bool in) {
        if (!f32 && whole_packets(rows, c.K, in)) return Laid{(const char*)src, ld, ((in ? rows : c.K) - 1) * ld * 2 + (in ? c.K : rows) * 2, 0};
        const Laid l{scratch, packed_ld(in ? c.K : rows), (int64_t)packed_bytes(rows, c.K, in, planes), (in ? rows : c.K) * packed_ld(in ? c.K : rows) * 2};
        if (f32) pack<float>(src, ld, scratch, rows, c.K, in, st);
        else pack<uint16_t>(src, ld, scratch, rows, c.K, in, st);
        scratch += l.size;
        return l;
    };
    const Laid la = lay(c.a, c.a_ld, c.rows, c.a_in), lb = lay(c.b, c.b_ld, c.cols, c.b_in);
    p.a = la.p; p.a_ld = la.ld; p.a_size = la.size; p.a_plane = la.plane;
    p.b = lb.p; p.b_ld = lb.ld; p.b_size = lb.size; p.b_plane = lb.plane;
    p.rows = (int)c.rows; p.cols = (int)c.cols; p.K = (int)c.K;
    p.planes = planes;
    p.steps = g.steps; p.per_split = g.per_split; p.splits = g.splits;
    p.tiles_i = g.tiles_i; p.tiles_j = g.tiles_j;
    p.group = 8;
    const bool second = g.splits > 1 || f32;
    p.part = (float*)scratch;
    p.part_ld = (int)part_ld(c.cols);
    p.out = c.out; p.out_ld = c.out_ld; p.out_f32 = c.out_dtype == PURINE_F32;
    p.bias = c.bias; p.res = c.res; p.res_ld = c.res_ld; p.pre = c.pre; p.pre_ld = c.pre_ld; p.slope = c.slope; p.slope_ld = c.slope_ld;
    p.accumulate = c.accumulate;
    p.vectors = c.out_ld % 8 == 0 && (!c.res || c.res_ld % 8 == 0) && (!c.pre || c.pre_ld % 8 == 0) && (!c.slope || c.slope_ld % 8 == 0);
    const int act = second ? lin::PART : c.b_in || c.slope ? c.act : PURINE_ACT_NONE;
    hipError_t e;
    {
        ProbeScope probe(st);
        switch (g.tile * 10 + g.bufs) {
            case 2562: e = lin::gemm_256_2(p, c.a_in, c.b_in, act, st); break;
            case 1282: e = lin::gemm_128_2(p, c.a_in, c.b_in, act, st); break;
            case 1284: e = lin::gemm_128_4(p, c.a_in, c.b_in, act, st); break;
            case 642: e = lin::gemm_64_2(p, c.a_in, c.b_in, act, st); break;
            default: e = lin::gemm_64_4(p, c.a_in, c.b_in, act, st); break;
        }
    }
    if (e != hipSuccess || !second) return e;
    JoinParams q{p.part, f, a, b, p.rows, p.cols, p.K, p.splits, 1};
    if (f32) return join<float, float>(q, st);
    return c.out_dtype == PURINE_F32 ? join<uint16_t, float>(q, st) : join<uint16_t, uint16_t>(q, st);
}

}  // namespace

size_t linear_ws_bytes(int64_t rows, int64_t cols, int64_t K, bool a_in, bool b_in, int dtype) {
    if (rows <= MOST && cols <= MOST) return piece_ws_bytes(rows, cols, K, a_in, b_in, dtype);
    size_t most = 0;
    for (const int64_t r : {rows < MOST ? rows : MOST, rows % MOST})
        for (const int64_t c : {cols < MOST ? cols : MOST, cols % MOST}) {
            const size_t n = r && c ? piece_ws_bytes(r, c, K, a_in, b_in, dtype) : 0;
            if (n > most) most = n;
        }
    return most;
}

hipError_t launch_linear(const LinearCall& c, void* ws, hipStream_t st) {
    if (c.rows <= MOST && c.cols <= MOST) return launch_piece(c, ws, st);
    return by_parts(c, MOST, MOST, [&](const LinearCall& q) { return launch_piece(q, ws, st); });
}

size_t act_bwd_ws_bytes(int64_t N, int64_t K) {
    int64_t slices = 0;
    for (int V : {1, 4, 8}) {
        const int64_t rows = act_rows(N, K, V), n = (N + rows - 1) / rows;
        if (n > slices) slices = n;
    }
    return (size_t)slices * K * 4;
}

namespace {
template <typename T, int V>
void act_bwd(const ActParams& q, int act, hipStream_t st) {
    ActParams p = q;
    p.tiles = (p.K / V - 1) / ANT + 1;
    const unsigned grid = (unsigned)((int64_t)p.slices * p.tiles);
    switch (act) {
        case PURINE_ACT_RELU: hipLaunchKernelGGL((act_bwd_kernel<T, V, PURINE_ACT_RELU>), dim3(grid), dim3(ANT), 0, st, p); break;
        case PURINE_ACT_SILU: hipLaunchKernelGGL((act_bwd_kernel<T, V, PURINE_ACT_SILU>), dim3(grid), dim3(ANT), 0, st, p); break;
        case PURINE_ACT_GELU: hipLaunchKernelGGL((act_bwd_kernel<T, V, PURINE_ACT_GELU>), dim3(grid), dim3(ANT), 0, st, p); break;
        case PURINE_ACT_GELU_TANH: hipLaunchKernelGGL((act_bwd_kernel<T, V, PURINE_ACT_GELU_TANH>), dim3(grid), dim3(ANT), 0, st, p); break;
        default: hipLaunchKernelGGL((act_bwd_kernel<T, V, PURINE_ACT_NONE>), dim3(grid), dim3(ANT), 0, st, p); break;
    }
}
}  // namespace

hipError_t launch_act_bwd(int dtype, const void* pre, int64_t pre_ld, const void* dy, int64_t dy_ld, void* g, int64_t g_ld, void* db, int db_dtype,
                          bool accumulate, int64_t N, int64_t K, int act, void* ws, hipStream_t st) {
    if (!pre) act = PURINE_ACT_NONE;
    const int64_t all = K | dy_ld | (pre ? pre_ld : 0) | (g ? g_ld : 0);
    const int V = dtype == PURINE_F32 ? (all % 4 ? 1 : 4) : all % 8 ? 1 : 8;
    ActParams p{pre, dy, g, db ? (float*)ws : nullptr, pre_ld, dy_ld, g_ld, (int)N, (int)K, act_rows(N, K, V), 0, 1};
    p.slices = (int)((N + p.rows - 1) / p.rows);
    (void)hipGetLastError();
    {
        ProbeScope probe(st);
        if (dtype == PURINE_F32) V == 4 ? act_bwd<float, 4>(p, act, st) : act_bwd<float, 1>(p, act, st);
        else V == 8 ? act_bwd<uint16_t, 8>(p, act, st) : act_bwd<uint16_t, 1>(p, act, st);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !db) return e;
    return db_dtype == PURINE_F32 ? column_sums(p.part, (float*)db, p.slices, (int)K, accumulate, st) : column_sums(p.part, (uint16_t*)db, p.slices, (int)K, accumulate, st);
}

}  // namespace purine
