// The matrix products of the block operators on the bf16 matrix cores:
//
//     out[i][j] = epilogue(sum over k of A(i, k) B(j, k))
//
// A workgroup of four wavefronts owns BI x BJ results, a wavefront a quarter (2 x 2). Steps of 64 of the reduction go through LDS in two buffers,
// filled by direct-to-LDS loads one step ahead; fragments are read one half step ahead of the MFMAs (16x16x32) that use them,
// so that a wavefront waits once per step, where all four meet.
//
// An operand whose reduction is its inner axis lies in LDS in rows of 64 (128 bytes), their eight 16-byte packets exchanged by the row's
// number so that the rows of a fragment fall into different banks. One whose reduction is its outer axis lies there as in memory,
// rows of BI (or BJ) elements of one k; ds_read_b64_tr_b16 hands a lane four k of its column. Its rows are put a step of the
// banks apart (SKEW), with k, k + 32, ... next to each other because a 1024-byte load cannot be taken apart.
//
// B is the MFMA's first operand: a lane's four results of a tile are neighbouring columns j of one row i. The columns are dealt to
// pairs of tiles so that the lane holds eight neighbours, 16 bytes of bf16, and the four lanes of a row 64.
#pragma once
#include "activation.h"
#include "bf16.h"
#include "block.h"

#include <utility>

namespace purine {
namespace lin {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int BK = 64;                     // reduction elements of a step
constexpr unsigned NOWHERE = 0x80000000u;  // an offset that no operand reaches: reads as zero
constexpr int PART = -1;                   // epilogue: none, fp32 partial sums

struct GemmParams {
    const char* a; const char* b;
    int64_t a_size, b_size;                // bytes from the operand's first to past its last element
    int64_t a_plane, b_plane;              // bytes between the parts of an fp32 operand
    int64_t a_ld, b_ld;                    // elements between rows
    int rows, cols, K;
    int steps, per_split, splits;
    int planes;                            // 1, or 3: fp32 operands in three bf16 parts
    int tiles_i, tiles_j, group;           // group: row tiles that share their columns' panels in L2
    float* part;                           // [split][rows][cols]
    void* out; const void* bias; const void* res; void* pre; const void* slope;
    int64_t out_ld, res_ld, pre_ld, slope_ld;
    int out_f32, accumulate;
    int vectors;                           // every row of every epilogue matrix begins at 16 bytes
};

// f(0), ..., f(N - 1) with constant arguments: accumulators are indexed by nothing else.
template <typename F, int... I>
__device__ __forceinline__ void each_of(F&& f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>()), ...); }
template <int N, typename F>
__device__ __forceinline__ void each(F&& f) { each_of(f, std::make_integer_sequence<int, N>()); }

// An operand's tile in LDS: R rows (or columns) of a step.
template <int R, bool IN, int SKEW>
struct Stage {
    static constexpr int UNITS = R / 8;                        // 1024-byte loads
    static constexpr int UNIT = IN ? 1024 : 1024 + SKEW;       // bytes between them
    static constexpr int BYTES = UNITS * UNIT;
    static constexpr int PER_ROW = R / 8;                      // packets in a row of an outer-axis operand
};

// Which of the R rows this lane reads, as the first operand's tiles deal them (see above) or in order.
template <bool DEALT> __device__ __forceinline__ int row_of(int r) { return DEALT ? 8 * (r >> 2) + (r & 3) : r; }
template <bool DEALT> __device__ __forceinline__ int exchange(int row) { return DEALT ? (row & 3) | (row >> 1 & 4) : row & 7; }

template <int R, bool IN, bool DEALT, int SKEW>
struct Operand {
    typedef Stage<R, IN, SKEW> S;
    static constexpr int LOADS = S::UNITS / 4;
    unsigned off[LOADS];                   // bytes from the step's base
    int k_at[LOADS];                       // first k of the packet (IN) or its k
    const char* base;                      // of the current step's first plane
    const char* end;
    int64_t k_bytes;                       // per step
    int frag;                              // LDS bytes of this lane's first fragment

    __device__ void init(const char* p, int64_t size, int64_t ld, int first, int limit, int lane, int wave) {
        base = p + (IN ? first * ld * 2 : (int64_t)first * 2);
        end = p + size;
        k_bytes = IN ? BK * 2 : BK * ld * 2;
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const int unit = u * 4 + wave;
            if constexpr (IN) {
                const int row = unit * 8 + (lane >> 3), c = (lane & 7) ^ exchange<DEALT>(row);
                off[u] = (unsigned)(min(row, limit - first - 1) * ld * 2) + c * 16;      // (rows past the last read it again)
                k_at[u] = c * 8;
            } else {
                const int k = unit + lane / S::PER_ROW * S::UNITS, c = min(lane % S::PER_ROW, (limit - first - 1) / 8);
                off[u] = (unsigned)(k * ld * 2) + c * 16;
                k_at[u] = k;
            }
        }
        const int r = lane & 15, q = lane >> 4;
        if constexpr (IN) {
            const int row = row_of<DEALT>(r);
            frag = row * 128 + ((q ^ exchange<DEALT>(row)) * 16);
        } else {
            const int k = 8 * q + (r >> 2);
            frag = (k % S::UNITS) * S::UNIT + (k / S::UNITS) * (R * 2) + (DEALT ? 8 * (r & 3) : 4 * (r & 3)) * 2;
        }
    }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t resource(const char* at) const {
        const int64_t room = end - at;
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(at), (short)0, (int)(room < 0x7fffffff ? room : 0x7fffffff), 0x00020000);
    }
    // one load of a step's tile; `left` elements of the reduction remain from the step's first on
    template <int U>
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, unsigned char* lds, int wave, int left) const {
        const unsigned o = k_at[U] < left ? off[U] : NOWHERE;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(lds + (U * 4 + wave) * S::UNIT), 16, o, 0, 0, 0);
    }
    // LDS offset of tile t (16 rows) from this lane's first fragment
    static constexpr int tile_at(int t) {
        const int tile = DEALT ? (t >> 1) * 32 + (t & 1) * 4 : t * 16;
        return IN ? tile * 128 : tile * 2;
    }
    static constexpr int HALF = 4 * S::UNIT;       // outer axis: from four k of a fragment to the next four
    // ... and of the first fragment in half step kk
    __device__ __forceinline__ static int half_at(int frag, int kk) { return IN ? frag ^ (kk * 64) : frag + kk * 512; }
};

// One fragment's read. The wait is at the end of the same asm block (see block()).
#define LIN_READ_IN(F, AT, OFF) "ds_read_b128 " F ", " AT " offset:" OFF "\n\t"
#define LIN_READ_OUT(LO, HI, AT, OFF, OFF2) "ds_read_b64_tr_b16 " LO ", " AT " offset:" OFF "\n\tds_read_b64_tr_b16 " HI ", " AT " offset:" OFF2 "\n\t"
#define LIN_MFMA(ACC, B) "v_mfma_f32_16x16x32_bf16 " ACC ", " B ", %[a], " ACC "\n\t"

// A fragment as it is read: 16 bytes, or two times 8.
template <bool IN> struct Frag { bf16x8 v; };
template <> struct Frag<false> { shortx4 lo, hi; };
__device__ __forceinline__ bf16x8 value(const Frag<true>& f) { return f.v; }
__device__ __forceinline__ bf16x8 value(const Frag<false>& f) { return __builtin_bit_cast(bf16x8, __builtin_shufflevector(f.lo, f.hi, 0, 1, 2, 3, 4, 5, 6, 7)); }

template <int BI, int BJ, bool AIN, bool BIN>
struct Shape {
    static constexpr int A_SKEW = 32, B_SKEW = 64;
    typedef Operand<BI, AIN, false, A_SKEW> A;
    typedef Operand<BJ, BIN, true, B_SKEW> B;
    static constexpr int A_BYTES = A::S::BYTES, STAGE = A_BYTES + B::S::BYTES, LDS = 2 * STAGE;
    static constexpr int TI = BI / 32, TJ = BJ / 32;
};

// Multiplies a row tile with every column tile, and reads tile I of both operands for the half step after: the reads have the MFMAs'
// time before the wait at the end of the same asm block, so that no read is in flight that the compiler does not know of.
#define LIN_ACC2 [c0] "+a"(c[0]), [c1] "+a"(c[1])
#define LIN_ACC4 LIN_ACC2, [c2] "+a"(c[2]), [c3] "+a"(c[3])
#define LIN_ACC8 LIN_ACC4, [c4] "+a"(c[4]), [c5] "+a"(c[5]), [c6] "+a"(c[6]), [c7] "+a"(c[7])
#define LIN_B2 [b0] "v"(b[0]), [b1] "v"(b[1])
#define LIN_B4 LIN_B2, [b2] "v"(b[2]), [b3] "v"(b[3])
#define LIN_B8 LIN_B4, [b4] "v"(b[4]), [b5] "v"(b[5]), [b6] "v"(b[6]), [b7] "v"(b[7])
#define LIN_M2 LIN_MFMA("%[c0]", "%[b0]") LIN_MFMA("%[c1]", "%[b1]")
#define LIN_M4 LIN_M2 LIN_MFMA("%[c2]", "%[b2]") LIN_MFMA("%[c3]", "%[b3]")
#define LIN_M8 LIN_M4 LIN_MFMA("%[c4]", "%[b4]") LIN_MFMA("%[c5]", "%[b5]") LIN_MFMA("%[c6]", "%[b6]") LIN_MFMA("%[c7]", "%[b7]")
#define LIN_WAIT "s_waitcnt lgkmcnt(0)"
#define LIN_BLOCK(M, ACC, B)                                                                                                                   \
    if constexpr (AIN && BIN)                                                                                                              \
            asm volatile(LIN_READ_IN("%[na]", "%[pa]", "%[ao]") LIN_READ_IN("%[nb]", "%[pb]", "%[bo]") M LIN_WAIT                              \
                         : ACC, [na] "=&v"(na.v), [nb] "=&v"(nb.v)                                                                             \
                         : B, [a] "v"(a), [pa] "v"(a_at), [pb] "v"(b_at), [ao] "n"(ao), [bo] "n"(bo) : "memory");                              \
        else if constexpr (AIN)                                                                                                                \
            asm volatile(LIN_READ_IN("%[na]", "%[pa]", "%[ao]") LIN_READ_OUT("%[nl]", "%[nh]", "%[pb]", "%[bo]", "%[bh]") M LIN_WAIT           \
                         : ACC, [na] "=&v"(na.v), [nl] "=&v"(nb.lo), [nh] "=&v"(nb.hi)                                                         \
                         : B, [a] "v"(a), [pa] "v"(a_at), [pb] "v"(b_at), [ao] "n"(ao), [bo] "n"(bo), [bh] "n"(bh) : "memory");                \
        else                                                                                                                                   \
            asm volatile(LIN_READ_OUT("%[al]", "%[ahi]", "%[pa]", "%[ao]", "%[ah]") LIN_READ_OUT("%[nl]", "%[nh]", "%[pb]", "%[bo]", "%[bh]") M LIN_WAIT \
                         : ACC, [al] "=&v"(na.lo), [ahi] "=&v"(na.hi), [nl] "=&v"(nb.lo), [nh] "=&v"(nb.hi)                                    \
                         : B, [a] "v"(a), [pa] "v"(a_at), [pb] "v"(b_at), [ao] "n"(ao), [ah] "n"(ah), [bo] "n"(bo), [bh] "n"(bh) : "memory")
template <typename T, bool AIN, bool BIN, int I, int TJ>
__device__ __forceinline__ void block(floatx4 (&c)[TJ], const Frag<AIN>& fa, const Frag<BIN> (&fb)[TJ], Frag<AIN>& na, Frag<BIN>& nb, int a_at, int b_at) {
    constexpr int ao = T::A::tile_at(I), bo = T::B::tile_at(I), ah = ao + T::A::HALF, bh = bo + T::B::HALF;
    bf16x8 b[TJ];
#pragma unroll
    for (int j = 0; j < TJ; ++j) b[j] = value(fb[j]);
    const bf16x8 a = value(fa);
    if constexpr (TJ == 8) { LIN_BLOCK(LIN_M8, LIN_ACC8, LIN_B8); }
    else if constexpr (TJ == 4) { LIN_BLOCK(LIN_M4, LIN_ACC4, LIN_B4); }
    else { LIN_BLOCK(LIN_M2, LIN_ACC2, LIN_B2); }
}
// One fragment, waited for.
template <int OFF, int>
__device__ __forceinline__ void read_now(Frag<true>& f, int at) { asm volatile(LIN_READ_IN("%0", "%1", "%2") LIN_WAIT : "=&v"(f.v) : "v"(at), "n"(OFF) : "memory"); }
template <int OFF, int HALF>
__device__ __forceinline__ void read_now(Frag<false>& f, int at) {
    asm volatile(LIN_READ_OUT("%0", "%1", "%2", "%3", "%4") LIN_WAIT : "=&v"(f.lo), "=&v"(f.hi) : "v"(at), "n"(OFF), "n"(OFF + HALF) : "memory");
}
// A lane's write of an accumulator and the MFMA that reads it, and the other way round, want some cycles between them, which the
// compiler does not see to: it does not know these MFMAs.
template <int TJ>
__device__ __forceinline__ void settle(floatx4 (&c)[TJ]) {
    if constexpr (TJ == 8) asm volatile("s_nop 15\n\ts_nop 15" : LIN_ACC8);
    else if constexpr (TJ == 4) asm volatile("s_nop 15\n\ts_nop 15" : LIN_ACC4);
    else asm volatile("s_nop 15\n\ts_nop 15" : LIN_ACC2);
}

// Eight values of a row, from and to memory: whole (16-byte aligned), or those of the first `n`.
__device__ __forceinline__ void get8(const uint16_t* p, bool whole, int n, float (&v)[8]) {
    if (whole) {
        const u32x4 k = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[2 * e] = __uint_as_float(k[e] << 16); v[2 * e + 1] = __uint_as_float(k[e] & 0xffff0000u); }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < n ? bf2f(p[e]) : 0.0f;
    }
}
__device__ __forceinline__ void get8(const float* p, bool whole, int n, float (&v)[8]) {
    if (whole) {
        const floatx4 a = reinterpret_cast<const floatx4*>(p)[0], b = reinterpret_cast<const floatx4*>(p)[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < n ? p[e] : 0.0f;
    }
}
__device__ __forceinline__ void put8(uint16_t* p, bool whole, int n, const float (&v)[8]) {
    if (whole) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        typedef float floatx2 __attribute__((ext_vector_type(2)));
        u32x4 k;
#pragma unroll
        for (int e = 0; e < 4; ++e) { const floatx2 f = {v[2 * e], v[2 * e + 1]}; k[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2)); }
        *reinterpret_cast<u32x4*>(p) = k;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) if (e < n) p[e] = f2bf(v[e]);
    }
}
__device__ __forceinline__ void put8(float* p, bool whole, int n, const float (&v)[8]) {
    if (whole) {
        reinterpret_cast<floatx4*>(p)[0] = floatx4{v[0], v[1], v[2], v[3]};
        reinterpret_cast<floatx4*>(p)[1] = floatx4{v[4], v[5], v[6], v[7]};
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) if (e < n) p[e] = v[e];
    }
}

// V neighbouring values: 16 bytes or one.
template <typename T, int V>
__device__ __forceinline__ void get_v(const T* p, float (&v)[V]) {
    if constexpr (V == 8) get8(p, true, 8, v);
    else if constexpr (V == 4) { const floatx4 k = *reinterpret_cast<const floatx4*>(p); v[0] = k[0]; v[1] = k[1]; v[2] = k[2]; v[3] = k[3]; }
    else if constexpr (sizeof(T) == 2) v[0] = bf2f(p[0]);
    else v[0] = p[0];
}
template <typename T, int V>
__device__ __forceinline__ void put_v(T* p, const float (&v)[V]) {
    if constexpr (V == 8) put8(p, true, 8, v);
    else if constexpr (V == 4) *reinterpret_cast<floatx4*>(p) = floatx4{v[0], v[1], v[2], v[3]};
    else if constexpr (sizeof(T) == 2) p[0] = f2bf(v[0]);
    else p[0] = v[0];
}

// The tile of a workgroup: consecutive workgroups go to the eight dies in turn, so a die takes a consecutive eighth of the tiles;
// there, `group` row tiles go through the column tiles together.
__device__ __forceinline__ void tile_of(const GemmParams& p, int& ti, int& tj, int& split) {
    const int total = gridDim.x, per = total >> 3, b = blockIdx.x;
    const int id = per > 0 && b < per * 8 ? (b & 7) * per + (b >> 3) : b;
    const int tiles = p.tiles_i * p.tiles_j;
    split = id / tiles;
    const int t = id - split * tiles, span = p.group * p.tiles_j, g = t / span, in = t - g * span;
    const int h = min(p.group, p.tiles_i - g * p.group);
    tj = in / h;
    ti = g * p.group + in - tj * h;
}

// EPI: PART; with B's reduction inner, act of y = act(. + bias) + res; else act of the slope that the sum is multiplied with.
template <int BI, int BJ, bool AIN, bool BIN, int EPI>
__global__ __launch_bounds__(256, BI == 256 ? 1 : BI == 128 ? 2 : 4) void linear_gemm_kernel(const GemmParams p) {
    typedef Shape<BI, BJ, AIN, BIN> T;
    constexpr int TI = T::TI, TJ = T::TJ;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wi = wave >> 1, wj = wave & 1;
    int ti, tj, split;
    tile_of(p, ti, tj, split);
    const int i0 = ti * BI, j0 = tj * BJ;

    typename T::A A;
    typename T::B B;
    A.init(p.a, p.a_size, p.a_ld, i0, p.rows, lane, wave);
    B.init(p.b, p.b_size, p.b_ld, j0, p.cols, lane, wave);
    // this wavefront's quarter
    const int a_frag = A.frag + (AIN ? wi * (BI / 2) * 128 : wi * (BI / 2) * 2);
    const int b_frag = B.frag + (BIN ? wj * (BJ / 2) * 128 : wj * (BJ / 2) * 2);

    // steps of this split; fp32 operands: the six products of their parts one after the other, the small ones first
    const int s0 = split * p.per_split, s1 = min(s0 + p.per_split, p.steps), len = s1 - s0;
    const int total = p.planes == 1 ? len : 6 * len;
    // the next step to be requested: its place in the reduction, the operands' first bytes, and for fp32 which parts
    int k_next = s0, left = total, pair = 0;
    const char *a_next = A.base + s0 * A.k_bytes, *b_next = B.base + s0 * B.k_bytes;
    const char *const a_first = a_next, *const b_first = b_next;
    if (p.planes != 1) { a_next += p.a_plane; b_next += p.b_plane; }
    // (always as many loads, so that the loop has no branches; past the end they fetch nothing)
    int room = 0;
    unsigned char* to = smem;
    __amdgpu_buffer_rsrc_t ra, rb;
    auto begin_request = [&](int buf) {
        room = left > 0 ? p.K - k_next * BK : 0;
        to = smem + buf * T::STAGE;
        ra = A.resource(a_next);
        rb = B.resource(b_next);
    };
    auto request_one = [&](auto K) {
        constexpr int k = K.value;
        if constexpr (k < T::A::LOADS) A.template load<k>(ra, to, wave, room);
        else B.template load<k - T::A::LOADS>(rb, to + T::A_BYTES, wave, room);
    };
    auto end_request = [&]() {
        --left;
        ++k_next;
        a_next += A.k_bytes;
        b_next += B.k_bytes;
        if (EPI == PART && p.planes != 1 && k_next == s1) {
            // parts (1, 1), (2, 0), (0, 2), (1, 0), (0, 1), (0, 0) of A and B
            constexpr unsigned PA = 1u | 2u << 2 | 0u << 4 | 1u << 6 | 0u << 8 | 0u << 10, PB = 1u | 0u << 2 | 2u << 4 | 0u << 6 | 1u << 8 | 0u << 10;
            ++pair;
            a_next = a_first + (PA >> (2 * pair) & 3u) * p.a_plane;
            b_next = b_first + (PB >> (2 * pair) & 3u) * p.b_plane;
            k_next = s0;
        }
        if (left <= 0) { a_next = a_first; b_next = b_first; }
    };
    auto request = [&](int buf) {
        begin_request(buf);
        each<T::A::LOADS + T::B::LOADS>(request_one);
        end_request();
    };

    floatx4 acc[TI][TJ];
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};

    // two sets of fragments: one is multiplied while the other is read
    Frag<AIN> fa[2][TI];
    Frag<BIN> fb[2][TJ];
    // this wavefront's loads have landed and its LDS reads are done; then all meet
    auto meet = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070);        // vmcnt(0) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    const int lds = (int)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    auto a_at = [&](int buf, int kk) { return lds + buf * T::STAGE + T::A::half_at(a_frag, kk); };
    auto b_at = [&](int buf, int kk) { return lds + buf * T::STAGE + T::A_BYTES + T::B::half_at(b_frag, kk); };

    request(0);
    meet();
    request(1);
    each<TI>([&](auto I) {
        read_now<T::A::tile_at(I.value), T::A::HALF>(fa[0][I.value], a_at(0, 0));
        read_now<T::B::tile_at(I.value), T::B::HALF>(fb[0][I.value], b_at(0, 0));
        settle(acc[I.value]);
    });
    for (int s = 0, buf = 0; s < total; ++s, buf ^= 1) {
        const int a1 = a_at(buf, 1), b1 = b_at(buf, 1), a0 = a_at(buf ^ 1, 0), b0 = b_at(buf ^ 1, 0);
        each<TI>([&](auto I) {
            constexpr int i = I.value;
            block<T, AIN, BIN, i>(acc[i], fa[0][i], fb[0], fa[1][i], fb[1][i], a1, b1);
        });
        meet();                                    // step s + 1 is in the other buffer, and nobody reads this one any more
        begin_request(buf);
        each<TI>([&](auto I) {
            constexpr int i = I.value, n = (T::A::LOADS + T::B::LOADS) / TI;
            each<n>([&](auto K) { request_one(std::integral_constant<int, i * n + K.value>()); });
            block<T, AIN, BIN, i>(acc[i], fa[1][i], fb[1], fa[0][i], fb[0][i], a0, b0);
        });
        end_request();
    }
    each<TI>([&](auto I) { settle(acc[I.value]); });
    // (the loads past the end write zeros into LDS: they are over before the workgroup's LDS is another's)
    __builtin_amdgcn_s_waitcnt(0x0070);

    // results: row i0 + wi * BI / 2 + i * 16 + (lane & 15), eight columns from j0 + wj * BJ / 2 + pair * 32 + (lane >> 4) * 8
    const int row0 = i0 + wi * (BI / 2) + (lane & 15), col0 = j0 + wj * (BJ / 2) + (lane >> 4) * 8;
    each<TJ / 2>([&](auto JP) {
        constexpr int jp = JP.value;
        const int col = col0 + jp * 32, n = p.cols - col;
        if (n <= 0) return;
        const bool whole = p.vectors && n >= 8;
        float bias[8];
        if constexpr (EPI != PART && BIN) {
#pragma unroll
            for (int e = 0; e < 8; ++e) bias[e] = 0.0f;
            if (p.bias) get8((const uint16_t*)p.bias + col, n >= 8, n, bias);
        }
        each<TI>([&](auto I) {
            constexpr int i = I.value;
            const int row = row0 + i * 16;
            if (row >= p.rows) return;
            float v[8], t[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = acc[i][jp * 2 + (e >> 2)][e & 3];
            if constexpr (EPI == PART) {
                put8(p.part + ((int64_t)split * p.rows + row) * p.cols + col, n >= 8 && p.cols % 4 == 0, n, v);
            } else {
                if constexpr (BIN) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] += bias[e];
                    if (p.pre) put8((uint16_t*)p.pre + row * p.pre_ld + col, whole, n, v);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = act_of<EPI>(v[e]);
                    if (p.res) {
                        get8((const uint16_t*)p.res + row * p.res_ld + col, whole, n, t);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] += t[e];
                    }
                } else if constexpr (EPI != PURINE_ACT_NONE) {
                    get8((const uint16_t*)p.slope + row * p.slope_ld + col, whole, n, t);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] *= act_slope<EPI>(t[e]);
                }
                if (p.out_f32) {
                    float* o = (float*)p.out + row * p.out_ld + col;
                    if (p.accumulate) {
                        get8(o, whole, n, t);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] += t[e];
                    }
                    put8(o, whole, n, v);
                } else {
                    uint16_t* o = (uint16_t*)p.out + row * p.out_ld + col;
                    if (p.accumulate) {
                        get8(o, whole, n, t);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] += t[e];
                    }
                    put8(o, whole, n, v);
                }
            }
        });
    });
}

template <int BI, int BJ, bool AIN, bool BIN, int EPI>
hipError_t launch_gemm(const GemmParams& p, hipStream_t st) {
    typedef Shape<BI, BJ, AIN, BIN> T;
    const int64_t grid = (int64_t)p.tiles_i * p.tiles_j * p.splits;
    if (grid < 1 || grid > 0x7fffffff) return hipErrorInvalidValue;
    const auto kernel = &linear_gemm_kernel<BI, BJ, AIN, BIN, EPI>;
    if (T::LDS > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(256), T::LDS, st, p);
    return hipGetLastError();
}

// One tile extent's kernels (linear_gemm_<tile>.hip). act: PART or an activation.
hipError_t gemm_256(const GemmParams& p, bool a_in, bool b_in, int act, hipStream_t st);
hipError_t gemm_128(const GemmParams& p, bool a_in, bool b_in, int act, hipStream_t st);
hipError_t gemm_64(const GemmParams& p, bool a_in, bool b_in, int act, hipStream_t st);

template <int BI, int BJ>
hipError_t gemm_any(const GemmParams& p, bool a_in, bool b_in, int act, hipStream_t st) {
    if (a_in && b_in) {
        switch (act) {
            case PART: return launch_gemm<BI, BJ, true, true, PART>(p, st);
            case PURINE_ACT_NONE: return launch_gemm<BI, BJ, true, true, PURINE_ACT_NONE>(p, st);
            case PURINE_ACT_RELU: return launch_gemm<BI, BJ, true, true, PURINE_ACT_RELU>(p, st);
            case PURINE_ACT_SILU: return launch_gemm<BI, BJ, true, true, PURINE_ACT_SILU>(p, st);
            case PURINE_ACT_GELU: return launch_gemm<BI, BJ, true, true, PURINE_ACT_GELU>(p, st);
            case PURINE_ACT_GELU_TANH: return launch_gemm<BI, BJ, true, true, PURINE_ACT_GELU_TANH>(p, st);
        }
    } else if (a_in) {
        switch (act) {
            case PART: return launch_gemm<BI, BJ, true, false, PART>(p, st);
            case PURINE_ACT_NONE: return launch_gemm<BI, BJ, true, false, PURINE_ACT_NONE>(p, st);
            case PURINE_ACT_RELU: return launch_gemm<BI, BJ, true, false, PURINE_ACT_RELU>(p, st);
            case PURINE_ACT_SILU: return launch_gemm<BI, BJ, true, false, PURINE_ACT_SILU>(p, st);
            case PURINE_ACT_GELU: return launch_gemm<BI, BJ, true, false, PURINE_ACT_GELU>(p, st);
            case PURINE_ACT_GELU_TANH: return launch_gemm<BI, BJ, true, false, PURINE_ACT_GELU_TANH>(p, st);
        }
    } else if (!b_in) {
        return act == PART ? launch_gemm<BI, BJ, false, false, PART>(p, st) : launch_gemm<BI, BJ, false, false, PURINE_ACT_NONE>(p, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace lin
}  // namespace purine
