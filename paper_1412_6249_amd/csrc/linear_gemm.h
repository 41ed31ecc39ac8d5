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
// Bound: the matrix cores at large products, the operands' way through the caches at few rows. us at 8192 x 4096 x 8192 bf16 (0.55 PFLOP), tiles of 256: data
// gradient 370, weight gradient 370 (1.48 PFLOP/s, a library product's rate on this card), forward with GELU, residual and the stored sum 500: a compute unit holds one
// workgroup, so that a tile's epilogue (13 us, 12 more of vector instructions for GELU) is not overlapped. Tiles of 128 take 465 - 480. Operands whose rows are a power of two
// of bytes apart, both with the reduction inner, lose 15% to memory channels.
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
    float* part;                           // [split][rows][part_ld]: rows of whole 16-byte packets
    int part_ld;
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
    unsigned off[LOADS];                   // bytes of this lane's packets from the step's base ...
    unsigned now[LOADS];                   // ... or NOWHERE past the reduction's end
    int k_at;                              // first k of the first packet (IN: of all)
    const char* base;
    const char* end;
    int64_t k_bytes;                       // per step
    int frag;                              // LDS bytes of this lane's first fragment

    __device__ __forceinline__ void init(const char* p, int64_t size, int64_t ld, int first, int limit, int lane, int wave) {
        base = p + (IN ? first * ld * 2 : (int64_t)first * 2);
        end = p + size;
        k_bytes = IN ? BK * 2 : BK * ld * 2;
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const int unit = u * 4 + wave;
            if constexpr (IN) {
                const int row = unit * 8 + (lane >> 3), c = (lane & 7) ^ exchange<DEALT>(row);      // (the same c for every u)
                off[u] = (unsigned)(min(row, limit - first - 1) * ld * 2) + c * 16;      // (rows past the last read it again)
                if (u == 0) k_at = c * 8;
            } else {
                const int k = unit + lane / S::PER_ROW * S::UNITS, c = min(lane % S::PER_ROW, (limit - first - 1) / 8);
                off[u] = (unsigned)(k * ld * 2) + c * 16;
                if (u == 0) k_at = k;
            }
            now[u] = off[u];
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
    // only the first `left` elements of a step exist
    __device__ __forceinline__ void mask(int left) {
#pragma unroll
        for (int u = 0; u < LOADS; ++u) now[u] = k_at + (IN ? 0 : 4 * u) < left ? off[u] : NOWHERE;
    }
    __device__ __forceinline__ u32x4 resource(const char* at) const {
        const int64_t room = end - at;
        const uint64_t p = (uint64_t)(uintptr_t)at;
        return u32x4{(uint32_t)p, (uint32_t)(p >> 32) & 0xffffu, room < 0x7fffffff ? (uint32_t)room : 0x7fffffffu, 0x00020000u};
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
#define LIN_WAIT "s_waitcnt lgkmcnt(0)"

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
    static constexpr int A_BYTES = A::S::BYTES, STAGE = A_BYTES + B::S::BYTES;
    static constexpr int TI = BI / 32, TJ = BJ / 32;
};

// One asm block multiplies two row tiles from I on with every column tile. Between its MFMAs, in whose 16 cycles other instructions issue for nothing,
// it reads two tiles of both operands for the half step after, and (LOAD) requests a part of a later step's tiles. The reads have
// the remaining MFMAs' time before the wait at the block's end, so that no read is in flight that the compiler does not know of;
// the requests fill no register, and meet() waits for them. (8192 x 4096 x 8192 with these in front of the MFMAs instead: data gradient 401 us,
// with a block for each row tile besides: LDS reads take longer than 128 cycles beside three other wavefronts'.)
#define LIN_C2(N, R) [N##0] "+a"(c[R][0]), [N##1] "+a"(c[R][1])
#define LIN_C4(N, R) LIN_C2(N, R), [N##2] "+a"(c[R][2]), [N##3] "+a"(c[R][3])
#define LIN_C8(N, R) LIN_C4(N, R), [N##4] "+a"(c[R][4]), [N##5] "+a"(c[R][5]), [N##6] "+a"(c[R][6]), [N##7] "+a"(c[R][7])
#define LIN_B2() [b0] "v"(b[0]), [b1] "v"(b[1])
#define LIN_B4() LIN_B2(), [b2] "v"(b[2]), [b3] "v"(b[3])
#define LIN_B8() LIN_B4(), [b4] "v"(b[4]), [b5] "v"(b[5]), [b6] "v"(b[6]), [b7] "v"(b[7])
#define LIN_M(N, J, A) "v_mfma_f32_16x16x32_bf16 %[" #N #J "], %[b" #J "], %[" #A "], %[" #N #J "]\n\t"
// a request: where in LDS, an instruction between, the load
#define LIN_TO(K) "s_mov_b32 m0, %[m" #K "]\n\t"
#define LIN_GET(K) "buffer_load_dwordx4 %[v" #K "], %[r" #K "], 0 offen lds\n\t"
#define LIN_NO(K) ""
// the MFMAs of a block of 2 x 8, 2 x 4 or 2 x 2 tiles, with the reads R0..R3 and the requests
#define LIN_SEQ8(R0, R1, R2, R3, T, G) LIN_M(c, 0, a0) R0 LIN_M(c, 1, a0) R1 LIN_M(c, 2, a0) R2 LIN_M(c, 3, a0) R3 T(0) LIN_M(c, 4, a0) G(0) LIN_M(c, 5, a0) T(1) \
    LIN_M(c, 6, a0) G(1) LIN_M(c, 7, a0) T(2) LIN_M(d, 0, a1) G(2) LIN_M(d, 1, a1) T(3) LIN_M(d, 2, a1) G(3) LIN_M(d, 3, a1) LIN_M(d, 4, a1) LIN_M(d, 5, a1)     \
    LIN_M(d, 6, a1) LIN_M(d, 7, a1)
#define LIN_SEQ4(R0, R1, R2, R3, T, G) LIN_M(c, 0, a0) R0 R1 LIN_M(c, 1, a0) R2 R3 T(0) LIN_M(c, 2, a0) G(0) T(1) LIN_M(c, 3, a0) G(1) T(2) LIN_M(d, 0, a1) G(2) T(3) \
    LIN_M(d, 1, a1) G(3) LIN_M(d, 2, a1) LIN_M(d, 3, a1)
#define LIN_SEQ2(R0, R1, R2, R3, T, G) R0 R1 R2 R3 T(0) LIN_M(c, 0, a0) G(0) T(1) LIN_M(c, 1, a0) G(1) T(2) LIN_M(d, 0, a1) G(2) T(3) LIN_M(d, 1, a1) G(3)
// operand X (a or b), tile number R of the block: reading it, what it is read to, where from
#define LIN_IN(X, R) LIN_READ_IN("%[n" #X #R "]", "%[p" #X "]", "%[o" #X #R "]")
#define LIN_OUT(X, R) LIN_READ_OUT("%[n" #X #R "]", "%[h" #X #R "]", "%[p" #X "]", "%[o" #X #R "]", "%[q" #X #R "]")
#define LIN_IN_D(X, R, F) [n##X##R] "=&v"(F[I + R].v)
#define LIN_OUT_D(X, R, F) [n##X##R] "=&v"(F[I + R].lo), [h##X##R] "=&v"(F[I + R].hi)
#define LIN_IN_O(X, O, R) [o##X##R] "n"(O::tile_at(I + R))
#define LIN_OUT_O(X, O, R) [o##X##R] "n"(O::tile_at(I + R)), [q##X##R] "n"(O::tile_at(I + R) + O::HALF)
#define LIN_REQ(K) [m##K] "s"(q[K].to), [v##K] "v"(q[K].off), [r##K] "s"(q[K].from)
#define LIN_ASM(X, Y, SEQ, C, B)                                                                                                               \
    if constexpr (LOAD)                                                                                                                        \
        asm volatile(SEQ(LIN_##X(a, 0), LIN_##Y(b, 0), LIN_##X(a, 1), LIN_##Y(b, 1), LIN_TO, LIN_GET) LIN_WAIT                                 \
                     : C(c, I), C(d, I + 1), LIN_##X##_D(a, 0, na), LIN_##X##_D(a, 1, na), LIN_##Y##_D(b, 0, nb), LIN_##Y##_D(b, 1, nb)        \
                     : B(), [a0] "v"(a[0]), [a1] "v"(a[1]), [pa] "v"(a_at), [pb] "v"(b_at), LIN_##X##_O(a, A, 0), LIN_##X##_O(a, A, 1),          \
                       LIN_##Y##_O(b, O, 0), LIN_##Y##_O(b, O, 1), LIN_REQ(0), LIN_REQ(1), LIN_REQ(2), LIN_REQ(3) : "memory");           \
    else                                                                                                                                       \
        asm volatile(SEQ(LIN_##X(a, 0), LIN_##Y(b, 0), LIN_##X(a, 1), LIN_##Y(b, 1), LIN_NO, LIN_NO) LIN_WAIT                                  \
                     : C(c, I), C(d, I + 1), LIN_##X##_D(a, 0, na), LIN_##X##_D(a, 1, na), LIN_##Y##_D(b, 0, nb), LIN_##Y##_D(b, 1, nb)        \
                     : B(), [a0] "v"(a[0]), [a1] "v"(a[1]), [pa] "v"(a_at), [pb] "v"(b_at), LIN_##X##_O(a, A, 0), LIN_##X##_O(a, A, 1),          \
                       LIN_##Y##_O(b, O, 0), LIN_##Y##_O(b, O, 1) : "memory")
#define LIN_BLOCK(SEQ, C, B)                                      \
    if constexpr (AIN && BIN) { LIN_ASM(IN, IN, SEQ, C, B); }     \
    else if constexpr (AIN) { LIN_ASM(IN, OUT, SEQ, C, B); }      \
    else { LIN_ASM(OUT, OUT, SEQ, C, B); }

// A 1024-byte load: LDS address, this lane's offset, the buffer. (M0 is the asm blocks' own here. The compiler reserves it and
// warns of a clobber; that nothing else in these kernels uses it is tested on the code that it made.)
struct Request { int to; unsigned off; u32x4 from; };
__device__ __forceinline__ void request_now(const Request& q) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(q.to), "v"(q.off), "s"(q.from) : "memory");
}

template <typename T, bool AIN, bool BIN, bool LOAD, int I, int TI, int TJ>
__device__ __forceinline__ void block(floatx4 (&c)[TI][TJ], const Frag<AIN> (&fa)[TI], const Frag<BIN> (&fb)[TJ], Frag<AIN> (&na)[TI], Frag<BIN> (&nb)[TJ], int a_at,
                                      int b_at, const Request (&q)[4]) {
    typedef typename T::A A;
    typedef typename T::B O;
    bf16x8 b[TJ];
#pragma unroll
    for (int j = 0; j < TJ; ++j) b[j] = value(fb[j]);
    const bf16x8 a[2] = {value(fa[I]), value(fa[I + 1])};
    if constexpr (TJ == 8) { LIN_BLOCK(LIN_SEQ8, LIN_C8, LIN_B8) }
    else if constexpr (TJ == 4) { LIN_BLOCK(LIN_SEQ4, LIN_C4, LIN_B4) }
    else { LIN_BLOCK(LIN_SEQ2, LIN_C2, LIN_B2) }
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
template <int I, int TI, int TJ>
__device__ __forceinline__ void settle(floatx4 (&c)[TI][TJ]) {
    if constexpr (TJ == 8) asm volatile("s_nop 15\n\ts_nop 15" : LIN_C8(c, I));
    else if constexpr (TJ == 4) asm volatile("s_nop 15\n\ts_nop 15" : LIN_C4(c, I));
    else asm volatile("s_nop 15\n\ts_nop 15" : LIN_C2(c, I));
}

__device__ __forceinline__ void widen8(const u32x4& k, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[2 * e] = __uint_as_float(k[e] << 16); v[2 * e + 1] = __uint_as_float(k[e] & 0xffff0000u); }
}
// Eight values of a row, from and to memory: whole (16-byte aligned), or those of the first `n`.
__device__ __forceinline__ void get8(const uint16_t* p, bool whole, int n, float (&v)[8]) {
    if (whole) {
        widen8(*reinterpret_cast<const u32x4*>(p), v);
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
__device__ __forceinline__ u32x4 pack8(const float (&v)[8]) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    typedef float floatx2 __attribute__((ext_vector_type(2)));
    u32x4 k;
#pragma unroll
    for (int e = 0; e < 4; ++e) { const floatx2 f = {v[2 * e], v[2 * e + 1]}; k[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2)); }
    return k;
}
__device__ __forceinline__ void put8(uint16_t* p, bool whole, int n, const float (&v)[8]) {
    if (whole) {
        *reinterpret_cast<u32x4*>(p) = pack8(v);
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
// BUFS: steps in LDS, all but the one in use on their way.
template <int BI, int BJ, int BUFS, bool AIN, bool BIN, int EPI>
__global__ __launch_bounds__(256, BI * BUFS > 256 ? 1 : BI * BUFS > 128 ? 2 : 4) void linear_gemm_kernel(const GemmParams p) {
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
    const int lds = (int)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    constexpr int LOADS = T::A::LOADS + T::B::LOADS;
    // (always as many loads; past the end they fetch nothing)
    int to = 0;
    bool masked = false;
    u32x4 ra, rb;
    auto begin_request = [&](int buf) {
        const int room = left > 0 ? p.K - k_next * BK : 0;
        if (room < BK || masked) {
            A.mask(room);
            B.mask(room);
            masked = room < BK;
        }
        to = lds + buf * T::STAGE;
        ra = A.resource(a_next);
        rb = B.resource(b_next);
    };
    auto request_of = [&](auto K) {
        constexpr int k = K.value;
        if constexpr (k < T::A::LOADS) return Request{to + (k * 4 + wave) * T::A::S::UNIT, A.now[k], ra};
        else return Request{to + T::A_BYTES + ((k - T::A::LOADS) * 4 + wave) * T::B::S::UNIT, B.now[k - T::A::LOADS], rb};
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
        each<LOADS>([&](auto K) { request_now(request_of(K)); });
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
    // this wavefront's loads have landed, all but those of the `YOUNGER` last steps, and its LDS reads are done; then all meet
    auto meet = [&](auto YOUNGER) {
        constexpr int n = decltype(YOUNGER)::value * LOADS;
        static_assert(n < 64, "the counter's range");
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070 | (n & 15) | (n >> 4) << 14);        // vmcnt(n) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    typedef std::integral_constant<int, 0> None;
    auto a_at = [&](int buf, int kk) { return lds + buf * T::STAGE + T::A::half_at(a_frag, kk); };
    auto b_at = [&](int buf, int kk) { return lds + buf * T::STAGE + T::A_BYTES + T::B::half_at(b_frag, kk); };

    each<BUFS>([&](auto B_) { request(B_.value); });
    meet(std::integral_constant<int, BUFS - 1>());
    each<TI>([&](auto I) {
        read_now<T::A::tile_at(I.value), T::A::HALF>(fa[0][I.value], a_at(0, 0));
        read_now<T::B::tile_at(I.value), T::B::HALF>(fb[0][I.value], b_at(0, 0));
        settle<I.value>(acc);
    });
    for (int s = 0, buf = 0; s < total; ++s) {
        const int other = buf + 1 == BUFS ? 0 : buf + 1;
        const int a1 = a_at(buf, 1), b1 = b_at(buf, 1), a0 = a_at(other, 0), b0 = b_at(other, 0);
        const Request none[4] = {};
        each<TI / 2>([&](auto I) { block<T, AIN, BIN, false, 2 * I.value>(acc, fa[0], fb[0], fa[1], fb[1], a1, b1, none); });
        meet(std::integral_constant<int, BUFS - 2>());     // step s + 1 is in the next buffer, and nobody reads this one any more
        begin_request(buf);
        each<TI / 2>([&](auto I) {
            constexpr int i = 4 * I.value;
            static_assert(LOADS == TI / 2 * 4, "four requests in every block");
            const Request q[4] = {request_of(std::integral_constant<int, i>()), request_of(std::integral_constant<int, i + 1>()),
                                  request_of(std::integral_constant<int, i + 2>()), request_of(std::integral_constant<int, i + 3>())};
            block<T, AIN, BIN, true, 2 * I.value>(acc, fa[1], fb[1], fa[0], fb[0], a0, b0, q);
        });
        end_request();
        buf = other;
    }
    each<TI>([&](auto I) { settle<I.value>(acc); });
    meet(None());                                  // (the loads past the end wrote zeros) LDS is free

    // Results: through LDS into rows, so that a lane has eight columns of one row and a few lanes whole lines of memory. The loop over them is a
    // loop: unrolled over the accumulators, every tile fetched 40 KB of instructions anew (22 - 44 us a tile).
    constexpr int WJ = BJ / 2, PACKS = WJ / 8, ROWS = (TI < 4 ? TI : 4) * 16, ITEMS = ROWS * PACKS / 64, BATCH = ITEMS < 4 ? ITEMS : 4;
    unsigned char* const mine = smem + wave * (ROWS * WJ * 4);
    auto cell = [&](int row, int chunk) { return reinterpret_cast<floatx4*>(mine + row * (WJ * 4) + ((chunk ^ (row & 7)) * 16)); };
    const int col = j0 + wj * WJ + lane % PACKS * 8, n = p.cols - col;
    const bool inside = p.vectors && j0 + BJ <= p.cols;        // every lane's eight columns exist and are 16 bytes
    float bias[8];
    if constexpr (EPI != PART && BIN) {
#pragma unroll
        for (int e = 0; e < 8; ++e) bias[e] = 0.0f;
        if (p.bias && n > 0) get8((const uint16_t*)p.bias + col, n >= 8, n, bias);
    }
    // what is read from memory besides the sums: the residual, or what the slope is taken of
    const uint16_t* const other = (const uint16_t*)(BIN ? p.res : p.slope);
    const int64_t other_ld = BIN ? p.res_ld : p.slope_ld;
    const bool reads = EPI != PART && (BIN ? p.res != nullptr : EPI != PURINE_ACT_NONE);
    auto combine = [&](float (&v)[8], const float (&t)[8], float (&pre)[8]) {
        if constexpr (EPI != PART && BIN) {
#pragma unroll
            for (int e = 0; e < 8; ++e) { pre[e] = v[e] + bias[e]; v[e] = act_of<EPI, false>(pre[e]); }
            if (reads)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += t[e];
        } else if constexpr (EPI != PART && EPI != PURINE_ACT_NONE) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= act_slope<EPI, false>(t[e]);
        }
    };
    each<TI * 16 / ROWS>([&](auto H) {
        constexpr int h = H.value;
        asm volatile("" ::: "memory");             // (a wavefront's LDS operations are carried out in order)
        each<ROWS / 16>([&](auto I) {
            each<TJ>([&](auto J) {
                *cell(I.value * 16 + (lane & 15), J.value / 2 * 8 + (lane >> 4) * 2 + J.value % 2) = acc[h * (ROWS / 16) + I.value][J.value];
            });
        });
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
        const int first = i0 + wi * (BI / 2) + h * ROWS;
        auto item = [&](int k, float (&v)[8]) {
            const int r = k * (64 / PACKS) + lane / PACKS, c = lane % PACKS * 2;
            const floatx4 x = *cell(r, c), y = *cell(r, c + 1);
#pragma unroll
            for (int e = 0; e < 4; ++e) { v[e] = x[e]; v[4 + e] = y[e]; }
            return first + r;
        };
        if (EPI != PART && inside && !p.out_f32) {
            // everything that is read is asked for before any of it is used, without a branch between (rows past the last read it)
#pragma unroll 1
            for (int it = 0; it < ITEMS; it += BATCH) {
                float v[BATCH][8];
                u32x4 t[BATCH], o[BATCH];
                int row[BATCH];
#pragma unroll
                for (int u = 0; u < BATCH; ++u) row[u] = first + (it + u) * (64 / PACKS) + lane / PACKS;
                if (reads)
#pragma unroll
                    for (int u = 0; u < BATCH; ++u) t[u] = *reinterpret_cast<const u32x4*>(other + min(row[u], p.rows - 1) * other_ld + col);
                if (p.accumulate)
#pragma unroll
                    for (int u = 0; u < BATCH; ++u) o[u] = *reinterpret_cast<const u32x4*>((const uint16_t*)p.out + min(row[u], p.rows - 1) * p.out_ld + col);
#pragma unroll
                for (int u = 0; u < BATCH; ++u) item(it + u, v[u]);
#pragma unroll
                for (int u = 0; u < BATCH; ++u) {
                    float w[8], pre[8];
                    if (reads) widen8(t[u], w);
                    combine(v[u], w, pre);
                    if (p.accumulate) {
                        widen8(o[u], w);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[u][e] += w[e];
                    }
                    if (row[u] < p.rows) {
                        if (BIN && p.pre) put8((uint16_t*)p.pre + row[u] * p.pre_ld + col, true, 8, pre);
                        put8((uint16_t*)p.out + row[u] * p.out_ld + col, true, 8, v[u]);
                    }
                }
            }
        } else {
            const bool whole = n >= 8 && (EPI == PART || p.vectors);
#pragma unroll 1
            for (int it = 0; it < ITEMS; ++it) {
                float v[8], t[8], pre[8];
                const int row = item(it, v);
                if (row >= p.rows || n <= 0) continue;
                if constexpr (EPI == PART) {
                    put8(p.part + ((int64_t)split * p.rows + row) * p.part_ld + col, whole, n, v);
                } else {
                    if (reads) get8(other + row * other_ld + col, whole, n, t);
                    combine(v, t, pre);
                    if (BIN && p.pre) put8((uint16_t*)p.pre + row * p.pre_ld + col, whole, n, pre);
                    if (p.accumulate) {
                        if (p.out_f32) get8((const float*)p.out + row * p.out_ld + col, whole, n, t);
                        else get8((const uint16_t*)p.out + row * p.out_ld + col, whole, n, t);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] += t[e];
                    }
                    if (p.out_f32) put8((float*)p.out + row * p.out_ld + col, whole, n, v);
                    else put8((uint16_t*)p.out + row * p.out_ld + col, whole, n, v);
                }
            }
        }
    });
}

template <int BI, int BJ, int BUFS, bool AIN, bool BIN, int EPI>
hipError_t launch_gemm(const GemmParams& p, hipStream_t st) {
    constexpr int LDS = Shape<BI, BJ, AIN, BIN>::STAGE * BUFS;
    const int64_t grid = (int64_t)p.tiles_i * p.tiles_j * p.splits;
    if (grid < 1 || grid > 0x7fffffff) return hipErrorInvalidValue;
    const auto kernel = &linear_gemm_kernel<BI, BJ, BUFS, AIN, BIN, EPI>;
    if (LDS > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(256), LDS, st, p);
    return hipGetLastError();
}

// One tile extent's kernels, with two steps in LDS or four (linear_gemm_<tile>_<steps>.hip). act: PART or an activation.
hipError_t gemm_256_2(const GemmParams& p, bool a_in, bool b_in, int act, hipStream_t st);
hipError_t gemm_128_2(const GemmParams& p, bool a_in, bool b_in, int act, hipStream_t st);
hipError_t gemm_128_4(const GemmParams& p, bool a_in, bool b_in, int act, hipStream_t st);
hipError_t gemm_64_2(const GemmParams& p, bool a_in, bool b_in, int act, hipStream_t st);
hipError_t gemm_64_4(const GemmParams& p, bool a_in, bool b_in, int act, hipStream_t st);

template <int BI, int BJ, int BUFS>
hipError_t gemm_any(const GemmParams& p, bool a_in, bool b_in, int act, hipStream_t st) {
    if (a_in && b_in) {
        switch (act) {
            case PART: return launch_gemm<BI, BJ, BUFS, true, true, PART>(p, st);
            case PURINE_ACT_NONE: return launch_gemm<BI, BJ, BUFS, true, true, PURINE_ACT_NONE>(p, st);
            case PURINE_ACT_RELU: return launch_gemm<BI, BJ, BUFS, true, true, PURINE_ACT_RELU>(p, st);
            case PURINE_ACT_SILU: return launch_gemm<BI, BJ, BUFS, true, true, PURINE_ACT_SILU>(p, st);
            case PURINE_ACT_GELU: return launch_gemm<BI, BJ, BUFS, true, true, PURINE_ACT_GELU>(p, st);
            case PURINE_ACT_GELU_TANH: return launch_gemm<BI, BJ, BUFS, true, true, PURINE_ACT_GELU_TANH>(p, st);
        }
    } else if (a_in) {
        switch (act) {
            case PART: return launch_gemm<BI, BJ, BUFS, true, false, PART>(p, st);
            case PURINE_ACT_NONE: return launch_gemm<BI, BJ, BUFS, true, false, PURINE_ACT_NONE>(p, st);
            case PURINE_ACT_RELU: return launch_gemm<BI, BJ, BUFS, true, false, PURINE_ACT_RELU>(p, st);
            case PURINE_ACT_SILU: return launch_gemm<BI, BJ, BUFS, true, false, PURINE_ACT_SILU>(p, st);
            case PURINE_ACT_GELU: return launch_gemm<BI, BJ, BUFS, true, false, PURINE_ACT_GELU>(p, st);
            case PURINE_ACT_GELU_TANH: return launch_gemm<BI, BJ, BUFS, true, false, PURINE_ACT_GELU_TANH>(p, st);
        }
    } else if (!b_in) {
        return act == PART ? launch_gemm<BI, BJ, BUFS, false, false, PART>(p, st) : launch_gemm<BI, BJ, BUFS, false, false, PURINE_ACT_NONE>(p, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace lin
}  // namespace purine
