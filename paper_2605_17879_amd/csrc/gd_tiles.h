// Tiled products C[q][p] = sum_k P[p][k] Q[q][k] of matrices whose rows lie along k, 128 bytes of a row (a
// block) at a time: 64 numbers of f16, or 128 codes of 8 bits with a power of two for each row's block.
//
// Sixteen rows of an operand make a fragment of the matrix cores.  Here they are every fourth row: fragment i of a
// group of 64 rows holds rows 4 c + i, lane l row c = l % 16.  So what a lane needs of four fragments lies next to each
// other: the rows' powers of two are the four bytes of a word that the scaled instruction picks from, and of a
// product a lane holds columns 16 (l / 16) + 4 r + i, r, i = 0..3, of the rows 4 (l % 16) + j -- sixteen numbers
// next to each other of a row of C, four next to each other of a row of its transpose: 128 bytes of a row of the transpose by sixteen
// lanes, and with an exchange between four neighbours (below) 128 of a row of C.
//
// Which k a lane's bytes stand for does not matter to a sum as long as both operands agree: the quarter l / 16 of a
// wave takes the 16-byte chunks l / 16 and 4 + l / 16 of a block.
#ifndef GD_TILES_H_
#define GD_TILES_H_

#include <type_traits>
#include <utility>

#include "gd_operators.h"

namespace gd_tiles {

constexpr uint32_t BYTES = 128;                  // of a row in a block

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef gd_f16 f16x8 __attribute__((ext_vector_type(8)));
typedef gd_bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef gd_bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void lds_void;

template <int N, typename F, int... I>
__device__ __forceinline__ void each_of(F&& f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, typename F>
__device__ __forceinline__ void each(F&& f) { each_of<N>(f, std::make_integer_sequence<int, N>{}); }

// A lane's 32 bytes of a row's block.
struct fragment {
    gd_u32x4 h[2];
};

// ---- the two kinds of products ---------------------------------------------------------------

// Numbers of 16 bits.
__device__ __forceinline__ f32x4 multiply_16(f16x8 p, f16x8 q, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(p, q, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 multiply_16(bf16x8 p, bf16x8 q, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(p, q, c, 0, 0, 0); }

// A kind of product is STEPS instructions on a pair of fragments: one after the other on one sum they would wait for each other,
// so that a tile takes a step for all of its sums before the next.
template <typename X8>
struct of_16 {
    static constexpr bool SCALED = false;
    static constexpr int STEPS = 2;
    template <int STEP, int I, int J>
    static __device__ __forceinline__ f32x4 multiply(const fragment& p, const fragment& q, f32x4 c, uint32_t, uint32_t) {
        return multiply_16(__builtin_bit_cast(X8, p.h[STEP]), __builtin_bit_cast(X8, q.h[STEP]), c);
    }
};
typedef of_16<f16x8> of_f16;
typedef of_16<bf16x8> of_bf16;

// Numbers hi + lo of two f16 each, 32 hi and then their 32 lo in a block: lo hi + hi lo + hi hi.  A lane's first chunk of a block is hi, its
// second the lo of the same numbers.
struct of_pairs {
    static constexpr bool SCALED = false;
    static constexpr int STEPS = 3;
    template <int STEP, int I, int J>
    static __device__ __forceinline__ f32x4 multiply(const fragment& p, const fragment& q, f32x4 c, uint32_t, uint32_t) {
        return multiply_16(__builtin_bit_cast(f16x8, p.h[STEP == 0]), __builtin_bit_cast(f16x8, q.h[STEP == 1]), c);
    }
};

// Codes of P and of Q: 0 for e4m3, 1 for e5m2.  Byte I of `pe` is the power of two of the lane's row of P, byte J of `qe`
// that of Q.  The 8-bit matrix cores cut the products of eight neighbouring k toward zero, to multiples of 2^(E - 13), before they
// add them, E the largest sum of two codes' exponents (a subnormal code's is the least of its type); the eights' sums are added in fp32.
// A sum is off by up to 7 * 2^(E - 13) an eight, in the norm by 1.5e-5 for normal numbers and 9e-5 for such of wide range.
template <int P_CODES, int Q_CODES>
struct of_codes {
    static constexpr bool SCALED = true;
    static constexpr int STEPS = 1;
    template <int STEP, int I, int J>
    static __device__ __forceinline__ f32x4 multiply(const fragment& p, const fragment& q, f32x4 c, uint32_t pe, uint32_t qe) {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(__builtin_bit_cast(i32x8, p), __builtin_bit_cast(i32x8, q), c, P_CODES, Q_CODES,
                                                                I, (int)pe, J, (int)qe);
    }
};

// Sixteen scaled instructions, c[i][j] += p[i] q[j], in a piece of assembly: the compiler gives this instruction's sum a
// register apart from the addend's, runs out of runs of eight registers with it, and keeps sums in scratch memory inside the loop
// (a tile of 256 x 256: 365 registers).  The waits stand with it: 2 cycles from a vector instruction's result to its use, 20
// from the last sum to a vector instruction that reads it, which is as long as the matrix cores take to finish.
#define GD_SCALED(c, p, q, low, high) \
    "v_mfma_scale_f32_16x16x128_f8f6f4 %" #c ", %" #p ", %" #q ", %" #c ", %24, %25 op_sel:[" low ",0] op_sel_hi:[" high ",0] cbsz:%26 blgp:%27\n"
template <int P_CODES, int Q_CODES>
__device__ __forceinline__ void multiply_sixteen(f32x4 (&c)[4][4], const fragment (&p)[4], const fragment (&q)[4], uint32_t pe, uint32_t qe) {
    const i32x8 p0 = __builtin_bit_cast(i32x8, p[0]), p1 = __builtin_bit_cast(i32x8, p[1]), p2 = __builtin_bit_cast(i32x8, p[2]), p3 = __builtin_bit_cast(i32x8, p[3]);
    const i32x8 q0 = __builtin_bit_cast(i32x8, q[0]), q1 = __builtin_bit_cast(i32x8, q[1]), q2 = __builtin_bit_cast(i32x8, q[2]), q3 = __builtin_bit_cast(i32x8, q[3]);
    asm volatile("s_nop 1\n"
            GD_SCALED(0, 16, 20, "0,0", "0,0")
            GD_SCALED(1, 16, 21, "0,1", "0,0")
            GD_SCALED(2, 16, 22, "0,0", "0,1")
            GD_SCALED(3, 16, 23, "0,1", "0,1")
            GD_SCALED(4, 17, 20, "1,0", "0,0")
            GD_SCALED(5, 17, 21, "1,1", "0,0")
            GD_SCALED(6, 17, 22, "1,0", "0,1")
            GD_SCALED(7, 17, 23, "1,1", "0,1")
            GD_SCALED(8, 18, 20, "0,0", "1,0")
            GD_SCALED(9, 18, 21, "0,1", "1,0")
            GD_SCALED(10, 18, 22, "0,0", "1,1")
            GD_SCALED(11, 18, 23, "0,1", "1,1")
            GD_SCALED(12, 19, 20, "1,0", "1,0")
            GD_SCALED(13, 19, 21, "1,1", "1,0")
            GD_SCALED(14, 19, 22, "1,0", "1,1")
            GD_SCALED(15, 19, 23, "1,1", "1,1")
                 "s_nop 15\ns_nop 3"
                 : "+v"(c[0][0]), "+v"(c[0][1]), "+v"(c[0][2]), "+v"(c[0][3]), "+v"(c[1][0]), "+v"(c[1][1]), "+v"(c[1][2]), "+v"(c[1][3]),
                   "+v"(c[2][0]), "+v"(c[2][1]), "+v"(c[2][2]), "+v"(c[2][3]), "+v"(c[3][0]), "+v"(c[3][1]), "+v"(c[3][2]), "+v"(c[3][3])
                 : "v"(p0), "v"(p1), "v"(p2), "v"(p3), "v"(q0), "v"(q1), "v"(q2), "v"(q3), "v"(pe), "v"(qe), "n"(P_CODES), "n"(Q_CODES));
}
#undef GD_SCALED

// Eight codes, from byte `from` of a fragment's half on, times 2^(e - 127): exact in bf16 (but for what lies below 2^-126).
template <int CODES>
__device__ __forceinline__ bf16x8 numbers_of(uint32_t lo, uint32_t hi, float two) {
    union {
        bf16x2 two_of[4];
        bf16x8 x;
    } u;
    if constexpr (CODES == 0) {
        u.two_of[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, two, false);
        u.two_of[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, two, true);
        u.two_of[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, two, false);
        u.two_of[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, two, true);
    } else {
        u.two_of[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, two, false);
        u.two_of[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, two, true);
        u.two_of[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, two, false);
        u.two_of[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, two, true);
    }
    return u.x;
}
// 2^(e - 127) as a conversion takes it, which reads the exponent's bits alone: those of 0 are 2^-127 there, as in the scaled instruction.
// NaN for 255, of any code.
__device__ __forceinline__ float power_of(uint32_t e) { return __builtin_bit_cast(float, e == 255 ? 0x7FC00000u : e << 23); }

// The same products by the 16-bit matrix cores, with sums of fp32.
template <int P_CODES, int Q_CODES>
struct of_codes_in_16 {
    static constexpr bool SCALED = true;
    template <int FP, int FQ>
    static __device__ __forceinline__ void multiply_all(const fragment (&p)[FP], const fragment (&q)[FQ], f32x4 (&acc)[FP][FQ], uint32_t pe, uint32_t qe) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {                // eight codes of each row at a time
            bf16x8 x[FP];
#pragma unroll
            for (int i = 0; i < FP; ++i) x[i] = numbers_of<P_CODES>(p[i].h[w / 2][w % 2 * 2], p[i].h[w / 2][w % 2 * 2 + 1], power_of(pe >> (8 * i) & 255));
#pragma unroll
            for (int j = 0; j < FQ; ++j) {
                const bf16x8 y = numbers_of<Q_CODES>(q[j].h[w / 2][w % 2 * 2], q[j].h[w / 2][w % 2 * 2 + 1], power_of(qe >> (8 * j) & 255));
#pragma unroll
                for (int i = 0; i < FP; ++i) acc[i][j] = multiply_16(x[i], y, acc[i][j]);
            }
        }
    }
};

template <typename MUL, int FP, int FQ>
__device__ __forceinline__ void multiply_all(const fragment (&p)[FP], const fragment (&q)[FQ], f32x4 (&acc)[FP][FQ], uint32_t pe, uint32_t qe) {
    each<MUL::STEPS>([&](auto of_step) {
        each<FP>([&](auto of_p) {
            each<FQ>([&](auto of_q) {
                constexpr int s = decltype(of_step)::value, i = decltype(of_p)::value, j = decltype(of_q)::value;
                acc[i][j] = MUL::template multiply<s, i, j>(p[i], q[j], acc[i][j], pe, qe);
            });
        });
    });
}

template <typename MUL> struct sixteen {
    static __device__ __forceinline__ void multiply(f32x4 (&c)[4][4], const fragment (&p)[4], const fragment (&q)[4], uint32_t pe, uint32_t qe) {
        multiply_all<MUL>(p, q, c, pe, qe);
    }
};
template <int P, int Q> struct sixteen<of_codes<P, Q>> {
    static __device__ __forceinline__ void multiply(f32x4 (&c)[4][4], const fragment (&p)[4], const fragment (&q)[4], uint32_t pe, uint32_t qe) {
        multiply_sixteen<P, Q>(c, p, q, pe, qe);
    }
};

template <typename MUL> struct requires_all : std::false_type {};
template <int P, int Q> struct requires_all<of_codes_in_16<P, Q>> : std::true_type {};

// ---- operands ----------------------------------------------------------------------------------

struct operand {
    const uint8_t* p;
    uint64_t pitch;        // bytes between rows, a multiple of 16
    uint32_t rows;         // that are there, at least one
    uint32_t row_bytes;    // that a row has along k, up to whole chunks of 16, at least one chunk
    const uint8_t* exp;    // powers of two, [block][row], 4-byte aligned, or unused
    uint64_t exp_pitch;    // a multiple of 4
};

struct passage {
    uint32_t blocks;       // of k
    uint32_t ends;         // bytes of the last block that are there; 0: all
};

// Of a row's chunk in the last block, of which `ends` bytes are there: zeros behind them.
__device__ __forceinline__ void cut(gd_u32x4& x, uint32_t ends, uint32_t chunk) {
    const int left = (int)ends - (int)(chunk * 16);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int bytes = left - 4 * w;
        x[w] &= bytes >= 4 ? 0xFFFFFFFFu : bytes <= 0 ? 0u : (1u << (8 * bytes)) - 1;
    }
}
__device__ __forceinline__ void cut(fragment& f, uint32_t ends, uint32_t lane) {
#pragma unroll
    for (int h = 0; h < 2; ++h) cut(f.h[h], ends, h * 4 + (lane >> 4));
}

// Bytes from a row on to the end of an operand, at most 2^30, and a pointer, in scalar registers: a buffer's description in
// vector registers would be loaded with in a loop over the lanes.
__device__ __forceinline__ uint32_t left_of(const operand& o, uint32_t row) {
    const uint64_t left = (o.rows - 1 - row) * o.pitch + o.row_bytes;
    return __builtin_amdgcn_readfirstlane(row >= o.rows ? 0u : left >> 30 ? 1u << 30 : (uint32_t)left);
}
// What is left behind `skip` bytes.  (Signed: the difference of unsigned numbers that ends at 0 is a vector instruction.)
__device__ __forceinline__ int behind(uint32_t left, uint32_t skip) { return max((int)left - (int)skip, 0); }
__device__ __forceinline__ const uint8_t* scalar(const uint8_t* p) {
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    return reinterpret_cast<const uint8_t*>((uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(a >> 32)) << 32 |
                                            (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)a));
}

// s_waitcnt operands: all but `n` loads (n below 64); all LDS reads
constexpr int loads_but(int n) { return 0x0F70 | (n & 15) | (n >> 4) << 14; }
constexpr int LDS_READ = 0xC07F;

// Loads of a workgroup of NT lanes that stage ROWS rows of an operand, straight to the LDS.  The rows of a fragment lie
// next to each other there, and chunk k of place r at k ^ (r % 8), so that a read of sixteen rows meets every bank once
// (rows in their order, of which a read takes every fourth, met half of them twice: 8 192 x 8 192 x 8 192 469 us).  What lies behind the last row's last chunk
// comes as zeros (the buffer ends there); behind the end of another row lies the next one, which is cut off where it
// would count.  A lane has one offset, the rest is scalar and does not change from block to block.
template <int ROWS, int NT>
struct stager {
    static constexpr int LOADS = ROWS * 8 / NT, EACH = NT / 8;   // 16 bytes a lane, so many rows a load: 32 or 64
    __amdgpu_buffer_rsrc_t from[LOADS];           // a load's rows to the end of the operand
    const uint8_t* base;
    uint64_t pitch;
    uint32_t at, chunk;                           // this lane's chunk of the first block: bytes from base, and which of its row
    uint32_t left[LOADS];                         // bytes from a load's first row to the end, at most 2^30
    uint32_t to;                                  // where the wave's part begins in a buffer

    __device__ __forceinline__ void init(const operand& o, uint32_t first, uint32_t wave) {
        base = scalar(o.p + first * o.pitch);
        pitch = o.pitch;
        chunk = (threadIdx.x ^ (threadIdx.x / 8)) & 7;
        at = (threadIdx.x / 8 % 16 * 4 + threadIdx.x / 128) * (uint32_t)o.pitch + chunk * 16;
        to = wave * 1024;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            left[j] = left_of(o, first + row_of(j));
            from[j] = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base + row_of(j) * pitch), 0, (int)left[j], 0x00020000);
        }
    }
    // The first row of a load: 64 of them are two loads of 256 lanes, fragments 0 and 1, 2 and 3, or one of 512.
    static __device__ __forceinline__ constexpr uint32_t row_of(int j) { return EACH == 64 ? 64 * j : j / 2 * 64 + j % 2 * 2; }
    // The whole block that begins `skip` bytes into the rows.  (An offset beside the lane's own is not held against the buffer's end:
    // that is right for whole blocks, whose chunks are there where the row is.)
    __device__ __forceinline__ void stage(uint8_t* s, uint32_t skip) const {
#pragma unroll
        for (int j = 0; j < LOADS; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from[j], (lds_void*)(s + to + j * NT * 16), 16, at, skip, 0, 0);
    }
    // The last block, of which `ends` bytes are there: through registers, with zeros behind them.  (Every load before these is
    // there behind it too: they return in order.  What is written has to be waited for.)
    __device__ __forceinline__ void stage_end(uint8_t* s, uint32_t t, uint32_t ends) const {
        const uint32_t skip = t * BYTES;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const __amdgpu_buffer_rsrc_t rsrc =
                __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base + skip + row_of(j) * pitch), 0, behind(left[j], skip), 0x00020000);
            gd_u32x4 x = __builtin_bit_cast(gd_u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, 0, 0));
            cut(x, ends, chunk);
            *reinterpret_cast<gd_u32x4*>(s + (j * NT + threadIdx.x) * 16) = x;
        }
    }
};

// The powers of two of a block: P_ROWS bytes, then Q_ROWS, sixteen words a wave.  (A word that begins in front of the
// last row ends behind it: it is aligned, so that it lies in the same line as the row.)
template <int P_ROWS, int Q_ROWS, int NT>
struct exp_stager {
    static_assert(P_ROWS + Q_ROWS == NT, "a byte a lane");
    const uint8_t* base;
    uint64_t pitch;
    uint32_t at;
    __device__ __forceinline__ void init(const operand& p, uint32_t p0, const operand& q, uint32_t q0, uint32_t lane, uint32_t wave) {
        const bool of_q = wave * 64 >= P_ROWS;
        base = scalar(of_q ? q.exp : p.exp);
        pitch = (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(of_q ? q.exp_pitch : p.exp_pitch));
        const uint32_t row = (of_q ? q0 + wave * 64 - P_ROWS : p0 + wave * 64) + (lane & 15) * 4;
        at = min(row, ((of_q ? q.rows : p.rows) - 1) & ~3u);
    }
    __device__ __forceinline__ void stage(uint8_t* s, uint32_t t, uint32_t lane, uint32_t wave) const {
        __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base + t * pitch), 0, 0xFFFFFFFF, 0x00020000);
        if (lane < 16) __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)(s + wave * 64), 4, at, 0, 0, 0);
    }
};

// Fragment i of the 64 rows from `row` on.
__device__ __forceinline__ fragment read_fragment(const uint8_t* s, uint32_t row, int i, uint32_t lane) {
    const uint32_t r = row + 16 * i + (lane & 15);
    fragment f;
#pragma unroll
    for (int h = 0; h < 2; ++h) f.h[h] = *reinterpret_cast<const gd_u32x4*>(s + r * BYTES + (((h * 4 + (lane >> 4)) ^ (lane & 7)) * 16));
    return f;
}

// ---- tiles -------------------------------------------------------------------------------------

// 256 x 256 by eight waves, one workgroup a CU, two waves a SIMD that take turns: while the waves of one
// group multiply, those of the other read their operands from the LDS, and a barrier changes the roles.  A block takes
// two turns of a wave: Q and the upper half of P's rows, then the lower half.  The buffers of Q and of P's upper
// half are free again behind the first turn and are filled for the block after the next at once, those of the lower
// half behind the second: every load has three turns of both groups, one and a half blocks, to arrive.
//
//   turn          g0 reads    g1 reads     loads issued (each group in its reading turn)
//   4 t           Q, upper    (lower t-1)  g0: lower t+1
//   4 t + 1                   Q, upper     g1: lower t+1
//   4 t + 2       lower                    g0: Q, upper t+2
//   4 t + 3                   lower        g1: Q, upper t+2
//
// What is read in turns 4 t and on was issued before the latest loads of one block; the wait stands before the barrier in
// front of the even turns, which g0 reaches multiplying and g1 reading.
//
// The matrix cores bound it, and their clock, which falls under this load: 8 192 x 8 192 x 8 192 of codes 404 to 435 us, 2 530 to 2 720 TFLOP/s (the
// library's plain 8-bit product 2 840 to 3 040, the instruction alone 3 200), of bf16 700 to 855, 1 290 to 1 570 (library 1 580).  A tile's ends, first
// loads and C, are some 8 us, during which the matrix cores rest: 8 192 x 8 192 x 1 024 of codes 77 to 84 us, 1 640 to 1 780 TFLOP/s.
template <typename MUL>
struct large_tile {
    static constexpr int BP = 256, BQ = 256, WP = 2, WQ = 4, NT = 512, FP = 8, FQ = 4;
    // The first of the 64 rows of P that fragments 4 g .. 4 g + 3 of a wave hold, and of Q.
    static __device__ __forceinline__ uint32_t p_of(uint32_t wave, int g) { return g * 128 + (wave / WQ) * 64; }
    static __device__ __forceinline__ uint32_t q_of(uint32_t wave) { return (wave % WQ) * 64; }

    static __device__ __forceinline__ void run(const operand& op, const operand& oq, uint32_t p0, uint32_t q0, const passage& way,
                                               f32x4 (&acc)[FP][FQ]) {
        __shared__ __attribute__((aligned(16))) uint8_t up0[128 * BYTES], low0[128 * BYTES], sq0[BQ * BYTES];
        __shared__ __attribute__((aligned(16))) uint8_t up1[128 * BYTES], low1[128 * BYTES], sq1[BQ * BYTES];
        __shared__ __attribute__((aligned(16))) uint8_t se0[BP + BQ], se1[BP + BQ];
        const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        const uint32_t wp = wave / WQ, group = wp;           // (waves w and w + 4 share a SIMD)
        const uint32_t blocks = way.blocks;
        if (blocks == 0) return;
        constexpr int ALL = MUL::SCALED ? 9 : 8;             // loads of a wave in a block, two of them the lower half's
        stager<128, NT> lu, ll;
        stager<BQ, NT> lq;
        exp_stager<BP, BQ, NT> le;
        lu.init(op, p0, wave);
        ll.init(op, p0 + 128, wave);
        lq.init(oq, q0, wave);
        if (MUL::SCALED) le.init(op, p0, oq, q0, lane, wave);
        fragment fp[4], fq[FQ];
        uint32_t eu = 0, el = 0, eq = 0;
        // `inner`: this is not the last block
        auto stage_low = [&](bool inner, uint8_t* low, uint32_t t) {
            if (MUL::SCALED && !inner && way.ends != 0 && t + 1 == blocks) ll.stage_end(low, t, way.ends);
            else ll.stage(low, t * BYTES);
        };
        auto stage_up = [&](bool inner, uint8_t* up, uint8_t* sq, uint8_t* se, uint32_t t) {
            if (MUL::SCALED) le.stage(se, t, lane, wave);
            if (MUL::SCALED && !inner && way.ends != 0 && t + 1 == blocks) {
                lq.stage_end(sq, t, way.ends);
                lu.stage_end(up, t, way.ends);
            } else {
                lq.stage(sq, t * BYTES);
                lu.stage(up, t * BYTES);
            }
        };
        auto read_p = [&](const uint8_t* s) {
#pragma unroll
            for (int i = 0; i < 4; ++i) fp[i] = read_fragment(s, wp * 64, i, lane);
        };
        // `newer`: how many of the wave's loads were issued behind those that the next turn reads
        auto turn_over = [&](bool wait, uint32_t newer) {
            asm volatile("" ::: "memory");
            if (wait) {
                if (newer == ALL) __builtin_amdgcn_s_waitcnt(loads_but(ALL));
                else if (newer == 2) __builtin_amdgcn_s_waitcnt(loads_but(2));
                else __builtin_amdgcn_s_waitcnt(loads_but(0));
            }
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
        };
        auto multiply_half = [&](f32x4 (&c)[4][FQ], uint32_t e) {
            __builtin_amdgcn_s_setprio(1);
            sixteen<MUL>::multiply(c, fp, fq, e, eq);
            __builtin_amdgcn_s_setprio(0);
            __builtin_amdgcn_sched_barrier(0);
        };
        // With `more` three blocks follow at least, and no question is asked.
        auto block = [&](auto more, uint8_t* up, uint8_t* low, uint8_t* sq, uint8_t* se, uint8_t* nlow, uint32_t t) {
            constexpr bool MORE = decltype(more)::value;
            const uint32_t newer_up = MORE || t + 1 < blocks ? ALL : 0, newer_low = MORE || t + 2 < blocks ? ALL : t + 1 < blocks ? 2 : 0;
#pragma unroll
            for (int j = 0; j < FQ; ++j) fq[j] = read_fragment(sq, q_of(wave), j, lane);
            read_p(up);
            if (MUL::SCALED) {
                eu = *reinterpret_cast<const uint32_t*>(se + wp * 64 + 4 * (lane & 15));
                el = *reinterpret_cast<const uint32_t*>(se + 128 + wp * 64 + 4 * (lane & 15));
                eq = *reinterpret_cast<const uint32_t*>(se + BP + q_of(wave) + 4 * (lane & 15));
            }
            if (MORE || t + 1 < blocks) stage_low(MORE, nlow, t + 1);
            __builtin_amdgcn_s_waitcnt(LDS_READ);
            turn_over(group == 1, newer_up);
            multiply_half(*reinterpret_cast<f32x4 (*)[4][FQ]>(&acc[0]), eu);
            turn_over(group == 0, newer_up);
            read_p(low);
            if (MORE || t + 2 < blocks) stage_up(MORE, up, sq, se, t + 2);
            __builtin_amdgcn_s_waitcnt(LDS_READ);
            turn_over(group == 1, newer_low);
            multiply_half(*reinterpret_cast<f32x4 (*)[4][FQ]>(&acc[4]), el);
            turn_over(group == 0, newer_low);
        };
        auto start = [&](uint8_t* up, uint8_t* low, uint8_t* sq, uint8_t* se, uint8_t* nup, uint8_t* nsq, uint8_t* nse) {
            stage_up(false, up, sq, se, 0);
            stage_low(false, low, 0);
            if (blocks > 1) {
                stage_up(false, nup, nsq, nse, 1);
                __builtin_amdgcn_s_waitcnt(loads_but(ALL - 2));
            } else {
                __builtin_amdgcn_s_waitcnt(loads_but(0));
            }
            __builtin_amdgcn_s_waitcnt(LDS_READ);
            turn_over(false, 0);
            if (group == 1) turn_over(false, 0);             // one turn behind
        };
        // blocks go through the buffers in turn and end with the second one
        const std::true_type more;
        const std::false_type last;
        uint32_t t = blocks & 1;
        if (t) {
            start(up1, low1, sq1, se1, up0, sq0, se0);
            block(last, up1, low1, sq1, se1, low0, 0);
        } else {
            start(up0, low0, sq0, se0, up1, sq1, se1);
        }
        for (; t + 4 < blocks; t += 2) {
            block(more, up0, low0, sq0, se0, low1, t);
            block(more, up1, low1, sq1, se1, low0, t + 1);
        }
        for (; t < blocks; t += 2) {
            block(last, up0, low0, sq0, se0, low1, t);
            block(last, up1, low1, sq1, se1, low0, t + 1);
        }
        if (group == 0) turn_over(false, 0);
    }
};

// 128 x 128 by four waves, two workgroups a CU.  A step multiplies one fragment of P by the wave's four of Q; P's are read
// three steps ahead, Q's a block ahead, so that the matrix cores do not wait for the LDS behind the barrier.  The LDS bounds it: each byte of
// it feeds half as many products as in a large tile (an update of a matrix of 4 096 x 4 096 with
// pairs of f16 4.29 ms, with large tiles 3.96).
template <typename MUL>
struct small_tile {
    static constexpr int BP = 128, BQ = 128, WP = 2, WQ = 2, NT = 256, FP = 4, FQ = 4;
    static __device__ __forceinline__ uint32_t p_of(uint32_t wave, int) { return (wave / WQ) * 64; }
    static __device__ __forceinline__ uint32_t q_of(uint32_t wave) { return (wave % WQ) * 64; }

    static __device__ __forceinline__ void run(const operand& op, const operand& oq, uint32_t p0, uint32_t q0, const passage& way,
                                               f32x4 (&acc)[FP][FQ]) {
        __shared__ __attribute__((aligned(16))) uint8_t sp0[BP * BYTES], sq0[BQ * BYTES], se0[BP + BQ];
        __shared__ __attribute__((aligned(16))) uint8_t sp1[BP * BYTES], sq1[BQ * BYTES], se1[BP + BQ];
        const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        const uint32_t blocks = way.blocks;
        if (blocks == 0) return;
        stager<BP, NT> lp;
        stager<BQ, NT> lq;
        exp_stager<BP, BQ, NT> le;
        lp.init(op, p0, wave);
        lq.init(oq, q0, wave);
        if (MUL::SCALED) le.init(op, p0, oq, q0, lane, wave);
        auto stage = [&](bool inner, uint8_t* sp, uint8_t* sq, uint8_t* se, uint32_t t) {
            if (MUL::SCALED) le.stage(se, t, lane, wave);
            if (MUL::SCALED && !inner && way.ends != 0 && t + 1 == blocks) {
                lp.stage_end(sp, t, way.ends);
                lq.stage_end(sq, t, way.ends);
            } else {
                lp.stage(sp, t * BYTES);
                lq.stage(sq, t * BYTES);
            }
        };
        fragment fp[4], fq[2][FQ];
        uint32_t ep[2] = {0, 0}, eq[2] = {0, 0};
        auto read_q = [&](const uint8_t* sq, const uint8_t* se, int b) {
#pragma unroll
            for (int j = 0; j < FQ; ++j) fq[b][j] = read_fragment(sq, q_of(wave), j, lane);
            if (MUL::SCALED) {
                ep[b] = *reinterpret_cast<const uint32_t*>(se + p_of(wave, 0) + 4 * (lane & 15));
                eq[b] = *reinterpret_cast<const uint32_t*>(se + BP + q_of(wave) + 4 * (lane & 15));
            }
        };
        // What every wave has staged is there behind this: the wait for a wave's own loads is written out, a barrier orders
        // only what goes through registers.
        auto staged_by_all = [&]() {
            __builtin_amdgcn_s_waitcnt(loads_but(0));
            __syncthreads();
        };
        // Block t from the buffers of b, then the first fragments of the one behind it from the others: where there is
        // none they are read for nothing.
        auto block = [&](auto b, auto more, uint8_t* sp, uint8_t* sq, uint8_t* se, uint8_t* np, uint8_t* nq, uint8_t* ne, uint32_t t) {
            constexpr bool MORE = decltype(more)::value;
            each<4>([&](auto step) {
                constexpr int i = decltype(step)::value, B = decltype(b)::value;
                if (i == 0) fp[3] = read_fragment(sp, p_of(wave, 0), 3, lane);
                if (i == 1) {
                    staged_by_all();                         // (the next block is there, this one read by all)
                    if (MORE || t + 2 < blocks) stage(MORE, sp, sq, se, t + 2);
                    read_q(nq, ne, 1 - B);
                }
                each<MUL::STEPS>([&](auto of_step) {
                    each<FQ>([&](auto of_q) {
                        constexpr int s = decltype(of_step)::value, j = decltype(of_q)::value;
                        acc[i][j] = MUL::template multiply<s, i, j>(fp[i], fq[B][j], acc[i][j], ep[B], eq[B]);
                    });
                });
                if (i > 0) fp[(i + 3) % 4] = read_fragment(np, p_of(wave, 0), (i + 3) % 4, lane);
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        auto start = [&](int b, uint8_t* sp, uint8_t* sq, uint8_t* se, uint8_t* np, uint8_t* nq, uint8_t* ne) {
            stage(false, sp, sq, se, 0);
            staged_by_all();
            if (blocks > 1) stage(false, np, nq, ne, 1);
            read_q(sq, se, b);
#pragma unroll
            for (int i = 0; i < 3; ++i) fp[i] = read_fragment(sp, p_of(wave, 0), i, lane);
        };
        const std::integral_constant<int, 0> zero;
        const std::integral_constant<int, 1> one;
        const std::true_type more;
        const std::false_type last;
        uint32_t t = blocks & 1;
        if (t) {
            start(1, sp1, sq1, se1, sp0, sq0, se0);
            block(one, last, sp1, sq1, se1, sp0, sq0, se0, 0);
        } else {
            start(0, sp0, sq0, se0, sp1, sq1, se1);
        }
        for (; t + 4 < blocks; t += 2) {
            block(zero, more, sp0, sq0, se0, sp1, sq1, se1, t);
            block(one, more, sp1, sq1, se1, sp0, sq0, se0, t + 1);
        }
        for (; t < blocks; t += 2) {
            block(zero, last, sp0, sq0, se0, sp1, sq1, se1, t);
            block(one, last, sp1, sq1, se1, sp0, sq0, se0, t + 1);
        }
        __syncthreads();                                     // (the last block read for the next by all)
    }
};

// 64 x 16 FQ by eight waves (or four, two workgroups a CU) that share k, for products of few tiles, and of few rows of Q, where every byte of P is read once.
// Each wave stages blocks of its own in a part of the LDS that no other wave touches, so that it waits for nothing but its
// own loads: the next block is on its way while this one, read into registers, is multiplied.  What the waves have
// summed is joined in the LDS, in their order.  (Fragments read from memory straight into registers took half as long again:
// neighbouring lanes hold rows apart, and the loads' addresses are taken four lanes at a time.)  Fragments of Q hold
// rows FQ c + j.
template <typename MUL, int FQ_, int WAVES_>
struct direct_tile {
    static constexpr int FP = 4, FQ = FQ_, BP = 64, BQ = 16 * FQ, WAVES = WAVES_, NT = 64 * WAVES;
    static constexpr int PART = (BP + BQ) * BYTES, EXPS = 128;
    typedef f32x4 sums[FQ][FP][64];
    static_assert(sizeof(sums) <= PART, "the sums take the place of the blocks");

    // Blocks from `first` up to `end`.  Behind it waves 0 .. FQ - 1 have the sums of column j = wave in `sum`, the others nothing.
    // Returned: room in the LDS that the waves have read (each its own column j of each wave's sums).
    static __device__ __forceinline__ sums* run(const operand& op, const operand& oq, uint32_t p0, uint32_t q0, const passage& way,
                                                uint32_t first, uint32_t end, f32x4 (&sum)[FP]) {
        __shared__ __attribute__((aligned(16))) uint8_t rows[WAVES * PART], exps[WAVES * EXPS];
        const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        const uint32_t blocks = way.blocks, c = lane & 15;
        f32x4 acc[FP][FQ] = {};
        // Eight places of the LDS a load, a row's chunk a lane: place 16 i + c holds row FP c + i, chunk k at k ^ (c % 8).
        constexpr int PL = BP / 8, QL = BQ / 8;
        const uint32_t chunk = ((lane ^ (lane / 8)) & 7) * 16;
        uint32_t p_at[PL], q_at[QL];
#pragma unroll
        for (int j = 0; j < PL; ++j) p_at[j] = (min(p0 + FP * (j % 2 * 8 + lane / 8) + j / 2, op.rows - 1) - min(p0, op.rows - 1)) * (uint32_t)op.pitch;
#pragma unroll
        for (int j = 0; j < QL; ++j) q_at[j] = (min(q0 + FQ * (j % 2 * 8 + lane / 8) + j / 2, oq.rows - 1) - min(q0, oq.rows - 1)) * (uint32_t)oq.pitch;
        const uint8_t *p_base = scalar(op.p + min(p0, op.rows - 1) * op.pitch), *q_base = scalar(oq.p + min(q0, oq.rows - 1) * oq.pitch);
        const uint32_t pe_at = min(p0 + 4 * lane, (op.rows - 1) & ~3u), qe_at = min(q0 + 4 * lane, (oq.rows - 1) & ~3u);
        auto whole_buffer = [](const uint8_t* p) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, -1, 0x00020000); };
        auto load = [](__amdgpu_buffer_rsrc_t from, uint8_t* to, uint32_t at) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_void*)to, 16, at, 0, 0, 0);
        };
        uint8_t *const to = rows + wave * PART, *const to_exp = exps + wave * EXPS;
        auto stage = [&](uint32_t t) {
            const uint32_t in = t * BYTES;
            if (MUL::SCALED) {
                if (lane < BP / 4)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(whole_buffer(scalar(op.exp + t * op.exp_pitch)), (lds_void*)to_exp, 4, pe_at, 0, 0, 0);
                if (lane < BQ / 4)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(whole_buffer(scalar(oq.exp + t * oq.exp_pitch)), (lds_void*)(to_exp + BP), 4, qe_at, 0, 0, 0);
            }
            // (chunks behind the row's end: its last one again, which is cut off)
            const uint32_t here = min(chunk, op.row_bytes - 16 - in), there = min(chunk, oq.row_bytes - 16 - in);
            const __amdgpu_buffer_rsrc_t from_p = whole_buffer(p_base + in), from_q = whole_buffer(q_base + in);
#pragma unroll
            for (int j = 0; j < PL; ++j) load(from_p, to + j * 1024, p_at[j] + here);
#pragma unroll
            for (int j = 0; j < QL; ++j) load(from_q, to + BP * BYTES + j * 1024, q_at[j] + there);
        };
        uint32_t t = first + wave;
        if (t < end) stage(t);
        for (; t < end; t += WAVES) {
            __builtin_amdgcn_s_waitcnt(loads_but(0));
            asm volatile("" ::: "memory");
            fragment p[FP], q[FQ];
#pragma unroll
            for (int i = 0; i < FP; ++i) p[i] = read_fragment(to, 0, i, lane);
#pragma unroll
            for (int j = 0; j < FQ; ++j) q[j] = read_fragment(to + BP * BYTES, 0, j, lane);
            uint32_t pe = 0, qe = 0;
            if (MUL::SCALED) {
                pe = *reinterpret_cast<const uint32_t*>(to_exp + 4 * c);
                if (FQ == 4) qe = *reinterpret_cast<const uint32_t*>(to_exp + BP + 4 * c);
                else if (FQ == 2) qe = *reinterpret_cast<const uint16_t*>(to_exp + BP + 2 * c);
                else qe = to_exp[BP + c];
            }
            __builtin_amdgcn_s_waitcnt(LDS_READ);            // (read: there is room for the next)
            asm volatile("" ::: "memory");
            if (t + WAVES < end) stage(t + WAVES);
            if (MUL::SCALED && way.ends != 0 && t + 1 == blocks) {
#pragma unroll
                for (int i = 0; i < FP; ++i) cut(p[i], way.ends, lane);
#pragma unroll
                for (int j = 0; j < FQ; ++j) cut(q[j], way.ends, lane);
            }
            if constexpr (requires_all<MUL>::value) MUL::multiply_all(p, q, acc, pe, qe);
            else multiply_all<MUL>(p, q, acc, pe, qe);
        }
        __syncthreads();
        sums* shared = reinterpret_cast<sums*>(rows);
#pragma unroll
        for (int i = 0; i < FP; ++i)
#pragma unroll
            for (int j = 0; j < FQ; ++j) shared[wave][j][i][lane] = acc[i][j];
        __syncthreads();
        if (wave < FQ) {
#pragma unroll
            for (int i = 0; i < FP; ++i) {
                sum[i] = shared[0][wave][i][lane];
#pragma unroll
                for (int w = 1; w < WAVES; ++w) sum[i] += shared[w][wave][i][lane];
            }
        }
        return shared;
    }
};

// A row's neighbours: the lanes whose number differs in the lowest bits hold the same columns of the rows 4 and 8 further on.
// N pieces of 16 bytes of each lane's row become piece lane % N of the rows of the N lanes, so that what the lanes write
// at once lies next to each other: 128 bytes of a row instead of four times 16 (a C of 8 192 x 8 192 in bf16: 21 us, 70 with stores
// that go through and were split so).
template <int BIT>
__device__ __forceinline__ uint32_t from_neighbour(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, BIT == 1 ? 0xB1 : 0x4E, 0xF, 0xF, true);
}
template <int N>
__device__ __forceinline__ void exchange(gd_u32x4 (&x)[N], uint32_t lane) {
    static_assert(N == 2 || N == 4, "within four lanes");
    each<2>([&](auto of_bit) {
        constexpr int BIT = 1 << decltype(of_bit)::value;
        if constexpr (BIT < N) {
            const uint32_t set = lane & BIT ? ~0u : 0u;      // (choices by masks, as above)
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (!(i & BIT)) {
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint32_t a = x[i][w], b = x[i | BIT][w], got = from_neighbour<BIT>((a & set) | (b & ~set));
                        x[i][w] = (got & set) | (a & ~set);
                        x[i | BIT][w] = (b & set) | (got & ~set);
                    }
                }
        }
    });
}

// Tiles in an order in which those that run at the same time share operands: workgroups go to the
// eight chiplets in turn, each takes a stretch of the tiles, walked in strips of STRIP tiles of q.
__device__ __forceinline__ uint32_t stretch_of(uint32_t b, uint32_t tiles) {
    const uint32_t chip = b & 7, each = tiles / 8, more = tiles % 8;
    return chip * each + min(chip, more) + b / 8;
}
template <uint32_t STRIP>
__device__ __forceinline__ void tile_of(uint32_t t, uint32_t tiles_p, uint32_t tiles_q, uint32_t& tp, uint32_t& tq) {
    const uint32_t strip = t / (STRIP * tiles_p), in = t - strip * STRIP * tiles_p;
    const uint32_t width = min(STRIP, tiles_q - strip * STRIP);
    tq = strip * STRIP + in % width;
    tp = in / width;
}

}  // namespace gd_tiles
#endif  // GD_TILES_H_
