// Softmax cross entropy of hidden states H [n][d] projected onto a vocabulary W [V][d], and its
// gradients, in pieces of the vocabulary.
//
//   l_iv = s <H_i, W_v>;  lse_i = log sum_v exp l_iv;  loss_i = lse_i - l_i,target
//   G_iv = c_i (exp(l_iv - lse_i) - [v = target_i]);  dH = s G W;  dW = s G^T H
//
// Every product runs on one tiled matrix product, C[m][n] = sum_k A[m][k] B[n][k], on the matrix
// cores with fp32 accumulators; what differs is how an operand lies in memory (its rows along k, or k
// along its rows, read through the LDS's transposing loads) and what becomes of a tile:
//   forward   m = vocabulary, n = rows: the tile's largest logit and sum of exponentials per row, joined
//             over the tiles by a second kernel; logits never leave the registers
//   G         the same tile again, with lse known: one piece of G in the type of H
//   dH        m = width, n = rows, k = the piece's vocabulary: fp32 sums, the pieces added up
//   dW        m = width, n = the piece's vocabulary, k = rows: written as the piece's rows
// Up to FOLD rows fill half a block of k of dW, which takes two halves all the same: the second one holds the rows once more, against
// what the rounding of G has dropped, so that dW of few rows is not rounded twice.
// Of other rows' G what counts most is the element at the target, 1 less than a probability: what rounding drops of it is kept, and
// added to dH as a row of W times it, and to dW as a block of k more in the tiles whose words are targets, where it is not
// little.  With targets drawn from the softmax of logits of standard deviation 4, 2 000 rows x 20 000 x 512: dH and dW off by 0.00173
// and 0.00172 of themselves (0.00206 and 0.00205 without; 0.00166 are their own rounding), 240 -> 246 us; 8 192 x 131 072 x 4 096
// 26.56 -> 26.76 ms.  What remains is the other elements' rounding.
// For the gradients the rows that have one are gathered first: rows left out cost nothing, and what
// their hidden states hold (infinities, NaN) reaches no product.
//
// The matrix cores bound large products (8 192 x 131 072 x 4 096: logits 6.28 ms, 1 400 TFLOP/s), few rows the weights' stream (4 rows x
// 131 072 x 4 096: 171 us, 6.3 TB/s), and what lies between them what a tile takes beside its sum.
//
// Tiles are staged with loads that go from memory straight to the LDS, into one of two buffers while
// the other is multiplied.  Places in the LDS are exchanged by exclusive or within a row, so that reads
// of eight or sixteen rows at one k fall on different banks.
#include <type_traits>

#include "gd_lanes.h"
#include "gd_operators.h"
#include "gd_vocab_plan.h"

namespace {

using namespace vocab_plan;

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;
constexpr uint32_t FOLD = BK / 2;                 // most rows whose G is held in two numbers

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef gd_bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef gd_f16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

template <typename T> struct of_type;
template <> struct of_type<gd_bf16> { typedef bf16x8 x8; };
template <> struct of_type<gd_f16> { typedef f16x8 x8; };

__device__ __forceinline__ f32x4 multiply(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 multiply(f16x8 a, f16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// ---- what a launch needs -------------------------------------------------------------------

struct operand {
    const void* p;
    uint64_t stride;     // elements between rows
    uint32_t rows;       // rows that are there (beyond them the last one is read again)
    uint32_t cols;       // elements of a row that are there, a multiple of 8
};

// Written by prepare_rows for the launches of the gradients.
struct grad_head {
    uint32_t count;      // rows with a gradient
    float back, more;    // what the products with G have to be multiplied by
};

struct product_args {
    operand a, b;
    uint32_t m, n, k;               // sizes; k is rounded up to BK by the staging; m: the launch's words, for logits
    uint32_t tiles_m, tiles_n;
    const grad_head* head;          // or null: n (or k) is as given
    // forward and G
    float scale2;                   // s * log2(e)
    float scale;
    uint32_t v0;                    // the launch's first row of W
    gd_token_list targets;          // forward
    float* target_logit;            // [n]
    float2* part;                   // [n][parts]
    uint32_t parts, part0;
    const float* row_lse2;          // G: per gathered row, in units of log 2
    const float* row_coef;
    const int32_t* row_target;
    float* row_rest;                // what rounding drops of a row's G at its target (rest_of): written with G, read for dW
    const uint2* list;              // dW: rows and their targets in order of the targets' groups, or null
    const uint32_t* list_at;        // [groups + 1] where a group's begin
    uint32_t groups;
    uint32_t fold;                  // G: row FOLD + i is what rounding drops of row i
    // outputs
    void* c;  uint64_t ldc;         // G, slabs, dW
    uint64_t slab;                  // elements between two slabs of dH
    uint32_t add;                   // dH: add to what is there
    uint32_t splits;                // dH: parts of k, a slab each
};

enum { EPI_LSE, EPI_G, EPI_SLAB, EPI_OUT };

// ---- staging ---------------------------------------------------------------------------------

// LDS images, 16 bytes (8 elements) a chunk.
// Rows along k: ROWS rows of 8 chunks; chunk c of row r lies at c ^ (r & 7).
// k along the rows: BK rows of ROWS / 8 chunks; chunk c of row k lies at c ^ turn(k).
__device__ __forceinline__ constexpr uint32_t turn(uint32_t k) { return 2 * ((k & 3) + 4 * ((k >> 3) & 3)); }

// APART (k along the rows, 128 of them): 64 rows and, behind the next 64, 64 more.
template <int ROWS, bool ALONG_K, int NT, bool APART = false>
struct stager {
    static constexpr int LOADS = ROWS * 8 / NT;   // of 16 bytes, per lane
    const uint8_t* base;                          // of the tile at k = k0
    uint32_t at[LOADS];                           // this lane's chunks: byte offsets within a block of k
    uint32_t place[LOADS];                        // chunk of the row (ALONG_K) or row of k
    uint32_t pitch;                               // bytes between rows
    uint32_t last;                                // chunks (ALONG_K) or rows that are there from k0 on, less one

    // first: the tile's first row (ALONG_K) or column, a row that is there; ROWS rows from first + more on are
    // staged.  k0 < cols where rows lie along k.
    __device__ __forceinline__ void init(const operand& o, uint32_t first, uint32_t more, uint32_t k0) {
        pitch = (uint32_t)o.stride * 2;
        base = static_cast<const uint8_t*>(o.p) + (ALONG_K ? (uint64_t)first * pitch + (uint64_t)k0 * 2 : 0);
        last = ALONG_K ? (o.cols - k0) / 8 - 1 : o.rows - 1;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const uint32_t i = j * NT + threadIdx.x;
            if (ALONG_K) {
                const uint32_t r = i / 8;
                place[j] = (i & 7) ^ (r & 7);
                at[j] = min(more + r, o.rows - 1 - first) * pitch;
            } else {
                place[j] = i / (ROWS / 8);
                const uint32_t c = (i % (ROWS / 8)) ^ (turn(place[j]) % (ROWS / 8));
                at[j] = min((first + more) / 8 + c + (APART ? c & 8 : 0), o.cols / 8 - 1) * 16;
            }
        }
    }

    // Block kt of k (from k0 on) into the buffer s.  What is not there is read from the nearest
    // place that is: the multiplication leaves it out, or meets zeros in the other operand.
    __device__ __forceinline__ void stage(uint8_t* s, uint32_t k0, uint32_t kt) const {
        const uint32_t row = min(k0 + kt * BK, last);             // (k along the rows)
        const uint8_t* from = base + (ALONG_K ? (uint64_t)kt * (BK * 2) : (uint64_t)row * pitch);
        __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(from), 0, 0x7FFFFFFF, 0x00020000);
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const uint32_t off = at[j] + (ALONG_K ? min(place[j], last - kt * 8) * 16 : min(place[j], last - row) * pitch);
            uint8_t* to = s + (j * NT + (threadIdx.x & ~63u)) * 16;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)to, 16, off, 0, 0, 0);
        }
    }
};

// Sixteen rows (from `row`) and 32 elements of k (from 32 * half) as a matrix operand: lane l holds row
// l % 16, k = 8 (l / 16) + 0..7.
template <int ROWS, bool ALONG_K, typename X8>
__device__ __forceinline__ X8 fragment(const uint8_t* s, uint32_t row, uint32_t half, uint32_t lane) {
    if (ALONG_K) {
        const uint32_t r = row + (lane & 15), c = half * 4 + (lane >> 4);
        return *reinterpret_cast<const X8*>(s + r * 128 + ((c ^ (r & 7)) * 16));
    } else {
        // each group of 16 lanes reads 4 rows of k of 16 elements, four a lane, and gets them transposed
        union { s16x4 q[2]; X8 x; } u;
#pragma unroll
        for (uint32_t h = 0; h < 2; ++h) {
            const uint32_t k = half * 32 + (lane >> 4) * 8 + h * 4 + ((lane & 15) >> 2);
            const uint32_t e = row + (lane & 3) * 4, c = (e / 8) ^ (turn(k) % (ROWS / 8));
            u.q[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(s + k * (ROWS * 2) + c * 16 + (e & 4) * 2));
        }
        return u.x;
    }
}

// ---- the tiled product ---------------------------------------------------------------------

// Tiles in an order in which those that run at the same time share operands: workgroups go to the
// eight chiplets in turn, each takes a stretch of the tiles, walked in strips of STRIP tiles of n.
template <uint32_t STRIP>
__device__ __forceinline__ void tile_of(uint32_t b, uint32_t tiles_m, uint32_t tiles_n, uint32_t& tm, uint32_t& tn) {
    const uint32_t tiles = tiles_m * tiles_n, chip = b & 7, each = tiles / 8, more = tiles % 8;
    const uint32_t t = chip * each + min(chip, more) + b / 8;
    const uint32_t strip = t / (STRIP * tiles_m), in = t - strip * STRIP * tiles_m;
    const uint32_t width = min(STRIP, tiles_n - strip * STRIP);
    tn = strip * STRIP + in % width;
    tm = in / width;
}

// s_waitcnt operands: all but `n` loads (n below 16); all LDS reads
constexpr int loads_but(int n) { return 0x0F70 | n; }
constexpr int LDS_READ = 0xC07F;

// A barrier behind which what every wave has staged is there.  The wait for a wave's own loads to the LDS is written out: a
// barrier by itself orders what a wave has written, and leaves loads that go past its registers to the compiler, which waits
// where it sees this wave read them, in front of the barrier or not.
__device__ __forceinline__ void staged_by_all() {
    __builtin_amdgcn_s_waitcnt(loads_but(0));
    __syncthreads();
}

// Behind the sum the buffers of B are free, `room`; of the first one a wave has SPARE bytes to itself.
constexpr uint32_t SPARE = 4096;

// The sum over k for tiles of 128 x 128 by four waves, two workgroups a CU.  Sixteen rows of A at a
// time (a step) are multiplied by all of the wave's columns, over the first half of the block's k, then the
// second.  A's fragments are read AHEAD steps before they are multiplied, B's half a block before; the
// last steps of a block already read from the next one, so that the matrix cores do not wait for the LDS
// behind the barrier.
template <typename T, bool A_ALONG, bool B_ALONG>
struct small_tile {
    static constexpr int BM = 128, BN = 128, WM = 2, WN = 2, NT = 256, FM = 4, FN = 4;
    typedef typename of_type<T>::x8 X8;

    // Rows (columns) of the tile that fragment i of wave wm (j of wn) begins at.
    static __device__ __forceinline__ uint32_t row_of(uint32_t wm, int i) { return wm * 64 + i * 16; }
    static __device__ __forceinline__ uint32_t col_of(uint32_t wn, int j) { return wn * 64 + j * 16; }

    template <typename Meanwhile>
    static __device__ __forceinline__ void run(const operand& oa, const operand& ob, uint32_t m0, uint32_t n0, uint32_t kfirst,
                                               uint32_t blocks, uint32_t ends, f32x4 (&acc)[FM][FN], uint8_t* (&room)[2],
                                               Meanwhile meanwhile) {
        // (one array a buffer, so that the compiler knows which loads a read has to wait for)
        __shared__ __attribute__((aligned(16))) uint8_t sa0[BM * BK * 2], sb0[BN * BK * 2];
        __shared__ __attribute__((aligned(16))) uint8_t sa1[BM * BK * 2], sb1[BN * BK * 2];
        const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        const uint32_t wm = wave / WN, wn = wave % WN;
        room[0] = sb0;
        room[1] = sb1;
        if (blocks == 0) return;
        stager<BM, A_ALONG, NT> la;
        stager<BN, B_ALONG, NT> lb;
        la.init(oa, m0, 0, kfirst * BK);
        lb.init(ob, n0, 0, kfirst * BK);
        auto stage = [&](uint8_t* a, uint8_t* b, uint32_t kt) {
            la.stage(a, kfirst * BK, kt);
            lb.stage(b, kfirst * BK, kt);
        };
        auto end_rows = [&](uint8_t* a, uint8_t* b) {
            for (uint32_t i = threadIdx.x; i < BM * 8; i += NT)
                if (((i & 7) ^ ((i >> 3) & 7)) * 8 >= ends) *reinterpret_cast<X8*>(a + i * 16) = X8(0);
            for (uint32_t i = threadIdx.x; i < BN * 8; i += NT)
                if (((i & 7) ^ ((i >> 3) & 7)) * 8 >= ends) *reinterpret_cast<X8*>(b + i * 16) = X8(0);
            __syncthreads();
        };
        constexpr int STEPS = 2 * FM, AHEAD = 3, RING = AHEAD + 1;
        static_assert(STEPS % RING == 0, "fragments keep their registers from block to block");
        X8 fa[RING], fb[2][FN];
        auto read_a = [&](const uint8_t* a, int s) { fa[s % RING] = fragment<BM, A_ALONG, X8>(a, row_of(wm, s % FM), s / FM, lane); };
        auto read_b = [&](const uint8_t* b, int half) {
#pragma unroll
            for (int j = 0; j < FN; ++j) fb[half][j] = fragment<BN, B_ALONG, X8>(b, col_of(wn, j), half, lane);
        };
        // Block kt from (a, b), then the first fragments of the one behind it from (na, nb): where there is none
        // they are read for nothing.
        auto block = [&](uint8_t* a, uint8_t* b, uint8_t* na, uint8_t* nb, uint32_t kt) {
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                if (s == 1) read_b(b, 1);
                if (s + AHEAD == STEPS) {
                    staged_by_all();                         // (the next block is there, this one read by all)
                    if (ends != 0 && kt + 2 == blocks) end_rows(na, nb);
                    if (kt + 2 < blocks) stage(a, b, kt + 2);
                    read_b(nb, 0);
                }
                if (s + AHEAD < STEPS) read_a(a, s + AHEAD);
                else read_a(na, s + AHEAD - STEPS);
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[s % FM][j] = multiply(fa[s % RING], fb[s / FM][j], acc[s % FM][j]);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        // blocks go through the buffers in turn and end with the second one
        uint32_t kt = blocks & 1;
        auto start = [&](uint8_t* a, uint8_t* b, uint8_t* na, uint8_t* nb) {
            stage(a, b, 0);
            meanwhile();
            staged_by_all();
            if (ends != 0 && blocks == 1) end_rows(a, b);
            if (blocks > 1) stage(na, nb, 1);
            read_b(b, 0);
#pragma unroll
            for (int s = 0; s < AHEAD; ++s) read_a(a, s);
        };
        if (kt) {
            start(sa1, sb1, sa0, sb0);
            block(sa1, sb1, sa0, sb0, 0);
        } else {
            start(sa0, sb0, sa1, sb1);
        }
        for (; kt < blocks; kt += 2) {
            block(sa0, sb0, sa1, sb1, kt);
            block(sa1, sb1, sa0, sb0, kt + 1);
        }
        __syncthreads();                                     // (the last block read for the next by all)
    }
};

// The sum over k for tiles of 256 x 256 by eight waves, one workgroup a CU, two waves a SIMD that take
// turns: while the waves of one group multiply, those of the other read their operands from the LDS, and
// a barrier changes the roles.  A block of 64 k takes two turns of a wave: B and the upper half of A's rows,
// then the lower half.  The buffers of B and of A's upper half are free again behind the first turn and are
// filled for the block after the next at once, those of the lower half behind the second: every load has
// three turns of both groups, one and a half blocks, to arrive.
//
//   turn          g0 reads    g1 reads     loads issued (each group in its reading turn)
//   4 kt          B, upper    (lower kt-1) g0: lower kt+1
//   4 kt + 1                  B, upper     g1: lower kt+1
//   4 kt + 2      lower                    g0: B, upper kt+2
//   4 kt + 3                  lower        g1: B, upper kt+2
//
// A wave has eight loads a block.  What is read in turns 4 kt and on was issued before the latest eight; the wait
// stands before the barrier in front of the even turns, which g0 reaches multiplying and g1 reading.
template <typename T, bool A_ALONG, bool B_ALONG>
struct large_tile {
    static constexpr int BM = 256, BN = 256, WM = 2, WN = 4, NT = 512, FM = 8, FN = 4;
    typedef typename of_type<T>::x8 X8;

    // Which rows of A the halves hold: 128 next to each other, or for the weights' gradient 64 of each wave's 128 (each
    // wave then writes 256 bytes of a row instead of twice 128: 1 000 rows x 50 001 x 1 000 131 us against 149).
    static constexpr bool APART = !A_ALONG && !B_ALONG;
    static __device__ __forceinline__ uint32_t row_of(uint32_t wm, int i) {
        return APART ? wm * 128 + i * 16 : (i / 4) * 128 + wm * 64 + (i % 4) * 16;
    }
    static __device__ __forceinline__ uint32_t col_of(uint32_t wn, int j) { return wn * 64 + j * 16; }

    template <typename Meanwhile>
    static __device__ __forceinline__ void run(const operand& oa, const operand& ob, uint32_t m0, uint32_t n0, uint32_t kfirst,
                                               uint32_t blocks, uint32_t ends, f32x4 (&acc)[FM][FN], uint8_t* (&room)[2],
                                               Meanwhile meanwhile) {
        __shared__ __attribute__((aligned(16))) uint8_t up0[128 * BK * 2], low0[128 * BK * 2], sb0[BN * BK * 2];
        __shared__ __attribute__((aligned(16))) uint8_t up1[128 * BK * 2], low1[128 * BK * 2], sb1[BN * BK * 2];
        const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        const uint32_t wm = wave / WN, wn = wave % WN, group = wm;   // (waves w and w + 4 share a SIMD)
        room[0] = sb0;
        room[1] = sb1;
        if (blocks == 0) return;
        stager<128, A_ALONG, NT, APART> lu, ll;
        stager<BN, B_ALONG, NT> lb;
        lu.init(oa, m0, 0, kfirst * BK);
        ll.init(oa, m0, APART ? 64 : 128, kfirst * BK);
        lb.init(ob, n0, 0, kfirst * BK);
        X8 fa[4][2], fb[FN][2];
        auto read_a = [&](const uint8_t* a) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) fa[i][h] = fragment<128, A_ALONG, X8>(a, wm * 64 + i * 16, h, lane);
        };
        auto read_b = [&](const uint8_t* b) {
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) fb[j][h] = fragment<BN, B_ALONG, X8>(b, col_of(wn, j), h, lane);
        };
        // what lies behind the end of k: zeros
        auto cut = [&](X8 (&f)[4][2]) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (uint32_t h = 0; h < 2; ++h)
                    if (h * 32 + (lane >> 4) * 8 >= ends) f[i][h] = X8(0);
        };
        // `newer`: how many of the wave's loads were issued behind those that the next turn reads
        auto turn_over = [&](bool wait, uint32_t newer) {
            asm volatile("" ::: "memory");
            if (wait) {
                if (newer == 8) __builtin_amdgcn_s_waitcnt(loads_but(8));
                else if (newer == 2) __builtin_amdgcn_s_waitcnt(loads_but(2));
                else __builtin_amdgcn_s_waitcnt(loads_but(0));
            }
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
        };
        auto multiply_half = [&](int first) {
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j) acc[first + i][j] = multiply(fa[i][h], fb[j][h], acc[first + i][j]);
            __builtin_amdgcn_s_setprio(0);
            __builtin_amdgcn_sched_barrier(0);
        };
        auto block = [&](uint8_t* up, uint8_t* low, uint8_t* b, uint8_t* nlow, uint32_t kt) {
            const bool tail = ends != 0 && kt + 1 == blocks;
            const uint32_t newer_up = kt + 1 < blocks ? 8 : 0, newer_low = kt + 2 < blocks ? 8 : kt + 1 < blocks ? 2 : 0;
            read_b(b);
            read_a(up);
            if (kt > 0 && kt + 1 < blocks) ll.stage(nlow, kfirst * BK, kt + 1);
            if (tail) { cut(fa); cut(fb); }
            __builtin_amdgcn_s_waitcnt(LDS_READ);
            turn_over(group == 1, newer_up);
            multiply_half(0);
            turn_over(group == 0, newer_up);
            read_a(low);
            if (kt + 2 < blocks) {
                lb.stage(b, kfirst * BK, kt + 2);
                lu.stage(up, kfirst * BK, kt + 2);
            }
            if (tail) cut(fa);
            __builtin_amdgcn_s_waitcnt(LDS_READ);
            turn_over(group == 1, newer_low);
            multiply_half(4);
            turn_over(group == 0, newer_low);
        };
        auto start = [&](uint8_t* up, uint8_t* low, uint8_t* b, uint8_t* nup, uint8_t* nlow, uint8_t* nb) {
            lb.stage(b, kfirst * BK, 0);
            lu.stage(up, kfirst * BK, 0);
            ll.stage(low, kfirst * BK, 0);
            if (blocks > 1) {
                lb.stage(nb, kfirst * BK, 1);
                lu.stage(nup, kfirst * BK, 1);
                ll.stage(nlow, kfirst * BK, 1);
                meanwhile();
                __builtin_amdgcn_s_waitcnt(loads_but(8));
            } else {
                meanwhile();
                __builtin_amdgcn_s_waitcnt(loads_but(0));
            }
            turn_over(false, 0);
            if (group == 1) turn_over(false, 0);             // one turn behind
        };
        uint32_t kt = blocks & 1;
        if (kt) {
            start(up1, low1, sb1, up0, low0, sb0);
            block(up1, low1, sb1, low0, 0);
        } else {
            start(up0, low0, sb0, up1, low1, sb1);
        }
        for (; kt < blocks; kt += 2) {
            block(up0, low0, sb0, low1, kt);
            block(up1, low1, sb1, low0, kt + 1);
        }
        if (group == 0) turn_over(false, 0);
    }
};

// ---- what becomes of a tile ------------------------------------------------------------------

// Sums over parts of the vocabulary: x the largest logit (in units of log 2), y the sum of the exponentials
// relative to it.  Nothing at all is (-inf, 0).
__device__ __forceinline__ float2 join_sums(float2 a, float2 b) {
    const float top = fmaxf(a.x, b.x), from = top == -__builtin_inff() ? 0.0f : top;
    return make_float2(top, a.y * __builtin_amdgcn_exp2f(a.x - from) + b.y * __builtin_amdgcn_exp2f(b.x - from));
}

// Target i as it is seen from the launch's first word on; -1 where it has none there.
__device__ __forceinline__ int32_t target_from(const product_args& p, uint32_t i, uint32_t n) {
    const int64_t t = i < n ? gd_token(p.targets, i) : -1;
    return t >= (int64_t)p.v0 && t - (int64_t)p.v0 < (int64_t)p.m ? (int32_t)(t - p.v0) : -1;
}

// How many of the launch's words there are from `first` on, the same number each time: tiles may reach behind them, where the
// last one is staged again, and another launch's words may follow.  (Comparisons
// with it stay in the branches that need them.  Worked out once for all columns they fill the scalar registers: a tile of
// 256 x 256 spent 6.7 us behind its sum, with a wait for each column's targets, where it spends 3.5 now.)
__device__ __forceinline__ int32_t words_left(const product_args& p, uint32_t first) {
    int32_t left = (int32_t)p.m - (int32_t)first;
    asm volatile("" : "+v"(left));
    return left;
}

// Column j of a wave's tile, row i, over all of its words (words[f] + 0..3), the same in the four lanes that share the
// column.  `target` as from target_from.  What few tiles need stands behind branches that all lanes take alike:
// words behind the launch's last, and the target's logit, which is written where it is met.
template <int FM, int FN>
__device__ __forceinline__ float2 tile_sums(const product_args& p, f32x4 (&acc)[FM][FN], int j, const uint32_t (&words)[FM], uint32_t i,
                                            int32_t target, uint32_t lane) {
    if (__ballot(target >= (int32_t)words[0] && target < (int32_t)words[FM - 1] + 4)) {
        float logit = 0.0f;
        bool met = false;
#pragma unroll
        for (int f = 0; f < FM; ++f)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (target - (int32_t)words[0] == (int32_t)(words[f] - words[0]) + r) { logit = acc[f][j][r]; met = true; }
        if (met) p.target_logit[i] = logit * p.scale;
    }
    if (p.scale2 < 0.0f) {
#pragma unroll
        for (int f = 0; f < FM; ++f) acc[f][j] = -acc[f][j];
    }
    // (never 0: words that are not there are -inf, and their exponentials 0; a scale that is no number makes every sum none)
    const float up = fabsf(p.scale2) < 1.1754943508222875e-38f ? 1.1754943508222875e-38f : fabsf(p.scale2);
    float top = -__builtin_inff();
    if (__ballot((int32_t)(words[FM - 1] - words[0]) + 3 >= words_left(p, words[0]))) {
        const int32_t left = words_left(p, words[0]);
#pragma unroll
        for (int f = 0; f < FM; ++f)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if ((int32_t)(words[f] - words[0]) + r >= left) acc[f][j][r] = -__builtin_inff();
    }
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
        for (int r = 0; r < 4; ++r) top = fmaxf(top, acc[f][j][r]);
    top = fmaxf(top, __uint_as_float(gd_lane_xor<16>(__float_as_uint(top), lane)));
    top = fmaxf(top, __uint_as_float(gd_lane_xor<32>(__float_as_uint(top), lane)));
    const float from = top == -__builtin_inff() ? 0.0f : top * up;
    float sum = 0.0f;
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
        for (int r = 0; r < 4; ++r) sum += __builtin_amdgcn_exp2f(fmaf(acc[f][j][r], up, -from));
    sum += __uint_as_float(gd_lane_xor<16>(__float_as_uint(sum), lane));
    sum += __uint_as_float(gd_lane_xor<32>(__float_as_uint(sum), lane));
    return make_float2(top == -__builtin_inff() ? top : from, sum);
}

// A row of G: what all its words share.
struct alignas(16) g_row {
    float lse2, coef, low;           // 64 less than lse in units of log 2; the coefficient; 2^-64 of it
    int32_t target;                  // from the launch's first word on
};
// Rows without a gradient have a coefficient of 0.
__device__ __forceinline__ g_row g_row_of(const product_args& p, uint32_t i, bool there) {
    if (!there) return g_row{0.0f, 0.0f, 0.0f, -1};
    const float coef = p.row_coef[i];
    return g_row{p.row_lse2[i] - 64.0f, coef, coef * 5.421010862427522e-20f, p.row_target[i] - (int32_t)p.v0};
}

// The row whose place i is.
__device__ __forceinline__ uint32_t folded(const product_args& p, uint32_t i) { return p.fold && i >= FOLD && i < 2 * FOLD ? i - FOLD : i; }

// What rounding to T drops of an element of G, with a last bit of 1 where that is little, less than a sixteenth of what it may drop;
// 0 where it drops nothing or the result is no number.
template <typename T>
__device__ __forceinline__ float rest_of(float g) {
    const float rest = g - gd_to_f32(gd_from_f32<T>(g));
    const float little = fabsf(g) * (std::is_same<T, gd_f16>::value ? 0x1p-15f : 0x1p-12f);
    if (rest == 0.0f || !(fabsf(rest) < __builtin_inff())) return 0.0f;
    return __uint_as_float((__float_as_uint(rest) & ~1u) | (fabsf(rest) < little ? 1u : 0u));
}

// Column j of a wave's tile of logits, row i, to G.  The exponential's instruction drops subnormal results: it is taken 2^64
// times as large, and the coefficient as much smaller.  What the rounding to T drops at the row's target is kept.
template <typename T, int FM, int FN>
__device__ __forceinline__ void tile_g(const product_args& p, f32x4 (&acc)[FM][FN], int j, const uint32_t (&words)[FM], uint32_t i,
                                       const g_row row) {
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[f][j][r] = __builtin_amdgcn_exp2f(fmaf(acc[f][j][r], p.scale2, -row.lse2)) * row.low;
    const int32_t span = (int32_t)(words[FM - 1] - words[0]) + 3, left = words_left(p, words[0]), met = row.target - (int32_t)words[0];
    // (a row without a gradient is zeros, also against a word of infinities)
    const bool none = row.coef == 0.0f;
    if (__ballot((met >= 0 && met <= span) || span >= left || none)) {       // (all lanes alike)
        float g = 0.0f;
        bool here = false;
#pragma unroll
        for (int f = 0; f < FM; ++f)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int32_t w = (int32_t)(words[f] - words[0]) + r;
                acc[f][j][r] -= w == met ? row.coef : 0.0f;
                if (w >= left || none) acc[f][j][r] = 0.0f;
                if (w == met) { g = acc[f][j][r]; here = true; }
            }
        if (here) p.row_rest[i] = rest_of<T>(g);
    }
}

// Four numbers to the nearest ones of a type.
template <typename T>
__device__ __forceinline__ gd_vec<T, 4> four_of(const f32x4& x) {
    typedef T x4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(gd_vec<T, 4>, __builtin_convertvector(x, x4));
}

// What that drops; nothing where the result is no number.
template <typename T>
__device__ __forceinline__ f32x4 dropped_by(const f32x4& x) {
    const gd_vec<T, 4> q = four_of<T>(x);
    f32x4 d;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        d[r] = x[r] - gd_to_f32(q.v[r]);
        d[r] = d[r] == d[r] ? d[r] : 0.0f;
    }
    return d;
}

// ---- what the rounding of G drops at the targets, for dW ----------------------------------------------

constexpr uint32_t GROUP = 128;    // words of a group of the list of rows by their targets

// A row whose target is a word of the tile: which row, which word of the tile, what rounding has dropped there.
struct alignas(16) rest_of_row {
    uint32_t row, word;
    float rest;
};
// (those of rows that are not there are 0, and left out)
__device__ __forceinline__ rest_of_row rest_at(const product_args& p, uint32_t word0, uint32_t e, uint32_t to) {
    if (e >= to) return rest_of_row{0, 0, 0.0f};
    const uint2 x = p.list[e];
    return rest_of_row{x.x, x.y - word0, p.row_rest[x.x]};
}

// Added to a tile of the weights' gradient whose sum is taken: the rows whose targets are words of the tile, entries from..to of the
// list, where rounding has not dropped little, 64 at a time against a matrix with one number a row.  Most tiles
// have a few such rows, or none.  listed: one entry for each thread, the first ones in it; while a block is multiplied, the
// next one's rows are on their way.
template <typename T, typename TILE>
__device__ __forceinline__ void add_rests(const product_args& p, uint32_t m0, uint32_t n0, uint32_t from, uint32_t to, uint32_t wave, uint32_t lane,
                                          uint8_t* const (&room)[2], rest_of_row* listed, f32x4 (&acc)[TILE::FM][TILE::FN]) {
    typedef typename of_type<T>::x8 X8;
    constexpr uint32_t BM = TILE::BM, BN = TILE::BN, NT = TILE::NT, LOADS = BM * 8 / NT;
    static_assert(BM == BN, "a lane's chunks of the two operands are the same rows'");
    __shared__ uint32_t counts[NT / 64];
    uint8_t* const sa = room[1];                                 // as the sum's images: chunk c of row k at c ^ turn(k)
    uint8_t* const sb = room[0];
    const uint32_t wm = wave / TILE::WN, wn = wave % TILE::WN;
    for (uint32_t base = from; base < to; base += NT) {
        const rest_of_row mine = base == from ? listed[threadIdx.x] : rest_at(p, p.v0 + n0, base + threadIdx.x, to);
        const bool keep = mine.rest != 0.0f && !(__float_as_uint(mine.rest) & 1);
        const uint64_t who = __ballot(keep);
        if (lane == 0) counts[wave] = (uint32_t)__popcll(who);
        __syncthreads();
        uint32_t at = (uint32_t)__popcll(who & ((1ull << lane) - 1)), count = 0;
#pragma unroll
        for (uint32_t w = 0; w < NT / 64; ++w) { if (w < wave) at += counts[w]; count += counts[w]; }
        if (keep) listed[at] = mine;
        __syncthreads();
        X8 ahead[LOADS];
        const auto ask = [&](uint32_t e0) {
#pragma unroll
            for (uint32_t j = 0; j < LOADS; ++j) {
                const uint32_t i = j * NT + threadIdx.x, e = e0 + i / (BM / 8), c = min(m0 / 8 + i % (BM / 8), p.a.cols / 8 - 1);
                ahead[j] = X8(0);
                if (e < count) ahead[j] = *reinterpret_cast<const X8*>(static_cast<const T*>(p.a.p) + (uint64_t)listed[e].row * p.a.stride + c * 8);
            }
        };
        if (count > 0) ask(0);
        for (uint32_t e0 = 0; e0 < count; e0 += BK) {
#pragma unroll
            for (uint32_t j = 0; j < LOADS; ++j) {
                const uint32_t i = j * NT + threadIdx.x, k = i / (BM / 8), c = i % (BM / 8), to_k = k * (BM * 2) + ((c ^ (turn(k) % (BM / 8))) * 16);
                *reinterpret_cast<X8*>(sa + to_k) = ahead[j];
                const rest_of_row r = listed[min(e0 + k, count - 1)];
                const T value = gd_from_f32<T>(e0 + k < count ? r.rest : 0.0f);
                X8 x(0);
#pragma unroll
                for (uint32_t w = 0; w < 8; ++w) x[w] = r.word == c * 8 + w ? value : T(0.0f);
                *reinterpret_cast<X8*>(sb + to_k) = x;
            }
            __syncthreads();
            if (e0 + BK < count) ask(e0 + BK);
#pragma unroll
            for (uint32_t half = 0; half < 2; ++half) {
                if (e0 + half * 32 >= count) break;
                X8 fb[TILE::FN];
#pragma unroll
                for (int j = 0; j < TILE::FN; ++j) fb[j] = fragment<BN, false, X8>(sb, TILE::col_of(wn, j), half, lane);
#pragma unroll
                for (int i = 0; i < TILE::FM; ++i) {
                    const X8 fa = fragment<BM, false, X8>(sa, TILE::row_of(wm, i), half, lane);
#pragma unroll
                    for (int j = 0; j < TILE::FN; ++j) acc[i][j] = multiply(fa, fb[j], acc[i][j]);
                }
            }
            __syncthreads();
        }
    }
}

template <typename T, typename TILE, int EPI>
__global__ __launch_bounds__(TILE::NT, 512 / TILE::NT) void product_kernel(const product_args p) {
    constexpr int BM = TILE::BM, BN = TILE::BN, WM = TILE::WM, WN = TILE::WN, FM = TILE::FM, FN = TILE::FN;
    uint32_t tm, tn, n = p.n, k = p.k, tiles_n = p.tiles_n;
    if (EPI == EPI_G || EPI == EPI_SLAB) {                           // (the grid is made for every row)
        n = p.head->count;
        tiles_n = (n + BN - 1) / BN;
        if (blockIdx.x >= p.tiles_m * tiles_n) return;
    }
    if (EPI == EPI_OUT) k = p.head->count;
    // (strips of four for the weights' gradient: 6 970 against 7 150 us, 8 192 rows x 131 072 x 4 096; of eight otherwise)
    tile_of<EPI == EPI_OUT ? 4 : 8>(blockIdx.x, p.tiles_m, tiles_n, tm, tn);
    const uint32_t m0 = tm * BM, n0 = tn * BN;
    uint32_t blocks = (k + BK - 1) / BK, kfirst = 0;
    if (EPI == EPI_SLAB) {
        const uint32_t per = (blocks + p.splits - 1) / p.splits;
        kfirst = min(blocks, blockIdx.y * per);
        blocks = min(per, blocks - kfirst);
    }
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t wm = wave / WN, wn = wave % WN;
    f32x4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    // What the rows of a tile of logits need is loaded before everything else, and lies in the LDS while the sum is taken.
    typedef typename std::conditional<EPI == EPI_G, g_row, int32_t>::type row_data;
    __shared__ row_data row_of[EPI == EPI_LSE || EPI == EPI_G ? BN : 1];
    row_data mine{};
    if ((EPI == EPI_LSE || EPI == EPI_G) && threadIdx.x < BN) {
        const uint32_t i = n0 + threadIdx.x;
        if constexpr (EPI == EPI_G) mine = g_row_of(p, folded(p, i), folded(p, i) < n);
        else mine = target_from(p, i, n);
    }
    // So do the first rows whose targets are words of a tile of the weights' gradient.
    __shared__ rest_of_row listed[EPI == EPI_OUT ? TILE::NT : 1];
    uint2 entry = make_uint2(0, 0);
    uint32_t from = 0, to = 0;
    if (EPI == EPI_OUT && p.list) {
        const uint32_t group = (p.v0 + n0) / GROUP;
        from = p.list_at[group];
        to = p.list_at[min(group + BN / GROUP, p.groups)];
        if (from + threadIdx.x < to) entry = p.list[from + threadIdx.x];
    }
    // operands that lie along k end where their rows do
    uint8_t* room[2];
    TILE::run(p.a, p.b, m0, n0, kfirst, blocks, EPI == EPI_LSE || EPI == EPI_G ? k % BK : 0, acc, room, [&] {
        if ((EPI == EPI_LSE || EPI == EPI_G) && threadIdx.x < BN) row_of[threadIdx.x] = mine;
        if (EPI == EPI_OUT && from < to)
            listed[threadIdx.x] = rest_of_row{entry.x, entry.y - (p.v0 + n0), from + threadIdx.x < to ? p.row_rest[entry.x] : 0.0f};
    });
    if constexpr (EPI == EPI_OUT)
        if (from < to) add_rests<T, TILE>(p, m0, n0, from, to, wave, lane, room, listed, acc);
    uint8_t* const spare = room[0] + wave * SPARE;

    // lane l holds rows 4 (l / 16) + 0..3 and column l % 16 of each 16 x 16 block
    uint32_t row[FM], col[FN];
#pragma unroll
    for (int i = 0; i < FM; ++i) row[i] = m0 + TILE::row_of(wm, i) + (lane >> 4) * 4;
#pragma unroll
    for (int j = 0; j < FN; ++j) col[j] = n0 + TILE::col_of(wn, j) + (lane & 15);

    // Rows are what lies next to each other in memory: through the wave's part of the LDS, 16 columns at a time, lanes
    // that have four rows of a column each become lanes with eight, and whole lines are written.
    constexpr uint32_t CH = FM * 2;                              // 16-byte chunks of a column
    auto put = [&](uint32_t f, const gd_vec<T, 4>& q) {
        const uint32_t c = lane & 15, ch = f * 2 + (lane >> 5);
        *reinterpret_cast<gd_vec<T, 4>*>(spare + c * (CH * 16) + ((ch ^ (c & (CH - 1))) * 16) + ((lane >> 4) & 1) * 8) = q;
    };
    auto take = [&](auto write) {
#pragma unroll
        for (uint32_t it = 0; it < 16 * CH / 64; ++it) {
            const uint32_t at = it * 64 + lane, c = at / CH, ch = at % CH;
            const uint8_t* from = spare + c * (CH * 16) + ((ch ^ (c & (CH - 1))) * 16);
            write(c, m0 + TILE::row_of(wm, ch / 2) + ch % 2 * 8, *reinterpret_cast<const gd_vec<T, 8>*>(from));
        }
    };
    if constexpr (EPI == EPI_LSE) {
        __shared__ float2 join[WM * BN];
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const float2 q = tile_sums<FM, FN>(p, acc, j, row, col[j], row_of[col[j] - n0], lane);
            if (lane < 16) join[wm * BN + TILE::col_of(wn, j) + lane] = q;
        }
        __syncthreads();
        if (threadIdx.x < BN && n0 + threadIdx.x < n) {
            float2 q = join[threadIdx.x];
#pragma unroll
            for (int w = 1; w < WM; ++w) q = join_sums(q, join[w * BN + threadIdx.x]);
            p.part[(uint64_t)(n0 + threadIdx.x) * p.parts + p.part0 + tm] = q;
        }
    } else if constexpr (EPI == EPI_G) {
        T* g = static_cast<T*>(p.c);
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            tile_g<T, FM, FN>(p, acc, j, row, folded(p, col[j]), row_of[col[j] - n0]);
            if (p.fold && n0 + TILE::col_of(wn, j) >= FOLD)
#pragma unroll
                for (int f = 0; f < FM; ++f) acc[f][j] = dropped_by<T>(acc[f][j]);
#pragma unroll
            for (int f = 0; f < FM; ++f) put(f, four_of<T>(acc[f][j]));
            // (there is room for whole tiles of rows)
            take([&](uint32_t c, uint32_t m, const gd_vec<T, 8>& q) {
                *reinterpret_cast<gd_vec<T, 8>*>(g + (uint64_t)(n0 + TILE::col_of(wn, j) + c) * p.ldc + m) = q;
            });
        }
    } else if constexpr (EPI == EPI_SLAB) {
        float* slab = static_cast<float*>(p.c) + blockIdx.y * p.slab;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const uint32_t i = col[j];
            if (i >= n) continue;
#pragma unroll
            for (int f = 0; f < FM; ++f) {
                const uint32_t e = row[f];                       // slabs are padded to four columns
                if (e >= p.m) continue;
                f32x4* to = reinterpret_cast<f32x4*>(slab + (uint64_t)i * p.ldc + e);
                *to = p.add ? *to + acc[f][j] : acc[f][j];
            }
        }
    } else {
        T* out = static_cast<T*>(p.c);
        const float back = p.head->back, more = p.head->more * p.scale;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
#pragma unroll
            for (int f = 0; f < FM; ++f) put(f, four_of<T>(acc[f][j] * back * more));
            take([&](uint32_t c, uint32_t m, const gd_vec<T, 8>& q) {
                const uint32_t i = n0 + TILE::col_of(wn, j) + c;
                if (i >= p.n) return;
                T* to = out + (uint64_t)i * p.ldc + m;
                if (m + 8 <= p.m) {
                    gd_write_through(to, q);
                } else {
#pragma unroll
                    for (uint32_t r = 0; r < 8; ++r)
                        if (m + r < p.m) to[r] = q.v[r];
                }
            });
        }
    }
}

// ---- few rows ----------------------------------------------------------------------------------

// Eight elements of a row, wherever it begins.
template <typename T>
__device__ __forceinline__ typename of_type<T>::x8 eight_at(const T* p) {
    return __builtin_bit_cast(typename of_type<T>::x8, gd_read<T, 8>(p));
}
// Those from `at` on, zeros behind the row's end; no branch where the row has eight elements (`whole`): what lies in front
// of the end is read and moved down.
template <typename T>
__device__ __forceinline__ typename of_type<T>::x8 last_at(const T* row, int32_t at, int32_t end, bool whole) {
    typename of_type<T>::x8 x(0);
    if (whole) {
        const int32_t down = max(at + 8 - end, 0);
        struct { uint64_t lo, hi; } q = __builtin_bit_cast(decltype(q), eight_at(row + at - down));
        const uint32_t bits = (uint32_t)(down & 3) * 16;
        const uint64_t lo = down & 4 ? q.hi : q.lo, hi = down & 4 ? 0 : q.hi;
        q.lo = down >= 8 ? 0 : lo >> bits | (hi << 1) << (63 - bits);
        q.hi = down >= 8 ? 0 : hi >> bits;
        return __builtin_bit_cast(typename of_type<T>::x8, q);
    }
#pragma unroll
    for (int32_t j = 0; j < 8; ++j) {
        const T e = row[min(at + j, end - 1)];
        x[j] = at + j < end ? e : T(0.0f);
    }
    return x;
}

// Logits where rows and words make too few tiles for the chip: a workgroup takes 32 words and up to 64 rows, its
// four waves a block of 64 k each in turn, straight into registers and DEPTH blocks ahead, with no LDS and no
// barrier between the loads; their sums are added up through the LDS.  Rows are read where they lie, aligned or not.
template <typename T, int FN, int EPI>
__global__ __launch_bounds__(256) void few_rows_kernel(const product_args p) {
    typedef typename of_type<T>::x8 X8;
    constexpr int FM = 2, DEPTH = FN == 4 ? 2 : 4;
    constexpr uint32_t WAVES = 4, WORDS = 32;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t n = EPI == EPI_G ? p.head->count : p.n, n0 = blockIdx.y * (FN * 16);
    if (n0 >= n) return;
    const uint32_t m0 = blockIdx.x * WORDS, k = p.k;
    const T* a[FM];
    const T* b[FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
        a[i] = static_cast<const T*>(p.a.p) + (uint64_t)min(m0 + i * 16 + (lane & 15), p.a.rows - 1) * p.a.stride + (lane >> 4) * 8;
#pragma unroll
    for (int j = 0; j < FN; ++j)
        b[j] = static_cast<const T*>(p.b.p) + (uint64_t)min(n0 + j * 16 + (lane & 15), n - 1) * p.b.stride + (lane >> 4) * 8;
    f32x4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    X8 fa[DEPTH][FM][2], fb[DEPTH][FN][2];
    const uint32_t whole = k / BK, mine = whole > wave ? (whole - wave + WAVES - 1) / WAVES : 0;   // whole blocks
    auto load = [&](int d, uint32_t q) {
        const uint32_t at = (wave + q * WAVES) * BK;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < FM; ++i) fa[d][i][h] = eight_at(a[i] + at + h * 32);
#pragma unroll
            for (int j = 0; j < FN; ++j) fb[d][j][h] = eight_at(b[j] + at + h * 32);
        }
    };
    auto use = [&](int d) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = multiply(fa[d][i][h], fb[d][j][h], acc[i][j]);
    };
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if ((uint32_t)d < mine) load(d, d);
    for (uint32_t q0 = 0; q0 < mine; q0 += DEPTH) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
            if (q0 + d < mine) {
                use(d);
                if (q0 + d + DEPTH < mine) load(d, q0 + d + DEPTH);
            }
    }
    if (k % BK && whole % WAVES == wave) {                       // the last block ends inside: zeros behind the end
        // (a lane's rows are counted from its own place, which may lie behind their end)
        const int32_t at = (int32_t)(whole * BK), end = (int32_t)k - (int32_t)(lane >> 4) * 8;
        if (k % 8 == 0) {
#pragma unroll
            for (int32_t h = 0; h < 2; ++h) {
                const int32_t from = min(at + h * 32, end - 8);
                const bool in = at + h * 32 < end;
#pragma unroll
                for (int i = 0; i < FM; ++i) fa[0][i][h] = in ? eight_at(a[i] + from) : X8(0);
#pragma unroll
                for (int j = 0; j < FN; ++j) fb[0][j][h] = in ? eight_at(b[j] + from) : X8(0);
            }
        } else {
#pragma unroll
            for (int32_t h = 0; h < 2; ++h) {
#pragma unroll
                for (int i = 0; i < FM; ++i) fa[0][i][h] = last_at(a[i], at + h * 32, end, k >= 8);
#pragma unroll
                for (int j = 0; j < FN; ++j) fb[0][j][h] = last_at(b[j], at + h * 32, end, k >= 8);
            }
        }
        use(0);
    }
    __shared__ f32x4 sums[WAVES][FM * FN][64];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) sums[wave][i * FN + j][lane] = acc[i][j];
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (uint32_t w = 1; w < WAVES; ++w) acc[i][j] += sums[w][i * FN + j][lane];
    const uint32_t rows[FM] = {m0 + (lane >> 4) * 4, m0 + 16 + (lane >> 4) * 4};
    if (EPI == EPI_LSE) {
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const uint32_t i = n0 + j * 16 + (lane & 15);
            const float2 q = tile_sums<FM, FN>(p, acc, j, rows, i, target_from(p, i, n), lane);
            if (lane < 16 && i < n) p.part[(uint64_t)i * p.parts + p.part0 + blockIdx.x] = q;
        }
    } else {
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const uint32_t i = n0 + j * 16 + (lane & 15);        // (there is room for whole tiles)
            tile_g<T, FM, FN>(p, acc, j, rows, i, g_row_of(p, i, i < n));
#pragma unroll
            for (int f = 0; f < FM; ++f)
                *reinterpret_cast<gd_vec<T, 4>*>(static_cast<T*>(p.c) + (uint64_t)i * p.ldc + rows[f]) = four_of<T>(acc[f][j]);
        }
        // (the weights' gradient takes the rows in blocks of 64: what rounding drops, and zeros between)
        constexpr int HALF = FOLD / 16;
#pragma unroll
        for (int j = FN; j < 2 * HALF; ++j)
#pragma unroll
            for (int f = 0; f < FM; ++f) {
                const bool rest = FN <= HALF && j >= HALF && j - HALF < FN;
                const gd_vec<T, 4> q = rest ? four_of<T>(dropped_by<T>(acc[f][rest ? j - HALF : 0])) : gd_vec<T, 4>{};
                *reinterpret_cast<gd_vec<T, 4>*>(static_cast<T*>(p.c) + (uint64_t)(j * 16 + (lane & 15)) * p.ldc + rows[f]) = q;
            }
    }
}

// ---- around the products -------------------------------------------------------------------

// Rows of `in` (all, or those listed) into rows of a padded copy, eight elements a lane: zeros behind the row's end
// and, behind a list, up to the next 256 rows.
template <typename T>
__device__ __forceinline__ void pack_rows(const void* in, uint64_t stride, uint32_t width, const grad_head* head,
                                          const uint32_t* rows, uint32_t n, T* out, uint32_t ldo, bool fold, uint32_t packers) {
    if (head) n = head->count;
    const uint32_t last = head ? (n + 255) / 256 * 256 : n, chunks = ldo / 8;
    const uint64_t total = (uint64_t)last * chunks;
    for (uint64_t x = (uint64_t)blockIdx.x * 256 + threadIdx.x; x < total; x += (uint64_t)packers * 256) {
        const uint32_t r = (uint32_t)(x / chunks), c = (uint32_t)(x - (uint64_t)r * chunks) * 8;
        const uint32_t at = fold && r >= FOLD && r < 2 * FOLD ? r - FOLD : r;
        gd_vec<T, 8> q{};
        if (at < n) {
            const uint64_t row = rows ? rows[at] : at;
            if (c < width) q = __builtin_bit_cast(gd_vec<T, 8>, last_at(static_cast<const T*>(in) + row * stride, (int32_t)c, (int32_t)width, width >= 8));
        }
        *reinterpret_cast<gd_vec<T, 8>*>(out + (uint64_t)r * ldo + c) = q;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(const void* in, uint64_t stride, uint32_t width, uint32_t n, T* out, uint32_t ldo) {
    pack_rows<T>(in, stride, width, nullptr, nullptr, n, out, ldo, false, gridDim.x);
}

// The rows with a gradient into a copy and, by the workgroups behind the `packers`, their list in order of the targets' groups: workgroup
// g counts the rows whose targets lie in groups before g, then lists its own behind those, in order of the rows.  A wave looks
// at a stretch of the rows, 512 at once.
template <typename T>
__global__ __launch_bounds__(256) void gather_kernel(const void* in, uint64_t stride, uint32_t width, const grad_head* head, const uint32_t* rows,
                                                     T* out, uint32_t ldo, bool fold, uint32_t packers, const int32_t* target,
                                                     uint32_t groups, uint2* list, uint32_t* list_at) {
    if (blockIdx.x < packers) return pack_rows<T>(in, stride, width, head, rows, 0, out, ldo, fold, packers);
    constexpr uint32_t WAVES = 4, EACH = 8;
    __shared__ uint32_t before[WAVES], own[WAVES];
    const uint32_t n = head->count, g = blockIdx.x - packers, wave = threadIdx.x / 64, lane = threadIdx.x & 63;
    const uint32_t per = (n + WAVES - 1) / WAVES, from = min(wave * per, n), to = min(from + per, n);
    uint32_t t[EACH];
    const auto look = [&](uint32_t i0) {                         // (rows that are not there lie behind all words)
#pragma unroll
        for (uint32_t b = 0; b < EACH; ++b) t[b] = (uint32_t)target[min(i0 + b * 64 + lane, n - 1)];
#pragma unroll
        for (uint32_t b = 0; b < EACH; ++b)
            if (i0 + b * 64 + lane >= to) t[b] = 0xFFFFFFFFu;
    };
    uint32_t less = 0, mine = 0;
    for (uint32_t i0 = from; i0 < to; i0 += EACH * 64) {
        look(i0);
#pragma unroll
        for (uint32_t b = 0; b < EACH; ++b) {
            less += (uint32_t)__popcll(__ballot(t[b] / GROUP < g));
            mine += (uint32_t)__popcll(__ballot(t[b] / GROUP == g));
        }
    }
    if (lane == 0) { before[wave] = less; own[wave] = mine; }
    __syncthreads();
    uint32_t at = 0;
    for (uint32_t w = 0; w < WAVES; ++w) at += before[w];
    if (threadIdx.x == 0) {
        list_at[g] = at;
        if (g + 1 == groups) list_at[groups] = n;
    }
    for (uint32_t w = 0; w < wave; ++w) at += own[w];
    if (mine == 0) return;
    for (uint32_t i0 = from; i0 < to; i0 += EACH * 64) {
        if (per > EACH * 64) look(i0);                           // (else they are still here)
#pragma unroll
        for (uint32_t b = 0; b < EACH; ++b) {
            const uint64_t who = __ballot(t[b] / GROUP == g);
            if (t[b] / GROUP == g) list[at + (uint32_t)__popcll(who & ((1ull << lane) - 1))] = make_uint2(i0 + b * 64 + lane, t[b]);
            at += (uint32_t)__popcll(who);
        }
    }
}

// Sums joined over the lanes of a wave.
__device__ __forceinline__ float2 wave_sums(float2 q, uint32_t lane) {
    const auto with = [&](uint32_t x, uint32_t y) { q = join_sums(q, make_float2(__uint_as_float(x), __uint_as_float(y))); };
    with(gd_lane_xor<1>(__float_as_uint(q.x), lane), gd_lane_xor<1>(__float_as_uint(q.y), lane));
    with(gd_lane_xor<2>(__float_as_uint(q.x), lane), gd_lane_xor<2>(__float_as_uint(q.y), lane));
    with(gd_lane_xor<4>(__float_as_uint(q.x), lane), gd_lane_xor<4>(__float_as_uint(q.y), lane));
    with(gd_lane_xor<8>(__float_as_uint(q.x), lane), gd_lane_xor<8>(__float_as_uint(q.y), lane));
    with(gd_lane_xor<16>(__float_as_uint(q.x), lane), gd_lane_xor<16>(__float_as_uint(q.y), lane));
    with(gd_lane_xor<32>(__float_as_uint(q.x), lane), gd_lane_xor<32>(__float_as_uint(q.y), lane));
    return q;
}

struct join_args {
    const float2* part;
    uint32_t stride, parts;          // elements between rows; parts of a row
    gd_token_list targets;
    uint32_t vocab;
    const float* target_logit;
    float* loss;  float* lse;  float* mean;
};

// Every `step`-th part of row i from `from` on, four at a time.
__device__ __forceinline__ float2 parts_of(const join_args& a, uint32_t i, uint32_t from, uint32_t step) {
    const float2* q = a.part + (uint64_t)i * a.stride;
    float2 sum = make_float2(-__builtin_inff(), 0.0f);
    for (uint32_t c = from; c < a.parts; c += 4 * step) {
        float2 x[4];
#pragma unroll
        for (uint32_t b = 0; b < 4; ++b) x[b] = c + b * step < a.parts ? q[c + b * step] : make_float2(-__builtin_inff(), 0.0f);
#pragma unroll
        for (uint32_t b = 0; b < 4; ++b) sum = join_sums(sum, x[b]);
    }
    return sum;
}

// A row's results; returns its loss.
__device__ __forceinline__ float finish_row(const join_args& a, uint32_t i, float2 q) {
    const float l = (q.x + __builtin_amdgcn_logf(q.y)) * LN2;
    const int64_t t = gd_token(a.targets, i);
    const float loss = t < 0 ? 0.0f : t >= (int64_t)a.vocab ? __uint_as_float(0x7FC00000u) : l - a.target_logit[i];
    a.lse[i] = l;
    a.loss[i] = loss;
    return loss;
}

// The tiles' sums joined, one wave a row.
__global__ __launch_bounds__(256) void join_kernel(const join_args a) {
    const uint32_t i = blockIdx.x * 4 + threadIdx.x / 64, lane = threadIdx.x & 63;
    if (i >= a.targets.n) return;
    const float2 q = wave_sums(parts_of(a, i, lane, 64), lane);
    if (lane == 0) finish_row(a, i, q);
}

// The same and the mean for few rows and parts, by one workgroup of sixteen waves: `share` (a power of two) of
// them work on a row.
__global__ __launch_bounds__(1024) void join_alone(const join_args a, uint32_t share) {
    __shared__ float2 sums[16];
    __shared__ float losses[64];
    const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x & 63, n = a.targets.n, at_once = 16 / share;
    for (uint32_t i0 = 0; i0 < n; i0 += at_once) {
        const uint32_t i = i0 + wave / share;
        float2 q = make_float2(-__builtin_inff(), 0.0f);
        if (i < n) q = wave_sums(parts_of(a, i, (wave % share) * 64 + lane, share * 64), lane);
        if (lane == 0) sums[wave] = q;
        __syncthreads();
        if (lane == 0 && wave % share == 0 && i < n) {
            for (uint32_t w = 1; w < share; ++w) q = join_sums(q, sums[wave + w]);
            losses[i] = finish_row(a, i, q);
        }
        __syncthreads();
    }
    if (wave > 0) return;
    float sum = lane < n ? losses[lane] : 0.0f;
    const float count = (float)__popcll(__ballot(lane < n && gd_token(a.targets, min(lane, n - 1)) >= 0));
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if (lane == 0) {
        a.mean[0] = sum / fmaxf(count, 1.0f);
        a.mean[1] = count;
    }
}

// Mean over the rows not left out, one workgroup, in a fixed order, AT_ONCE rows a lane at once.
template <int AT_ONCE>
__global__ __launch_bounds__(1024) void mean_kernel(const float* loss, gd_token_list targets, float* mean) {
    __shared__ float s[16];
    __shared__ uint32_t c[16];
    const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x & 63;
    float sum = 0.0f;
    uint32_t count = 0;
    for (uint32_t i = threadIdx.x; i < targets.n; i += AT_ONCE * 1024) {
        int64_t t[AT_ONCE];
        float l[AT_ONCE];
        gd_tokens<AT_ONCE>(targets, i, 1024, t);
#pragma unroll
        for (int b = 0; b < AT_ONCE; ++b) l[b] = loss[min(i + b * 1024, targets.n - 1)];
#pragma unroll
        for (int b = 0; b < AT_ONCE; ++b)
            if (i + b * 1024 < targets.n) {
                sum += l[b];
                count += t[b] >= 0;
            }
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        sum += __shfl_xor(sum, d);
        count += __shfl_xor(count, d);
    }
    if (lane == 0) { s[wave] = sum; c[wave] = count; }
    __syncthreads();
    if (wave > 0) return;
    sum = lane < 16 ? s[lane] : 0.0f;
    count = lane < 16 ? c[lane] : 0;
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) {
        sum += __shfl_xor(sum, d);
        count += __shfl_xor(count, d);
    }
    if (lane == 0) {
        mean[0] = sum / fmaxf((float)count, 1.0f);
        mean[1] = (float)count;
    }
}

struct rows_args {
    gd_token_list targets;
    uint32_t vocab, half;             // half: G is f16
    const float* lse;  const float* mean;  const float* grad_mean;  const float* grad_rows;
    grad_head* head;
    uint32_t* rows;                   // [count] the rows with a gradient
    int32_t* slot;                    // [n] their places, -1 without a gradient
    float* row_lse2;  float* row_coef;  int32_t* row_target;
};

// What the coefficients are scaled by.  Gradients of a mean over many rows, and of improbable words, would underflow
// as G is rounded to 16 bits, and the -1 at the target would be rounded as well: coefficients are divided by the
// largest one and multiplied by 2^15 in f16 (G is at most that then) and by 2^40 in bf16 (where every
// probability that fp32 holds stays a normal number), which is undone behind the products.
struct coef_scale {
    float most, power;
    bool fine;                       // the largest one is a number, and not 0
    __device__ __forceinline__ coef_scale(uint32_t top, uint32_t half)
        : most(__uint_as_float(top)), power(half ? 32768.0f : 1099511627776.0f), fine(top < 0x7F800000u && top != 0) {}
    __device__ __forceinline__ float of(float c) const { return fine ? c / most * power : c; }
    __device__ __forceinline__ void write(grad_head* head, uint32_t count) const {
        // (two factors, so that neither is subnormal)
        head->count = count;
        head->back = fine ? (most >= 1.0f ? most / power : 1.0f / power) : 1.0f;
        head->more = fine && most < 1.0f ? most : 1.0f;
    }
};

__device__ __forceinline__ uint32_t wave_max(uint32_t v, uint32_t lane) {
    v = max(v, gd_lane_xor<1>(v, lane));  v = max(v, gd_lane_xor<2>(v, lane));
    v = max(v, gd_lane_xor<4>(v, lane));  v = max(v, gd_lane_xor<8>(v, lane));
    v = max(v, gd_lane_xor<16>(v, lane)); return max(v, gd_lane_xor<32>(v, lane));
}

// Lists the rows with a gradient and works out what their tiles need.  One workgroup, EACH rows a lane at once: the list
// is in order of the rows.
template <int EACH>
__global__ __launch_bounds__(1024) void prepare_rows(const rows_args a) {
    constexpr uint32_t ROUND = EACH * 1024, WAVES = 16;
    __shared__ uint32_t s[EACH * WAVES];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64, n = a.targets.n;
    const float each = a.grad_mean ? *a.grad_mean / fmaxf(a.mean[1], 1.0f) : 0.0f;
    float c[EACH], lse[EACH];
    int64_t t[EACH];
    const auto load = [&](uint32_t base) {
        const uint32_t from = base + threadIdx.x;
        gd_tokens<EACH>(a.targets, from, 1024, t);
#pragma unroll
        for (int b = 0; b < EACH; ++b) {
            lse[b] = a.lse[min(from + b * 1024, n - 1)];
            c[b] = 0.0f;
        }
        if (a.grad_rows)
#pragma unroll
            for (int b = 0; b < EACH; ++b) c[b] = a.grad_rows[min(from + b * 1024, n - 1)];
#pragma unroll
        for (int b = 0; b < EACH; ++b) {
            if (a.grad_mean) c[b] += each;
            if (from + b * 1024 >= n || t[b] < 0 || t[b] >= (int64_t)a.vocab) c[b] = 0.0f;
        }
    };
    uint32_t top = 0;
    for (uint32_t base = 0; base < n; base += ROUND) {
        load(base);
#pragma unroll
        for (int b = 0; b < EACH; ++b) top = max(top, __float_as_uint(c[b]) & 0x7FFFFFFFu);
    }
    top = wave_max(top, lane);
    if (lane == 0) s[wave] = top;
    __syncthreads();
    for (uint32_t w = 0; w < WAVES; ++w) top = max(top, s[w]);
    __syncthreads();
    const coef_scale scale(top, a.half);
    uint32_t count = 0;
    for (uint32_t base = 0; base < n; base += ROUND) {
        if (n > ROUND) load(base);                            // (else they are still here)
        uint64_t who[EACH];
#pragma unroll
        for (int b = 0; b < EACH; ++b) {
            who[b] = __ballot(c[b] != 0.0f);
            if (lane == 0) s[b * WAVES + wave] = (uint32_t)__popcll(who[b]);
        }
        __syncthreads();
#pragma unroll
        for (int b = 0; b < EACH; ++b) {
            uint32_t at = count;
            for (uint32_t w = 0; w < WAVES; ++w) { if (w < wave) at += s[b * WAVES + w]; count += s[b * WAVES + w]; }
            at += (uint32_t)__popcll(who[b] & ((1ull << lane) - 1));
            const uint32_t i = base + b * 1024 + threadIdx.x;
            const bool in = c[b] != 0.0f;
            if (in) {
                a.rows[at] = i;
                a.row_lse2[at] = lse[b] * LOG2E;
                a.row_coef[at] = scale.of(c[b]);
                a.row_target[at] = (int32_t)t[b];
            }
            if (i < n) a.slot[i] = in ? (int32_t)at : -1;
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) scale.write(a.head, count);
}

// dH from its slabs, added up in order, and what the rounding of G has dropped at the row's target; zeros where a row has
// no gradient.  Four columns a lane.
template <typename T>
__global__ __launch_bounds__(256) void finish_hidden(const float* slabs, uint32_t lds, uint64_t slab, uint32_t splits,
                                                     const grad_head* head, const int32_t* slot, const int32_t* row_target,
                                                     const float* row_rest, const T* weight, uint64_t ldw, float scale, uint32_t n,
                                                     uint32_t width, T* out, uint64_t ldo) {
    const uint32_t quads = lds / 4;
    const float back = head->back, more = head->more * scale;
    const uint64_t total = (uint64_t)n * quads;
    for (uint64_t x = (uint64_t)blockIdx.x * 256 + threadIdx.x; x < total; x += (uint64_t)gridDim.x * 256) {
        const uint32_t i = (uint32_t)(x / quads), c = (uint32_t)(x - (uint64_t)i * quads) * 4;
        const int32_t at = slot[i];
        f32x4 sum = f32x4(0.0f);
        if (at >= 0) {
            const float rest = row_rest[at];
            const T* word = weight + (uint64_t)row_target[at] * ldw + c;
            const float* from = slabs + (uint64_t)at * lds + c;
            uint32_t s = 0;
            for (; s + 8 <= splits; s += 8) {
                f32x4 q[8];
#pragma unroll
                for (uint32_t b = 0; b < 8; ++b) q[b] = *reinterpret_cast<const f32x4*>(from + (s + b) * slab);
#pragma unroll
                for (uint32_t b = 0; b < 8; ++b) sum += q[b];
            }
            if (s < splits) {
                f32x4 q[7];
#pragma unroll
                for (uint32_t b = 0; b < 7; ++b) q[b] = *reinterpret_cast<const f32x4*>(from + min(s + b, splits - 1) * slab);
#pragma unroll
                for (uint32_t b = 0; b < 7; ++b)
                    if (s + b < splits) sum += q[b];
            }
            if (rest != 0.0f) {
                if (c + 4 <= width) {
                    const gd_vec<T, 4> w = gd_read<T, 4>(word);
#pragma unroll
                    for (int r = 0; r < 4; ++r) sum[r] += rest * gd_to_f32(w.v[r]);
                } else {
#pragma unroll
                    for (uint32_t r = 0; r < 4; ++r)
                        if (c + r < width) sum[r] += rest * gd_to_f32(word[r]);
                }
            }
        }
        gd_vec<T, 4> q;
#pragma unroll
        for (int r = 0; r < 4; ++r) q.v[r] = gd_from_f32<T>(at >= 0 ? sum[r] * back * more : 0.0f);
        T* to = out + (uint64_t)i * ldo + c;
        if (c + 4 <= width) {
            __builtin_memcpy(to, &q, sizeof(q));
        } else {
#pragma unroll
            for (uint32_t r = 0; r < 4; ++r)
                if (c + r < width) to[r] = q.v[r];
        }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void zero_rows(T* out, uint64_t ldo, uint32_t rows, uint32_t width) {
    for (uint32_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (uint32_t c = threadIdx.x; c < width; c += 256) out[(uint64_t)r * ldo + c] = gd_from_f32<T>(0.0f);
}

// ---- host side ----------------------------------------------------------------------------

struct loss_layout {
    // forward and both
    size_t target_logit, part, hidden, weight;
    // gradients
    size_t head, rows, slot, lse2, coef, target, rest, list, list_at, g, slabs;
    size_t total;
    uint64_t padded_rows, ldh, piece, pack_piece, slab;
    split_plan split;
    uint32_t parts;
};

// Everything that depends on the sizes alone.
loss_layout layout_of(uint64_t n, uint64_t vocab, uint64_t width, bool with_grad) {
    loss_layout l;
    l.padded_rows = up_to(n, 256);
    l.ldh = up_to(width, 64);                                   // (copies have rows of whole lines)
    const uint64_t all = up_to(vocab, 256);
    l.pack_piece = PACK / l.ldh / 256 * 256;
    if (l.pack_piece < 256) l.pack_piece = 256;
    if (l.pack_piece > all) l.pack_piece = all;
    l.parts = (uint32_t)(few_tiles(n, vocab) ? up_to(vocab, 32) / 32 : up_to(vocab, 128) / 128);
    size_t o = 0;
    l.target_logit = o; o = gd_align256(o + n * 4);
    l.part = o;         o = gd_align256(o + n * l.parts * 8);
    size_t f = o;
    // a packed copy of the hidden states: where their rows are not aligned, and of the rows with a gradient
    l.hidden = f;  f = gd_align256(f + l.padded_rows * l.ldh * 2);
    l.weight = f;  f = gd_align256(f + l.pack_piece * l.ldh * 2);
    l.total = f;
    l.head = l.rows = l.slot = l.lse2 = l.coef = l.target = l.rest = l.list = l.list_at = l.g = l.slabs = 0;
    l.piece = l.slab = 0;
    if (!with_grad) return l;
    // pieces of G alike in size
    uint64_t most = PIECE / (l.padded_rows ? l.padded_rows : 256) / 256 * 256;
    if (most < 256) most = 256;
    const uint64_t pieces = (all + most - 1) / most;
    l.piece = up_to((all + pieces - 1) / pieces, 256);
    l.split = split_for(width, n, l.piece);
    l.slab = n * up_to(width, 4);
    l.head = f;   f = gd_align256(f + sizeof(grad_head));
    l.rows = f;   f = gd_align256(f + n * 4);
    l.slot = f;   f = gd_align256(f + n * 4);
    l.lse2 = f;   f = gd_align256(f + n * 4);
    l.coef = f;   f = gd_align256(f + n * 4);
    l.target = f; f = gd_align256(f + n * 4);
    l.rest = f;   f = gd_align256(f + n * 4);
    l.list = f;   f = gd_align256(f + n * 8);
    l.list_at = f; f = gd_align256(f + (up_to(vocab, GROUP) / GROUP + 1) * 4);
    l.g = f;      f = gd_align256(f + l.padded_rows * l.piece * 2);
    l.slabs = f;  f = gd_align256(f + l.split.splits * l.slab * 4);
    l.total = f;
    return l;
}

// Workgroups of 256 for so many items, in rounds where there are more than fill the chip.
uint32_t blocks_for(uint64_t items) {
    const uint64_t b = (items + 255) / 256;
    return (uint32_t)(b < 8192 ? b : 8192);
}

bool direct(const void* p, uint64_t stride, uint64_t width) { return (uintptr_t)p % 16 == 0 && stride % 8 == 0 && width % 8 == 0; }

template <typename T, typename TILE, int EPI>
void launch_tiles(product_args p, hipStream_t s) {
    p.tiles_m = (p.m + TILE::BM - 1) / TILE::BM;
    p.tiles_n = (p.n + TILE::BN - 1) / TILE::BN;
    if (EPI != EPI_SLAB) p.splits = 1;
    hipLaunchKernelGGL((product_kernel<T, TILE, EPI>), dim3(p.tiles_m * p.tiles_n, p.splits), dim3(TILE::NT), 0, s, p);
}

template <typename T, int FN, int EPI>
void launch_few(const product_args& p, hipStream_t s) {
    // (G is read in blocks of 64 words)
    const dim3 grid((uint32_t)up_to(p.m, EPI == EPI_G ? BK : 32) / 32, (p.n + FN * 16 - 1) / (FN * 16));
    hipLaunchKernelGGL((few_rows_kernel<T, FN, EPI>), grid, dim3(256), 0, s, p);
}

// The logits of a piece; returns how many parts of the vocabulary each row's sums come in.
template <typename T, int EPI>
uint32_t launch_logits(const product_args& p, bool few, hipStream_t s) {
    if (few) {
        if (p.n <= 16) launch_few<T, 1, EPI>(p, s);
        else if (p.n <= 32) launch_few<T, 2, EPI>(p, s);
        else launch_few<T, 4, EPI>(p, s);
        return parts_of_words(p.m, p.n, p.k, true);
    }
    const uint32_t large = (uint32_t)large_part(p.m, p.n, p.k);
    const uint32_t large_parts = (large + 255) / 256;
    if (large > 0) {
        product_args q = p;
        q.m = large;
        launch_tiles<T, large_tile<T, true, true>, EPI>(q, s);
    }
    if (large < p.m) {
        product_args q = p;
        q.m -= large; q.v0 += large; q.part0 += large_parts;
        q.a.p = static_cast<const T*>(p.a.p) + (uint64_t)large * p.a.stride;
        q.a.rows -= large;
        q.c = static_cast<T*>(p.c) + large;
        launch_tiles<T, small_tile<T, true, true>, EPI>(q, s);
    }
    return parts_of_words(p.m, p.n, p.k, false);
}

// The rows of the weights' gradient for a piece.
template <typename T>
void launch_weight_grad(const product_args& p, hipStream_t s) {
    const uint32_t large = (uint32_t)large_part(p.n, p.m, p.k);
    if (large > 0) {
        product_args q = p;
        q.n = large;
        launch_tiles<T, large_tile<T, false, false>, EPI_OUT>(q, s);
    }
    if (large < p.n) {
        product_args q = p;
        q.n -= large; q.v0 += large;
        q.b.p = static_cast<const T*>(p.b.p) + large;
        q.b.cols -= large;
        q.c = static_cast<T*>(p.c) + (uint64_t)large * p.ldc;
        launch_tiles<T, small_tile<T, false, false>, EPI_OUT>(q, s);
    }
}

template <typename T>
hipError_t forward(const gd_vocab_loss_args& a, hipStream_t s) {
    const uint32_t n = a.targets.n;
    const loss_layout l = layout_of(n, a.vocab, a.width, false);
    const uint32_t ldh = (uint32_t)l.ldh;
    T* hidden = reinterpret_cast<T*>(a.work + l.hidden);
    T* weight = reinterpret_cast<T*>(a.work + l.weight);
    product_args p = {};
    const bool few = few_tiles(n, a.vocab);
    p.b = operand{a.hidden, a.hidden_stride, n, a.width};
    if (!few && !direct(a.hidden, a.hidden_stride, a.width)) {
        hipLaunchKernelGGL((pack_kernel<T>), dim3(blocks_for((uint64_t)n * ldh / 8)), dim3(256), 0, s, a.hidden, a.hidden_stride, a.width, n,
                           hidden, ldh);
        p.b = operand{hidden, ldh, n, ldh};
    }
    const bool plain = few || direct(a.weight, a.weight_stride, a.width);
    p.k = few ? a.width : (uint32_t)up_to(a.width, 8);           // (rows of a copy go on with zeros)
    p.n = n; p.scale = a.scale; p.scale2 = a.scale * LOG2E; p.targets = a.targets;
    p.target_logit = reinterpret_cast<float*>(a.work + l.target_logit);
    p.part = reinterpret_cast<float2*>(a.work + l.part);
    p.parts = l.parts;
    const uint32_t piece = words_at_once(n, a.vocab, plain ? a.vocab : l.pack_piece);
    uint32_t parts = 0;
    for (uint32_t v0 = 0; v0 < a.vocab; v0 += piece) {
        const uint32_t here = a.vocab - v0 < piece ? a.vocab - v0 : piece;
        const T* w = static_cast<const T*>(a.weight) + (uint64_t)v0 * a.weight_stride;
        if (plain) {
            p.a = operand{w, a.weight_stride, here, a.width};
        } else {
            hipLaunchKernelGGL((pack_kernel<T>), dim3(blocks_for((uint64_t)here * ldh / 8)), dim3(256), 0, s, w, a.weight_stride, a.width, here,
                               weight, ldh);
            p.a = operand{weight, ldh, here, ldh};
        }
        p.m = here; p.v0 = v0; p.part0 = parts;
        parts += launch_logits<T, EPI_LSE>(p, few, s);
    }
    const join_args j{p.part, p.parts, parts, a.targets, a.vocab, p.target_logit, a.loss, a.lse, a.mean};
    if (n <= 64 && n * j.parts <= 16384) {
        uint32_t share = 1;
        while (share < 16 && share * 2 * n <= 16 && share * 64 < j.parts) share *= 2;
        hipLaunchKernelGGL(join_alone, dim3(1), dim3(1024), 0, s, j, share);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(join_kernel, dim3((n + 3) / 4), dim3(256), 0, s, j);
    if (n <= 1024) hipLaunchKernelGGL((mean_kernel<1>), dim3(1), dim3(1024), 0, s, a.loss, a.targets, a.mean);
    else hipLaunchKernelGGL((mean_kernel<8>), dim3(1), dim3(1024), 0, s, a.loss, a.targets, a.mean);
    return hipGetLastError();
}

template <typename T>
hipError_t backward(const gd_vocab_grad_args& a, hipStream_t s) {
    const uint32_t n = a.targets.n;
    const loss_layout l = layout_of(n, a.vocab, a.width, true);
    const uint32_t ldh = (uint32_t)l.ldh, lds = (uint32_t)up_to(a.width, 4);
    grad_head* head = reinterpret_cast<grad_head*>(a.work + l.head);
    T* hidden = reinterpret_cast<T*>(a.work + l.hidden);
    T* weight = reinterpret_cast<T*>(a.work + l.weight);
    T* g = reinterpret_cast<T*>(a.work + l.g);
    float* slabs = reinterpret_cast<float*>(a.work + l.slabs);
    rows_args r;
    r.targets = a.targets; r.vocab = a.vocab; r.half = a.dtype == GD_F16;
    r.lse = a.lse; r.mean = a.mean; r.grad_mean = a.grad_mean; r.grad_rows = a.grad_rows;
    r.head = head;
    r.rows = reinterpret_cast<uint32_t*>(a.work + l.rows);
    r.slot = reinterpret_cast<int32_t*>(a.work + l.slot);
    r.row_lse2 = reinterpret_cast<float*>(a.work + l.lse2);
    r.row_coef = reinterpret_cast<float*>(a.work + l.coef);
    r.row_target = reinterpret_cast<int32_t*>(a.work + l.target);
    float* rest = reinterpret_cast<float*>(a.work + l.rest);
    const uint32_t padded = (uint32_t)l.padded_rows;
    if (n <= 1024) hipLaunchKernelGGL((prepare_rows<1>), dim3(1), dim3(1024), 0, s, r);
    else hipLaunchKernelGGL((prepare_rows<8>), dim3(1), dim3(1024), 0, s, r);
    uint2* list = reinterpret_cast<uint2*>(a.work + l.list);
    uint32_t* list_at = reinterpret_cast<uint32_t*>(a.work + l.list_at);
    const bool listed = a.weight_grad && n > FOLD;
    const uint32_t packers = blocks_for((uint64_t)padded * ldh / 8), groups = (a.vocab + GROUP - 1) / GROUP;
    hipLaunchKernelGGL((gather_kernel<T>), dim3(packers + (listed ? groups : 0)), dim3(256), 0, s, a.hidden, a.hidden_stride, a.width, head, r.rows,
                       hidden, ldh, n <= FOLD, packers, r.row_target, groups, list, list_at);
    const bool plain = direct(a.weight, a.weight_stride, a.width);
    uint32_t piece = (uint32_t)l.piece;
    if (!plain && piece > l.pack_piece) piece = (uint32_t)l.pack_piece;
    const bool few = few_tiles(n, a.vocab);
    for (uint32_t v0 = 0; v0 < a.vocab; v0 += piece) {
        const uint32_t here = a.vocab - v0 < piece ? a.vocab - v0 : piece;
        const T* w = static_cast<const T*>(a.weight) + (uint64_t)v0 * a.weight_stride;
        operand wo{w, a.weight_stride, here, a.width};
        if (!plain && (a.hidden_grad || !few)) {
            hipLaunchKernelGGL((pack_kernel<T>), dim3(blocks_for((uint64_t)here * ldh / 8)), dim3(256), 0, s, w, a.weight_stride, a.width, here,
                               weight, ldh);
            wo = operand{weight, ldh, here, ldh};
        }
        const operand go{g, piece, padded, piece};
        product_args p = {};
        p.head = head;
        p.a = wo;
        p.b = operand{hidden, ldh, padded, ldh};
        p.m = here; p.n = n; p.k = few ? a.width : (uint32_t)up_to(a.width, 8);
        p.scale2 = a.scale * LOG2E; p.v0 = v0;
        p.row_lse2 = r.row_lse2; p.row_coef = r.row_coef; p.row_target = r.row_target; p.row_rest = rest;
        p.c = g; p.ldc = piece; p.fold = n <= FOLD;
        launch_logits<T, EPI_G>(p, few, s);
        const uint32_t padded_here = (uint32_t)up_to(here, BK);      // (the tiles of G have written so far at least)
        if (a.hidden_grad) {
            product_args q = {};
            q.head = head;
            q.a = wo;
            q.b = go;
            q.m = a.width; q.n = n; q.k = padded_here;
            q.c = slabs; q.ldc = lds; q.slab = l.slab; q.add = v0 > 0; q.splits = l.split.splits;
            if (l.split.large) launch_tiles<T, large_tile<T, false, true>, EPI_SLAB>(q, s);
            else launch_tiles<T, small_tile<T, false, true>, EPI_SLAB>(q, s);
        }
        if (a.weight_grad) {
            product_args q = {};
            q.head = head;
            q.a = operand{hidden, ldh, padded, ldh};
            q.b = go;
            q.m = a.width; q.n = here; q.k = n;
            q.scale = a.scale; q.v0 = v0;
            q.row_rest = rest;
            q.list = listed ? list : nullptr; q.list_at = list_at; q.groups = groups;
            q.c = static_cast<T*>(a.weight_grad) + (uint64_t)v0 * a.weight_grad_stride; q.ldc = a.weight_grad_stride;
            launch_weight_grad<T>(q, s);
        }
    }
    if (a.hidden_grad)
        hipLaunchKernelGGL((finish_hidden<T>), dim3(blocks_for((uint64_t)n * lds / 4)), dim3(256), 0, s, slabs, lds, l.slab, l.split.splits,
                           head, r.slot, r.row_target, rest, static_cast<const T*>(a.weight), a.weight_stride, a.scale, n, a.width, static_cast<T*>(a.hidden_grad), a.hidden_grad_stride);
    return hipGetLastError();
}

}  // namespace

size_t gd_vocab_loss_work(uint64_t n, uint64_t vocab, uint64_t width, bool with_grad) {
    return layout_of(n, vocab, width, with_grad).total;
}

hipError_t gd_launch_vocab_loss(const gd_vocab_loss_args& a, hipStream_t s) {
    if (a.targets.n == 0) {
        hipLaunchKernelGGL((mean_kernel<1>), dim3(1), dim3(1024), 0, s, a.loss, a.targets, a.mean);
        return hipGetLastError();
    }
    return a.dtype == GD_BF16 ? forward<gd_bf16>(a, s) : forward<gd_f16>(a, s);
}

hipError_t gd_launch_vocab_grad(const gd_vocab_grad_args& a, hipStream_t s) {
    if (a.targets.n == 0) {
        if (!a.weight_grad) return hipSuccess;
        const dim3 grid(a.vocab < 65536 ? a.vocab : 65536);
        if (a.dtype == GD_BF16)
            hipLaunchKernelGGL((zero_rows<gd_bf16>), grid, dim3(256), 0, s, static_cast<gd_bf16*>(a.weight_grad), a.weight_grad_stride, a.vocab, a.width);
        else
            hipLaunchKernelGGL((zero_rows<gd_f16>), grid, dim3(256), 0, s, static_cast<gd_f16*>(a.weight_grad), a.weight_grad_stride, a.vocab, a.width);
        return hipGetLastError();
    }
    return a.dtype == GD_BF16 ? backward<gd_bf16>(a, s) : backward<gd_f16>(a, s);
}
