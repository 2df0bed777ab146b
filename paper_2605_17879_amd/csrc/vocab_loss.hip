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
// For the gradients the rows that have one are gathered first: rows left out cost nothing, and what
// their hidden states hold (infinities, NaN) reaches no product.
//
// Tiles are staged with loads that go from memory straight to the LDS, into one of two buffers while
// the other is multiplied.  Places in the LDS are exchanged by exclusive or within a row, so that reads
// of eight or sixteen rows at one k fall on different banks.
#include <type_traits>

#include "gd_lanes.h"
#include "gd_operators.h"

namespace {

constexpr uint32_t BK = 64;                       // elements of k staged at a time
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;
constexpr uint64_t PIECE = 1ull << 28;            // the most elements of a piece of G
constexpr uint64_t PACK = 1ull << 27;             // the most elements of a packed piece of W

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
    uint32_t m, n, k;               // sizes; k is rounded up to BK by the staging
    uint32_t tiles_m, tiles_n;
    const grad_head* head;          // or null: n (or k) is as given
    // forward and G
    float scale2;                   // s * log2(e)
    float scale;
    uint32_t v0, vocab;             // the piece's first row of W; rows of W
    gd_token_list targets;          // forward
    float* target_logit;            // [n]
    float2* part;                   // [n][parts]
    uint32_t parts, part0;
    const float* row_lse2;          // G: per gathered row, in units of log 2
    const float* row_coef;
    const int32_t* row_target;
    // outputs
    void* c;  uint64_t ldc;         // G, slabs, dW
    uint64_t slab;                  // elements between two slabs of dH
    uint32_t add;                   // dH: add to what is there
    uint32_t splits;                // dH: parts of k, a slab each
    uint32_t large;                 // tiles of 256 x 256 instead of 128 x 128 (the host's choice)
};

enum { EPI_LSE, EPI_G, EPI_SLAB, EPI_OUT };

// ---- staging ---------------------------------------------------------------------------------

// LDS images, 16 bytes (8 elements) a chunk.
// Rows along k: ROWS rows of 8 chunks; chunk c of row r lies at c ^ (r & 7).
// k along the rows: BK rows of ROWS / 8 chunks; chunk c of row k lies at c ^ turn(k).
__device__ __forceinline__ constexpr uint32_t turn(uint32_t k) { return 2 * ((k & 3) + 4 * ((k >> 3) & 3)); }

template <int ROWS, bool ALONG_K, int NT>
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
                at[j] = min((first + more) / 8 + ((i % (ROWS / 8)) ^ (turn(place[j]) % (ROWS / 8))), o.cols / 8 - 1) * 16;
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
// eight chiplets in turn, each takes a stretch of the tiles, walked in strips of eight tiles of n.
__device__ __forceinline__ void tile_of(uint32_t b, uint32_t tiles_m, uint32_t tiles_n, uint32_t& tm, uint32_t& tn) {
    const uint32_t tiles = tiles_m * tiles_n, chip = b & 7, each = tiles / 8, more = tiles % 8;
    const uint32_t t = chip * each + min(chip, more) + b / 8;
    constexpr uint32_t STRIP = 8;
    const uint32_t strip = t / (STRIP * tiles_m), in = t - strip * STRIP * tiles_m;
    const uint32_t width = min(STRIP, tiles_n - strip * STRIP);
    tn = strip * STRIP + in % width;
    tm = in / width;
}

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

    static __device__ __forceinline__ void run(const operand& oa, const operand& ob, uint32_t m0, uint32_t n0, uint32_t kfirst,
                                               uint32_t blocks, uint32_t ends, f32x4 (&acc)[FM][FN]) {
        // (one array a buffer, so that the compiler knows which loads a read has to wait for)
        __shared__ __attribute__((aligned(16))) uint8_t sa0[BM * BK * 2], sb0[BN * BK * 2];
        __shared__ __attribute__((aligned(16))) uint8_t sa1[BM * BK * 2], sb1[BN * BK * 2];
        const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        const uint32_t wm = wave / WN, wn = wave % WN;
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
                    __syncthreads();                         // (the next block is there, this one read by all)
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
            __syncthreads();
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

    static __device__ __forceinline__ uint32_t row_of(uint32_t wm, int i) { return (i / 4) * 128 + wm * 64 + (i % 4) * 16; }
    static __device__ __forceinline__ uint32_t col_of(uint32_t wn, int j) { return wn * 64 + j * 16; }

    // s_waitcnt operands: all but `n` loads (n below 16); all LDS reads
    static constexpr int loads_but(int n) { return 0x0F70 | n; }
    static constexpr int LDS_READ = 0xC07F;

    static __device__ __forceinline__ void run(const operand& oa, const operand& ob, uint32_t m0, uint32_t n0, uint32_t kfirst,
                                               uint32_t blocks, uint32_t ends, f32x4 (&acc)[FM][FN]) {
        __shared__ __attribute__((aligned(16))) uint8_t up0[128 * BK * 2], low0[128 * BK * 2], sb0[BN * BK * 2];
        __shared__ __attribute__((aligned(16))) uint8_t up1[128 * BK * 2], low1[128 * BK * 2], sb1[BN * BK * 2];
        const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        const uint32_t wm = wave / WN, wn = wave % WN, group = wm;   // (waves w and w + 4 share a SIMD)
        stager<128, A_ALONG, NT> lu, ll;
        stager<BN, B_ALONG, NT> lb;
        lu.init(oa, m0, 0, kfirst * BK);
        ll.init(oa, m0, 128, kfirst * BK);
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
                __builtin_amdgcn_s_waitcnt(loads_but(8));
            } else {
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

template <typename T, typename TILE, int EPI>
__global__ __launch_bounds__(TILE::NT, 512 / TILE::NT) void product_kernel(const product_args p) {
    constexpr int BM = TILE::BM, BN = TILE::BN, WM = TILE::WM, WN = TILE::WN, FM = TILE::FM, FN = TILE::FN;
    uint32_t tm, tn;
    tile_of(blockIdx.x, p.tiles_m, p.tiles_n, tm, tn);
    uint32_t n = p.n, k = p.k;
    if (EPI == EPI_G || EPI == EPI_SLAB) n = p.head->count;
    if (EPI == EPI_OUT) k = p.head->count;
    const uint32_t m0 = tm * BM, n0 = tn * BN;
    if (EPI != EPI_LSE && EPI != EPI_OUT && n0 >= n) return;         // (the grid is made for every row)
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
    // operands that lie along k end where their rows do
    if (blocks > 0)
        TILE::run(p.a, p.b, m0, n0, kfirst, blocks, EPI == EPI_LSE || EPI == EPI_G ? k % BK : 0, acc);

    // lane l holds rows 4 (l / 16) + 0..3 and column l % 16 of each 16 x 16 block
    uint32_t row[FM], col[FN];
#pragma unroll
    for (int i = 0; i < FM; ++i) row[i] = m0 + TILE::row_of(wm, i) + (lane >> 4) * 4;
#pragma unroll
    for (int j = 0; j < FN; ++j) col[j] = n0 + TILE::col_of(wn, j) + (lane & 15);
    if (EPI == EPI_LSE) {
        __shared__ float2 join[WM * BN];
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const uint32_t i = col[j];
            const int64_t t = i < n ? gd_token(p.targets, i) : -1;
            float top = -__builtin_inff();
#pragma unroll
            for (int f = 0; f < FM; ++f)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const uint32_t v = p.v0 + row[f] + r;
                    if (v < p.vocab) {
                        if (t == (int64_t)v) p.target_logit[i] = acc[f][j][r] * p.scale;
                        acc[f][j][r] *= p.scale2;
                    } else {
                        acc[f][j][r] = -__builtin_inff();
                    }
                    top = fmaxf(top, acc[f][j][r]);
                }
            top = fmaxf(top, __uint_as_float(gd_lane_xor<16>(__float_as_uint(top), lane)));
            top = fmaxf(top, __uint_as_float(gd_lane_xor<32>(__float_as_uint(top), lane)));
            const float from = top == -__builtin_inff() ? 0.0f : top;
            float sum = 0.0f;
#pragma unroll
            for (int f = 0; f < FM; ++f)
#pragma unroll
                for (int r = 0; r < 4; ++r) sum += __builtin_amdgcn_exp2f(acc[f][j][r] - from);
            sum += __uint_as_float(gd_lane_xor<16>(__float_as_uint(sum), lane));
            sum += __uint_as_float(gd_lane_xor<32>(__float_as_uint(sum), lane));
            if (lane < 16) join[wm * BN + TILE::col_of(wn, j) + lane] = make_float2(top, sum);
        }
        __syncthreads();
        if (threadIdx.x < BN && n0 + threadIdx.x < n) {
            float2 q = join[threadIdx.x];
#pragma unroll
            for (int w = 1; w < WM; ++w) {
                const float2 o = join[w * BN + threadIdx.x];
                const float top = fmaxf(q.x, o.x), from = top == -__builtin_inff() ? 0.0f : top;
                q.y = q.y * __builtin_amdgcn_exp2f(q.x - from) + o.y * __builtin_amdgcn_exp2f(o.x - from);
                q.x = top;
            }
            p.part[(uint64_t)(n0 + threadIdx.x) * p.parts + p.part0 + tm] = q;
        }
    } else if (EPI == EPI_G) {
        T* g = static_cast<T*>(p.c);
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const uint32_t i = col[j];                          // (there is room for whole tiles of rows)
            const bool there = i < n;
            const float lse2 = there ? p.row_lse2[i] : 0.0f, coef = there ? p.row_coef[i] : 0.0f;
            const int32_t t = there ? p.row_target[i] : -1;
#pragma unroll
            for (int f = 0; f < FM; ++f) {
                gd_vec<T, 4> q;
                const uint32_t v = p.v0 + row[f];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float e = exp2f(acc[f][j][r] * p.scale2 - lse2);    // (the instruction alone drops subnormal results)
                    if ((int32_t)(v + r) == t) e -= 1.0f;
                    q.v[r] = gd_from_f32<T>(there && v + r < p.vocab ? coef * e : 0.0f);
                }
                *reinterpret_cast<gd_vec<T, 4>*>(g + (uint64_t)i * p.ldc + row[f]) = q;
            }
        }
    } else if (EPI == EPI_SLAB) {
        float* c = static_cast<float*>(p.c) + blockIdx.y * p.slab;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const uint32_t i = col[j];
            if (i >= n) continue;
#pragma unroll
            for (int f = 0; f < FM; ++f) {
                const uint32_t e = row[f];                      // slabs are padded to four columns
                if (e >= p.m) continue;
                f32x4* to = reinterpret_cast<f32x4*>(c + (uint64_t)i * p.ldc + e);
                *to = p.add ? *to + acc[f][j] : acc[f][j];
            }
        }
    } else {
        T* c = static_cast<T*>(p.c);
        const float back = p.head->back, more = p.head->more * p.scale;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const uint32_t i = col[j];
            if (i >= p.n) continue;
#pragma unroll
            for (int f = 0; f < FM; ++f) {
                const uint32_t e = row[f];
                T* to = c + (uint64_t)i * p.ldc + e;
                if (e + 4 <= p.m && (p.ldc & 3) == 0 && ((uintptr_t)c & 7) == 0) {
                    gd_vec<T, 4> q;
#pragma unroll
                    for (int r = 0; r < 4; ++r) q.v[r] = gd_from_f32<T>(acc[f][j][r] * back * more);
                    *reinterpret_cast<gd_vec<T, 4>*>(to) = q;
                } else {
#pragma unroll
                    for (uint32_t r = 0; r < 4; ++r)
                        if (e + r < p.m) to[r] = gd_from_f32<T>(acc[f][j][r] * back * more);
                }
            }
        }
    }
}

// ---- around the products -------------------------------------------------------------------

// Rows of `in` (all, or those listed) into rows of a padded copy: zeros behind the row's end and,
// up to `padded` rows, behind the last row.
template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(const void* in, uint64_t stride, uint32_t width, const grad_head* head,
                                                   const uint32_t* rows, uint32_t n, uint32_t padded, T* out, uint32_t ldo) {
    if (head) n = head->count;
    const uint32_t last = head ? min(padded, (n + 255) / 256 * 256) : padded;
    for (uint64_t r = blockIdx.x; r < last; r += gridDim.x) {
        const T* from = static_cast<const T*>(in) + (r < n ? (rows ? (uint64_t)rows[r] : r) : 0) * stride;
        T* to = out + r * ldo;
        if (((uintptr_t)in & 15) == 0 && stride % 8 == 0 && width % 8 == 0) {
            for (uint32_t c = threadIdx.x * 8; c < ldo; c += 256 * 8) {
                gd_vec<T, 8> q;
                if (r < n && c < width) q = *reinterpret_cast<const gd_vec<T, 8>*>(from + c);
                else
#pragma unroll
                    for (int j = 0; j < 8; ++j) q.v[j] = gd_from_f32<T>(0.0f);
                *reinterpret_cast<gd_vec<T, 8>*>(to + c) = q;
            }
        } else {
            for (uint32_t c = threadIdx.x; c < ldo; c += 256) to[c] = r < n && c < width ? from[c] : gd_from_f32<T>(0.0f);
        }
    }
}

// The tiles' sums of a row joined, one wave a row.
__global__ __launch_bounds__(256) void join_kernel(const float2* part, uint32_t stride, uint32_t parts, gd_token_list targets, uint32_t vocab,
                                                   const float* target_logit, float* loss, float* lse) {
    const uint32_t i = blockIdx.x * 4 + threadIdx.x / 64, lane = threadIdx.x & 63;
    if (i >= targets.n) return;
    const float2* q = part + (uint64_t)i * stride;
    float top = -__builtin_inff();
    bool nan = false;
    for (uint32_t c = lane; c < parts; c += 64) { top = fmaxf(top, q[c].x); nan |= q[c].x != q[c].x; }
    top = fmaxf(top, __uint_as_float(gd_lane_xor<1>(__float_as_uint(top), lane)));
    top = fmaxf(top, __uint_as_float(gd_lane_xor<2>(__float_as_uint(top), lane)));
    top = fmaxf(top, __uint_as_float(gd_lane_xor<4>(__float_as_uint(top), lane)));
    top = fmaxf(top, __uint_as_float(gd_lane_xor<8>(__float_as_uint(top), lane)));
    top = fmaxf(top, __uint_as_float(gd_lane_xor<16>(__float_as_uint(top), lane)));
    top = fmaxf(top, __uint_as_float(gd_lane_xor<32>(__float_as_uint(top), lane)));
    const float from = top == -__builtin_inff() ? 0.0f : top;
    float sum = 0.0f;
    for (uint32_t c = lane; c < parts; c += 64) sum += q[c].y * __builtin_amdgcn_exp2f(q[c].x - from);
    sum += __uint_as_float(gd_lane_xor<1>(__float_as_uint(sum), lane));
    sum += __uint_as_float(gd_lane_xor<2>(__float_as_uint(sum), lane));
    sum += __uint_as_float(gd_lane_xor<4>(__float_as_uint(sum), lane));
    sum += __uint_as_float(gd_lane_xor<8>(__float_as_uint(sum), lane));
    sum += __uint_as_float(gd_lane_xor<16>(__float_as_uint(sum), lane));
    sum += __uint_as_float(gd_lane_xor<32>(__float_as_uint(sum), lane));
    if (lane == 0) {
        float l = (top + __builtin_amdgcn_logf(sum)) * LN2;
        if (nan) l = __uint_as_float(0x7FC00000u);
        lse[i] = l;
        const int64_t t = gd_token(targets, i);
        loss[i] = t < 0 ? 0.0f : t >= (int64_t)vocab ? __uint_as_float(0x7FC00000u) : l - target_logit[i];
    }
}

// Mean over the rows not left out, one workgroup, in a fixed order.
__global__ __launch_bounds__(1024) void mean_kernel(const float* loss, gd_token_list targets, float* mean) {
    __shared__ float s[1024];
    __shared__ uint32_t c[1024];
    float sum = 0.0f;
    uint32_t count = 0;
    for (uint32_t i = threadIdx.x; i < targets.n; i += 1024) {
        sum += loss[i];
        count += gd_token(targets, i) >= 0;
    }
    s[threadIdx.x] = sum;
    c[threadIdx.x] = count;
    __syncthreads();
    for (uint32_t d = 512; d > 0; d >>= 1) {
        if (threadIdx.x < d) { s[threadIdx.x] += s[threadIdx.x + d]; c[threadIdx.x] += c[threadIdx.x + d]; }
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        mean[0] = s[0] / fmaxf((float)c[0], 1.0f);
        mean[1] = (float)c[0];
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

__device__ __forceinline__ float coef_of(const rows_args& a, uint32_t i) {
    const int64_t t = gd_token(a.targets, i);
    if (t < 0 || t >= (int64_t)a.vocab) return 0.0f;
    float c = a.grad_rows ? a.grad_rows[i] : 0.0f;
    if (a.grad_mean) c += *a.grad_mean / fmaxf(a.mean[1], 1.0f);
    return c;
}

// Lists the rows with a gradient and works out what their tiles need.  One workgroup: the list is in
// order of the rows.  Gradients of a mean over many rows, and of improbable words, would underflow as G
// is rounded to 16 bits, and the -1 at the target would be rounded as well: coefficients are divided by the
// largest one and multiplied by 2^15 in f16 (G is at most that then) and by 2^40 in bf16 (where every
// probability that fp32 holds stays a normal number), which is undone behind the products.
__global__ __launch_bounds__(1024) void prepare_rows(const rows_args a) {
    __shared__ uint32_t s[16];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64, n = a.targets.n;
    uint32_t top = 0;
    for (uint32_t i = threadIdx.x; i < n; i += 1024) top = max(top, __float_as_uint(coef_of(a, i)) & 0x7FFFFFFFu);
    top = max(top, gd_lane_xor<1>(top, lane));  top = max(top, gd_lane_xor<2>(top, lane));
    top = max(top, gd_lane_xor<4>(top, lane));  top = max(top, gd_lane_xor<8>(top, lane));
    top = max(top, gd_lane_xor<16>(top, lane)); top = max(top, gd_lane_xor<32>(top, lane));
    if (lane == 0) s[wave] = top;
    __syncthreads();
    for (int w = 0; w < 16; ++w) top = max(top, s[w]);
    __syncthreads();
    const float most = __uint_as_float(top), power = a.half ? 32768.0f : 1099511627776.0f;
    const bool fine = top < 0x7F800000u && top != 0;
    uint32_t count = 0;
    for (uint32_t base = 0; base < n; base += 1024) {
        const uint32_t i = base + threadIdx.x;
        const float c = i < n ? coef_of(a, i) : 0.0f;
        const bool in = c != 0.0f;
        const uint64_t who = __ballot(in);
        if (lane == 0) s[wave] = (uint32_t)__popcll(who);
        __syncthreads();
        uint32_t at = count;
        for (uint32_t w = 0; w < 16; ++w) { if (w < wave) at += s[w]; count += s[w]; }
        at += (uint32_t)__popcll(who & ((1ull << lane) - 1));
        if (in) {
            a.rows[at] = i;
            a.row_lse2[at] = a.lse[i] * LOG2E;
            a.row_coef[at] = fine ? c / most * power : c;
            a.row_target[at] = (int32_t)gd_token(a.targets, i);
        }
        if (i < n) a.slot[i] = in ? (int32_t)at : -1;
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        // (two factors, so that neither is subnormal)
        a.head->count = count;
        a.head->back = fine ? (most >= 1.0f ? most / power : 1.0f / power) : 1.0f;
        a.head->more = fine && most < 1.0f ? most : 1.0f;
    }
}

// dH from its slabs, added up in order; zeros where a row has no gradient.
template <typename T>
__global__ __launch_bounds__(256) void finish_hidden(const float* slabs, uint32_t lds, uint64_t slab, uint32_t splits,
                                                     const grad_head* head, const int32_t* slot, float scale, uint32_t n,
                                                     uint32_t width, T* out, uint64_t ldo) {
    const float back = head->back, more = head->more * scale;
    for (uint32_t i = blockIdx.x; i < n; i += gridDim.x) {
        const int32_t at = slot[i];
        for (uint32_t c = threadIdx.x; c < width; c += 256) {
            float sum = 0.0f;
            if (at >= 0)
                for (uint32_t s = 0; s < splits; ++s) sum += slabs[s * slab + (uint64_t)at * lds + c];
            out[(uint64_t)i * ldo + c] = gd_from_f32<T>(sum * back * more);
        }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void zero_rows(T* out, uint64_t ldo, uint32_t rows, uint32_t width) {
    for (uint32_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (uint32_t c = threadIdx.x; c < width; c += 256) out[(uint64_t)r * ldo + c] = gd_from_f32<T>(0.0f);
}

// ---- host side ----------------------------------------------------------------------------

uint64_t up_to(uint64_t v, uint64_t unit) { return (v + unit - 1) / unit * unit; }

struct loss_layout {
    // forward and both
    size_t target_logit, part, hidden, weight;
    // gradients
    size_t head, rows, slot, lse2, coef, target, g, slabs;
    size_t total;
    uint64_t padded_rows, ldh, piece, pack_piece, splits, slab;
    uint32_t parts;
};

// Everything that depends on the sizes alone.
loss_layout layout_of(uint64_t n, uint64_t vocab, uint64_t width, bool with_grad) {
    loss_layout l;
    l.padded_rows = up_to(n, 256);
    l.ldh = up_to(width, 8);
    const uint64_t all = up_to(vocab, 256);
    l.pack_piece = PACK / l.ldh / 256 * 256;
    if (l.pack_piece < 256) l.pack_piece = 256;
    if (l.pack_piece > all) l.pack_piece = all;
    l.parts = (uint32_t)(up_to(vocab, 128) / 128);
    size_t o = 0;
    l.target_logit = o; o = gd_align256(o + n * 4);
    l.part = o;         o = gd_align256(o + n * l.parts * 8);
    size_t f = o;
    // a packed copy of the hidden states: where their rows are not aligned, and of the rows with a gradient
    l.hidden = f;  f = gd_align256(f + l.padded_rows * l.ldh * 2);
    l.weight = f;  f = gd_align256(f + l.pack_piece * l.ldh * 2);
    l.total = f;
    l.head = l.rows = l.slot = l.lse2 = l.coef = l.target = l.g = l.slabs = 0;
    l.piece = l.splits = l.slab = 0;
    if (!with_grad) return l;
    l.piece = PIECE / (l.padded_rows ? l.padded_rows : 256) / 256 * 256;
    if (l.piece < 256) l.piece = 256;
    if (l.piece > all) l.piece = all;
    // as many parts of the vocabulary for dH as make some 512 tiles of 128 x 128
    const uint64_t tiles = up_to(n, 128) / 128 * (up_to(width, 128) / 128);
    l.splits = tiles ? 512 / tiles : 1;
    if (l.splits > l.piece / 512) l.splits = l.piece / 512;
    if (l.splits < 1) l.splits = 1;
    l.slab = n * up_to(width, 4);
    l.head = f;   f = gd_align256(f + sizeof(grad_head));
    l.rows = f;   f = gd_align256(f + n * 4);
    l.slot = f;   f = gd_align256(f + n * 4);
    l.lse2 = f;   f = gd_align256(f + n * 4);
    l.coef = f;   f = gd_align256(f + n * 4);
    l.target = f; f = gd_align256(f + n * 4);
    l.g = f;      f = gd_align256(f + l.padded_rows * l.piece * 2);
    l.slabs = f;  f = gd_align256(f + l.splits * l.slab * 4);
    l.total = f;
    return l;
}

bool direct(const void* p, uint64_t stride, uint64_t width) { return (uintptr_t)p % 16 == 0 && stride % 8 == 0 && width % 8 == 0; }

template <typename T, typename TILE, int EPI>
void launch_tiles(product_args& p, hipStream_t s) {
    p.tiles_m = (p.m + TILE::BM - 1) / TILE::BM;
    p.tiles_n = (p.n + TILE::BN - 1) / TILE::BN;
    if (EPI != EPI_SLAB) p.splits = 1;
    hipLaunchKernelGGL((product_kernel<T, TILE, EPI>), dim3(p.tiles_m * p.tiles_n, p.splits), dim3(TILE::NT), 0, s, p);
}

template <typename T, bool A_ALONG, bool B_ALONG, int EPI>
void launch_product(product_args& p, hipStream_t s) {
    if (p.large) launch_tiles<T, large_tile<T, A_ALONG, B_ALONG>, EPI>(p, s);
    else launch_tiles<T, small_tile<T, A_ALONG, B_ALONG>, EPI>(p, s);
}

// Tiles of 256 x 256 (half the reads of an operand, one workgroup a CU) where there are some for all CUs.
bool large_tiles(uint64_t m, uint64_t n) { return up_to(m, 256) / 256 * (up_to(n, 256) / 256) >= 256; }

template <typename T>
hipError_t forward(const gd_vocab_loss_args& a, hipStream_t s) {
    const uint32_t n = a.targets.n;
    const loss_layout l = layout_of(n, a.vocab, a.width, false);
    const uint32_t ldh = (uint32_t)l.ldh;
    T* hidden = reinterpret_cast<T*>(a.work + l.hidden);
    T* weight = reinterpret_cast<T*>(a.work + l.weight);
    product_args p = {};
    p.b = operand{a.hidden, a.hidden_stride, n, a.width};
    if (!direct(a.hidden, a.hidden_stride, a.width)) {
        hipLaunchKernelGGL((pack_kernel<T>), dim3(n < 65536 ? n : 65536), dim3(256), 0, s, a.hidden, a.hidden_stride, a.width,
                           (const grad_head*)nullptr, (const uint32_t*)nullptr, n, n, hidden, ldh);
        p.b = operand{hidden, ldh, n, ldh};
    }
    const bool plain = direct(a.weight, a.weight_stride, a.width);
    p.n = n; p.scale = a.scale; p.scale2 = a.scale * LOG2E; p.vocab = a.vocab; p.targets = a.targets;
    p.target_logit = reinterpret_cast<float*>(a.work + l.target_logit);
    p.part = reinterpret_cast<float2*>(a.work + l.part);
    p.parts = l.parts;
    const uint32_t piece = plain ? a.vocab : (uint32_t)l.pack_piece;
    for (uint32_t v0 = 0; v0 < a.vocab; v0 += piece) {
        const uint32_t here = a.vocab - v0 < piece ? a.vocab - v0 : piece;
        const T* w = static_cast<const T*>(a.weight) + (uint64_t)v0 * a.weight_stride;
        if (plain) {
            p.a = operand{w, a.weight_stride, here, a.width};
        } else {
            hipLaunchKernelGGL((pack_kernel<T>), dim3(here < 65536 ? here : 65536), dim3(256), 0, s, w, a.weight_stride, a.width,
                               (const grad_head*)nullptr, (const uint32_t*)nullptr, here, here, weight, ldh);
            p.a = operand{weight, ldh, here, ldh};
        }
        p.k = p.a.cols < p.b.cols ? p.b.cols : p.a.cols;
        p.m = here; p.v0 = v0;
        p.large = large_tiles(piece, n);
        p.part0 = v0 / (p.large ? 256 : 128);
        launch_product<T, true, true, EPI_LSE>(p, s);
    }
    const uint32_t tiles = (a.vocab + (p.large ? 255 : 127)) / (p.large ? 256 : 128);
    hipLaunchKernelGGL(join_kernel, dim3((n + 3) / 4), dim3(256), 0, s, p.part, p.parts, tiles, a.targets, a.vocab, p.target_logit, a.loss, a.lse);
    hipLaunchKernelGGL(mean_kernel, dim3(1), dim3(1024), 0, s, a.loss, a.targets, a.mean);
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
    hipLaunchKernelGGL(prepare_rows, dim3(1), dim3(1024), 0, s, r);
    const uint32_t padded = (uint32_t)l.padded_rows;
    hipLaunchKernelGGL((pack_kernel<T>), dim3(padded < 16384 ? padded : 16384), dim3(256), 0, s, a.hidden, a.hidden_stride, a.width,
                       head, r.rows, n, padded, hidden, ldh);
    const bool plain = direct(a.weight, a.weight_stride, a.width);
    uint32_t piece = (uint32_t)l.piece;
    if (!plain && piece > l.pack_piece) piece = (uint32_t)l.pack_piece;
    for (uint32_t v0 = 0; v0 < a.vocab; v0 += piece) {
        const uint32_t here = a.vocab - v0 < piece ? a.vocab - v0 : piece;
        const T* w = static_cast<const T*>(a.weight) + (uint64_t)v0 * a.weight_stride;
        operand wo{w, a.weight_stride, here, a.width};
        if (!plain) {
            hipLaunchKernelGGL((pack_kernel<T>), dim3(here < 65536 ? here : 65536), dim3(256), 0, s, w, a.weight_stride, a.width,
                               (const grad_head*)nullptr, (const uint32_t*)nullptr, here, here, weight, ldh);
            wo = operand{weight, ldh, here, ldh};
        }
        const operand go{g, piece, padded, piece};
        product_args p = {};
        p.head = head;
        p.a = wo;
        p.b = operand{hidden, ldh, padded, ldh};
        p.m = here; p.n = n; p.k = ldh;
        p.scale2 = a.scale * LOG2E; p.v0 = v0; p.vocab = a.vocab;
        p.row_lse2 = r.row_lse2; p.row_coef = r.row_coef; p.row_target = r.row_target;
        p.c = g; p.ldc = piece;
        p.large = large_tiles(piece, n);
        launch_product<T, true, true, EPI_G>(p, s);
        const uint32_t padded_here = (uint32_t)up_to(here, p.large ? 256 : 128);     // what the tiles of G have written
        if (a.hidden_grad) {
            product_args q = {};
            q.head = head;
            q.a = wo;
            q.b = go;
            q.m = a.width; q.n = n; q.k = padded_here;
            q.c = slabs; q.ldc = lds; q.slab = l.slab; q.add = v0 > 0; q.splits = (uint32_t)l.splits;
            q.large = large_tiles(q.m, q.n);
            launch_product<T, false, true, EPI_SLAB>(q, s);
        }
        if (a.weight_grad) {
            product_args q = {};
            q.head = head;
            q.a = operand{hidden, ldh, padded, ldh};
            q.b = go;
            q.m = a.width; q.n = here; q.k = n;
            q.scale = a.scale;
            q.c = static_cast<T*>(a.weight_grad) + (uint64_t)v0 * a.weight_grad_stride; q.ldc = a.weight_grad_stride;
            q.large = large_tiles(q.m, piece);
            launch_product<T, false, false, EPI_OUT>(q, s);
        }
    }
    if (a.hidden_grad)
        hipLaunchKernelGGL((finish_hidden<T>), dim3(n < 65536 ? n : 65536), dim3(256), 0, s, slabs, lds, l.slab, (uint32_t)l.splits,
                           head, r.slot, a.scale, n, a.width, static_cast<T*>(a.hidden_grad), a.hidden_grad_stride);
    return hipGetLastError();
}

}  // namespace

size_t gd_vocab_loss_work(uint64_t n, uint64_t vocab, uint64_t width, bool with_grad) {
    return layout_of(n, vocab, width, with_grad).total;
}

hipError_t gd_launch_vocab_loss(const gd_vocab_loss_args& a, hipStream_t s) {
    if (a.targets.n == 0) {
        hipLaunchKernelGGL(mean_kernel, dim3(1), dim3(1024), 0, s, a.loss, a.targets, a.mean);
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
