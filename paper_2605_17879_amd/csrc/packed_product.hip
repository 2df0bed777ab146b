// Products of packed matrices: C[n][m] = sum_k A[n][k] B[m][k], A and B codes of 8 bits with a power of two for each
// 128 of a row, C in fp32 or rounded once, added to what is there or not.
//
//   C_ij = sum over blocks b of 2^(ea_bi - 127 + eb_bj - 127) sum over the block's k of a_ik b_jk
//
// Sums are of fp32: by the 16-bit matrix cores, for which codes times powers of two are exact numbers of bf16.  The operands are written out as
// such first, or converted in registers where tiles are read straight into them.
//
// For a C of 16 bits the caller can ask for the scaled 8-bit instruction instead, which takes 128 of k at a time with their powers
// of two, so that a block costs what a plain 8-bit product costs, at twice the rate (8 192 x 8 192 x 8 192 410 us, 813 by the 16-bit cores).  Its own sums are short: the
// products of eight k are cut at 2^-13 of the largest (gd_tiles.h has the rule).  In the norm that costs 1.5e-5 to 9e-5, C's own rounding 1.7e-3 in
// bf16 and 2.1e-4 in f16; at its worst, seven small products beside a large one, 8.0e-4 of that product (half a step of bf16 is 3.9e-3, of
// f16 4.9e-4), and where large products cancel nothing of a small result may be left.
//
// Rows of B are the operand P (columns of C, which a lane holds sixteen of next to each other), rows of A the operand Q.
#include <algorithm>

#include "gd_tiles.h"

namespace {

using namespace gd_tiles;

struct product_args {
    operand p, q;
    passage way;
    uint32_t n, m;                 // rows and columns of C
    uint32_t tiles_p, tiles_q;
    uint32_t parts;                // of tiles of 256 x 256: the launch takes quarters of these, from this one on, plus 1; 0: its own tiles
    void* c;  uint64_t ldc;        // elements
    uint32_t add, type;            // type: of C, where the kernel is of any_type
    float* slab;                   // splits: [split][n][m4]; null: one split
    uint32_t m4, each;             // columns of a slab; blocks of k of a split
};

// Sixteen columns of a row of C: v[i][r] is column 4 r + i.
__device__ __forceinline__ float column(const f32x4 (&v)[4], int e) { return v[e % 4][e / 4]; }

// (Called by all lanes of a wave; the next lane's row is `apart` further on.)
template <typename T>
__device__ __forceinline__ void write_row(const product_args& a, uint32_t row, uint32_t col, const f32x4 (&v)[4], uint32_t apart, uint32_t lane) {
    constexpr int V = 16 / sizeof(T), N = 16 / V;
    T* to = static_cast<T*>(a.c) + row * a.ldc + col;
    if (col + 16 <= a.m) {
        gd_u32x4 x[N];
#pragma unroll
        for (int b = 0; b < N; ++b) {
            gd_vec<T, V> old = {}, q;
            if (a.add && row < a.n) old = gd_read<T, V>(to + b * V);
#pragma unroll
            for (int e = 0; e < V; ++e) q.v[e] = gd_from_f32<T>(a.add ? column(v, b * V + e) + gd_to_f32(old.v[e]) : column(v, b * V + e));
            x[b] = __builtin_bit_cast(gd_u32x4, q);
        }
        exchange<N>(x, lane);
        const uint32_t first = row - (lane % N) * apart;
#pragma unroll
        for (int b = 0; b < N; ++b) {
            const uint32_t r = first + b * apart;
            if (r < a.n) *reinterpret_cast<gd_u32x4_anywhere*>(static_cast<T*>(a.c) + r * a.ldc + col + lane % N * V) = x[b];
        }
    } else if (row < a.n) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (col + e < a.m) to[e] = gd_from_f32<T>(a.add ? column(v, e) + gd_to_f32(to[e]) : column(v, e));
    }
}

// A kernel of any_type asks what C is when its sums are ready (sixteen kernels of direct tiles instead of 48).
struct any_type {};
template <typename T> struct type_is {
    typedef T type;
};
template <typename T, typename F>
__device__ __forceinline__ void with_type(const product_args& a, F&& f) {
    if constexpr (!std::is_same<T, any_type>::value) f(type_is<T>{});
    else if (a.type == GD_F32) f(type_is<float>{});
    else if (a.type == GD_BF16) f(type_is<gd_bf16>{});
    else f(type_is<gd_f16>{});
}

template <typename MUL, typename T, template <typename> class TILE>
__global__ __launch_bounds__(TILE<MUL>::NT, 512 / TILE<MUL>::NT) void tiled_kernel(const product_args a) {
    typedef TILE<MUL> tile;
    uint32_t tp, tq, t = stretch_of(blockIdx.x, gridDim.x);
    const uint32_t quarter = t % 4;
    if (a.parts) t = a.parts - 1 + t / 4;
    tile_of<4>(t, a.tiles_p, a.tiles_q, tp, tq);
    if (a.parts) {
        tp = 2 * tp + quarter % 2;
        tq = 2 * tq + quarter / 2;
        if (tp * tile::BP >= a.m || tq * tile::BQ >= a.n) return;
    }
    f32x4 acc[tile::FP][tile::FQ] = {};
    tile::run(a.p, a.q, tp * tile::BP, tq * tile::BQ, a.way, acc);
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    with_type<T>(a, [&](auto of) {
#pragma unroll
        for (int j = 0; j < tile::FQ; ++j)
#pragma unroll
            for (int g = 0; g < tile::FP / 4; ++g) {
                const f32x4 v[4] = {acc[4 * g][j], acc[4 * g + 1][j], acc[4 * g + 2][j], acc[4 * g + 3][j]};
                write_row<typename decltype(of)::type>(a, tq * tile::BQ + tile::q_of(wave) + 4 * (lane & 15) + j,
                                                       tp * tile::BP + tile::p_of(wave, g) + 16 * (lane >> 4), v, 4, lane);
            }
    });
}

template <typename MUL, typename T, int FQ, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 8 / WAVES) void direct_kernel(const product_args a) {
    typedef direct_tile<MUL, FQ, WAVES> tile;
    const uint32_t b = blockIdx.x, tq = b % a.tiles_q, tp = b / a.tiles_q, split = blockIdx.y;
    const uint32_t first = split * a.each, blocks = a.way.blocks;
    f32x4 v[4];
    tile::run(a.p, a.q, tp * tile::BP, tq * tile::BQ, a.way, first, min(first + a.each, blocks), v);
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    if (wave >= FQ) return;
    const uint32_t row = tq * tile::BQ + FQ * (lane & 15) + wave, col = tp * tile::BP + 16 * (lane >> 4);
    if (!a.slab) {
        with_type<T>(a, [&](auto of) { write_row<typename decltype(of)::type>(a, row, col, v, FQ, lane); });
    } else if (row < a.n && col < a.m4) {
        float* to = a.slab + (split * (uint64_t)a.n + row) * a.m4 + col;
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (col + 4 * r < a.m4) *reinterpret_cast<f32x4*>(to + 4 * r) = f32x4{v[0][r], v[1][r], v[2][r], v[3][r]};
    }
}

// The splits' sums in their order: four columns a lane.
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(const product_args a, uint32_t splits) {
    const uint64_t i = blockIdx.x * 256ull + threadIdx.x, each = a.m4 / 4;
    if (i >= a.n * each) return;
    const uint32_t row = (uint32_t)(i / each), col = (uint32_t)(i % each) * 4;
    const float* from = a.slab + (uint64_t)row * a.m4 + col;
    f32x4 s = *reinterpret_cast<const f32x4*>(from);
    for (uint32_t p = 1; p < splits; ++p) s += *reinterpret_cast<const f32x4*>(from + p * (uint64_t)a.n * a.m4);
    T* to = static_cast<T*>(a.c) + row * a.ldc + col;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (col + e < a.m) to[e] = gd_from_f32<T>(a.add ? s[e] + gd_to_f32(to[e]) : s[e]);
}

// k = 0: a sum of nothing.
template <typename T>
__global__ __launch_bounds__(256) void zero_kernel(const product_args a) {
    for (uint32_t row = blockIdx.x; row < a.n; row += gridDim.x)
        for (uint32_t col = threadIdx.x; col < a.m; col += 256) static_cast<T*>(a.c)[row * a.ldc + col] = T(0);
}

// Codes as bf16, with zeros up to the end of a block of 64: sixteen a lane at a time, by at most as many lanes as the chip has at once.  (One for
// each sixteen would be 2^32 of them from (n + m) k = 2^36 on, and the runtime starts a launch without those that 32 bits do not count.  As fast:
// 8 192 x 8 192 x 8 192 803 us, so 798; 5 000 x 4 096 x 4 096 161 and 159.)
constexpr uint32_t NUMBERS_GRID = 2048;
struct numbers_args {
    const uint8_t* codes;  uint64_t stride;
    const uint8_t* exp;  uint64_t exp_stride;
    uint32_t rows, k, e5m2, pieces;    // of sixteen, of a row, to the end of a block
    uint64_t count;                    // pieces of all rows
    uint8_t* out;
};

__global__ __launch_bounds__(256) void numbers_kernel(const numbers_args a, const numbers_args b) {
    for (uint64_t at = blockIdx.x * 256ull + threadIdx.x; at < a.count + b.count; at += gridDim.x * 256ull) {
        const bool second = at >= a.count;
        const numbers_args& x = second ? b : a;
        const uint64_t i = second ? at - a.count : at;
        const uint32_t row = (uint32_t)(i / x.pieces), piece = (uint32_t)(i % x.pieces);
        bf16x8 q[2] = {};
        if (piece * 16 < x.k) {
            gd_u32x4 w = *reinterpret_cast<const gd_u32x4*>(x.codes + row * x.stride + piece * 16);
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const int bytes = (int)(x.k - piece * 16) - 4 * h;
                w[h] &= bytes >= 4 ? 0xFFFFFFFFu : bytes <= 0 ? 0u : (1u << (8 * bytes)) - 1;
            }
            const float two = power_of(x.exp[piece / 8 * x.exp_stride + row]);
#pragma unroll
            for (int h = 0; h < 2; ++h) q[h] = x.e5m2 ? numbers_of<1>(w[2 * h], w[2 * h + 1], two) : numbers_of<0>(w[2 * h], w[2 * h + 1], two);
        }
        gd_u32x4* to = reinterpret_cast<gd_u32x4*>(x.out + i * 32);
        to[0] = __builtin_bit_cast(gd_u32x4, q[0]);
        to[1] = __builtin_bit_cast(gd_u32x4, q[1]);
    }
}

// ---- which tiles ------------------------------------------------------------------------------

struct plan {
    enum { LARGE, SMALL, DIRECT } kind;
    uint32_t fq, splits, each;
};

uint32_t up(uint64_t a, uint64_t b) { return (uint32_t)((a + b - 1) / b); }

// For the 8-bit cores tiles of 64 x 64 and smaller up to 768 of them (2 000 x 1 500 x 1 000, 768: 12.1 us, tiles of 128 x 128 12.7, of 256 x 256 22.2;
// 2 048 x 2 048 x 2 048, 1 024: 20.3, 16.0, 27.7), then of 256 x 256 from where they fill more than half of the chip (3 000 x 3 000 x 3 000, 144 of
// them: 44 us, 50 with 128 x 128; 2 048 x 4 096 x 4 096, 128: 52 and 40).  For the 16-bit ones, where larger tiles need their operands written out in
// bf16 first, of 64 x 64 up to there (1 024 x 4 096 x 4 096, 1 024: 42 us, 65, 98; 2 500 x 2 500 x 1 000, 1 600: 27, 34, 42; 3 000 x 3 000 x 3 000: 84,
// 90, 80).
plan plan_of(uint64_t n, uint64_t m, uint64_t k, bool in_16) {
    const uint64_t blocks = up(k, BYTES);
    plan w{plan::DIRECT, n <= 16 ? 1u : n <= 32 ? 2u : 4u, 1, (uint32_t)blocks};
    // (narrower where there is room for them, but of more than 64 rows, as every band of rows reads B: 700 x 700 x 4 000 in two splits 14.8 us,
    // in 242 tiles of 64 x 32 10.0; 64 x 4 096 x 4 096 11.0 and 12.9 with tiles of 64 x 16)
    while (n > 64 && w.fq > 1 && (uint64_t)up(n, 16 * w.fq / 2) * up(m, 64) <= 256) w.fq /= 2;
    const uint64_t tiles = (uint64_t)up(n, 16 * w.fq) * up(m, 64);
    const bool large = (uint64_t)up(n, 256) * up(m, 256) >= 140;
    if (n > 64 && tiles > 768 && (large || !in_16)) {
        w.kind = large ? plan::LARGE : plan::SMALL;
        return w;
    }
    // workgroups for every CU, as long as a wave keeps two blocks
    const uint64_t most = std::max<uint64_t>(1, blocks / 16);
    w.splits = (uint32_t)std::min<uint64_t>(most, std::max<uint64_t>(1, 256 / tiles));
    w.each = up(blocks, w.splits);
    w.splits = std::max(1u, up(blocks, w.each));
    return w;
}

// Of the splits' sums, or of the operands in bf16.
uint64_t row_of_numbers(uint64_t k) { return (k + 63) / 64 * 128; }
uint64_t work_bytes(uint64_t n, uint64_t m, uint64_t k, bool in_16) {
    const plan w = plan_of(n, m, k, in_16);
    return w.kind != plan::DIRECT ? (in_16 ? (n + m) * row_of_numbers(k) : 0) : w.splits > 1 ? w.splits * n * gd_align256(m * 4) : 0;
}

template <typename MUL, typename T>
hipError_t launch_tiles(product_args& a, const plan& w, hipStream_t s) {
    const uint32_t edge = w.kind == plan::LARGE ? 256 : 128;
    a.tiles_p = up(a.m, edge);
    a.tiles_q = up(a.n, edge);
    const uint32_t tiles = a.tiles_p * a.tiles_q;
    if (w.kind == plan::SMALL) {
        tiled_kernel<MUL, T, small_tile><<<tiles, 256, 0, s>>>(a);
        return hipGetLastError();
    }
    // What is left behind whole rounds of the chip's 256 workgroups as quarters, where two of those a CU take all of it (5 000 x 4 096 x
    // 4 096, 320 tiles: 94 us, so 80; fp32 184 and 158; 4 096 x 6 144 x 4 096, 384: 97 and 89).
    const uint32_t left = tiles > 256 && tiles % 256 <= 128 ? tiles % 256 : 0;
    tiled_kernel<MUL, T, large_tile><<<tiles - left, 512, 0, s>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    if (left) {
        a.parts = tiles - left + 1;
        tiled_kernel<MUL, T, small_tile><<<4 * left, 256, 0, s>>>(a);
    }
    return hipGetLastError();
}

template <typename MUL, typename T>
hipError_t launch_direct(product_args& a, const plan& w, hipStream_t s) {
    a.tiles_p = up(a.m, 64);
    a.tiles_q = up(a.n, 16 * w.fq);
    a.each = w.each;
    if (w.splits == 1) a.slab = nullptr;
    const dim3 grid(a.tiles_p * a.tiles_q, w.splits);
    if (w.fq == 1) direct_kernel<MUL, T, 1, 8><<<grid, 512, 0, s>>>(a);
    else if (w.fq == 2) direct_kernel<MUL, T, 2, 8><<<grid, 512, 0, s>>>(a);
    else if (a.tiles_p * a.tiles_q <= 256) direct_kernel<MUL, T, 4, 8><<<grid, 512, 0, s>>>(a);
    else direct_kernel<MUL, T, 4, 4><<<grid, 256, 0, s>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    if (w.splits > 1) {
        const uint32_t groups = up((uint64_t)a.n * (a.m4 / 4), 256);
        if (a.type == GD_F32) join_kernel<float><<<groups, 256, 0, s>>>(a, w.splits);
        else if (a.type == GD_BF16) join_kernel<gd_bf16><<<groups, 256, 0, s>>>(a, w.splits);
        else join_kernel<gd_f16><<<groups, 256, 0, s>>>(a, w.splits);
    }
    return hipGetLastError();
}

// P_CODES, Q_CODES: 1 for e5m2.
template <int P_CODES, int Q_CODES>
hipError_t launch(product_args& a, const plan& w, const gd_packed_product_args& g, hipStream_t s) {
    if (g.short_sums) {
        if (w.kind == plan::DIRECT) {
            if (g.out_type == GD_BF16) return launch_direct<of_codes<P_CODES, Q_CODES>, gd_bf16>(a, w, s);
            return launch_direct<of_codes<P_CODES, Q_CODES>, gd_f16>(a, w, s);
        }
        if (g.out_type == GD_BF16) return launch_tiles<of_codes<P_CODES, Q_CODES>, gd_bf16>(a, w, s);
        return launch_tiles<of_codes<P_CODES, Q_CODES>, gd_f16>(a, w, s);
    }
    if (w.kind == plan::DIRECT) return launch_direct<of_codes_in_16<P_CODES, Q_CODES>, any_type>(a, w, s);
    const uint64_t pitch = row_of_numbers(g.k);
    const uint32_t pieces = (uint32_t)(pitch / 32);
    numbers_args x[2];
    for (int i = 0; i < 2; ++i) {
        operand& o = i ? a.q : a.p;
        x[i] = numbers_args{o.p, o.pitch, o.exp, o.exp_pitch, o.rows, g.k, (uint32_t)(i ? Q_CODES : P_CODES), pieces, (uint64_t)o.rows * pieces,
                            g.work + (i ? g.m * pitch : 0)};
        o = operand{x[i].out, pitch, o.rows, (uint32_t)pitch, nullptr, 0};
    }
    numbers_kernel<<<std::min<uint64_t>((x[0].count + x[1].count + 255) / 256, NUMBERS_GRID), 256, 0, s>>>(x[0], x[1]);
    if (hipError_t e = hipGetLastError()) return e;
    a.way.blocks = (uint32_t)(pitch / BYTES);
    a.way.ends = 0;
    return launch_tiles<of_bf16, any_type>(a, w, s);
}

}  // namespace

size_t gd_packed_product_work(uint64_t n, uint64_t m, uint64_t k) {
    return n && m && k ? gd_align256(std::max(work_bytes(n, m, k, false), work_bytes(n, m, k, true))) : 0;
}

hipError_t gd_launch_packed_product(const gd_packed_product_args& g, hipStream_t s) {
    product_args a = {};
    a.n = g.n; a.m = g.m;
    a.c = g.out; a.ldc = g.out_stride; a.add = g.accumulate; a.type = g.out_type;
    if (g.k == 0) {
        if (g.accumulate) return hipSuccess;
        const uint32_t grid = std::min<uint32_t>(g.n, 65536);
        if (g.out_type == GD_F32) zero_kernel<float><<<grid, 256, 0, s>>>(a);
        else zero_kernel<uint16_t><<<grid, 256, 0, s>>>(a);
        return hipGetLastError();
    }
    // (the distance to a row that is not there says nothing, and need not keep the loads' alignment)
    const uint32_t row = up(g.k, 16) * 16;
    a.p = operand{static_cast<const uint8_t*>(g.b), g.m > 1 ? g.b_stride : row, g.m, row, g.b_exp, g.b_exp_stride};
    a.q = operand{static_cast<const uint8_t*>(g.a), g.n > 1 ? g.a_stride : row, g.n, row, g.a_exp, g.a_exp_stride};
    a.way.blocks = up(g.k, BYTES); a.way.ends = g.k % BYTES;
    a.slab = reinterpret_cast<float*>(g.work);
    a.m4 = (uint32_t)(gd_align256(g.m * 4ull) / 4);
    const plan w = plan_of(g.n, g.m, g.k, !g.short_sums);
    if (g.a_codes == GD_E4M3) return g.b_codes == GD_E4M3 ? launch<0, 0>(a, w, g, s) : launch<1, 0>(a, w, g, s);
    return g.b_codes == GD_E4M3 ? launch<0, 1>(a, w, g, s) : launch<1, 1>(a, w, g, s);
}
