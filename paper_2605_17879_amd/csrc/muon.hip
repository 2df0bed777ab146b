// Update of matrices by their orthogonalised momentum.  For a matrix W with gradient G and momentum M, all
// of them of many matrices at once:
//
//   M = mu M + G;  U = G + mu M, or M;  X = U / (|U| + eps), |U| the root of the sum of squares
//   steps times:  X = a X + (b A + c A^2) X,  A = X X^T        (of the shorter side: X^T X for tall matrices)
//   W = W (1 - lr decay) - lr X
//
// An odd polynomial p(s) = a s + b s^3 + c s^5 is applied to the singular values of X: those of the first step lie in (0, 1],
// the coefficients bring them towards 1.
//
// The matrix cores bound it: 2 a^2 b numbers are multiplied for A, half of them since A is symmetric, a^3 likewise for
// A^2, and a^2 b for the product with X.  They take f16; X, A and B = b A + c A^2 are kept in numbers of f16 times a power of two
// that their largest singular values allow, as hi + lo, and a product is one of
//   GD_F32   lo hi + hi lo + hi hi: 22 digits of each operand (hi and lo of 32 numbers side by side, so that each is loaded once for the
//            three: lo hi, hi lo and hi hi one behind the other took 1.06 to 1.12 times as long)
//   GD_F16   hi hi.  The X that is a part of the next one keeps its lo: what rounding drops of it would lie in directions whose
//            singular values are small, and grow with them, up to a^steps = 485 times (512 x 512, 16 strong directions over a floor of
//            noise: 1.1e-2 off with X in f16, 1.7e-4 with hi + lo; bf16 9e-2).  In the product with B it matters little: X hi there
//            instead of hi + lo changes 1.2e-3 to 1.6e-3 for a matrix of normal numbers, and saves half of the product.
//
// Every product is C[q][p] = sum_k P[p][k] Q[q][k] of rows that lie along k, so X is kept both ways, R as the matrix lies and
// C transposed; a lane's part of a tile is written both ways in whole lines (gd_tiles.h).  Symmetric products are computed on and
// above the diagonal of tiles and written to both sides.  One launch does a step's product for all matrices.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <vector>

#include "gd_tiles.h"

namespace {

using namespace gd_tiles;

constexpr float ONE_X = 0x1p15f;                   // X and A are kept times 2^15: below 65 504 for values below 1.99
constexpr uint32_t CUS = 256;
constexpr uint32_t CHUNKS = 1024;                  // most pieces of a matrix that its sum of squares is taken in
constexpr uint32_t CHUNK = 4096;                   // elements of a piece: a multiple of it
enum { LARGE, SMALL, DIRECT, KINDS, TINY = KINDS };   // tiles of the products; TINY: a matrix in one workgroup, in one launch
constexpr uint32_t EDGE[KINDS + 1] = {256, 128, 64, 0};
constexpr uint32_t TINY_NT = 512, TINY_A = 64, TINY_B = 192;      // the longest sides of a tiny matrix

// ---- the table ---------------------------------------------------------------------------------

struct entry {
    void* param;  const void* grad;  float* m;  void* copy;
    double lr_scale, decay;
    uint32_t rows, cols;
    uint32_t param_type, grad_type, copy_type;
    uint32_t chunks, chunk;       // pieces, and elements of one
    uint32_t partial;             // the first of its sums
    uint64_t at[2];               // where its matrices begin in the work area, with products of f32 and of f16
};

struct head {
    uint64_t mark;                // of all that follows: a launch reads a table that has the mark of the host's, or none
    uint64_t bytes;
    uint32_t magic, n;
    uint32_t first[KINDS + 1];    // entries of a kind of tiles; behind the last one's lie the tiny ones
    uint32_t share[KINDS][2][8];  // tiles of a symmetric product, and of the others, that each XCD takes
    uint32_t most[KINDS][2];      // that an XCD takes
    uint32_t whole[3];            // of the large ones, what an XCD takes as such of X X^T, A A^T and the others; the rest is taken in parts
    uint32_t chunks, tiles;       // pieces of all matrices, and 64 x 64 of them
    uint64_t work[2];
};
constexpr uint32_t MAGIC = 0x6D756F6E;
// Lists of one number an entry: what begins where, and for each XCD, of the tiles of symmetric products and then of the others, where an
// entry's begin, and what added to a place makes the tile of the entry's own.
enum { OF_CHUNKS, OF_TILES, OF_SHARES, LISTS = OF_SHARES + 2 * 8 * 2 };

constexpr uint64_t HEAD = 512;
static_assert(sizeof(head) <= HEAD, "the table's head");

__host__ __device__ inline uint64_t up_to(uint64_t v, uint64_t unit) { return (v + unit - 1) / unit * unit; }
__host__ __device__ inline uint64_t list_at(uint32_t n, int list) { return HEAD + n * sizeof(entry) + (uint64_t)list * up_to(n * 4, 16); }

// How a matrix of numbers of hi and lo lies: with `pairs` 32 hi and their 32 lo in turn, else the hi of a row and, `lo` bytes behind
// them, its lo, if it has them.
struct plane {
    uint64_t pitch;               // bytes between rows
    uint32_t cols;                // numbers of a row with the zeros behind its end
    uint32_t lo;                  // bytes from a hi to its lo; 0: there are none
    uint32_t pairs;
    // The first of sixteen numbers that begin at a multiple of sixteen, or of fewer inside of them.
    __host__ __device__ uint32_t at(uint32_t col) const { return pairs ? col / 32 * 128 + col % 32 * 2 : col * 2; }
    __host__ __device__ uint32_t blocks() const { return pairs ? cols / 32 : cols / 64; }
};

// Where an entry's matrices lie from its place in the work area on.
struct layout {
    uint32_t a, b;                // the shorter and the longer side
    plane r, c, s;                // X as the matrix lies and transposed; A and B
    uint64_t of_r, of_c, sa, sb, total;
    __host__ __device__ layout(uint32_t rows, uint32_t cols, bool both) {
        a = rows < cols ? rows : cols;
        b = rows < cols ? cols : rows;
        r = plane_of(cols, both, true);
        c = plane_of(rows, both, both);          // (without pairs R alone is a part of the next X)
        s = plane_of(a, both, both);
        of_r = up_to(rows * r.pitch, 256);
        of_c = up_to(cols * c.pitch, 256);
        const uint64_t of_s = up_to(a * s.pitch, 256);
        sa = 2 * (of_r + of_c);
        sb = sa + of_s;
        total = sb + of_s;
    }
    static __host__ __device__ plane plane_of(uint32_t cols, bool pairs, bool lo) {
        plane p;
        p.pairs = pairs;
        p.cols = (uint32_t)up_to(cols, pairs ? 32 : 64);
        p.lo = !lo ? 0 : pairs ? 64 : p.cols * 2;
        p.pitch = (uint64_t)p.cols * (lo ? 4 : 2);
        // (rows a multiple of 256 bytes apart meet at the same channels of the memory: 8 matrices of 1 024 x 1 024 and 8 of 2 048 x 1 024
        // 2.39 ms with such, 2.21 without, 4 of 4 096 x 4 096 5.95 and 5.76)
        if (p.pitch % 256 == 0) p.pitch += 128;
        return p;
    }
    // The first and the second X, as the matrix lies and transposed.
    __host__ __device__ uint64_t r_at(uint32_t i) const { return i * of_r; }
    __host__ __device__ uint64_t c_at(uint32_t i) const { return 2 * of_r + i * of_c; }
};

struct muon_args {
    const uint8_t* table;
    uint64_t mark;
    uint32_t n, tiled;            // entries, those that are not tiny
    uint32_t first, count;        // entries of the launch's kind
    uint32_t kind;                // of tiles
    uint32_t parts;               // of tiles of 256 x 256: the launch takes its own tiles of an XCD's, from this one on, plus 1; 0: of its kind
    uint8_t* work;
    const float* grad_scale;
    uint32_t both;                // products of f32
    uint32_t from, to;            // which of the two X is read and written
    float a, b, c, one_b;         // coefficients, and the power of two that B is kept times
    float mu;
    double eps;
    uint32_t nesterov;
    double lr;
};

// An entry, in scalar registers.
__device__ __forceinline__ entry entry_at(const muon_args& g, uint32_t i) {
    const uint32_t* from = reinterpret_cast<const uint32_t*>(g.table + HEAD + i * sizeof(entry));
    struct words {
        uint32_t w[sizeof(entry) / 4];
    } x;
#pragma unroll
    for (uint32_t k = 0; k < sizeof(entry) / 4; ++k) x.w[k] = __builtin_amdgcn_readfirstlane(from[k]);
    return __builtin_bit_cast(entry, x);
}

// Which of `count` entries from `first` on has place t of a list: the last that does not begin behind it.  A wave looks at 64 of them at
// once, of more at 64 an equal way apart first (1 500 matrices of 130 x 70 0.99 ms, with all of them looked at in turn 1.25).
__device__ __forceinline__ uint32_t entry_of(const muon_args& g, int list, uint32_t first, uint32_t count, uint32_t t) {
    const uint32_t* at = reinterpret_cast<const uint32_t*>(g.table + list_at(g.n, list));
    const uint32_t lane = threadIdx.x & 63;
    for (uint32_t left = count;;) {
        const uint32_t apart = (left + 63) / 64, i = lane * apart;
        const uint64_t begun = __ballot(i < left && at[first + min(i, left - 1)] <= t);
        const uint32_t behind = ((uint32_t)__popcll(begun) - 1) * apart;
        first = __builtin_amdgcn_readfirstlane(first + behind);
        if (apart == 1) return first;
        left = min(apart, left - behind);
    }
}
__device__ __forceinline__ uint32_t number_at(const muon_args& g, int list, uint32_t k) {
    return __builtin_amdgcn_readfirstlane(reinterpret_cast<const uint32_t*>(g.table + list_at(g.n, list))[k]);
}
// t becomes the number of the entry's own.
__device__ __forceinline__ uint32_t find(const muon_args& g, int list, uint32_t& t) {
    const uint32_t k = entry_of(g, list, 0, g.tiled, t);
    t -= number_at(g, list, k);
    return k;
}

// Whether there is something to do: the table is the one that the launch was made for, the gradients' factor (in f) is finite.
__device__ __forceinline__ bool begins(const muon_args& g, float& f) {
    f = g.grad_scale ? *g.grad_scale : 1.0f;
    return reinterpret_cast<const head*>(g.table)->mark == g.mark && (__builtin_bit_cast(uint32_t, f) & 0x7F800000u) != 0x7F800000u;
}

__device__ __forceinline__ float grad_at(const entry& e, uint64_t i) {
    return e.grad_type == GD_F32 ? static_cast<const float*>(e.grad)[i]
         : e.grad_type == GD_BF16 ? gd_to_f32(static_cast<const gd_bf16*>(e.grad)[i]) : gd_to_f32(static_cast<const gd_f16*>(e.grad)[i]);
}

// ---- momentum and norm ---------------------------------------------------------------------------

// U from the new momentum.
__device__ __forceinline__ float update_of(const muon_args& g, float grad, float m) { return g.nesterov ? grad + g.mu * m : m; }

__device__ __forceinline__ double sum_of_all(double s) {
    __shared__ double part[16];
#pragma unroll
    for (int d = 32; d; d /= 2) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x / 64] = s;
    __syncthreads();
    s = 0;
    for (uint32_t w = 0; w < blockDim.x / 64; ++w) s += part[w];
    return s;
}

template <typename T, int V>
__device__ __forceinline__ double advance(const muon_args& g, const entry& e, uint64_t i, float f) {
    const gd_vec<T, V> grad = gd_read<T, V>(static_cast<const T*>(e.grad) + i);
    gd_vec<float, 4> m[V / 4];
    double s = 0;
#pragma unroll
    for (int h = 0; h < V / 4; ++h) {
        m[h] = gd_read<float, 4>(e.m + i + 4 * h);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const float gr = g.grad_scale ? gd_to_f32(grad.v[4 * h + x]) * f : gd_to_f32(grad.v[4 * h + x]);
            m[h].v[x] = m[h].v[x] * g.mu + gr;
            const double u = update_of(g, gr, m[h].v[x]);
            s += u * u;
        }
    }
#pragma unroll
    for (int h = 0; h < V / 4; ++h) *reinterpret_cast<gd_u32x4_anywhere*>(e.m + i + 4 * h) = __builtin_bit_cast(gd_u32x4, m[h]);
    return s;
}

// M, and the sums of squares of U, a piece a workgroup.  Memory bounds it: 4 of 4 096 x 4 096 with gradients in bf16, 671 MB, 112 us, 6.0 TB/s
// (a part comes from the last level's cache).
__global__ __launch_bounds__(512) void momentum_kernel(const muon_args g) {
    float f;
    if (!begins(g, f)) return;
    uint32_t t = blockIdx.x;
    const entry e = entry_at(g, find(g, OF_CHUNKS, t));
    const uint64_t size = (uint64_t)e.rows * e.cols, from = (uint64_t)t * e.chunk, end = min(from + e.chunk, size);
    double s = 0;
    uint64_t i = from + threadIdx.x * 8;
    for (; i + 8 <= end; i += 4096)
        s += e.grad_type == GD_F32 ? advance<float, 4>(g, e, i, f) + advance<float, 4>(g, e, i + 4, f)
           : e.grad_type == GD_BF16 ? advance<gd_bf16, 8>(g, e, i, f) : advance<gd_f16, 8>(g, e, i, f);
    for (uint64_t j = i; j < min(i + 8, end); ++j) {
        const float gr = g.grad_scale ? grad_at(e, j) * f : grad_at(e, j), m = e.m[j] * g.mu + gr;
        e.m[j] = m;
        const double u = update_of(g, gr, m);
        s += u * u;
    }
    s = sum_of_all(s);
    if (threadIdx.x == 0) reinterpret_cast<double*>(g.work)[e.partial + t] = s;
}

struct halves {
    gd_f16 hi, lo;
};
__device__ __forceinline__ halves split(float x) {
    const gd_f16 hi = (gd_f16)x;
    return {hi, (gd_f16)(x - (float)hi)};
}
__device__ __forceinline__ float whole(gd_f16 hi, gd_f16 lo) { return (float)hi + (float)lo; }

typedef gd_f16 f16x4 __attribute__((ext_vector_type(4)));

// U of four rows of four columns each, as far as they are there.
template <typename T>
__device__ __forceinline__ void updates_of(const muon_args& g, const entry& e, uint32_t row, uint32_t col, float f, float (&u)[4][4]) {
    gd_vec<T, 4> grad[4] = {};
    gd_vec<float, 4> m[4] = {};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (row + i >= e.rows) break;
        const uint64_t at = (uint64_t)(row + i) * e.cols + col;
        const T* from = static_cast<const T*>(e.grad) + at;
        if (col + 4 <= e.cols) {
            __builtin_memcpy(&grad[i], from, sizeof(grad[i]));
            m[i] = gd_read<float, 4>(e.m + at);
        } else {
#pragma unroll
            for (int j = 0; j < 3; ++j)
                if (col + j < e.cols) {
                    grad[i].v[j] = from[j];
                    m[i].v[j] = e.m[at + j];
                }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float gr = gd_to_f32(grad[i].v[j]);
            u[i][j] = update_of(g, g.grad_scale ? gr * f : gr, m[i].v[j]);
        }
}

// X of the first step, 64 x 64 a workgroup, both ways, with zeros up to the end of a block of k.  Memory bounds it: 4 of 4 096 x 4 096, 805
// MB, 176 us, 4.6 TB/s.
__global__ __launch_bounds__(256) void start_kernel(const muon_args g) {
    float f;
    if (!begins(g, f)) return;
    uint32_t t = blockIdx.x;
    const entry e = entry_at(g, find(g, OF_TILES, t));
    const uint32_t tiles_c = (e.cols + 63) / 64, row = t / tiles_c * 64 + threadIdx.x / 16 * 4, col = t % tiles_c * 64 + threadIdx.x % 16 * 4;
    const double* part = reinterpret_cast<const double*>(g.work) + e.partial;
    double s = 0;
    for (uint32_t i = threadIdx.x; i < e.chunks; i += 256) s += part[i];
    float u[4][4] = {};                            // (on its way beside the sum)
    if (row < e.rows && col < e.cols) {
        if (e.grad_type == GD_F32) updates_of<float>(g, e, row, col, f, u);
        else if (e.grad_type == GD_BF16) updates_of<gd_bf16>(g, e, row, col, f, u);
        else updates_of<gd_f16>(g, e, row, col, f, u);
    }
    const double size = sqrt(sum_of_all(s)) + g.eps, scale = size == 0 ? 0 : ONE_X / size;   // (in 64 bits: no gradient is too small)
    const layout l(e.rows, e.cols, g.both);
    uint8_t* base = g.work + e.at[!g.both];
    halves x[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) x[i][j] = split((float)(u[i][j] * scale));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (row + i < e.rows && col < l.r.cols) {
            uint8_t* to = base + l.r_at(0) + (row + i) * l.r.pitch + l.r.at(col);
            *reinterpret_cast<f16x4*>(to) = f16x4{x[i][0].hi, x[i][1].hi, x[i][2].hi, x[i][3].hi};
            *reinterpret_cast<f16x4*>(to + l.r.lo) = f16x4{x[i][0].lo, x[i][1].lo, x[i][2].lo, x[i][3].lo};
        }
        if (col + i < e.cols && row < l.c.cols) {
            uint8_t* to = base + l.c_at(0) + (col + i) * l.c.pitch + l.c.at(row);
            *reinterpret_cast<f16x4*>(to) = f16x4{x[0][i].hi, x[1][i].hi, x[2][i].hi, x[3][i].hi};
            if (l.c.lo) *reinterpret_cast<f16x4*>(to + l.c.lo) = f16x4{x[0][i].lo, x[1][i].lo, x[2][i].lo, x[3][i].lo};
        }
    }
}

// ---- products ------------------------------------------------------------------------------------

enum { OF_X, OF_A, STEP, LAST };                   // A = X X^T; B = b A + c A A; X = a X + B X; the same, and W

// What becomes of a tile: element (q, p) of a matrix D [rows][cols], and of its transpose.
struct target {
    uint8_t* d;  plane of_d;       // written as it lies
    uint8_t* t;  plane of_t;       // written transposed, or null
    const uint8_t* old;            // A or X, as d lies
    uint32_t rows, cols;
};

struct problem {
    operand p, q;
    passage way;
    target out;
};

template <int PHASE>
__device__ __forceinline__ problem problem_of(const muon_args& g, const entry& e, bool off_diagonal) {
    const layout l(e.rows, e.cols, g.both);
    uint8_t* base = g.work + e.at[!g.both];
    const bool tall = e.rows > e.cols;
    uint8_t *r0 = base + l.r_at(g.from), *c0 = base + l.c_at(g.from), *r1 = base + l.r_at(g.to), *c1 = base + l.c_at(g.to);
    uint8_t *sa = base + l.sa, *sb = base + l.sb;
    problem x;
    auto matrix = [](const uint8_t* p, const plane& l, uint32_t rows) { return operand{p, l.pitch, rows, (uint32_t)l.pitch, nullptr, 0}; };
    x.way.ends = 0;
    if (PHASE == OF_X || PHASE == OF_A) {
        if (PHASE == OF_X) x.p = tall ? matrix(c0, l.c, l.a) : matrix(r0, l.r, l.a);
        else x.p = matrix(sa, l.s, l.a);
        x.q = x.p;
        x.way.blocks = PHASE == OF_A ? l.s.blocks() : tall ? l.c.blocks() : l.r.blocks();
        uint8_t* to = PHASE == OF_X ? sa : sb;
        x.out = target{to, l.s, off_diagonal ? to : nullptr, l.s, sa, l.a, l.a};
    } else {
        const operand b = matrix(sb, l.s, l.a);
        x.p = tall ? b : matrix(c0, l.c, e.cols);
        x.q = tall ? matrix(r0, l.r, e.rows) : b;
        x.way.blocks = l.s.blocks();
        x.out = target{r1, l.r, c1, l.c, r0, e.rows, e.cols};
    }
    return x;
}

// What was at sixteen columns of a row, from `col` on.
struct old_row {
    gd_u32x4 hi[2], lo[2];
};
__device__ __forceinline__ void read_old(const target& o, uint32_t row, uint32_t col, old_row& old) {
#pragma unroll
    for (int h = 0; h < 2; ++h) old.hi[h] = old.lo[h] = gd_u32x4{};
    if (row < o.rows && col < o.of_d.cols) {
        const gd_u32x4* from = reinterpret_cast<const gd_u32x4*>(o.old + row * o.of_d.pitch + o.of_d.at(col));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            old.hi[h] = from[h];
            if (o.of_d.lo) old.lo[h] = from[o.of_d.lo / 16 + h];
        }
    }
}

// Sixteen columns, from `col` on, of a row: v[i][r] is column 4 r + i, and becomes what the row does.
template <int PHASE>
__device__ __forceinline__ void finish_row(const muon_args& g, const target& o, uint32_t row, uint32_t col, f32x4 (&v)[4], const old_row& was) {
    gd_vec<gd_f16, 8> hi[2], lo[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        hi[h] = __builtin_bit_cast(gd_vec<gd_f16, 8>, was.hi[h]);
        lo[h] = __builtin_bit_cast(gd_vec<gd_f16, 8>, was.lo[h]);
    }
#pragma unroll
    for (int x = 0; x < 16; ++x) {
        float w = v[x % 4][x / 4];
        const float old = whole(hi[x / 8].v[x % 8], lo[x / 8].v[x % 8]);
        if (PHASE == OF_X) w *= 1 / ONE_X;
        else if (PHASE == OF_A) w = (g.c * (w * (1 / (ONE_X * ONE_X))) + g.b * (old * (1 / ONE_X))) * g.one_b;
        else w = g.a * old + w * (1 / g.one_b);
        v[x % 4][x / 4] = row < o.rows && col + x < o.cols ? w : 0.0f;   // (zeros up to the end of a block)
    }
}

// (Called by all lanes of a wave; the next lane's row is `apart` further on.)
__device__ __forceinline__ void write_row(const target& o, uint32_t row, uint32_t col, const f32x4 (&v)[4], uint32_t apart, uint32_t lane) {
    if (col >= o.of_d.cols) return;                // (the same for lanes that exchange)
    gd_u32x4 hi[2], lo[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        gd_vec<gd_f16, 8> x, y;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const halves s = split(v[e % 4][2 * h + e / 4]);
            x.v[e] = s.hi;
            y.v[e] = s.lo;
        }
        hi[h] = __builtin_bit_cast(gd_u32x4, x);
        lo[h] = __builtin_bit_cast(gd_u32x4, y);
    }
    exchange<2>(hi, lane);
    if (o.of_d.lo) exchange<2>(lo, lane);
    const uint32_t first = row - lane % 2 * apart;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t r = first + apart * h;
        if (r >= o.rows) break;
        uint8_t* to = o.d + r * o.of_d.pitch + o.of_d.at(col) + lane % 2 * 16;
        *reinterpret_cast<gd_u32x4*>(to) = hi[h];
        if (o.of_d.lo) *reinterpret_cast<gd_u32x4*>(to + o.of_d.lo) = lo[h];
    }
}

// N rows from `row` on of a column, written next to each other.
template <int N>
__device__ __forceinline__ void write_column(const target& o, uint32_t row, uint32_t col, const float (&x)[N]) {
    if (!o.t || col >= o.cols || row >= o.of_t.cols) return;
    typedef gd_f16 some __attribute__((ext_vector_type(N)));
    uint8_t* to = o.t + col * o.of_t.pitch + o.of_t.at(row);
    some hi, lo;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const halves h = split(x[i]);
        hi[i] = h.hi;
        lo[i] = h.lo;
    }
    *reinterpret_cast<some*>(to) = hi;
    if (o.of_t.lo) *reinterpret_cast<some*>(to + o.of_t.lo) = lo;
}

template <typename T>
__device__ __forceinline__ void write_param(const entry& e, uint64_t at, uint32_t there, float keep, float rate, const f32x4 (&v)[4]) {
    T* p = static_cast<T*>(e.param) + at;
    gd_bf16* b = e.copy && e.copy_type == GD_BF16 ? static_cast<gd_bf16*>(e.copy) + at : nullptr;
    gd_f16* h = e.copy && e.copy_type == GD_F16 ? static_cast<gd_f16*>(e.copy) + at : nullptr;
    constexpr int V = 16 / sizeof(T);
    if (there >= 16) {
        float x[16];
#pragma unroll
        for (int q = 0; q < 16; q += V) {
            gd_vec<T, V> old = gd_read<T, V>(p + q);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                x[q + i] = gd_to_f32(old.v[i]) * keep - v[(q + i) % 4][(q + i) / 4] * rate;
                old.v[i] = gd_from_f32<T>(x[q + i]);
            }
            gd_write_through<T, V>(p + q, old);
        }
#pragma unroll
        for (int q = 0; q < 16; q += 8) {
            gd_vec<gd_bf16, 8> to_b;
            gd_vec<gd_f16, 8> to_h;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                to_b.v[i] = gd_from_f32<gd_bf16>(x[q + i]);
                to_h.v[i] = gd_from_f32<gd_f16>(x[q + i]);
            }
            if (b) gd_write_through<gd_bf16, 8>(b + q, to_b);
            if (h) gd_write_through<gd_f16, 8>(h + q, to_h);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (i < there) {
                const float x = gd_to_f32(p[i]) * keep - v[i % 4][i / 4] * rate;
                p[i] = gd_from_f32<T>(x);
                if (b) b[i] = gd_from_f32<gd_bf16>(x);
                if (h) h[i] = gd_from_f32<gd_f16>(x);
            }
    }
}

__device__ __forceinline__ void update_row(const muon_args& g, const entry& e, uint32_t row, uint32_t col, const f32x4 (&v)[4]) {
    if (row >= e.rows || col >= e.cols) return;
    const double rate = g.lr * e.lr_scale;
    const float keep = (float)(1.0 - rate * e.decay), move = (float)(rate / ONE_X);
    const uint64_t at = (uint64_t)row * e.cols + col;
    if (e.param_type == GD_F32) write_param<float>(e, at, e.cols - col, keep, move, v);
    else if (e.param_type == GD_BF16) write_param<gd_bf16>(e, at, e.cols - col, keep, move, v);
    else write_param<gd_f16>(e, at, e.cols - col, keep, move, v);
}

// Tile t of a triangle of them: column tq, row tp <= tq.
__device__ __forceinline__ void corner_of(uint32_t t, uint32_t& tp, uint32_t& tq) {
    uint32_t q = (uint32_t)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
    while (q * (q + 1) / 2 > t) --q;
    while ((q + 1) * (q + 2) / 2 <= t) ++q;
    tq = q;
    tp = t - q * (q + 1) / 2;
}

// The workgroup's tile, and which of the `bands` of its rows; false if there is none.
template <int PHASE>
__device__ __forceinline__ bool place_of(const muon_args& g, uint32_t edge, uint32_t bands, uint32_t& tp, uint32_t& tq, uint32_t& band, entry& e) {
    constexpr bool HALF = PHASE == OF_X || PHASE == OF_A;
    // (workgroup b is on XCD b % 8)
    const uint32_t chip = blockIdx.x % 8;
    const int list = OF_SHARES + ((HALF ? 0 : 8) + (int)chip) * 2;
    uint32_t t = blockIdx.x / 8;
    band = t % bands;
    t /= bands;
    const uint32_t cut = g.parts ? 256 / edge : 1, part = t % (cut * cut), own = edge;
    if (g.parts) {
        t = g.parts - 1 + t / (cut * cut);
        edge = 256;
    }
    if (t >= reinterpret_cast<const head*>(g.table)->share[g.kind][!HALF][chip]) return false;
    const uint32_t k = entry_of(g, list, g.first, g.count, t);
    t += number_at(g, list + 1, k);
    e = entry_at(g, k);
    if (HALF) corner_of(t, tq, tp);                // (columns at or behind the rows)
    else tile_of<4>(t, (e.cols + edge - 1) / edge, (e.rows + edge - 1) / edge, tp, tq);
    if (!g.parts) return true;
    tp = cut * tp + part % cut;
    tq = cut * tq + part / cut;
    const uint32_t a = min(e.rows, e.cols);
    return (HALF ? tp >= tq : true) && tq * own < (HALF ? a : e.rows) && tp * own < (HALF ? a : e.cols);
}

template <int PHASE, typename TILE>
__global__ __launch_bounds__(TILE::NT, 512 / TILE::NT) void tiled_kernel(const muon_args g) {
    typedef TILE tile;
    float f;
    if (!begins(g, f)) return;
    uint32_t tp, tq, band;
    entry e;
    if (!place_of<PHASE>(g, tile::BP, 1, tp, tq, band, e)) return;
    const problem x = problem_of<PHASE>(g, e, tp != tq);
    f32x4 acc[tile::FP][tile::FQ] = {};
    tile::run(x.p, x.q, tp * tile::BP, tq * tile::BQ, x.way, acc);
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t row = tq * tile::BQ + tile::q_of(wave) + 4 * (lane & 15);
#pragma unroll
    for (int h = 0; h < tile::FP / 4; ++h) {
        const uint32_t col = tp * tile::BP + tile::p_of(wave, h) + 16 * (lane >> 4);
        f32x4 v[4][4];
        // (four rows are asked for before one is waited for)
        old_row old[4] = {};
        if (PHASE != OF_X) {
#pragma unroll
            for (int j = 0; j < 4; ++j) read_old(x.out, row + j, col, old[j]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[j][i] = acc[4 * h + i][j];
            finish_row<PHASE>(g, x.out, row + j, col, v[j], old[j]);
            if (PHASE == LAST) update_row(g, e, row + j, col, v[j]);
            else write_row(x.out, row + j, col, v[j], 4, lane);
        }
        if (PHASE != LAST) {
#pragma unroll
            for (int c = 0; c < 16; ++c)
                write_column<4>(x.out, row, col + c, {v[0][c % 4][c / 4], v[1][c % 4][c / 4], v[2][c % 4][c / 4], v[3][c % 4][c / 4]});
        }
    }
}

// Tiles of 64 columns and 16 FQ rows.
template <int PHASE, typename MUL, int FQ, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 8 / WAVES) void direct_kernel(const muon_args g) {
    typedef direct_tile<MUL, FQ, WAVES> tile;
    float f;
    if (!begins(g, f)) return;
    uint32_t tp, tq, part;
    entry e;
    if (!place_of<PHASE>(g, 64, 4 / FQ, tp, tq, part, e)) return;
    const problem x = problem_of<PHASE>(g, e, tp != tq);
    f32x4 v[4];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), first = tq * 64 + part * tile::BQ;
    const uint32_t row = first + FQ * (lane & 15), col = tp * 64 + 16 * (lane >> 4);
    old_row old = {};
    if (PHASE != OF_X && wave < FQ) read_old(x.out, row + wave, col, old);  // (on its way beside the sum)
    typename tile::sums* room = tile::run(x.p, x.q, tp * 64, first, x.way, 0, x.way.blocks, v);
    if (wave < FQ) {
        finish_row<PHASE>(g, x.out, row + wave, col, v, old);
        if (PHASE == LAST) update_row(g, e, row + wave, col, v);
        else write_row(x.out, row + wave, col, v, FQ, lane);
    }
    if (PHASE == LAST || !x.out.t) return;
    // the rows of a lane together, for the transpose: wave r has columns 4 r .. 4 r + 3
    if (wave < FQ) {
#pragma unroll
        for (int i = 0; i < 4; ++i) room[0][wave][i][lane] = v[i];
    }
    __syncthreads();
    if (wave < 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float some[FQ];
#pragma unroll
            for (int j = 0; j < FQ; ++j) some[j] = room[0][j][i][lane][wave];
            write_column<FQ>(x.out, row, col + 4 * wave + i, some);
        }
    }
}

// steps = 0: W from X of the start.
__global__ __launch_bounds__(256) void apply_kernel(const muon_args g) {
    float f;
    if (!begins(g, f)) return;
    uint32_t t = blockIdx.x;
    const entry e = entry_at(g, find(g, OF_TILES, t));
    const layout l(e.rows, e.cols, g.both);
    const uint8_t* base = g.work + e.at[!g.both] + l.r_at(0);
    const uint32_t tiles_c = (e.cols + 63) / 64, row = t / tiles_c * 64 + threadIdx.x / 4, col = t % tiles_c * 64 + threadIdx.x % 4 * 16;
    if (row >= e.rows || col >= e.cols) return;
    const gd_f16* from = reinterpret_cast<const gd_f16*>(base + row * l.r.pitch + l.r.at(col));
    f32x4 v[4];
#pragma unroll
    for (int x = 0; x < 16; ++x) v[x % 4][x / 4] = whole(from[x], from[l.r.lo / 2 + x]);
    update_row(g, e, row, col, v);
}

// ---- tiny matrices -------------------------------------------------------------------------------

// A matrix of up to 64 x 192 (or 192 x 64), momentum to parameters: X as a lane holds it, in fp32, in registers, and as
// operands in the LDS, hi and lo, both ways (R [i][j], C [j][i], i along the shorter side), A and B [i][i'].  A wave has pieces of 16 x 16 of a product: a
// lane four neighbouring j of one i of X.  Five steps are 15 products one behind the other, which with the launches of
// the larger matrices took 6 to 8 us each (six of 96 x 64: 105 us, so 24).  By their count the matrix instructions are some 3 us of that; how the
// rest falls on the reads, the writes and the four barriers of a step has not been measured.
struct tiny_lds {
    static constexpr uint32_t R = 2 * 2 * TINY_B, C = 2 * 2 * TINY_A, S = C;   // bytes of a row: hi, lo
    uint8_t r[TINY_A * R], c[TINY_B * C];
    union {
        struct {
            uint8_t a[TINY_A * S], b[TINY_A * S];
        };
        float u[TINY_A * TINY_B];                  // before the steps U, behind them X, as the matrix lies
    };
};

// Rows of 256 bytes for each 64 numbers: 128 of hi, 128 of lo.  In rows 8 to 15 of each 16 they change places, and of
// each 128 bytes chunk c lies at c ^ (row % 8), so that a read of sixteen rows meets every bank once (they bound the products: rows that met
// half of the banks 28.3 us for six of 96 x 64).  `at` is where a row's first 64 bytes of hi are; this is `shared` bytes of hi (a multiple of 32, the
// same for all lanes) further on; lo is at ^ 128.
__device__ __forceinline__ uint32_t tiny_further(uint32_t at, uint32_t shared) { return (at ^ (shared & 96)) + (shared & ~127u) * 2; }
__device__ __forceinline__ constexpr uint32_t tiny_turn(uint32_t row) { return (row & 15) * 16; }

// N products of 16 rows of P and the same 16 of Q, k_bytes (a multiple of 64) of each along k: side by side, so that one's sums and reads
// are under way while another's are waited for.
template <uint32_t P_PITCH, uint32_t Q_PITCH, int N>
__device__ __forceinline__ void tiny_products(f32x4 (&out)[N], const uint8_t* p, const uint32_t (&p0)[N], uint32_t p_row, const uint8_t* q,
                                              uint32_t q0, uint32_t q_row, uint32_t k_bytes, bool both) {
    f32x4 low[N] = {}, high[N] = {};
    q_row += q0 * Q_PITCH;
    for (uint32_t k = 0; k < k_bytes; k += 64) {
        const uint32_t pk = tiny_further(p_row, k), qk = tiny_further(q_row, k);
        f16x8 ph[N], pl[N];
        const f16x8 qh = *reinterpret_cast<const f16x8*>(q + qk);
#pragma unroll
        for (int n = 0; n < N; ++n) ph[n] = *reinterpret_cast<const f16x8*>(p + pk + p0[n] * P_PITCH);
        if (both) {
            const f16x8 ql = *reinterpret_cast<const f16x8*>(q + (qk ^ 128));
#pragma unroll
            for (int n = 0; n < N; ++n) pl[n] = *reinterpret_cast<const f16x8*>(p + (pk ^ 128) + p0[n] * P_PITCH);
#pragma unroll
            for (int n = 0; n < N; ++n) low[n] = multiply_16(pl[n], qh, low[n]);
#pragma unroll
            for (int n = 0; n < N; ++n) low[n] = multiply_16(ph[n], ql, low[n]);
        }
#pragma unroll
        for (int n = 0; n < N; ++n) high[n] = multiply_16(ph[n], qh, high[n]);
    }
#pragma unroll
    for (int n = 0; n < N; ++n) out[n] = high[n] + low[n];
}

// Four neighbouring numbers of a row, as four hi and four lo.
struct four_halves {
    f16x4 hi, lo;
};
__device__ __forceinline__ four_halves split_four(const f32x4& x) {
    const halves a = split(x[0]), b = split(x[1]), c = split(x[2]), d = split(x[3]);
    return {f16x4{a.hi, b.hi, c.hi, d.hi}, f16x4{a.lo, b.lo, c.lo, d.lo}};
}
template <uint32_t PITCH>
__device__ __forceinline__ void tiny_write(uint8_t* m, uint32_t row0, uint32_t at, uint32_t col0, const four_halves& x) {
    const uint32_t to = row0 * PITCH + tiny_further(at, col0 * 2);
    *reinterpret_cast<f16x4*>(m + to) = x.hi;
    *reinterpret_cast<f16x4*>(m + (to ^ 128)) = x.lo;
}

// Numbers from, from + TINY_NT, ... of a gradient of `all`.
template <int N>
__device__ __forceinline__ void grads_of(const entry& e, uint32_t from, uint32_t all, float (&x)[N]) {
    if (e.grad_type == GD_F32) {
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = static_cast<const float*>(e.grad)[min(from + TINY_NT * k, all - 1)];
    } else {
        uint16_t q[N];
#pragma unroll
        for (int k = 0; k < N; ++k) q[k] = static_cast<const uint16_t*>(e.grad)[min(from + TINY_NT * k, all - 1)];
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = e.grad_type == GD_BF16 ? gd_to_f32(__builtin_bit_cast(gd_bf16, q[k])) : gd_to_f32(__builtin_bit_cast(gd_f16, q[k]));
    }
}

template <typename T>
__device__ __forceinline__ void tiny_update(const entry& e, const float* x, uint32_t all, float keep, float move) {
    constexpr int N = 8;
    T* p = static_cast<T*>(e.param);
    for (uint32_t from = threadIdx.x; from < all; from += TINY_NT * N) {
        T q[N];
#pragma unroll
        for (int k = 0; k < N; ++k) q[k] = p[min(from + TINY_NT * k, all - 1)];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const uint32_t i = from + TINY_NT * k;
            if (i >= all) break;
            const float w = gd_to_f32(q[k]) * keep - x[i] * move;
            p[i] = gd_from_f32<T>(w);
            if (e.copy && e.copy_type == GD_BF16) static_cast<gd_bf16*>(e.copy)[i] = gd_from_f32<gd_bf16>(w);
            if (e.copy && e.copy_type == GD_F16) static_cast<gd_f16*>(e.copy)[i] = gd_from_f32<gd_f16>(w);
        }
    }
}

struct tiny_steps {
    uint32_t steps;
    float c[GD_MUON_MAX_STEPS][4];                 // a, b, c, and the power of two that B is kept times
};

__global__ __launch_bounds__(TINY_NT) void tiny_kernel(const muon_args g, const tiny_steps way) {
    __shared__ __attribute__((aligned(16))) tiny_lds lds;
    constexpr uint32_t WAVES = TINY_NT / 64;
    constexpr int MINE = TINY_A / 16 * (TINY_B / 16) / WAVES, SQUARES = TINY_A / 16 * (TINY_A / 16) / WAVES;
    float f;
    if (!begins(g, f)) return;
    const entry e = entry_at(g, g.first + blockIdx.x);
    const bool tall = e.rows > e.cols, both = g.both;
    const uint32_t a = tall ? e.cols : e.rows, b = tall ? e.rows : e.cols;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t ni = (a + 31) / 32 * 2, nj = (b + 31) / 32 * 2;      // pieces: whole steps of k of 32
    // piece t: i from 16 (t % ni) on, j from 16 (t / ni) on
    auto i_of = [&](uint32_t t) { return t % ni * 16 + (lane & 15); };
    auto j_of = [&](uint32_t t) { return t / ni * 16 + 4 * (lane >> 4); };
    auto place = [&](uint32_t i, uint32_t j) { return tall ? j * e.cols + i : i * e.cols + j; };
    // Eight numbers of a lane are asked for before one is written.  (All code is read from memory once a workgroup: loops that are
    // unrolled to 52 KB took as long as what they did.)
    constexpr int AT_ONCE = 8;
    const uint32_t all = a * b;
    double sum = 0;
    for (uint32_t from = threadIdx.x; from < all; from += TINY_NT * AT_ONCE) {
        float gr[AT_ONCE], m[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) m[k] = e.m[min(from + TINY_NT * k, all - 1)];
        grads_of<AT_ONCE>(e, from, all, gr);
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            if (g.grad_scale) gr[k] *= f;
            m[k] = m[k] * g.mu + gr[k];
            if (from + TINY_NT * k >= all) break;
            e.m[from + TINY_NT * k] = m[k];
            const float u = update_of(g, gr[k], m[k]);
            lds.u[from + TINY_NT * k] = u;
            sum += (double)u * u;
        }
    }
    f32x4 x[MINE];
    const double size = sqrt(sum_of_all(sum)) + g.eps, scale = size == 0 ? 0 : ONE_X / size;
    // Where a lane reads of an operand (row lane % 16, 16 bytes of 64) and writes of a result (row lane % 16, 8 bytes of 32; two
    // bytes of 32 of each of four rows, transposed)
    const uint32_t row = lane & 15, quarter = lane >> 4, chunk = quarter * 16 ^ tiny_turn(row);
    const uint32_t r_read = row * tiny_lds::R + chunk, c_read = row * tiny_lds::C + chunk;
    const uint32_t piece = (quarter / 2 * 16 ^ tiny_turn(row)) + quarter % 2 * 8;
    const uint32_t r_write = row * tiny_lds::R + piece, s_write = row * tiny_lds::S + piece;
    auto keep_x = [&]() {
#pragma unroll
        for (int k = 0; k < MINE; ++k) {
            const uint32_t t = wave + WAVES * k;
            if (t >= ni * nj) break;
            const uint32_t i0 = t % ni * 16, j0 = t / ni * 16;
            const four_halves h = split_four(x[k]);
            tiny_write<tiny_lds::R>(lds.r, i0, r_write, j0, h);
#pragma unroll
            for (uint32_t r = 0; r < 4; ++r) {
                const uint32_t at = (4 * quarter + r) * tiny_lds::C + (row / 8 * 16 ^ tiny_turn(4 * quarter + r)) + row % 8 * 2;
                const uint32_t to = j0 * tiny_lds::C + tiny_further(at, i0 * 2);
                *reinterpret_cast<gd_f16*>(lds.c + to) = h.hi[r];
                *reinterpret_cast<gd_f16*>(lds.c + (to ^ 128)) = h.lo[r];
            }
        }
        __syncthreads();
    };
#pragma unroll
    for (int k = 0; k < MINE; ++k) {
        const uint32_t t = wave + WAVES * k, i = i_of(t), j = j_of(t);
#pragma unroll
        for (int r = 0; r < 4; ++r) x[k][r] = t < ni * nj && i < a && j + r < b ? (float)(lds.u[place(i, j + r)] * scale) : 0.0f;
    }
    __syncthreads();
    if (way.steps) keep_x();
    for (uint32_t s = 0; s < way.steps; ++s) {
        const float ca = way.c[s][0], cb = way.c[s][1], cc = way.c[s][2], one_b = way.c[s][3];
        // (a wave's pieces have the same rows of Q: 8 is a multiple of ni; one that is not there has the last one's of P)
        const uint32_t from = wave % ni * 16;
        uint32_t to[SQUARES];
#pragma unroll
        for (int k = 0; k < SQUARES; ++k) to[k] = min(wave + WAVES * k, ni * ni - 1) / ni * 16;
        f32x4 mine[SQUARES], square[SQUARES];
        // A, of which a piece's row is along Q
        tiny_products<tiny_lds::R, tiny_lds::R>(mine, lds.r, to, r_read, lds.r, from, r_read, nj * 32, both);
#pragma unroll
        for (int k = 0; k < SQUARES; ++k) {
            mine[k] *= 1 / ONE_X;
            if (wave + WAVES * k < ni * ni) tiny_write<tiny_lds::S>(lds.a, from, s_write, to[k], split_four(mine[k]));
        }
        __syncthreads();
        tiny_products<tiny_lds::S, tiny_lds::S>(square, lds.a, to, c_read, lds.a, from, c_read, ni * 32, both);
#pragma unroll
        for (int k = 0; k < SQUARES; ++k)
            if (wave + WAVES * k < ni * ni)
                tiny_write<tiny_lds::S>(lds.b, from, s_write, to[k], split_four((square[k] * (cc / (ONE_X * ONE_X)) + mine[k] * (cb / ONE_X)) * one_b));
        __syncthreads();
#pragma unroll
        for (int first = 0; first < MINE; first += 3) {
            if (wave + WAVES * first >= ni * nj) break;
            uint32_t j0[3];
#pragma unroll
            for (int k = 0; k < 3; ++k) j0[k] = min(wave + WAVES * (first + k), ni * nj - 1) / ni * 16;
            f32x4 bx[3];
            tiny_products<tiny_lds::C, tiny_lds::S>(bx, lds.c, j0, c_read, lds.b, from, c_read, ni * 32, both);
#pragma unroll
            for (int k = 0; k < 3; ++k) x[first + k] = x[first + k] * ca + bx[k] * (1 / one_b);
        }
        if (s + 1 < way.steps) {
            __syncthreads();                       // (X read by all)
            keep_x();
        }
    }
    __syncthreads();                               // (A and B read by all)
#pragma unroll
    for (int k = 0; k < MINE; ++k) {
        const uint32_t t = wave + WAVES * k, i = i_of(t), j = j_of(t);
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (t < ni * nj && i < a && j + r < b) lds.u[place(i, j + r)] = x[k][r];
    }
    __syncthreads();
    const double rate = g.lr * e.lr_scale;
    const float keep = (float)(1.0 - rate * e.decay), move = (float)(rate / ONE_X);
    if (e.param_type == GD_F32) tiny_update<float>(e, lds.u, all, keep, move);
    else if (e.param_type == GD_BF16) tiny_update<gd_bf16>(e, lds.u, all, keep, move);
    else tiny_update<gd_f16>(e, lds.u, all, keep, move);
}

template <int PHASE, typename MUL>
void launch_phase_of(muon_args g, const head& h, hipStream_t s) {
    for (int k = 0; k < KINDS; ++k) {
        const uint32_t most = h.most[k][PHASE == OF_X || PHASE == OF_A ? 0 : 1];
        if (!most) continue;
        g.first = h.first[k];
        g.count = h.first[k + 1] - h.first[k];
        g.kind = (uint32_t)k;
        if (k == LARGE) {
            const uint32_t whole = h.whole[PHASE == OF_X ? 0 : PHASE == OF_A ? 1 : 2];
            if (whole) tiled_kernel<PHASE, large_tile<MUL>><<<8 * whole, 512, 0, s>>>(g);
            if (whole < most) {
                g.parts = whole + 1;
                // (so few that two workgroups a CU take them as tiles of 64 x 64: of 4 096 x 4 352, 272 tiles, the last 16 as quarters 1.95 ms
                // for all, so 1.79)
                if (16 * 8 * (most - whole) <= 2 * CUS) direct_kernel<PHASE, MUL, 4, 4><<<8 * 16 * (most - whole), 256, 0, s>>>(g);
                else tiled_kernel<PHASE, small_tile<MUL>><<<8 * 4 * (most - whole), 256, 0, s>>>(g);
                g.parts = 0;
            }
        }
        else if (k == SMALL) tiled_kernel<PHASE, small_tile<MUL>><<<8 * most, 256, 0, s>>>(g);
        // (bands of 16 or 32 rows of a tile where there are CUs for them: 4 of 1 000 x 333 193 us, so 170; 1 of 512 x 512 162, 126; 8 of
        // 128 x 128 117, 93)
        else if (4 * 8 * most <= CUS) direct_kernel<PHASE, MUL, 1, 8><<<4 * 8 * most, 512, 0, s>>>(g);
        else if (2 * 8 * most <= CUS) direct_kernel<PHASE, MUL, 2, 8><<<2 * 8 * most, 512, 0, s>>>(g);
        else if (8 * most <= CUS) direct_kernel<PHASE, MUL, 4, 8><<<8 * most, 512, 0, s>>>(g);
        else direct_kernel<PHASE, MUL, 4, 4><<<8 * most, 256, 0, s>>>(g);
    }
}

template <int PHASE>
void launch_phase(const muon_args& g, const head& h, hipStream_t s) {
    if (g.both) launch_phase_of<PHASE, of_pairs>(g, h, s);
    else launch_phase_of<PHASE, of_f16>(g, h, s);
}

uint64_t tiles_of(const gd_muon_tensor& t, uint64_t edge) { return ((t.rows + edge - 1) / edge) * ((t.cols + edge - 1) / edge); }

// Which tiles the matrices take.  Tiles of 256 x 256 where they fill the chip (1 of 4 096 x 4 096, 256: 3.96 ms, with tiles of 128 x 128
// 4.29; 4 of 2 048 x 2 048, 256: 2.27 and 2.33; 8 of 1 024 x 1 024, 128: 1.10 and 0.80) and are not mostly empty; else tiles of 128 x 128
// where those of 64 x 64 would be two rounds of the chip and more (64 of 256 x 256, 1 024: 0.30 and 0.33; 8 of 1 024 x 1 024, 2 048: 0.80 and
// 0.87; 8 of 333 x 500, 384: 0.26 and 0.17) of matrices that are not long, whose products over the long side are few tiles of many blocks (4 of
// 512 x 2 048, 1 024: 0.45 and 0.32; 2 of 1 024 x 4 096, 2 048: 0.86 and 0.79).
void choose_kinds(const gd_muon_tensor* t, uint32_t n, std::vector<int>& kinds) {
    kinds.assign(n, DIRECT);
    auto side = [&](uint32_t i) { return std::min(t[i].rows, t[i].cols); };
    auto fills = [&](uint32_t i) { return side(i) >= 512 && tiles_of(t[i], 256) * 4 * 10 <= tiles_of(t[i], 128) * 13; };
    uint64_t large = 0, direct = 0;
    for (uint32_t i = 0; i < n; ++i)
        if (side(i) <= TINY_A && std::max(t[i].rows, t[i].cols) <= TINY_B) kinds[i] = TINY;
    for (uint32_t i = 0; i < n; ++i)
        if (fills(i)) large += tiles_of(t[i], 256);
    for (uint32_t i = 0; i < n; ++i)
        if (large >= 240 && fills(i)) kinds[i] = LARGE;
        else if (side(i) > 64) direct += tiles_of(t[i], 64);
    for (uint32_t i = 0; i < n; ++i)
        if (kinds[i] == DIRECT && side(i) > 64 && direct >= 1024 && std::max(t[i].rows, t[i].cols) < 3 * side(i)) kinds[i] = SMALL;
}

int bits_of(uint64_t v) { return v ? 64 - __builtin_clzll(v) : 0; }

// A kind's matrices, and for the tiles of symmetric products and for the others what each XCD takes of them.
struct dealt {
    std::vector<uint32_t> order;
    std::vector<uint32_t> begins[2][8], shift[2][8];
    uint32_t share[2][8] = {};
};

// Each XCD takes a stretch of the tiles of all matrices alike in the bits of their sides, those with the longer ones first: as much work
// as the others, and rows that it has in its L2 (2 of 4 096 x 4 096, 4 of 4 096 x 1 024 and 4 of 1 024 x
// 1 024: 8.3 ms; eighths of the list as the caller has it, with all the long ones on one half of the chip: 9.4).
void deal_out(const gd_muon_tensor* t, uint64_t edge, dealt& d) {
    auto a = [&](uint32_t i) { return std::min(t[i].rows, t[i].cols); };
    auto b = [&](uint32_t i) { return std::max(t[i].rows, t[i].cols); };
    auto like = [&](uint32_t i) { return bits_of(a(i)) * 64 + bits_of(b(i)); };
    std::stable_sort(d.order.begin(), d.order.end(), [&](uint32_t x, uint32_t y) { return like(x) > like(y); });
    for (int full = 0; full < 2; ++full) {
        double load[8] = {};
        auto tiles = [&](uint32_t i) {
            const uint64_t ta = (a(i) + edge - 1) / edge, tb = (b(i) + edge - 1) / edge;
            return full ? ta * tb : ta * (ta + 1) / 2;
        };
        size_t end;
        for (size_t begin = 0; begin < d.order.size(); begin = end) {
            uint64_t all = 0;
            for (end = begin; end < d.order.size() && like(d.order[end]) == like(d.order[begin]); ++end) all += tiles(d.order[end]);
            // (what an eighth leaves goes where there is the least so far)
            int chips[8] = {0, 1, 2, 3, 4, 5, 6, 7};
            std::stable_sort(chips, chips + 8, [&](int x, int y) { return load[x] < load[y]; });
            uint64_t from[9] = {}, behind = 0;
            for (uint64_t r = 0; r < 8; ++r) from[chips[r] + 1] = all / 8 + (r < all % 8);
            for (int x = 0; x < 8; ++x) {
                load[x] += (double)from[x + 1] * (double)(full ? a(d.order[begin]) : a(d.order[begin]) + b(d.order[begin]));
                from[x + 1] += from[x];
            }
            for (size_t k = begin; k < end; ++k) {
                const uint64_t here = tiles(d.order[k]);
                for (int x = 0; x < 8; ++x) {
                    const uint64_t first = std::max(behind, from[x]), last = std::min(behind + here, from[x + 1]);
                    d.begins[full][x].push_back(d.share[full][x]);
                    d.shift[full][x].push_back((uint32_t)(first - behind) - d.share[full][x]);
                    if (last > first) d.share[full][x] += (uint32_t)(last - first);
                }
                behind += here;
            }
        }
    }
}

// Tiles of 256 x 256 that have a k of `cost`, with what their ends take; quarters of them that are there.
struct large_tiles {
    double cost;
    uint64_t tiles, quarters;
};

// How many of a launch's large tiles are taken as such, a multiple of 256; UINT64_MAX: all.  One a CU, or two quarters: a round of those
// takes 0.6 of the time, 0.35 if there is but one for a CU.  All tiles, whole rounds and the rest in parts, or parts alone: what is a tenth
// faster by that count (12 of 2 048 x 1 024, X X^T and A A^T of 120 tiles as 432 quarters, the others of 384 as 256 and 512 quarters: 2.07
// ms -> 1.72; 4 of 4 096 x 4 096, X X^T, 544: 315 us as three rounds, 292 as two and 128 quarters).
uint64_t whole_of(std::vector<large_tiles> list) {
    std::stable_sort(list.begin(), list.end(), [](const large_tiles& x, const large_tiles& y) { return x.cost > y.cost; });
    uint64_t all = 0;
    for (const auto& l : list) all += l.tiles;
    auto time = [&](uint64_t whole) {
        double sum = 0, last = 0;
        uint64_t at = 0, quarters = 0;
        for (const auto& l : list) {
            const uint64_t w = std::min(l.tiles, whole - std::min(whole, at));
            sum += l.cost * (double)((at + w + CUS - 1) / CUS - (at + CUS - 1) / CUS);
            at += w;
            if (w == l.tiles) continue;
            const uint64_t q = l.quarters - l.quarters * w / l.tiles;
            sum += 0.6 * l.cost * (double)((quarters + q + 2 * CUS - 1) / (2 * CUS) - (quarters + 2 * CUS - 1) / (2 * CUS));
            if (quarters / (2 * CUS) != (quarters + q) / (2 * CUS) || quarters % (2 * CUS) == 0) last = l.cost;
            quarters += q;
        }
        if (quarters % (2 * CUS) != 0 && quarters % (2 * CUS) <= CUS) sum -= 0.25 * last;
        return sum;
    };
    uint64_t best = all;
    for (uint64_t whole : {all / CUS * CUS, (uint64_t)0})
        if (time(whole) < (best == all ? 0.9 : 1.0) * time(best)) best = whole;
    return best == all ? UINT64_MAX : best;
}

// The largest magnitude of a polynomial c1 x + c3 x^3 + c5 x^5, and of b x^2 + c x^4, over [0, s].
double most_of(double c1, double c3, double c5, double s) {
    double most = 0;
    auto look = [&](double x2) {
        if (x2 > 0 && x2 <= s * s) most = std::max(most, std::fabs(std::sqrt(x2) * (c1 + x2 * (c3 + x2 * c5))));
    };
    look(s * s);
    const double d = 9 * c3 * c3 - 20 * c5 * c1;
    if (c5 == 0) {
        if (c3 != 0) look(-c1 / (3 * c3));
    } else if (d >= 0) {
        look((-3 * c3 + std::sqrt(d)) / (10 * c5));
        look((-3 * c3 - std::sqrt(d)) / (10 * c5));
    }
    return most;
}
double most_of_even(double b, double c, double s) {
    double most = std::fabs(s * s * (b + s * s * c));
    if (c != 0) {
        const double x2 = -b / (2 * c);
        if (x2 > 0 && x2 < s * s) most = std::max(most, std::fabs(x2 * (b + x2 * c)));
    }
    return most;
}

// FNV-1a, 64 bits.
uint64_t mark_of(const uint8_t* p, size_t n) {
    uint64_t x = 0xCBF29CE484222325ull;
    for (size_t i = 0; i < n; ++i) x = (x ^ p[i]) * 0x100000001B3ull;
    return x;
}

}  // namespace

size_t gd_muon_table(const gd_muon_tensor* t, uint32_t n, void* out) {
    dealt of[KINDS + 1];
    std::vector<int> kinds;
    choose_kinds(t, n, kinds);
    uint32_t there = 0;
    for (uint32_t i = 0; i < n; ++i)
        if (t[i].rows && t[i].cols) {
            of[kinds[i]].order.push_back(i);
            ++there;
        }
    const size_t bytes = gd_align256(list_at(there, LISTS));
    uint8_t* to = static_cast<uint8_t*>(out);
    if (to) memset(to, 0, bytes);
    head h = {};
    h.bytes = bytes;
    h.magic = MAGIC;
    h.n = there;
    uint64_t chunks = 0, tiles = 0, work[2];
    uint32_t k = 0;
    // the sums of squares first
    for (uint32_t i = 0; i < n; ++i) chunks += (t[i].rows * t[i].cols + CHUNK - 1) / CHUNK;   // (an upper bound)
    work[0] = work[1] = gd_align256(std::min<uint64_t>(chunks, (uint64_t)there * CHUNKS) * 8);
    chunks = 0;
    std::vector<large_tiles> large[3];
    for (int kind = 0; kind <= KINDS; ++kind) {
        uint64_t half = 0, full = 0;
        h.first[kind] = k;
        for (uint32_t i : of[kind].order) {
            const uint64_t edge = std::max(EDGE[kind], 1u), tr = (t[i].rows + edge - 1) / edge, tc = (t[i].cols + edge - 1) / edge, ta = std::min(tr, tc);
            half += ta * (ta + 1) / 2;
            full += tr * tc;
        }
        // (launches of fewer than 2^32 threads)
        if (kind != TINY && (half >= 1u << 23 || full >= 1u << 23)) return 0;
        if (kind != TINY) deal_out(t, EDGE[kind], of[kind]);
        for (uint32_t i : of[kind].order) {
            const gd_muon_tensor& x = t[i];
            const uint64_t size = x.rows * x.cols;
            entry e = {};
            e.param = x.d_param; e.grad = x.d_grad; e.m = static_cast<float*>(x.d_m); e.copy = x.d_copy;
            e.lr_scale = x.lr_scale; e.decay = x.weight_decay;
            e.rows = (uint32_t)x.rows; e.cols = (uint32_t)x.cols;
            e.param_type = x.param_type; e.grad_type = x.grad_type; e.copy_type = x.copy_type;
            e.chunk = (uint32_t)up_to((size + CHUNKS - 1) / CHUNKS, CHUNK);
            e.chunks = (uint32_t)((size + e.chunk - 1) / e.chunk);
            e.partial = (uint32_t)chunks;
            if (to) {
                for (int b = 0; b < 2; ++b) e.at[b] = work[b];
                memcpy(to + HEAD + k * sizeof(entry), &e, sizeof(e));
                auto note = [&](int list, uint64_t v) {
                    const uint32_t number = (uint32_t)v;
                    memcpy(to + list_at(there, list) + 4ull * k, &number, 4);
                };
                note(OF_CHUNKS, chunks);
                note(OF_TILES, tiles);
                for (int l = 0; l < 16 && kind != TINY; ++l) {
                    note(OF_SHARES + 2 * l, of[kind].begins[l / 8][l % 8][k - h.first[kind]]);
                    note(OF_SHARES + 2 * l + 1, of[kind].shift[l / 8][l % 8][k - h.first[kind]]);
                }
            }
            ++k;
            if (kind == TINY) continue;
            for (int b = 0; b < 2; ++b) work[b] += layout(e.rows, e.cols, b == 0).total;
            chunks += e.chunks;
            tiles += ((x.rows + 63) / 64) * ((x.cols + 63) / 64);
            if (kind == LARGE) {
                // (a tile's ends take as long as 800 of k)
                const uint64_t tr = (x.rows + 255) / 256, tc = (x.cols + 255) / 256, ta = std::min(tr, tc);
                const uint64_t qr = (x.rows + 127) / 128, qc = (x.cols + 127) / 128, qa = std::min(qr, qc);
                const double k_x = 800.0 + (double)std::max(x.rows, x.cols), k_a = 800.0 + (double)std::min(x.rows, x.cols);
                large[0].push_back({k_x, ta * (ta + 1) / 2, qa * (qa + 1) / 2});
                large[1].push_back({k_a, ta * (ta + 1) / 2, qa * (qa + 1) / 2});
                large[2].push_back({k_a, tr * tc, qr * qc});
            }
        }
        if (k >= 1u << 22) return 0;
        if (kind == TINY) break;
        memcpy(h.share[kind], of[kind].share, sizeof(h.share[kind]));
        for (int l = 0; l < 2; ++l) h.most[kind][l] = *std::max_element(h.share[kind][l], h.share[kind][l] + 8);
    }
    if (chunks >= 1u << 23 || tiles >= 1u << 24) return 0;
    for (int phase = 0; phase < 3; ++phase) {
        const uint32_t most = h.most[LARGE][phase == 2];
        h.whole[phase] = (uint32_t)std::min<uint64_t>(most, whole_of(large[phase]) / 8);
    }
    h.chunks = (uint32_t)chunks;
    h.tiles = (uint32_t)tiles;
    h.work[0] = work[0];
    h.work[1] = work[1];
    if (to) {
        memcpy(to, &h, sizeof(h));
        h.mark = mark_of(to + sizeof(h.mark), bytes - sizeof(h.mark));
        memcpy(to, &h.mark, sizeof(h.mark));
    }
    return bytes;
}

bool gd_muon_table_fits(const void* host_table, size_t bytes) {
    head h;
    if (bytes < HEAD) return false;
    memcpy(&h, host_table, sizeof(h));
    return h.magic == MAGIC && h.bytes == bytes && list_at(h.n, LISTS) <= bytes;
}

size_t gd_muon_work(const void* host_table, bool both) {
    head h;
    memcpy(&h, host_table, sizeof(h));
    return h.work[both ? 0 : 1];
}

bool gd_muon_coefficients_fit(const double* c, uint32_t steps) {
    double s = 1.001;
    for (uint32_t i = 0; i < steps; ++i) {
        if (!(std::isfinite(c[3 * i]) && std::isfinite(c[3 * i + 1]) && std::isfinite(c[3 * i + 2]))) return false;
        s = most_of(c[3 * i], c[3 * i + 1], c[3 * i + 2], s) * 1.001;
        if (!(s <= 1.35)) return false;
    }
    return true;
}

hipError_t gd_launch_muon(const gd_muon_args& m, hipStream_t s) {
    head h;
    memcpy(&h, m.host_table, sizeof(h));
    if (h.n == 0) return hipSuccess;
    muon_args g = {};
    g.table = m.table; g.mark = h.mark; g.n = h.n; g.work = m.work; g.grad_scale = m.grad_scale;
    g.both = m.both; g.mu = m.momentum; g.eps = m.eps; g.nesterov = m.nesterov; g.lr = m.lr;
    g.tiled = h.first[TINY];
    if (g.tiled) {
        momentum_kernel<<<h.chunks, 512, 0, s>>>(g);
        start_kernel<<<h.tiles, 256, 0, s>>>(g);
        if (m.steps == 0) apply_kernel<<<h.tiles, 256, 0, s>>>(g);
    }
    tiny_steps way;
    way.steps = m.steps;
    double most = 1.001;
    for (uint32_t i = 0; i < m.steps; ++i) {
        const double* c = m.coefficients + 3 * i;
        g.a = (float)c[0]; g.b = (float)c[1]; g.c = (float)c[2];
        // B's singular values are below `b_most`: times the largest power of two that leaves them half of f16's range
        const double b_most = most_of_even(c[1], c[2], most);
        g.one_b = (float)std::exp2(std::min(15.0, std::floor(std::log2(32768.0 / std::max(b_most, 1e-30)))));
        most = most_of(c[0], c[1], c[2], most) * 1.001;
        const float of_step[4] = {g.a, g.b, g.c, g.one_b};
        memcpy(way.c[i], of_step, sizeof(of_step));
        if (!g.tiled) continue;
        g.from = i & 1;
        g.to = 1 - g.from;
        launch_phase<OF_X>(g, h, s);
        launch_phase<OF_A>(g, h, s);
        if (i + 1 < m.steps) launch_phase<STEP>(g, h, s);
        else launch_phase<LAST>(g, h, s);
    }
    if (h.n > g.tiled) {
        g.first = g.tiled;
        tiny_kernel<<<h.n - g.tiled, TINY_NT, 0, s>>>(g, way);
    }
    return hipGetLastError();
}
