// Embedding lookup, out[i] = round(scale * W[t_i]), and its gradient,
// dW[v] (+)= round(scale * sum of dOut[i] over the i with t_i = v).
//
// The lookup moves rows and computes next to nothing: lanes hold 16 bytes of a row each, a row or more a workgroup, and the
// memory bounds it (16 384 x 2 048 fp32, 182 MB: 31 us, 5.8 TB/s).
//
// The gradient must not depend on the order in which workgroups run, so there are no float
// atomics: the (token, position) pairs are sorted by token, stably, and the sorted list is cut into
// stretches.  A workgroup sums the rows of one stretch, one column vector per lane, and writes a
// token's sum when the next token begins.  A token that goes on over a stretch's end leaves fp32
// partial sums (one at the front and one at the back of each stretch), which a second kernel adds up in
// order, in pairs, fours, ... of sixteen parts and these one behind another.  There are at most MOST_STRETCHES, so that the longest chain
// of additions of n rows is that of n / 4 096 rows and 256 more (1 000 000 rows x 256 bf16 233 us; in stretches of 32 rows all of them
// 340, and a token of 4 194 304 rows was off by 1e-3).  The sums run at the memory's rate (16 384 x 4 096 bf16 added: 41 us,
// 6 TB/s); the rest of the time are short launches one behind another (85 us in all).
// The parts of one token are one workgroup's for 1 024 columns: a list that one token dominates takes longer (32 768 x 2 048, no token /
// one on half / on all of the rows: 127 / 157 / 186 us; 16 384 x 4 096 added: 84 / 116 / 127).
//
// Short lists cost launches, not work: up to FEW rows each row's workgroup looks for its token in the whole list and,
// if the row is the token's first, sums them all, in one launch (1 000 x 1 000 fp32, no token / one on half / on all of the rows: 8.6 / 24 / 49
// us; 2 048 x 512: 8.8 / 39 / 76).
//
// The gradient's zeros are written by workgroups of the sorting launches that have no keys: sorting is
// a chain of short launches that leaves the memory idle.
#include "gd_operators.h"

namespace {

constexpr uint32_t NT = 256;
constexpr uint32_t BITS = 9, DIGITS = 1u << BITS;   // of a sorting pass: two passes up to 262 143 rows
constexpr uint32_t SORT_KEYS = 1024;      // keys of a workgroup in a sorting pass
constexpr uint32_t ONE_SORT = 4096;       // most keys that one workgroup sorts by itself
// Workgroups of a sorting pass (us for two passes of n rows x 1 000, all launches): up to SELF_COUNT each counts all keys itself (5 000
// rows 30.3 against 36.9, 16 384 47.2 against 44.9), up to SELF_SCAN each adds up the counts of a first launch, else a third one does.
constexpr uint32_t SELF_COUNT = 8, SELF_SCAN = 64;
// Most rows whose tokens are compared with each other instead of sorted, and most workgroups that this may take (us for rows
// of 1 000 bf16 added, few / sorted: 1 100 rows 9.4 / 17.2, 2 000 13.4 / 18.0; of 4 096 fp32, 8 workgroups a row: 1 100 21.8 / 20.7,
// 2 000 33.9 / 26.6).
constexpr uint32_t FEW = 2048, FEW_GROUPS = 8192;
constexpr uint32_t MOST_GROUPS = 1u << 21;  // of a launch: HIP takes less than 2^32 threads in a dimension
constexpr uint32_t BATCH = 8;             // rows on their way at once in the sums
constexpr uint32_t MOST_STRETCHES = 4096;
constexpr uint32_t FILL_ROWS = 16384;     // most rows that one of its workgroups fills with zeros
constexpr uint32_t NO_ROW = 0xFFFFFFFFu;

// ---- lookup ------------------------------------------------------------------------------------

// A lane's V columns from c on.  The last lane of a row that is no multiple of V long reads (and sums) the row's last V
// columns, `skip` of which are its neighbour's, and writes the others.  Rows have V columns at least.
struct columns {
    uint32_t at, skip;
};
template <int V>
__device__ __forceinline__ columns columns_of(uint32_t c, uint32_t width) {
    const uint32_t at = min(c, width - V);
    return columns{at, c - at};
}
template <typename T, int V>
__device__ __forceinline__ void write_own(T* p, const gd_vec<T, V>& q, uint32_t skip) {
    if (skip == 0) {
        gd_write_through(p, q);
    } else if constexpr (sizeof(q) == 16) {                   // (in pieces of 8, 4 and 2 bytes, from a copy moved down)
        const auto w = __builtin_bit_cast(uint4, q);
        const uint64_t lo = (uint64_t)w.y << 32 | w.x, hi = (uint64_t)w.w << 32 | w.z;
        const uint32_t bits = skip * sizeof(T) * 8, left = 16 - skip * (uint32_t)sizeof(T);
        uint64_t rest = bits < 64 ? lo >> bits | hi << (64 - bits) : hi >> (bits - 64);
        uint8_t* to = reinterpret_cast<uint8_t*>(p + skip);
        if (left & 8) { __builtin_memcpy(to, &rest, 8); to += 8; rest = hi >> (bits & 63); }
        if (left & 4) { const uint32_t x = (uint32_t)rest; __builtin_memcpy(to, &x, 4); to += 4; rest >>= 32; }
        if (left & 2) { const uint16_t x = (uint16_t)rest; __builtin_memcpy(to, &x, 2); }
    } else {
#pragma unroll
        for (uint32_t j = 1; j < V; ++j)
            if (j >= skip) p[j] = q.v[j];
    }
}

// tx lanes side by side on a row, NT / tx rows a workgroup; V elements a lane at a time.
template <typename T, int V>
__global__ __launch_bounds__(NT) void embed_kernel(const gd_embed_args a, uint32_t log_tx) {
    const uint32_t tx = 1u << log_tx, lane = threadIdx.x & (tx - 1);
    const uint32_t rows = NT >> log_tx;
    for (uint32_t i = blockIdx.x * rows + (threadIdx.x >> log_tx); i < a.tokens.n; i += gridDim.x * rows) {
        const int64_t t = gd_token(a.tokens, i);
        T* out = static_cast<T*>(a.out) + i * a.out_stride;
        const bool row = t >= 0 && t < (int64_t)a.vocab;
        const T* w = static_cast<const T*>(a.weight) + (row ? (uint64_t)t : 0) * a.weight_stride;
        const float other = t < 0 ? 0.0f : __uint_as_float(0x7FC00000u);
        for (uint32_t c0 = lane * V; c0 < a.width; c0 += tx * V) {
            const columns c = columns_of<V>(c0, a.width);
            gd_vec<T, V> q;
            if (row) q = gd_read<T, V>(w + c.at);
#pragma unroll
            for (int j = 0; j < V; ++j) q.v[j] = gd_from_f32<T>(row ? gd_to_f32(q.v[j]) * a.scale : other);
            write_own<T, V>(out + c.at, q, c.skip);
        }
    }
}

template <typename T, int V>
hipError_t launch_embed(const gd_embed_args& a, hipStream_t s) {
    uint32_t log_tx = 0;
    while (log_tx < 8 && (1u << log_tx) * V < a.width) ++log_tx;
    const uint32_t rows = NT >> log_tx, groups = (a.tokens.n + rows - 1) / rows;
    hipLaunchKernelGGL((embed_kernel<T, V>), dim3(groups < MOST_GROUPS ? groups : MOST_GROUPS), dim3(NT), 0, s, a, log_tx);
    return hipGetLastError();
}

// ---- the stable sort by token ---------------------------------------------------------------

struct sort_args {
    gd_token_list tokens;
    uint32_t* key[2];
    uint32_t* pos[2];
    uint32_t* hist;      // [blocks + 1][DIGITS] counts; where they were scanned, those before a block, and totals
    uint32_t n, vocab, blocks, from, shift, scanned;
};

// Zeros that a launch writes beside its own work: rows from..to of the gradient.
struct fill_args {
    void* p;  uint64_t stride;
    uint32_t width, from, to;
};

// Tokens to keys: those without a row get the largest one and sort behind all others.
__device__ __forceinline__ uint32_t key_of(int64_t t, uint32_t vocab) { return t >= 0 && t < (int64_t)vocab ? (uint32_t)t : vocab; }

// The keys of positions from, from + step, ...; those behind the list's end are the last one's.
template <int N>
__device__ __forceinline__ void keys_of(const sort_args& a, uint32_t from, uint32_t step, uint32_t (&k)[N]) {
    if (a.shift) {
#pragma unroll
        for (int b = 0; b < N; ++b) k[b] = a.key[a.from][min(from + b * step, a.n - 1)];
    } else {
        int64_t t[N];
        gd_tokens<N>(a.tokens, from, step, t);
#pragma unroll
        for (int b = 0; b < N; ++b) k[b] = key_of(t[b], a.vocab);
    }
}

// For each lane: which lanes of the wave hold the same digit (among those with a key).
__device__ __forceinline__ uint64_t same_digit(uint32_t d, bool there) {
    uint64_t same = __ballot(there);
#pragma unroll
    for (uint32_t b = 0; b < BITS; ++b) {
        const uint64_t with = __ballot((d >> b) & 1);
        same &= ((d >> b) & 1) ? with : ~with;
    }
    return same;
}

// Workgroup `block` of `blocks` fills its share: of rows next to each other 16 bytes a lane and, below 8 GB, no more (512 MB: 79 us; 16 bytes
// again and again by 2 048 workgroups 112 us), of rows apart every blocks-th row.
template <typename T, int V, int THREADS>
__device__ __forceinline__ void fill_rows(const fill_args& f, uint32_t block, uint32_t blocks) {
    if (f.stride == f.width) {
        T* const begin = static_cast<T*>(f.p) + (uint64_t)f.from * f.width;
        T* const end = static_cast<T*>(f.p) + (uint64_t)f.to * f.width;
        typedef gd_vec<T, 16 / sizeof(T)> line;
        T* p = reinterpret_cast<T*>(((uintptr_t)begin & ~(uintptr_t)15) + ((uint64_t)block * THREADS + threadIdx.x) * 16);
        for (; p < end; p += (uint64_t)blocks * THREADS * (16 / sizeof(T))) {
            if (p >= begin && p + 16 / sizeof(T) <= end) {
                gd_write_through(p, line{});
            } else {
#pragma unroll
                for (uint32_t j = 0; j < 16 / sizeof(T); ++j)
                    if (p + j >= begin && p + j < end) p[j] = gd_from_f32<T>(0.0f);
            }
        }
    } else {
        for (uint32_t r = f.from + block; r < f.to; r += blocks)
            for (uint32_t c = threadIdx.x * V; c < f.width; c += THREADS * V)
                gd_write_through(static_cast<T*>(f.p) + (uint64_t)r * f.stride + columns_of<V>(c, f.width).at, gd_vec<T, V>{});
    }
}
template <typename T, int THREADS>
uint32_t fillers(const fill_args& f) {
    if (f.from == f.to) return 0;
    if (f.stride != f.width) return f.to - f.from < 8192 ? f.to - f.from : 8192;
    // (one more where the first line begins before the first row)
    const uint64_t groups = ((uint64_t)(f.to - f.from) * f.width * sizeof(T) + 14) / 16 / THREADS + 1;
    return (uint32_t)(groups < MOST_GROUPS ? groups : MOST_GROUPS);
}

// All passes by one workgroup of sixteen waves, the keys in its registers and, between passes, in the LDS.
// A wave owns a stretch of keys, 64 a round.
template <typename T, int V>
__global__ __launch_bounds__(1024) void sort_alone(sort_args a, fill_args f) {
    if (blockIdx.x > 0) return fill_rows<T, V, 1024>(f, blockIdx.x - 1, gridDim.x - 1);
    constexpr uint32_t WAVES = 16, ROUNDS = ONE_SORT / 1024;
    __shared__ uint32_t skey[ONE_SORT];
    __shared__ uint16_t spos[ONE_SORT];
    __shared__ uint16_t next[WAVES][DIGITS];
    __shared__ uint32_t part[DIGITS / 64];
    const uint32_t rounds = (a.n + 1023) / 1024;
    const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x & 63, base = wave * rounds * 64;
    uint32_t key[ROUNDS], pos[ROUNDS];
    // (rounds that there are not have no keys: every lane is behind the end)
    const auto there = [&](uint32_t r) { return r < rounds && base + r * 64 + lane < a.n; };
    keys_of<ROUNDS>(a, base + lane, 64, key);
#pragma unroll
    for (uint32_t r = 0; r < ROUNDS; ++r) pos[r] = base + r * 64 + lane;
    for (uint32_t shift = 0; shift == 0 || (a.vocab >> shift) > 0; shift += BITS) {
        for (uint32_t i = threadIdx.x; i < WAVES * DIGITS; i += 1024) (&next[0][0])[i] = 0;
        __syncthreads();
        uint32_t before[ROUNDS] = {};
#pragma unroll
        for (uint32_t r = 0; r < ROUNDS; ++r) {
            // (the wave's own counter: its lanes read it before the first of them adds)
            const uint32_t d = (key[r] >> shift) & (DIGITS - 1);
            if (r >= rounds) continue;
            const uint64_t same = same_digit(d, there(r));
            const uint32_t mine = (uint32_t)__popcll(same & ((1ull << lane) - 1));
            before[r] = next[wave][d] + mine;
            __builtin_amdgcn_wave_barrier();
            if (there(r) && mine == 0) next[wave][d] = (uint16_t)(next[wave][d] + (uint32_t)__popcll(same));
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        // counts to places: of the waves before, then of the digits before
        uint32_t total = 0, sum = 0;
        if (threadIdx.x < DIGITS) {
#pragma unroll
            for (uint32_t w = 0; w < WAVES; ++w) {
                const uint32_t c = next[w][threadIdx.x];
                next[w][threadIdx.x] = (uint16_t)total;
                total += c;
            }
            sum = total;
#pragma unroll
            for (uint32_t d = 1; d < 64; d <<= 1) {
                const uint32_t v = __shfl_up(sum, d);
                if (lane >= d) sum += v;
            }
            if (lane == 63) part[wave] = sum;
        }
        __syncthreads();
        if (threadIdx.x < DIGITS) {
            uint32_t at = sum - total;
            for (uint32_t w = 0; w < wave; ++w) at += part[w];
#pragma unroll
            for (uint32_t w = 0; w < WAVES; ++w) next[w][threadIdx.x] = (uint16_t)(next[w][threadIdx.x] + at);
        }
        __syncthreads();
#pragma unroll
        for (uint32_t r = 0; r < ROUNDS; ++r)
            if (there(r)) {
                const uint32_t at = next[wave][(key[r] >> shift) & (DIGITS - 1)] + before[r];
                skey[at] = key[r];
                spos[at] = (uint16_t)pos[r];
            }
        __syncthreads();
#pragma unroll
        for (uint32_t r = 0; r < ROUNDS; ++r) {
            const uint32_t i = base + r * 64 + lane;
            if (there(r)) { key[r] = skey[i]; pos[r] = spos[i]; }
        }
    }
#pragma unroll
    for (uint32_t r = 0; r < ROUNDS; ++r) {
        const uint32_t i = base + r * 64 + lane;
        if (there(r)) { a.key[0][i] = key[r]; a.pos[0][i] = pos[r]; }
    }
}

// A whole pass in one launch where there are few blocks: each workgroup of sixteen waves counts all keys itself, those
// before its own apart.
template <typename T, int V>
__global__ __launch_bounds__(1024) void sort_pass(sort_args a, fill_args f) {
    if (blockIdx.x >= a.blocks) return fill_rows<T, V, 1024>(f, blockIdx.x - a.blocks, gridDim.x - a.blocks);
    constexpr uint32_t WAVES = 16, ASK = 8;
    __shared__ uint32_t count[2][DIGITS];                     // of the keys in blocks before this one; of the others
    __shared__ uint32_t next[WAVES][DIGITS];
    __shared__ uint32_t part[DIGITS / 64];
    static_assert(SORT_KEYS == 1024, "a key a lane");
    const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x & 63, mine = blockIdx.x * SORT_KEYS + threadIdx.x;
    const auto digit = [&](uint32_t k) { return (k >> a.shift) & (DIGITS - 1); };
    (&count[0][0])[threadIdx.x] = 0;
    for (uint32_t i = threadIdx.x; i < WAVES * DIGITS; i += 1024) (&next[0][0])[i] = 0;
    const bool there = mine < a.n;
    uint32_t own[1];
    keys_of<1>(a, mine, 0, own);
    const uint32_t key = own[0], pos = there && a.shift ? a.pos[a.from][mine] : mine;
    __syncthreads();
    for (uint32_t b0 = 0; b0 < a.blocks; b0 += ASK) {
        uint32_t k[ASK];
        keys_of<ASK>(a, b0 * SORT_KEYS + threadIdx.x, SORT_KEYS, k);
#pragma unroll
        for (uint32_t b = 0; b < ASK; ++b) {
            const bool in = (b0 + b) * SORT_KEYS + threadIdx.x < a.n;
            const uint32_t d = digit(k[b]);
            const uint64_t who = __ballot(in);
            if (who == 0) continue;
            uint32_t* to = count[b0 + b < blockIdx.x ? 0 : 1];
            // (a frequent token's keys come in runs from the second pass on: one addition for a wave of them)
            if (__ballot(in && d == (uint32_t)__builtin_amdgcn_readfirstlane(d)) == who) {
                if (lane == 0) atomicAdd(&to[d], (uint32_t)__popcll(who));
            } else if (in) {
                atomicAdd(&to[d], 1u);
            }
        }
    }
    const uint64_t same = same_digit(digit(key), there);
    const uint32_t before = (uint32_t)__popcll(same & ((1ull << lane) - 1));
    if (there && before == 0) next[wave][digit(key)] = (uint32_t)__popcll(same);
    __syncthreads();
    // places of each digit's keys, then of each wave's
    uint32_t total = 0, sum = 0;
    if (threadIdx.x < DIGITS) {
        total = sum = count[0][threadIdx.x] + count[1][threadIdx.x];
#pragma unroll
        for (uint32_t d = 1; d < 64; d <<= 1) {
            const uint32_t v = __shfl_up(sum, d);
            if (lane >= d) sum += v;
        }
        if (lane == 63) part[wave] = sum;
    }
    __syncthreads();
    if (threadIdx.x < DIGITS) {
        uint32_t at = sum - total + count[0][threadIdx.x], c[WAVES];
        for (uint32_t w = 0; w < wave; ++w) at += part[w];
#pragma unroll
        for (uint32_t w = 0; w < WAVES; ++w) c[w] = next[w][threadIdx.x];
#pragma unroll
        for (uint32_t w = 0; w < WAVES; ++w) { next[w][threadIdx.x] = at; at += c[w]; }
    }
    __syncthreads();
    if (there) {
        const uint32_t to = next[wave][digit(key)] + before;
        a.key[a.from ^ 1][to] = key;
        a.pos[a.from ^ 1][to] = pos;
    }
}

template <typename T, int V>
__global__ __launch_bounds__(NT) void sort_count(sort_args a, fill_args f) {
    if (blockIdx.x >= a.blocks) return fill_rows<T, V, NT>(f, blockIdx.x - a.blocks, gridDim.x - a.blocks);
    __shared__ uint32_t h[DIGITS];
    for (uint32_t d = threadIdx.x; d < DIGITS; d += NT) h[d] = 0;
    __syncthreads();
    uint32_t key[SORT_KEYS / NT];
    keys_of<SORT_KEYS / NT>(a, blockIdx.x * SORT_KEYS + threadIdx.x, NT, key);
#pragma unroll
    for (uint32_t r = 0; r < SORT_KEYS / NT; ++r)
        if (blockIdx.x * SORT_KEYS + r * NT + threadIdx.x < a.n) atomicAdd(&h[(key[r] >> a.shift) & (DIGITS - 1)], 1u);
    __syncthreads();
    for (uint32_t d = threadIdx.x; d < DIGITS; d += NT) a.hist[(uint64_t)blockIdx.x * DIGITS + d] = h[d];
}

// A digit's counts to the counts of the blocks before each, workgroup d for digit d; its total goes into the
// row behind the last block's.
__global__ __launch_bounds__(NT) void sort_scan(uint32_t* h, uint32_t blocks) {
    __shared__ uint32_t s[NT];
    uint32_t sum = 0;
    for (uint32_t base = 0; base < blocks; base += NT) {
        const uint32_t b = base + threadIdx.x;
        const uint32_t c = b < blocks ? h[(uint64_t)b * DIGITS + blockIdx.x] : 0;
        s[threadIdx.x] = c;
        __syncthreads();
        for (uint32_t d = 1; d < NT; d <<= 1) {
            const uint32_t v = threadIdx.x >= d ? s[threadIdx.x - d] : 0;
            __syncthreads();
            s[threadIdx.x] += v;
            __syncthreads();
        }
        if (b < blocks) h[(uint64_t)b * DIGITS + blockIdx.x] = sum + s[threadIdx.x] - c;
        sum += s[NT - 1];
        __syncthreads();
    }
    if (threadIdx.x == 0) h[(uint64_t)blocks * DIGITS + blockIdx.x] = sum;
}

template <typename T, int V>
__global__ __launch_bounds__(NT) void sort_scatter(sort_args a, fill_args f) {
    if (blockIdx.x >= a.blocks) return fill_rows<T, V, NT>(f, blockIdx.x - a.blocks, gridDim.x - a.blocks);
    constexpr uint32_t WAVES = NT / 64, ROUNDS = SORT_KEYS / NT, PER = DIGITS / NT;
    __shared__ uint32_t next[WAVES][DIGITS];
    __shared__ uint32_t part[WAVES];
    const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x & 63;
    const uint32_t base = blockIdx.x * SORT_KEYS + wave * (SORT_KEYS / WAVES);
    for (uint32_t i = threadIdx.x; i < WAVES * DIGITS; i += NT) (&next[0][0])[i] = 0;
    __syncthreads();
    uint32_t key[ROUNDS], pos[ROUNDS], before[ROUNDS];
    keys_of<ROUNDS>(a, base + lane, 64, key);
#pragma unroll
    for (uint32_t r = 0; r < ROUNDS; ++r) {
        const uint32_t i = base + r * 64 + lane;
        pos[r] = a.shift ? a.pos[a.from][min(i, a.n - 1)] : i;
    }
#pragma unroll
    for (uint32_t r = 0; r < ROUNDS; ++r) {
        const uint32_t d = (key[r] >> a.shift) & (DIGITS - 1);
        const bool there = base + r * 64 + lane < a.n;
        const uint64_t same = same_digit(d, there);
        const uint32_t mine = (uint32_t)__popcll(same & ((1ull << lane) - 1));
        before[r] = next[wave][d] + mine;
        __builtin_amdgcn_wave_barrier();
        if (there && mine == 0) next[wave][d] += (uint32_t)__popcll(same);
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    // lane t has the digits PER * t and on: places of the block's keys, then of each wave's
    uint32_t total = 0, at[PER], all[PER];
#pragma unroll
    for (uint32_t e = 0; e < PER; ++e) {
        const uint32_t* h = a.hist + threadIdx.x * PER + e;
        at[e] = a.scanned ? h[(uint64_t)blockIdx.x * DIGITS] : 0;
        all[e] = a.scanned ? h[(uint64_t)a.blocks * DIGITS] : 0;
    }
    static_assert(PER == 2, "two digits a lane");
    if (!a.scanned)
        for (uint32_t b0 = 0; b0 < a.blocks; b0 += 16) {         // (sixteen loads on their way at once)
            uint2 c[16];
#pragma unroll
            for (uint32_t b = 0; b < 16; ++b)
                c[b] = b0 + b < a.blocks ? reinterpret_cast<const uint2*>(a.hist + (uint64_t)(b0 + b) * DIGITS)[threadIdx.x] : make_uint2(0, 0);
#pragma unroll
            for (uint32_t b = 0; b < 16; ++b) {
                all[0] += c[b].x; all[1] += c[b].y;
                if (b0 + b < blockIdx.x) { at[0] += c[b].x; at[1] += c[b].y; }
            }
        }
#pragma unroll
    for (uint32_t e = 0; e < PER; ++e) total += all[e];
    uint32_t sum = total;
#pragma unroll
    for (uint32_t d = 1; d < 64; d <<= 1) {
        const uint32_t v = __shfl_up(sum, d);
        if (lane >= d) sum += v;
    }
    if (lane == 63) part[wave] = sum;
    __syncthreads();
    sum -= total;
    for (uint32_t w = 0; w < wave; ++w) sum += part[w];
#pragma unroll
    for (uint32_t e = 0; e < PER; ++e) { at[e] += sum; sum += all[e]; }
#pragma unroll
    for (uint32_t e = 0; e < PER; ++e)
#pragma unroll
        for (uint32_t w = 0; w < WAVES; ++w) {
            uint32_t& slot = next[w][threadIdx.x * PER + e];
            const uint32_t c = slot;
            slot = at[e];
            at[e] += c;
        }
    __syncthreads();
#pragma unroll
    for (uint32_t r = 0; r < ROUNDS; ++r)
        if (base + r * 64 + lane < a.n) {
            const uint32_t to = next[wave][(key[r] >> a.shift) & (DIGITS - 1)] + before[r];
            a.key[a.from ^ 1][to] = key[r];
            a.pos[a.from ^ 1][to] = pos[r];
        }
}

template <typename T, int V>
__global__ __launch_bounds__(NT) void fill_kernel(fill_args f) { fill_rows<T, V, NT>(f, blockIdx.x, gridDim.x); }

// ---- sums over stretches of the sorted list -----------------------------------------------

// A token's row of the gradient from its sum and, where that is added to, its old values.
template <typename T, int V>
__device__ __forceinline__ void write_sum(const gd_embed_grad_args& a, uint32_t token, columns c, const float sum[V], bool add,
                                          const gd_vec<T, V>& old) {
    gd_vec<T, V> q;
#pragma unroll
    for (int j = 0; j < V; ++j) q.v[j] = gd_from_f32<T>(add ? gd_to_f32(old.v[j]) + a.scale * sum[j] : a.scale * sum[j]);
    write_own<T, V>(static_cast<T*>(a.weight_grad) + (uint64_t)token * a.weight_grad_stride + c.at, q, c.skip);
}
template <typename T, int V>
__device__ __forceinline__ gd_vec<T, V> old_row(const gd_embed_grad_args& a, uint32_t token, columns c) {
    return gd_read<T, V>(static_cast<const T*>(a.weight_grad) + (uint64_t)token * a.weight_grad_stride + c.at);
}

// Stretch blockIdx.x of `span` entries, columns by blockIdx.y.  partial: [stretch][2][width], the sums of
// a token that began before the stretch and of one that goes on behind it.  Rows are asked for BATCH at a
// time, whatever their tokens: with ADD together with the tokens' old rows (one after another, each was waited for),
// without it a batch ahead.
template <typename T, int V, bool ADD>
__global__ __launch_bounds__(NT) void grad_sum(gd_embed_grad_args a, const uint32_t* __restrict__ key, const uint32_t* __restrict__ pos,
                                               float* partial, uint32_t n, uint32_t span) {
    const uint32_t c0 = (blockIdx.y * NT + threadIdx.x) * V;
    const uint32_t from = blockIdx.x * span, to = min(from + span, n);
    const uint32_t begin = key[from];
    if (begin == a.vocab || c0 >= a.width) return;            // tokens without a row stand at the end
    const columns c = columns_of<V>(c0, a.width);
    const uint32_t before = from ? key[from - 1] : NO_ROW, behind = to < n ? key[to] : NO_ROW;
    const T* rows = static_cast<const T*>(a.out_grad) + c.at;
    float sum[V];
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] = 0.0f;
    uint32_t token = begin, k[BATCH];
    gd_vec<T, V> q[BATCH], old[ADD ? BATCH : 1], held{};
    auto ask = [&](uint32_t i0) {
#pragma unroll
        for (uint32_t b = 0; b < BATCH; ++b) {
            const uint32_t i = i0 + b;
            k[b] = i < to ? key[i] : a.vocab;
            // (one without a row: the stretch's first row once more)
            const bool row = k[b] != a.vocab;
            q[b] = gd_read<T, V>(rows + (uint64_t)pos[row ? i : from] * a.out_grad_stride);
            // (asked for without a condition, behind which it would be waited for)
            if constexpr (ADD) old[b] = old_row<T, V>(a, row ? k[b] : begin, c);
        }
    };
    // The token's rows here are summed up.
    auto finish = [&]() {
        if (token == before || token == behind) {            // (the stretch's first one, or its last)
            // (the last two lanes of a row write the same sums where they overlap)
            float* p = partial + ((uint64_t)blockIdx.x * 2 + (token == before ? 0 : 1)) * a.width + c.at;
            __builtin_memcpy(p, sum, sizeof(sum));
        } else {
            write_sum<T, V>(a, token, c, sum, ADD, held);
        }
    };
    if (!ADD) ask(from);
    for (uint32_t i0 = from; i0 < to; i0 += BATCH) {
        if (ADD) ask(i0);
        uint32_t now_k[BATCH];
        gd_vec<T, V> now_q[BATCH];
#pragma unroll
        for (uint32_t b = 0; b < BATCH; ++b) { now_k[b] = k[b]; now_q[b] = q[b]; }
        if (!ADD && i0 + BATCH < to) ask(i0 + BATCH);
#pragma unroll
        for (uint32_t b = 0; b < BATCH; ++b) {
            if (now_k[b] != token && token != a.vocab) {
                finish();
#pragma unroll
                for (int j = 0; j < V; ++j) sum[j] = 0.0f;
            }
            token = now_k[b];
            if constexpr (ADD) held = old[b];
            if (token != a.vocab)
#pragma unroll
                for (int j = 0; j < V; ++j) sum[j] += gd_to_f32(now_q[b].v[j]);
        }
    }
    if (token != a.vocab) finish();
}

// The token that begins in stretch blockIdx.x and goes on behind it: its parts in order.
template <typename T, int V>
__global__ __launch_bounds__(NT) void grad_join(gd_embed_grad_args a, const uint32_t* __restrict__ key, const float* __restrict__ partial,
                                                uint32_t n, uint32_t span) {
    const uint32_t c0 = (blockIdx.y * NT + threadIdx.x) * V;
    const uint32_t from = blockIdx.x * span, to = min(from + span, n);
    if (to >= n) return;
    const uint32_t token = key[to - 1];
    if (token != key[to] || token == a.vocab) return;
    if (from && key[from - 1] == token) return;              // began earlier
    // stretches that the token reaches into, 64 looked at at once
    const uint32_t stretches = (n + span - 1) / span, lane = threadIdx.x & 63;
    uint32_t hi = blockIdx.x + 1;
    while (true) {
        const uint32_t at = hi + lane;
        const uint64_t other = __ballot(at >= stretches || key[(uint64_t)min(at, stretches - 1) * span] != token);
        if (other) { hi += (uint32_t)__builtin_ctzll(other); break; }
        hi += 64;
    }
    if (c0 >= a.width) return;
    const columns c = columns_of<V>(c0, a.width);
    const gd_vec<float, V> first = gd_read<float, V>(partial + ((uint64_t)blockIdx.x * 2 + 1) * a.width + c.at);
    constexpr uint32_t PARTS = 16;                            // on their way at once
    float sum[V];
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] = first.v[j];
    for (uint32_t s0 = blockIdx.x + 1; s0 < hi; s0 += PARTS) {
        gd_vec<float, V> q[PARTS];
#pragma unroll
        for (uint32_t b = 0; b < PARTS; ++b)
            q[b] = gd_read<float, V>(partial + (uint64_t)min(s0 + b, hi - 1) * 2 * a.width + c.at);
        // (in pairs first: the sum of 4 096 parts is a chain of 256 additions then)
#pragma unroll
        for (uint32_t b = 0; b < PARTS; ++b)
            if (s0 + b >= hi) q[b] = gd_vec<float, V>{};
#pragma unroll
        for (uint32_t d = 1; d < PARTS; d *= 2)
#pragma unroll
            for (uint32_t b = 0; b < PARTS; b += 2 * d)
#pragma unroll
                for (int j = 0; j < V; ++j) q[b].v[j] += q[b + d].v[j];
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] += q[0].v[j];
    }
    write_sum<T, V>(a, token, c, sum, a.accumulate, a.accumulate ? old_row<T, V>(a, token, c) : gd_vec<T, V>{});
}

// ---- few rows: no list ------------------------------------------------------------------------

// Workgroup i * across + y: row i and the columns of y, 64 * V << log_sub of them; those behind write zeros into the rows
// without a token.  A token's rows are summed in order of their positions, more than BATCH of them in four parts
// of the list, a wave each.
template <typename T, int V, bool ADD, uint32_t ROUNDS>
__global__ __launch_bounds__(NT) void grad_few(gd_embed_grad_args a, uint32_t across, uint32_t log_sub, uint32_t log_tx) {
    constexpr uint32_t WAVES = NT / 64, MARKS = FILL_ROWS / 32;
    __shared__ uint32_t marks[MARKS];
    __shared__ uint16_t list[ROUNDS * NT];
    __shared__ uint32_t counts[ROUNDS * WAVES];
    __shared__ float sums[WAVES - 1][V][64];
    const uint32_t n = a.tokens.n, wave = threadIdx.x / 64, lane = threadIdx.x & 63;
    int64_t t[ROUNDS];
    gd_tokens<ROUNDS>(a.tokens, threadIdx.x, NT, t);
#pragma unroll
    for (uint32_t r = 0; r < ROUNDS; ++r)
        if (r * NT + threadIdx.x >= n) t[r] = -1;
    if (blockIdx.x >= n * across) {
        const uint64_t block = blockIdx.x - n * across, blocks = gridDim.x - n * across;
        const uint32_t from = (uint32_t)(a.vocab * block / blocks), to = (uint32_t)(a.vocab * (block + 1) / blocks);
        for (uint32_t i = threadIdx.x; i < MARKS; i += NT) marks[i] = 0;
        __syncthreads();
#pragma unroll
        for (uint32_t r = 0; r < ROUNDS; ++r)
            if (t[r] >= (int64_t)from && t[r] < (int64_t)to) atomicOr(&marks[((uint32_t)t[r] - from) / 32], 1u << (((uint32_t)t[r] - from) & 31));
        __syncthreads();
        const uint32_t tx = 1u << log_tx;
        for (uint32_t r = threadIdx.x >> log_tx; r < to - from; r += NT >> log_tx)
            if (!(marks[r / 32] >> (r & 31) & 1))
                for (uint32_t c = (threadIdx.x & (tx - 1)) * V; c < a.width; c += tx * V)
                    gd_write_through(static_cast<T*>(a.weight_grad) + (uint64_t)(from + r) * a.weight_grad_stride + columns_of<V>(c, a.width).at, gd_vec<T, V>{});
        return;
    }
    const uint32_t i = blockIdx.x / across;
    const int64_t token = gd_token(a.tokens, i);
    if (token < 0 || token >= (int64_t)a.vocab) return;
    constexpr uint32_t EARLIER = 1u << 31;
    uint64_t who[ROUNDS];
#pragma unroll
    for (uint32_t r = 0; r < ROUNDS; ++r) {
        who[r] = __ballot(t[r] == token);
        const uint32_t first = r * NT + wave * 64 + (who[r] ? (uint32_t)__builtin_ctzll(who[r]) : 0);
        if (lane == 0) counts[r * WAVES + wave] = (uint32_t)__popcll(who[r]) | (who[r] && first < i ? EARLIER : 0);
    }
    __syncthreads();
    uint32_t count = 0;
#pragma unroll
    for (uint32_t k = 0; k < ROUNDS * WAVES; ++k) count |= counts[k];
    if (count & EARLIER) return;                              // the token's first row sums them all
    count = 0;
#pragma unroll
    for (uint32_t k = 0; k < ROUNDS * WAVES; ++k) {
        if (k % WAVES == wave && (who[k / WAVES] >> lane & 1))
            list[count + (uint32_t)__popcll(who[k / WAVES] & ((1ull << lane) - 1))] = (uint16_t)(k / WAVES * NT + threadIdx.x);
        count += counts[k];
    }
    __syncthreads();
    const T* rows = static_cast<const T*>(a.out_grad);
    const auto sum_of = [&](uint32_t from, uint32_t to, columns c, float (&sum)[V]) {
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] = 0.0f;
        for (uint32_t k0 = from; k0 < to; k0 += BATCH) {
            gd_vec<T, V> q[BATCH];
#pragma unroll
            for (uint32_t b = 0; b < BATCH; ++b)
                if (k0 + b < to) q[b] = gd_read<T, V>(rows + (uint64_t)list[k0 + b] * a.out_grad_stride + c.at);
#pragma unroll
            for (uint32_t b = 0; b < BATCH; ++b)
                if (k0 + b < to)
#pragma unroll
                    for (int j = 0; j < V; ++j) sum[j] += gd_to_f32(q[b].v[j]);
        }
    };
    const uint32_t subs = 1u << log_sub, c0 = (blockIdx.x % across) * (64 * V) * subs + lane * V;
    float sum[V];
    if (count <= BATCH) {
        for (uint32_t sub = wave; sub < subs; sub += WAVES) {
            if (c0 + sub * (64 * V) >= a.width) return;
            const columns c = columns_of<V>(c0 + sub * (64 * V), a.width);
            gd_vec<T, V> old{};
            if constexpr (ADD) old = old_row<T, V>(a, (uint32_t)token, c);
            sum_of(0, count, c, sum);
            write_sum<T, V>(a, (uint32_t)token, c, sum, ADD, old);
        }
        return;
    }
    const uint32_t per = (count + WAVES - 1) / WAVES, from = min(wave * per, count), to = min(from + per, count);
    for (uint32_t sub = 0; sub < subs; ++sub) {
        const bool in = c0 + sub * (64 * V) < a.width;
        const columns c = columns_of<V>(c0 + sub * (64 * V), a.width);
        if (in) {
            sum_of(from, to, c, sum);
            if (wave > 0)
#pragma unroll
                for (int j = 0; j < V; ++j) sums[wave - 1][j][lane] = sum[j];
        }
        __syncthreads();
        if (wave == 0 && in) {
#pragma unroll
            for (uint32_t w = 0; w < WAVES - 1; ++w)
#pragma unroll
                for (int j = 0; j < V; ++j) sum[j] += sums[w][j][lane];
            write_sum<T, V>(a, (uint32_t)token, c, sum, ADD, ADD ? old_row<T, V>(a, (uint32_t)token, c) : gd_vec<T, V>{});
        }
        __syncthreads();
    }
}

// Two blocks of columns a workgroup where single ones are more workgroups than the chip holds at once.
uint32_t few_across(uint32_t width, uint32_t v, uint32_t log_sub) { return (width + ((64 * v) << log_sub) - 1) / ((64 * v) << log_sub); }
uint32_t few_log_sub(uint32_t n, uint32_t width, uint32_t v) { return (uint64_t)n * few_across(width, v, 0) > 2048 ? 1 : 0; }
bool few_rows(uint32_t n, uint32_t width, uint32_t v) {
    return n <= FEW && (uint64_t)n * few_across(width, v, few_log_sub(n, width, v)) <= FEW_GROUPS;
}

template <typename T, int V, uint32_t ROUNDS>
hipError_t launch_few(const gd_embed_grad_args& a, hipStream_t s) {
    const uint32_t log_sub = few_log_sub(a.tokens.n, a.width, V), across = few_across(a.width, V, log_sub), sums = a.tokens.n * across;
    uint32_t log_tx = 0;
    if (a.accumulate) {
        hipLaunchKernelGGL((grad_few<T, V, true, ROUNDS>), dim3(sums), dim3(NT), 0, s, a, across, log_sub, log_tx);
        return hipGetLastError();
    }
    while (log_tx < 8 && (1u << log_tx) * V < a.width) ++log_tx;
    // workgroups that fill have 16 KB each to write, or a row
    const uint64_t bytes = (uint64_t)a.vocab * a.width * sizeof(T), least = (a.vocab + FILL_ROWS - 1) / FILL_ROWS;
    uint64_t fill = (bytes + 16383) / 16384;
    if (fill > a.vocab) fill = a.vocab;
    if (fill > MOST_GROUPS) fill = MOST_GROUPS;
    if (fill < least) fill = least;
    hipLaunchKernelGGL((grad_few<T, V, false, ROUNDS>), dim3(sums + (uint32_t)fill), dim3(NT), 0, s, a, across, log_sub, log_tx);
    return hipGetLastError();
}

struct grad_layout {
    size_t key[2], pos[2], hist, partial, total;
    uint32_t blocks, span;
};

grad_layout layout_of(uint64_t n, uint64_t width) {
    grad_layout l;
    l.blocks = (uint32_t)((n + SORT_KEYS - 1) / SORT_KEYS);
    // stretches: 1 024 of them, that all CUs have some, between one batch and four; no more than MOST_STRETCHES, since a
    // token's parts are added up one behind another
    l.span = n <= 1024 * BATCH ? BATCH : n <= 2048 * BATCH ? 2 * BATCH : 4 * BATCH;
    if (n > (uint64_t)MOST_STRETCHES * l.span) l.span = (uint32_t)((n + (uint64_t)MOST_STRETCHES * BATCH - 1) / ((uint64_t)MOST_STRETCHES * BATCH)) * BATCH;
    size_t o = 0;
    for (int i = 0; i < 2; ++i) {
        l.key[i] = o; o = gd_align256(o + n * 4);
        l.pos[i] = o; o = gd_align256(o + n * 4);
    }
    l.hist = o;    o = gd_align256(o + (size_t)(l.blocks + 1) * DIGITS * 4);
    l.partial = o; o = gd_align256(o + (n + l.span - 1) / l.span * 2 * width * 4);
    l.total = o;
    return l;
}

template <typename T, int V>
hipError_t launch_grad(const gd_embed_grad_args& a, hipStream_t s) {
    const uint32_t n = a.tokens.n;
    const grad_layout l = layout_of(n, a.width);
    fill_args f;
    f.p = a.weight_grad; f.stride = a.weight_grad_stride; f.width = a.width; f.from = 0; f.to = 0;
    if (n == 0) {
        if (a.accumulate) return hipSuccess;
        f.to = a.vocab;
        hipLaunchKernelGGL((fill_kernel<T, V>), dim3(fillers<T, NT>(f)), dim3(NT), 0, s, f);
        return hipGetLastError();
    }
    if (few_rows(n, a.width, V)) return n <= FEW / 2 ? launch_few<T, V, FEW / 2 / NT>(a, s) : launch_few<T, V, FEW / NT>(a, s);
    sort_args b;
    for (int i = 0; i < 2; ++i) {
        b.key[i] = reinterpret_cast<uint32_t*>(a.work + l.key[i]);
        b.pos[i] = reinterpret_cast<uint32_t*>(a.work + l.pos[i]);
    }
    b.hist = reinterpret_cast<uint32_t*>(a.work + l.hist);
    b.tokens = a.tokens; b.n = n; b.vocab = a.vocab; b.blocks = l.blocks; b.from = 1; b.shift = 0;
    uint32_t sorted = 0;
    if (n <= ONE_SORT) {
        if (!a.accumulate) f.to = a.vocab;
        hipLaunchKernelGGL((sort_alone<T, V>), dim3(1 + fillers<T, 1024>(f)), dim3(1024), 0, s, b, f);
    } else {
        uint32_t passes = 1;
        while (((uint64_t)a.vocab >> (passes * BITS)) > 0) ++passes;
        const bool self = l.blocks <= SELF_COUNT;
        b.scanned = l.blocks > SELF_SCAN;
        const uint32_t launches = self ? passes : 2 * passes;
        for (uint32_t i = 0; i < launches; ++i) {             // (each fills its share)
            f.from = f.to;
            if (!a.accumulate) f.to = (uint32_t)((uint64_t)a.vocab * (i + 1) / launches);
            if (self) {
                b.shift = i * BITS;
                hipLaunchKernelGGL((sort_pass<T, V>), dim3(l.blocks + fillers<T, 1024>(f)), dim3(1024), 0, s, b, f);
                b.from ^= 1;
            } else if (i % 2 == 0) {
                b.shift = i / 2 * BITS;
                hipLaunchKernelGGL((sort_count<T, V>), dim3(l.blocks + fillers<T, NT>(f)), dim3(NT), 0, s, b, f);
                if (b.scanned) hipLaunchKernelGGL(sort_scan, dim3(DIGITS), dim3(NT), 0, s, b.hist, l.blocks);
            } else {
                hipLaunchKernelGGL((sort_scatter<T, V>), dim3(l.blocks + fillers<T, NT>(f)), dim3(NT), 0, s, b, f);
                b.from ^= 1;
            }
        }
        sorted = b.from;
    }
    float* partial = reinterpret_cast<float*>(a.work + l.partial);
    const dim3 grid((n + l.span - 1) / l.span, (a.width + NT * V - 1) / (NT * V));
    if (a.accumulate)
        hipLaunchKernelGGL((grad_sum<T, V, true>), grid, dim3(NT), 0, s, a, b.key[sorted], b.pos[sorted], partial, n, l.span);
    else
        hipLaunchKernelGGL((grad_sum<T, V, false>), grid, dim3(NT), 0, s, a, b.key[sorted], b.pos[sorted], partial, n, l.span);
    if (n > l.span) {
        constexpr int W = V < 4 ? V : 4;                      // (16 bytes of fp32)
        const dim3 join(grid.x, (a.width + NT * W - 1) / (NT * W));
        hipLaunchKernelGGL((grad_join<T, W>), join, dim3(NT), 0, s, a, b.key[sorted], partial, n, l.span);
    }
    return hipGetLastError();
}

}  // namespace

size_t gd_embed_grad_work(uint64_t n, uint64_t width) { return layout_of(n, width).total; }

hipError_t gd_launch_embed(const gd_embed_args& a, hipStream_t s) {
    if (a.tokens.n == 0 || a.width == 0) return hipSuccess;
    const auto launch = [&](auto zero) {                          // (rows shorter than 16 bytes: an element a lane)
        typedef decltype(zero) T;
        constexpr int V = 16 / sizeof(T);
        return a.width >= V ? launch_embed<T, V>(a, s) : launch_embed<T, 1>(a, s);
    };
    return a.dtype == GD_F32 ? launch(0.0f) : a.dtype == GD_BF16 ? launch(gd_bf16(0.0f)) : launch(gd_f16(0.0f));
}

hipError_t gd_launch_embed_grad(const gd_embed_grad_args& a, hipStream_t s) {
    if (a.width == 0 || a.vocab == 0) return hipSuccess;
    const auto launch = [&](auto zero) {
        typedef decltype(zero) T;
        constexpr int V = 16 / sizeof(T);
        return a.width >= V ? launch_grad<T, V>(a, s) : launch_grad<T, 1>(a, s);
    };
    return a.dtype == GD_F32 ? launch(0.0f) : a.dtype == GD_BF16 ? launch(gd_bf16(0.0f)) : launch(gd_f16(0.0f));
}
