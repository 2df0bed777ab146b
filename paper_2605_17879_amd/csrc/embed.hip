// Embedding lookup, out[i] = round(scale * W[t_i]), and its gradient,
// dW[v] (+)= round(scale * sum of dOut[i] over the i with t_i = v).
//
// The lookup moves rows and computes next to nothing: lanes hold 16 bytes of a row each.
//
// The gradient must not depend on the order in which workgroups run, so there are no float
// atomics: the (token, position) pairs are sorted by token, stably, and the sorted list is cut into
// stretches.  A workgroup sums the rows of one stretch, one column vector per lane, and writes a
// token's sum when the next token begins.  A token that goes on over a stretch's end leaves fp32
// partial sums (one at the front and one at the back of each stretch), which a second kernel adds up in
// order: however often a token occurs, the work stays even.
//
// The gradient's zeros are written by workgroups of the sorting launches that have no keys: sorting is
// a chain of short launches that leaves the memory idle.
#include "gd_operators.h"

namespace {

constexpr uint32_t NT = 256;
constexpr uint32_t BITS = 9, DIGITS = 1u << BITS;   // of a sorting pass: two passes up to 262 143 rows
constexpr uint32_t SORT_KEYS = 1024;      // keys of a workgroup in a sorting pass
constexpr uint32_t ONE_SORT = 4096;       // most keys that one workgroup sorts by itself
constexpr uint32_t SELF_SCAN = 64;        // most workgroups of a pass that add up the counts before them themselves
constexpr uint32_t BATCH = 8;             // rows on their way at once in the sums
constexpr uint32_t NO_ROW = 0xFFFFFFFFu;

// ---- lookup ------------------------------------------------------------------------------------

// tx lanes side by side on a row, NT / tx rows a workgroup; V elements a lane at a time.
template <typename T, int V>
__global__ __launch_bounds__(NT) void embed_kernel(const gd_embed_args a, uint32_t log_tx) {
    const uint32_t tx = 1u << log_tx, lane = threadIdx.x & (tx - 1);
    const uint64_t i = (uint64_t)blockIdx.x * (NT >> log_tx) + (threadIdx.x >> log_tx);
    if (i >= a.tokens.n) return;
    const int64_t t = gd_token(a.tokens, i);
    T* out = static_cast<T*>(a.out) + i * a.out_stride;
    const bool row = t >= 0 && t < (int64_t)a.vocab;
    const T* w = static_cast<const T*>(a.weight) + (row ? (uint64_t)t : 0) * a.weight_stride;
    const float other = t < 0 ? 0.0f : __uint_as_float(0x7FC00000u);
    for (uint32_t c = (blockIdx.y * tx + lane) * V; c < a.width; c += gridDim.y * tx * V) {
        gd_vec<T, V> q;
        if (row) q = *reinterpret_cast<const gd_vec<T, V>*>(w + c);
#pragma unroll
        for (int j = 0; j < V; ++j) q.v[j] = gd_from_f32<T>(row ? gd_to_f32(q.v[j]) * a.scale : other);
        gd_write_through(out + c, q);
    }
}

template <typename T, int V>
hipError_t launch_embed(const gd_embed_args& a, hipStream_t s) {
    uint32_t log_tx = 0;
    while (log_tx < 8 && (1u << log_tx) * V < a.width) ++log_tx;
    const uint32_t rows = NT >> log_tx;
    hipLaunchKernelGGL((embed_kernel<T, V>), dim3((a.tokens.n + rows - 1) / rows), dim3(NT), 0, s, a, log_tx);
    return hipGetLastError();
}

// The most elements (a power of two, 16 bytes at most) that every row of both matrices can be read
// and written by at once.
uint32_t vector_of(const void* p, uint64_t ps, const void* q, uint64_t qs, uint64_t width, uint32_t size) {
    uint32_t v = 16 / size;
    while (v > 1 && ((uintptr_t)p % (v * size) || (uintptr_t)q % (v * size) || ps % v || qs % v || width % v)) v /= 2;
    return v;
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
__device__ __forceinline__ uint32_t key_of(const gd_token_list& l, uint32_t i, uint32_t vocab) {
    const int64_t t = gd_token(l, i);
    return t >= 0 && t < (int64_t)vocab ? (uint32_t)t : vocab;
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

// Workgroup `block` of `blocks` fills its share.
template <typename T, int V, int THREADS>
__device__ __forceinline__ void fill_rows(const fill_args& f, uint32_t block, uint32_t blocks) {
    gd_vec<T, V> zero;
#pragma unroll
    for (int j = 0; j < V; ++j) zero.v[j] = gd_from_f32<T>(0.0f);
    if (f.stride == f.width) {                                // one stretch of memory
        T* p = static_cast<T*>(f.p);
        const uint64_t end = (uint64_t)f.to * f.width;
        for (uint64_t i = (uint64_t)f.from * f.width + ((uint64_t)block * THREADS + threadIdx.x) * V; i < end;
             i += (uint64_t)blocks * THREADS * V)
            gd_write_through(p + i, zero);
    } else {
        for (uint32_t r = f.from + block; r < f.to; r += blocks)
            for (uint32_t c = threadIdx.x * V; c < f.width; c += THREADS * V)
                gd_write_through(static_cast<T*>(f.p) + (uint64_t)r * f.stride + c, zero);
    }
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
#pragma unroll
    for (uint32_t r = 0; r < ROUNDS; ++r) {
        pos[r] = base + r * 64 + lane;
        key[r] = there(r) ? key_of(a.tokens, pos[r], a.vocab) : 0;
    }
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

template <typename T, int V>
__global__ __launch_bounds__(NT) void sort_count(sort_args a, fill_args f) {
    if (blockIdx.x >= a.blocks) return fill_rows<T, V, NT>(f, blockIdx.x - a.blocks, gridDim.x - a.blocks);
    __shared__ uint32_t h[DIGITS];
    for (uint32_t d = threadIdx.x; d < DIGITS; d += NT) h[d] = 0;
    __syncthreads();
#pragma unroll
    for (uint32_t r = 0; r < SORT_KEYS / NT; ++r) {
        const uint32_t i = blockIdx.x * SORT_KEYS + r * NT + threadIdx.x;
        if (i < a.n) {
            const uint32_t key = a.shift ? a.key[a.from][i] : key_of(a.tokens, i, a.vocab);
            atomicAdd(&h[(key >> a.shift) & (DIGITS - 1)], 1u);
        }
    }
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
#pragma unroll
    for (uint32_t r = 0; r < ROUNDS; ++r) {
        const uint32_t i = base + r * 64 + lane;
        key[r] = i < a.n ? (a.shift ? a.key[a.from][i] : key_of(a.tokens, i, a.vocab)) : 0;
        pos[r] = i < a.n && a.shift ? a.pos[a.from][i] : i;
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
__device__ __forceinline__ void write_sum(const gd_embed_grad_args& a, uint32_t token, uint32_t c, const float sum[V], bool add,
                                          const gd_vec<T, V>& old) {
    gd_vec<T, V> q;
#pragma unroll
    for (int j = 0; j < V; ++j) q.v[j] = gd_from_f32<T>(add ? gd_to_f32(old.v[j]) + a.scale * sum[j] : a.scale * sum[j]);
    gd_write_through(static_cast<T*>(a.weight_grad) + (uint64_t)token * a.weight_grad_stride + c, q);
}
template <typename T, int V>
__device__ __forceinline__ gd_vec<T, V> old_row(const gd_embed_grad_args& a, uint32_t token, uint32_t c) {
    return *reinterpret_cast<const gd_vec<T, V>*>(static_cast<const T*>(a.weight_grad) + (uint64_t)token * a.weight_grad_stride + c);
}

// Stretch blockIdx.x of `span` entries, columns by blockIdx.y.  partial: [stretch][2][width], the sums of
// a token that began before the stretch and of one that goes on behind it.  Rows are asked for BATCH at a
// time, whatever their tokens: with ADD together with the tokens' old rows (one after another, each was waited for),
// without it a batch ahead.
template <typename T, int V, bool ADD>
__global__ __launch_bounds__(NT) void grad_sum(gd_embed_grad_args a, const uint32_t* __restrict__ key, const uint32_t* __restrict__ pos,
                                               float* partial, uint32_t n, uint32_t span) {
    const uint32_t c = (blockIdx.y * NT + threadIdx.x) * V;
    const uint32_t from = blockIdx.x * span, to = min(from + span, n);
    const uint32_t begin = key[from];
    if (begin == a.vocab || c >= a.width) return;             // tokens without a row stand at the end
    const uint32_t before = from ? key[from - 1] : NO_ROW, behind = to < n ? key[to] : NO_ROW;
    const T* rows = static_cast<const T*>(a.out_grad) + c;
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
            q[b] = *reinterpret_cast<const gd_vec<T, V>*>(rows + (uint64_t)pos[row ? i : from] * a.out_grad_stride);
            if constexpr (ADD)
                if (row && k[b] != before && k[b] != behind) old[b] = old_row<T, V>(a, k[b], c);
        }
    };
    // The token's rows here are summed up.
    auto finish = [&]() {
        if (token == before || token == behind) {            // (the stretch's first one, or its last)
            float* p = partial + ((uint64_t)blockIdx.x * 2 + (token == before ? 0 : 1)) * a.width + c;
#pragma unroll
            for (int j = 0; j < V; ++j) p[j] = sum[j];
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
    const uint32_t c = (blockIdx.y * NT + threadIdx.x) * V;
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
    if (c >= a.width) return;
    const float* p = partial + ((uint64_t)blockIdx.x * 2 + 1) * a.width + c;
    constexpr uint32_t PARTS = 16;                            // on their way at once
    float sum[V];
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] = p[j];
    for (uint32_t s0 = blockIdx.x + 1; s0 < hi; s0 += PARTS) {
        gd_vec<float, V> q[PARTS];
#pragma unroll
        for (uint32_t b = 0; b < PARTS; ++b)
            q[b] = *reinterpret_cast<const gd_vec<float, V>*>(partial + (uint64_t)min(s0 + b, hi - 1) * 2 * a.width + c);
#pragma unroll
        for (uint32_t b = 0; b < PARTS; ++b)
            if (s0 + b < hi)
#pragma unroll
                for (int j = 0; j < V; ++j) sum[j] += q[b].v[j];
    }
    write_sum<T, V>(a, token, c, sum, a.accumulate, a.accumulate ? old_row<T, V>(a, token, c) : gd_vec<T, V>{});
}

struct grad_layout {
    size_t key[2], pos[2], hist, partial, total;
    uint32_t blocks, span;
};

grad_layout layout_of(uint64_t n, uint64_t width) {
    grad_layout l;
    l.blocks = (uint32_t)((n + SORT_KEYS - 1) / SORT_KEYS);
    // stretches: 1 024 of them, that all CUs have some, between one batch and four
    l.span = n <= 1024 * BATCH ? BATCH : n <= 2048 * BATCH ? 2 * BATCH : 4 * BATCH;
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
    // workgroups that fill: enough for the memory, no more than have 4 KB each to write
    const auto fillers = [&](const fill_args& g, uint32_t threads) {
        const uint64_t w = ((uint64_t)(g.to - g.from) * g.width * sizeof(T) + 4095) / 4096, most = 2048 * 256 / threads;
        return (uint32_t)(w < most ? w : most);
    };
    if (n == 0) {
        if (a.accumulate) return hipSuccess;
        f.to = a.vocab;
        hipLaunchKernelGGL((fill_kernel<T, V>), dim3(fillers(f, NT)), dim3(NT), 0, s, f);
        return hipGetLastError();
    }
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
        hipLaunchKernelGGL((sort_alone<T, V>), dim3(1 + fillers(f, 1024)), dim3(1024), 0, s, b, f);
    } else {
        uint32_t passes = 1;
        while (((uint64_t)a.vocab >> (passes * BITS)) > 0) ++passes;
        b.scanned = l.blocks > SELF_SCAN;
        for (uint32_t i = 0; i < passes; ++i) {
            b.shift = i * BITS;
            for (uint32_t half = 0; half < 2; ++half) {       // (each launch fills its share)
                f.from = f.to;
                if (!a.accumulate) f.to = (uint32_t)((uint64_t)a.vocab * (2 * i + half + 1) / (2 * passes));
                const dim3 grid(l.blocks + fillers(f, NT));
                if (half == 0) hipLaunchKernelGGL((sort_count<T, V>), grid, dim3(NT), 0, s, b, f);
                else hipLaunchKernelGGL((sort_scatter<T, V>), grid, dim3(NT), 0, s, b, f);
                if (half == 0 && b.scanned) hipLaunchKernelGGL(sort_scan, dim3(DIGITS), dim3(NT), 0, s, b.hist, l.blocks);
            }
            b.from ^= 1;
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
    const uint32_t size = a.dtype == GD_F32 ? 4 : 2;
    const uint32_t v = vector_of(a.weight, a.weight_stride, a.out, a.out_stride, a.width, size);
    if (a.dtype == GD_F32) return v == 4 ? launch_embed<float, 4>(a, s) : launch_embed<float, 1>(a, s);
    if (a.dtype == GD_BF16) return v == 8 ? launch_embed<gd_bf16, 8>(a, s) : v >= 2 ? launch_embed<gd_bf16, 2>(a, s) : launch_embed<gd_bf16, 1>(a, s);
    return v == 8 ? launch_embed<gd_f16, 8>(a, s) : v >= 2 ? launch_embed<gd_f16, 2>(a, s) : launch_embed<gd_f16, 1>(a, s);
}

hipError_t gd_launch_embed_grad(const gd_embed_grad_args& a, hipStream_t s) {
    if (a.width == 0 || a.vocab == 0) return hipSuccess;
    const uint32_t size = a.dtype == GD_F32 ? 4 : 2;
    const uint32_t v = vector_of(a.out_grad, a.out_grad_stride, a.weight_grad, a.weight_grad_stride, a.width, size);
    if (a.dtype == GD_F32) return v == 4 ? launch_grad<float, 4>(a, s) : launch_grad<float, 1>(a, s);
    if (a.dtype == GD_BF16) return v == 8 ? launch_grad<gd_bf16, 8>(a, s) : v >= 2 ? launch_grad<gd_bf16, 2>(a, s) : launch_grad<gd_bf16, 1>(a, s);
    return v == 8 ? launch_grad<gd_f16, 8>(a, s) : v >= 2 ? launch_grad<gd_f16, 2>(a, s) : launch_grad<gd_f16, 1>(a, s);
}
