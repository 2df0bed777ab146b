// Embedding lookup, out[i] = round(scale * W[t_i]), and its gradient,
// dW[v] (+)= round(scale * sum of dOut[i] over the i with t_i = v).
//
// The lookup moves rows and computes next to nothing: lanes hold 16 bytes of a row each.
//
// The gradient must not depend on the order in which workgroups run, so there are no float
// atomics: the (token, position) pairs are sorted by token, stably, and the sorted list is cut into
// stretches of SPAN.  A workgroup sums the rows of one stretch, one column vector per lane, and writes a
// token's sum when the next token begins.  A token that goes on over a stretch's end leaves fp32
// partial sums (one at the front and one at the back of each stretch), which a second kernel adds up in
// order: however often a token occurs, the work stays even.
#include "gd_operators.h"

namespace {

constexpr uint32_t NT = 256;
constexpr uint32_t SPAN = 32;             // sorted entries of a workgroup
constexpr uint32_t DIGITS = 256;          // of a sorting pass
constexpr uint32_t SORT_KEYS = 4096;      // keys of a workgroup in a sorting pass
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
        *reinterpret_cast<gd_vec<T, V>*>(out + c) = q;
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

struct sort_buffers {
    uint32_t* key[2];
    uint32_t* pos[2];
    uint32_t* hist;      // [DIGITS][blocks], then its exclusive prefix sums
    uint32_t blocks;
};

// Tokens to keys: NO_ROW for those without a row, which sort behind all others.
__device__ __forceinline__ uint32_t key_of(const gd_token_list& l, uint32_t i, uint32_t vocab) {
    const int64_t t = gd_token(l, i);
    return t >= 0 && t < (int64_t)vocab ? (uint32_t)t : vocab;
}

// Keys of a wave stand in order of (wave, round, lane): each wave owns a stretch of the block's keys.
constexpr uint32_t SORT_ROUNDS = SORT_KEYS / NT;

// For each lane: which lanes of the wave hold the same digit (among those with a key).
__device__ __forceinline__ uint64_t same_digit(uint32_t d, bool there) {
    uint64_t same = __ballot(there);
#pragma unroll
    for (int b = 0; b < 8; ++b) {
        const uint64_t with = __ballot((d >> b) & 1);
        same &= ((d >> b) & 1) ? with : ~with;
    }
    return same;
}

template <bool FIRST>
__global__ __launch_bounds__(NT) void sort_count(sort_buffers b, gd_token_list tokens, uint32_t n, uint32_t vocab, uint32_t from,
                                                 uint32_t shift) {
    __shared__ uint32_t h[DIGITS];
    h[threadIdx.x] = 0;
    __syncthreads();
    const uint32_t base = blockIdx.x * SORT_KEYS;
    for (uint32_t r = 0; r < SORT_ROUNDS; ++r) {
        const uint32_t i = base + r * NT + threadIdx.x;
        if (i < n) atomicAdd(&h[((FIRST ? key_of(tokens, i, vocab) : b.key[from][i]) >> shift) & (DIGITS - 1)], 1u);
    }
    __syncthreads();
    b.hist[threadIdx.x * b.blocks + blockIdx.x] = h[threadIdx.x];
}

// Exclusive prefix sums of `count` words, one workgroup.
__global__ __launch_bounds__(1024) void sort_scan(uint32_t* h, uint32_t count) {
    __shared__ uint32_t part[1024];
    const uint32_t per = (count + 1023) / 1024, from = threadIdx.x * per;
    uint32_t sum = 0;
    for (uint32_t i = from; i < from + per && i < count; ++i) sum += h[i];
    part[threadIdx.x] = sum;
    __syncthreads();
    for (uint32_t d = 1; d < 1024; d <<= 1) {
        const uint32_t v = threadIdx.x >= d ? part[threadIdx.x - d] : 0;
        __syncthreads();
        part[threadIdx.x] += v;
        __syncthreads();
    }
    uint32_t at = part[threadIdx.x] - sum;
    for (uint32_t i = from; i < from + per && i < count; ++i) { const uint32_t v = h[i]; h[i] = at; at += v; }
}

template <bool FIRST>
__global__ __launch_bounds__(NT) void sort_scatter(sort_buffers b, gd_token_list tokens, uint32_t n, uint32_t vocab, uint32_t from,
                                                   uint32_t shift) {
    constexpr uint32_t WAVES = NT / 64;
    __shared__ uint32_t next[WAVES][DIGITS];
    const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x & 63;
    const uint32_t base = blockIdx.x * SORT_KEYS + wave * (SORT_KEYS / WAVES);
#pragma unroll
    for (uint32_t w = 0; w < WAVES; ++w) next[w][threadIdx.x] = 0;
    __syncthreads();
    uint32_t key[SORT_ROUNDS];
#pragma unroll
    for (uint32_t r = 0; r < SORT_ROUNDS; ++r) {
        const uint32_t i = base + r * 64 + lane;
        key[r] = i < n ? (FIRST ? key_of(tokens, i, vocab) : b.key[from][i]) : 0;
        if (i < n) atomicAdd(&next[wave][(key[r] >> shift) & (DIGITS - 1)], 1u);
    }
    __syncthreads();
    {   // where each wave's keys of a digit begin
        uint32_t at = b.hist[threadIdx.x * b.blocks + blockIdx.x];
#pragma unroll
        for (uint32_t w = 0; w < WAVES; ++w) { const uint32_t c = next[w][threadIdx.x]; next[w][threadIdx.x] = at; at += c; }
    }
    __syncthreads();
#pragma unroll
    for (uint32_t r = 0; r < SORT_ROUNDS; ++r) {
        const uint32_t i = base + r * 64 + lane;
        const bool there = i < n;
        const uint32_t d = (key[r] >> shift) & (DIGITS - 1);
        const uint64_t same = same_digit(d, there);
        const uint32_t before = (uint32_t)__popcll(same & ((1ull << lane) - 1));
        uint32_t at = 0;
        if (there) at = next[wave][d] + before;
        __builtin_amdgcn_wave_barrier();
        if (there && before == 0) next[wave][d] += (uint32_t)__popcll(same);
        __builtin_amdgcn_wave_barrier();
        if (there) {
            b.key[from ^ 1][at] = key[r];
            b.pos[from ^ 1][at] = FIRST ? i : b.pos[from][i];
        }
    }
}

// ---- sums over stretches of the sorted list -----------------------------------------------

template <typename T, int V>
__global__ __launch_bounds__(NT) void grad_zero(gd_embed_grad_args a) {
    const uint32_t vecs = a.width / V;
    const uint64_t total = (uint64_t)a.vocab * vecs;
    for (uint64_t i = (uint64_t)blockIdx.x * NT + threadIdx.x; i < total; i += (uint64_t)gridDim.x * NT) {
        gd_vec<T, V> q;
#pragma unroll
        for (int j = 0; j < V; ++j) q.v[j] = gd_from_f32<T>(0.0f);
        const uint64_t row = i / vecs;
        *reinterpret_cast<gd_vec<T, V>*>(static_cast<T*>(a.weight_grad) + row * a.weight_grad_stride + (i - row * vecs) * V) = q;
    }
}

template <typename T, int V>
__device__ __forceinline__ void write_sum(const gd_embed_grad_args& a, uint32_t token, uint32_t c, const float sum[V]) {
    gd_vec<T, V>* p = reinterpret_cast<gd_vec<T, V>*>(static_cast<T*>(a.weight_grad) + (uint64_t)token * a.weight_grad_stride + c);
    gd_vec<T, V> q;
    if (a.accumulate) {
        q = *p;
#pragma unroll
        for (int j = 0; j < V; ++j) q.v[j] = gd_from_f32<T>(gd_to_f32(q.v[j]) + a.scale * sum[j]);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) q.v[j] = gd_from_f32<T>(a.scale * sum[j]);
    }
    *p = q;
}

// Stretch blockIdx.x, columns by blockIdx.y.  partial: [stretch][2][width], the sums of a token that
// began before the stretch and of one that goes on behind it.
template <typename T, int V>
__global__ __launch_bounds__(NT) void grad_sum(gd_embed_grad_args a, const uint32_t* key, const uint32_t* pos, float* partial,
                                               uint32_t n) {
    const uint32_t c = (blockIdx.y * NT + threadIdx.x) * V;
    const uint32_t from = blockIdx.x * SPAN, to = min(from + SPAN, n);
    if (c >= a.width) return;
    const uint32_t before = from ? key[from - 1] : NO_ROW, behind = to < n ? key[to] : NO_ROW;
    const uint32_t begin = key[from];
    float sum[V];
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] = 0.0f;
    uint32_t token = begin;
    for (uint32_t i = from; i < to; ++i) {
        const uint32_t k = key[i];
        if (k != token) {
            if (token == before) {                           // (only the stretch's first token can be)
                float* p = partial + ((uint64_t)blockIdx.x * 2) * a.width + c;
#pragma unroll
                for (int j = 0; j < V; ++j) p[j] = sum[j];
            } else {
                write_sum<T, V>(a, token, c, sum);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) sum[j] = 0.0f;
            token = k;
        }
        if (k == a.vocab) break;                             // tokens without a row stand at the end
        const gd_vec<T, V> q =
            *reinterpret_cast<const gd_vec<T, V>*>(static_cast<const T*>(a.out_grad) + (uint64_t)pos[i] * a.out_grad_stride + c);
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] += gd_to_f32(q.v[j]);
    }
    if (token == a.vocab) return;
    if (token == behind || token == before) {
        // goes on behind the stretch (its back) or ends with it (its front)
        float* p = partial + ((uint64_t)blockIdx.x * 2 + (token == before ? 0 : 1)) * a.width + c;
#pragma unroll
        for (int j = 0; j < V; ++j) p[j] = sum[j];
    } else {
        write_sum<T, V>(a, token, c, sum);
    }
}

// The token that begins in stretch blockIdx.x and goes on behind it: its parts in order.
template <typename T, int V>
__global__ __launch_bounds__(NT) void grad_join(gd_embed_grad_args a, const uint32_t* key, const float* partial, uint32_t n) {
    const uint32_t c = (blockIdx.y * NT + threadIdx.x) * V;
    const uint32_t from = blockIdx.x * SPAN, to = min(from + SPAN, n);
    if (to >= n || c >= a.width) return;
    const uint32_t token = key[to - 1];
    if (token != key[to] || token == a.vocab) return;
    if (from && key[from - 1] == token) return;              // began earlier
    const float* p = partial + ((uint64_t)blockIdx.x * 2 + 1) * a.width + c;
    float sum[V];
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] = p[j];
    for (uint32_t s = blockIdx.x + 1; (uint64_t)s * SPAN < n && key[s * SPAN] == token; ++s) {
        p = partial + ((uint64_t)s * 2) * a.width + c;
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] += p[j];
    }
    write_sum<T, V>(a, token, c, sum);
}

struct grad_layout {
    size_t key[2], pos[2], hist, partial, total;
    uint32_t blocks;
};

grad_layout layout_of(uint64_t n, uint64_t width) {
    grad_layout l;
    l.blocks = (uint32_t)((n + SORT_KEYS - 1) / SORT_KEYS);
    size_t o = 0;
    for (int i = 0; i < 2; ++i) {
        l.key[i] = o; o = gd_align256(o + n * 4);
        l.pos[i] = o; o = gd_align256(o + n * 4);
    }
    l.hist = o;    o = gd_align256(o + (size_t)l.blocks * DIGITS * 4);
    l.partial = o; o = gd_align256(o + (n + SPAN - 1) / SPAN * 2 * width * 4);
    l.total = o;
    return l;
}

template <typename T, int V>
hipError_t launch_grad(const gd_embed_grad_args& a, hipStream_t s) {
    const uint32_t n = a.tokens.n;
    const grad_layout l = layout_of(n, a.width);
    if (!a.accumulate) {
        const uint64_t vecs = (uint64_t)a.vocab * (a.width / V), blocks = (vecs + NT - 1) / NT;
        hipLaunchKernelGGL((grad_zero<T, V>), dim3((uint32_t)(blocks < 8192 ? blocks : 8192)), dim3(NT), 0, s, a);
    }
    if (n == 0) return hipGetLastError();
    sort_buffers b;
    for (int i = 0; i < 2; ++i) {
        b.key[i] = reinterpret_cast<uint32_t*>(a.work + l.key[i]);
        b.pos[i] = reinterpret_cast<uint32_t*>(a.work + l.pos[i]);
    }
    b.hist = reinterpret_cast<uint32_t*>(a.work + l.hist);
    b.blocks = l.blocks;
    uint32_t from = 1;
    bool first = true;
    for (uint32_t shift = 0; shift == 0 || ((uint64_t)a.vocab >> shift) > 0; shift += 8) {
        if (first) hipLaunchKernelGGL((sort_count<true>), dim3(l.blocks), dim3(NT), 0, s, b, a.tokens, n, a.vocab, from, shift);
        else hipLaunchKernelGGL((sort_count<false>), dim3(l.blocks), dim3(NT), 0, s, b, a.tokens, n, a.vocab, from, shift);
        hipLaunchKernelGGL(sort_scan, dim3(1), dim3(1024), 0, s, b.hist, l.blocks * DIGITS);
        if (first) hipLaunchKernelGGL((sort_scatter<true>), dim3(l.blocks), dim3(NT), 0, s, b, a.tokens, n, a.vocab, from, shift);
        else hipLaunchKernelGGL((sort_scatter<false>), dim3(l.blocks), dim3(NT), 0, s, b, a.tokens, n, a.vocab, from, shift);
        first = false;
        from ^= 1;
    }
    float* partial = reinterpret_cast<float*>(a.work + l.partial);
    const dim3 grid((n + SPAN - 1) / SPAN, (a.width + NT * V - 1) / (NT * V));
    hipLaunchKernelGGL((grad_sum<T, V>), grid, dim3(NT), 0, s, a, b.key[from], b.pos[from], partial, n);
    hipLaunchKernelGGL((grad_join<T, V>), grid, dim3(NT), 0, s, a, b.key[from], partial, n);
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
