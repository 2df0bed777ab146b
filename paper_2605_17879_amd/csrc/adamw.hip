// AdamW over many tensors in one launch.
//
// For each element, in fp32, every operation rounded by itself:
//   g = grad * grad_scale;  m = m b1 + g (1 - b1);  v = v b2 + (g (1 - b2)) g;  r = sqrt(v)
//   p = p (1 - lr wd) - (m lr / (1 - b1^t)) / (r / sqrt(1 - b2^t) + eps)
// 8-bit states hold m and r as e4m3 codes under a power of two per block of 256 elements, so that
// decoding and scaling are exact and the only rounding is the one to four significant bits.
//
// The tensors are cut into pieces of elements that a table on the device lists; a workgroup
// takes piece after piece.  A lane holds eight elements at a time, so that 32 lanes hold one block of an
// 8-bit state, whose largest magnitude then takes five exchanges between lanes and no LDS.  The memory bounds it: 28 bytes an element
// with 32-bit states, a bf16 gradient and a bf16 copy, 16 with 8-bit ones (200 M elements 1 030 us, 5.5 TB/s; 540 M 1 715, 5.0 TB/s).
#include "gd_lanes.h"
#include "gd_operators.h"

namespace {

constexpr uint32_t NT = 256;
constexpr uint32_t V = 8;                 // elements of a lane at a time
constexpr uint32_t ROUND = NT * V;
// Elements of a piece: two rounds of a workgroup with 32-bit states (200 M elements 1 029 us; four rounds 1 085, one 1 110,
// eight 1 048), four with 8-bit ones (540 M 1 757; two 1 839, one 1 762, eight 1 822).
__host__ __device__ constexpr uint32_t chunk_of(bool eight) { return eight ? 8192 : 4096; }
constexpr uint32_t BLOCK_LANES = GD_STATE_BLOCK / V;

struct table_head {
    uint64_t bytes;         // of the whole table
    uint32_t n_tensors, n_chunks;
};
struct table_tensor {
    void* param;  const void* grad;  void* m;  void* v;
    uint8_t* m_exp;  uint8_t* v_exp;  void* copy;
    uint64_t n, first_index;
    double lr_scale, weight_decay;
    uint8_t param_type, grad_type, copy_type, eight;
    uint8_t pad[4];
};
struct table_chunk {
    uint32_t tensor, chunk;
};
constexpr size_t HEAD = 64;

__host__ __device__ inline size_t chunks_at(uint32_t n_tensors) { return HEAD + (size_t)n_tensors * sizeof(table_tensor); }

// The table's pointers are to device memory; said to the compiler, which otherwise asks the LDS as well at every access.
// Gradients and copies are marked as passing through once, and with 8-bit states all that is written (200 M elements with
// 32-bit states 933 -> 910 us on one card, 540 M with 8-bit ones 1 661 -> 1 626; all loads marked 1 091 against 1 048, no copies 964 / 930).
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// (read and written at once wherever a tensor begins: such an access needs no more alignment than its elements have)
typedef u32x4 u32x4_anywhere __attribute__((aligned(1)));
typedef u32x2 u32x2_anywhere __attribute__((aligned(1)));
template <typename X>
using in_memory = __attribute__((address_space(1))) X;
template <typename X> __device__ __forceinline__ const in_memory<X>* memory(const void* p) { return (const in_memory<X>*)(uintptr_t)p; }
template <typename X> __device__ __forceinline__ in_memory<X>* memory(void* p) { return (in_memory<X>*)(uintptr_t)p; }

// V numbers of an array as they lie in memory.
template <typename T> struct raw { gd_vec<T, 16 / sizeof(T)> q[V * sizeof(T) / 16]; };
template <> struct raw<uint8_t> { uint2 q; };

template <bool ONCE>
__device__ __forceinline__ u32x4 get16(const void* p) {
    if constexpr (ONCE) return __builtin_nontemporal_load(memory<u32x4_anywhere>(p));
    else return *memory<u32x4_anywhere>(p);
}
template <bool ONCE>
__device__ __forceinline__ u32x2 get8(const void* p) {
    if constexpr (ONCE) return __builtin_nontemporal_load(memory<u32x2_anywhere>(p));
    else return *memory<u32x2_anywhere>(p);
}
template <bool ONCE>
__device__ __forceinline__ void set16(void* p, u32x4 x) {
    if constexpr (ONCE) __builtin_nontemporal_store(x, memory<u32x4_anywhere>(p));
    else *memory<u32x4_anywhere>(p) = x;
}

template <typename T, bool ONCE>
__device__ __forceinline__ raw<T> load_raw(const void* p, uint64_t at) {
    raw<T> r;
    if constexpr (sizeof(T) == 1) {
        const u32x2 x = get8<ONCE>(static_cast<const T*>(p) + at);
        r.q = make_uint2(x.x, x.y);
    } else {
#pragma unroll
        for (int i = 0; i < (int)(V * sizeof(T) / 16); ++i) {
            const u32x4 x = get16<ONCE>(static_cast<const T*>(p) + at + i * (16 / sizeof(T)));
            r.q[i] = __builtin_bit_cast(gd_vec<T, 16 / sizeof(T)>, x);
        }
    }
    return r;
}
template <typename T>
__device__ __forceinline__ void to_floats(const raw<T>& r, float x[V]) {
    constexpr int E = 16 / sizeof(T);
#pragma unroll
    for (int j = 0; j < (int)V; ++j) x[j] = gd_to_f32(r.q[j / E].v[j % E]);
}
// The first n of them: all at once (`vec`) or one by one, zeros behind.
template <typename T, bool ONCE>
__device__ __forceinline__ void load_some(const void* p, uint64_t at, uint32_t n, bool vec, float x[V]) {
    if (vec) {
        to_floats<T>(load_raw<T, ONCE>(p, at), x);
    } else {
#pragma unroll
        for (uint32_t j = 0; j < V; ++j) x[j] = j < n ? gd_to_f32((T)memory<T>(p)[at + j]) : 0.0f;
    }
}
template <typename T, bool ONCE>
__device__ __forceinline__ void store(void* p, uint64_t at, uint32_t n, bool vec, const float x[V]) {
    if (vec) {
        constexpr int E = 16 / sizeof(T);
        raw<T> r;
#pragma unroll
        for (int j = 0; j < (int)V; ++j) r.q[j / E].v[j % E] = gd_from_f32<T>(x[j]);
#pragma unroll
        for (int i = 0; i < (int)V / E; ++i)
            set16<ONCE>(static_cast<T*>(p) + at + i * E, __builtin_bit_cast(u32x4, r.q[i]));
    } else {
#pragma unroll
        for (uint32_t j = 0; j < V; ++j)
            if (j < n) memory<T>(p)[at + j] = gd_from_f32<T>(x[j]);
    }
}
__device__ __forceinline__ uint2 load_some_codes(const void* p, uint64_t at, uint32_t n, bool vec) {
    if (vec) return load_raw<uint8_t, true>(p, at).q;
    const in_memory<uint8_t>* b = memory<uint8_t>(p) + at;
    uint32_t c[2] = {0, 0};
#pragma unroll
    for (uint32_t j = 0; j < V; ++j)
        if (j < n) c[j / 4] |= (uint32_t)b[j] << (8 * (j & 3));
    return make_uint2(c[0], c[1]);
}
__device__ __forceinline__ void store_codes(void* p, uint64_t at, uint32_t n, bool vec, uint32_t c0, uint32_t c1) {
    in_memory<uint8_t>* b = memory<uint8_t>(p) + at;
    if (vec) {
        __builtin_nontemporal_store(u32x2{c0, c1}, (in_memory<u32x2_anywhere>*)b);
    } else {
#pragma unroll
        for (uint32_t j = 0; j < V; ++j)
            if (j < n) b[j] = (uint8_t)((j < 4 ? c0 : c1) >> (8 * (j & 3)));
    }
}

// e4m3 codes times their block's power of two (byte e): exact.
__device__ __forceinline__ void decode(uint2 c, uint32_t e, float x[V]) {
    const float two = e == 255 ? __uint_as_float(0x7FC00000u) : __uint_as_float(e << 23);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int w = (int)(h ? c.y : c.x);
        x[4 * h] = __builtin_amdgcn_cvt_f32_fp8(w, 0) * two;
        x[4 * h + 1] = __builtin_amdgcn_cvt_f32_fp8(w, 1) * two;
        x[4 * h + 2] = __builtin_amdgcn_cvt_f32_fp8(w, 2) * two;
        x[4 * h + 3] = __builtin_amdgcn_cvt_f32_fp8(w, 3) * two;
    }
}

// The largest of a value over the lanes of a block (half a wave).
static_assert(BLOCK_LANES == 32, "block_max");
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t lane) {
    v = max(v, gd_lane_xor<1>(v, lane));  v = max(v, gd_lane_xor<2>(v, lane));
    v = max(v, gd_lane_xor<4>(v, lane));  v = max(v, gd_lane_xor<8>(v, lane));
    return max(v, gd_lane_xor<16>(v, lane));
}

// The byte of the power of two that brings a magnitude (as bits) into (224, 448], at least 1.
__device__ __forceinline__ uint32_t block_exponent(uint32_t bits) {
    if (bits == 0) return 0;
    if (bits >= 0x7F800000u) return 255;
    const int32_t e = (int32_t)(bits >> 23) - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return e < 1 ? 1u : (uint32_t)e;
}

// Four numbers to codes under the block's power of two.  The conversion with a dither adds the upper 20
// bits of its second operand, in units of 2^-20 of a step, to the magnitude and drops what is below the step
// (2^-9 for numbers below 2^-6), subnormal codes included: a lower neighbour becomes the upper one
// as often as the number is near to that.  `hash`: two 16-bit numbers a word, one for each state.
template <bool ROOT>
__device__ __forceinline__ uint32_t encode4(const float x[4], uint32_t e, const uint32_t hash[4]) {
    if (e == 255) return 0x7F7F7F7Fu;                        // NaN
    const float up = __uint_as_float(e == 0 ? 0u : (254u - e) << 23);
    uint32_t d[4];
    float q[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        q[j] = x[j] * up;
        d[j] = (ROOT ? hash[j] & 0xFFFF0000u : hash[j] << 16) | 0x8000u;
    }
    int c = __builtin_amdgcn_cvt_sr_fp8_f32(q[0], d[0], 0, 0);
    c = __builtin_amdgcn_cvt_sr_fp8_f32(q[1], d[1], c, 1);
    c = __builtin_amdgcn_cvt_sr_fp8_f32(q[2], d[2], c, 2);
    c = __builtin_amdgcn_cvt_sr_fp8_f32(q[3], d[3], c, 3);
    if (ROOT) {                                              // no root above 0 becomes 0
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (((uint32_t)c >> (8 * j) & 255u) == 0 && q[j] > 0.0f) c |= 1 << (8 * j);
    }
    return (uint32_t)c;
}

// Well-mixed words from the indexes of V elements next to each other and the seed: a multiplicative
// start, then two rounds of shift, exclusive or and multiplication by odd numbers.
__device__ __forceinline__ void index_hash(uint64_t i, uint32_t seed, uint32_t h[V]) {
    const uint32_t lo = (uint32_t)i, start = lo * 0x9E3779B1u + (uint32_t)(i >> 32) * 0x7F4A7C15u + seed * 0x85157AF5u;
#pragma unroll
    for (uint32_t j = 0; j < V; ++j) {
        uint32_t x = start + j * 0x9E3779B1u;
        if (lo + j < lo) x += 0x7F4A7C15u;                   // (the index's upper word counts on)
        x = (x ^ (x >> 16)) * 0x58F38DEDu;
        x = (x ^ (x >> 15)) * 0x1AC2F6EBu;
        h[j] = x ^ (x >> 16);
    }
}

// What one lane holds of a round.
template <typename P, typename G, typename S>
struct round_data {
    raw<P> p;
    raw<G> g;
    raw<S> m, v;
    uint32_t me, ve;
};

template <typename P, typename G, typename S>
__device__ __forceinline__ void load_round(const table_tensor& t, uint64_t at, round_data<P, G, S>& d) {
    d.p = load_raw<P, false>(t.param, at);
    d.g = load_raw<G, true>(t.grad, at);
    d.m = load_raw<S, false>(t.m, at);
    d.v = load_raw<S, false>(t.v, at);
    if (sizeof(S) == 1) {
        d.me = memory<uint8_t>(t.m_exp)[at / GD_STATE_BLOCK];
        d.ve = memory<uint8_t>(t.v_exp)[at / GD_STATE_BLOCK];
    }
}

struct factors {
    float keep, size, gs;
    bool scaled;
};

// One lane's elements: updated and written back.  WHOLE: all V of them are there and loaded (d);
// else the first n, `vec` where that are all V of them.
template <typename P, typename G, typename S, bool WHOLE>
__device__ __forceinline__ void update(const table_tensor& t, const gd_adamw_args& a, const factors& f, uint64_t at, uint32_t n,
                                       bool vec, const round_data<P, G, S>* d) {
    constexpr bool EIGHT = sizeof(S) == 1;
    const uint32_t lane = threadIdx.x & 63;
    float p[V], g[V], m[V], v[V], root[V];
    if constexpr (WHOLE) {
        to_floats<P>(d->p, p);
        to_floats<G>(d->g, g);
        if constexpr (EIGHT) {
            decode(d->m.q, d->me, m);
            decode(d->v.q, d->ve, v);
        } else {
            to_floats<S>(d->m, m);
            to_floats<S>(d->v, v);
        }
    } else {
        load_some<P, EIGHT>(t.param, at, n, vec, p);
        load_some<G, EIGHT>(t.grad, at, n, vec, g);
        if constexpr (EIGHT) {
            decode(load_some_codes(t.m, at, n, vec), memory<uint8_t>(t.m_exp)[at / GD_STATE_BLOCK], m);
            decode(load_some_codes(t.v, at, n, vec), memory<uint8_t>(t.v_exp)[at / GD_STATE_BLOCK], v);
        } else {
            load_some<S, EIGHT>(t.m, at, n, vec, m);
            load_some<S, EIGHT>(t.v, at, n, vec, v);
        }
    }
#pragma unroll
    for (int j = 0; j < (int)V; ++j) {
        const float gj = f.scaled ? g[j] * f.gs : g[j];
        if (EIGHT) v[j] = v[j] * v[j];
        m[j] = m[j] * a.fbeta1 + gj * a.one_beta1;
        v[j] = v[j] * a.fbeta2 + (gj * a.one_beta2) * gj;
        root[j] = sqrtf(v[j]);
        p[j] = p[j] * f.keep - (m[j] * f.size) / (root[j] * a.inv_root_c2 + a.eps);
    }
    store<P, EIGHT>(t.param, at, n, vec, p);
    if (t.copy) {
        if (t.copy_type == GD_BF16) store<gd_bf16, true>(t.copy, at, n, vec, p);
        else store<gd_f16, true>(t.copy, at, n, vec, p);
    }
    if constexpr (EIGHT) {
        // elements behind the end count as zeros
        uint32_t mm = 0, mv = 0, hash[V];
#pragma unroll
        for (uint32_t j = 0; j < V; ++j) {
            if (!WHOLE && j >= n) m[j] = root[j] = 0.0f;
            mm = max(mm, __float_as_uint(m[j]) & 0x7FFFFFFFu);
            mv = max(mv, __float_as_uint(root[j]) & 0x7FFFFFFFu);
        }
        index_hash(t.first_index + at, a.seed, hash);
        const uint32_t em = block_exponent(block_max(mm, lane)), ev = block_exponent(block_max(mv, lane));
        store_codes(t.m, at, n, vec, encode4<false>(m, em, hash), encode4<false>(m + 4, em, hash + 4));
        store_codes(t.v, at, n, vec, encode4<true>(root, ev, hash), encode4<true>(root + 4, ev, hash + 4));
        if ((lane & (BLOCK_LANES - 1)) == 0 && (WHOLE || n > 0)) {
            memory<uint8_t>(t.m_exp)[at / GD_STATE_BLOCK] = (uint8_t)em;
            memory<uint8_t>(t.v_exp)[at / GD_STATE_BLOCK] = (uint8_t)ev;
        }
    } else {
        store<float, false>(t.m, at, n, vec, m);
        store<float, false>(t.v, at, n, vec, v);
    }
}

template <typename P, typename G, typename S>
__device__ __forceinline__ void update_chunk(const table_tensor& t, uint32_t chunk, const gd_adamw_args& a, float gs, bool scaled) {
    factors f;
    f.keep = (float)(1.0 - a.lr * t.lr_scale * t.weight_decay);
    f.size = (float)(a.lr * t.lr_scale / a.c1);
    f.gs = gs;
    f.scaled = scaled;
    constexpr uint32_t CHUNK = chunk_of(sizeof(S) == 1), ROUNDS = CHUNK / ROUND;
    const uint64_t base = (uint64_t)chunk * CHUNK;
    if (base + CHUNK <= t.n) {
        // the next round's loads are on their way while this one is worked out
        round_data<P, G, S> d[2];
        uint64_t at = base + threadIdx.x * V;
        load_round(t, at, d[0]);
#pragma unroll
        for (uint32_t r = 0; r < ROUNDS; ++r, at += ROUND) {
            if (r + 1 < ROUNDS) load_round(t, at + ROUND, d[(r + 1) & 1]);
            update<P, G, S, true>(t, a, f, at, V, true, &d[r & 1]);
        }
        return;
    }
    for (uint32_t r = 0; r < ROUNDS; ++r) {
        const uint64_t at = base + r * ROUND + threadIdx.x * V;
        // a wave is in or out as a whole, for the exchanges of an 8-bit block; lanes of a block that is not
        // there read the exponents of the last one and write nothing
        if (base + r * ROUND + (threadIdx.x & ~63u) * V >= t.n) break;
        const uint32_t n = at >= t.n ? 0u : (uint32_t)(t.n - at < V ? t.n - at : V);
        const uint64_t block = at & ~(uint64_t)(GD_STATE_BLOCK - 1);
        update<P, G, S, false>(t, a, f, block < t.n ? at : t.n - 1, n, n == V, nullptr);
    }
}

template <typename P, typename S>
__device__ __forceinline__ void by_grad(const table_tensor& t, uint32_t chunk, const gd_adamw_args& a, float gs, bool scaled) {
    switch (t.grad_type) {
        case GD_F32: update_chunk<P, float, S>(t, chunk, a, gs, scaled); break;
        case GD_BF16: update_chunk<P, gd_bf16, S>(t, chunk, a, gs, scaled); break;
        default: update_chunk<P, gd_f16, S>(t, chunk, a, gs, scaled); break;
    }
}
template <typename S>
__device__ __forceinline__ void by_param(const table_tensor& t, uint32_t chunk, const gd_adamw_args& a, float gs, bool scaled) {
    switch (t.param_type) {
        case GD_F32: by_grad<float, S>(t, chunk, a, gs, scaled); break;
        case GD_BF16: by_grad<gd_bf16, S>(t, chunk, a, gs, scaled); break;
        default: by_grad<gd_f16, S>(t, chunk, a, gs, scaled); break;
    }
}

__global__ __launch_bounds__(NT) void adamw_kernel(const gd_adamw_args a) {
    const table_head* head = reinterpret_cast<const table_head*>(a.table);
    if (head->bytes != a.table_bytes) return;               // not a table of this size
    float gs = 1.0f;
    if (a.grad_scale) {
        gs = *a.grad_scale;
        if (!(fabsf(gs) <= 3.4028235e38f)) return;           // an overflow somewhere: no update
    }
    const table_chunk* chunks = reinterpret_cast<const table_chunk*>(a.table + chunks_at(head->n_tensors));
    const table_tensor* tensors = reinterpret_cast<const table_tensor*>(a.table + HEAD);
    for (uint32_t c = blockIdx.x; c < head->n_chunks; c += gridDim.x) {
        const table_tensor& t = tensors[chunks[c].tensor];
        if (t.eight) by_param<uint8_t>(t, chunks[c].chunk, a, gs, a.grad_scale != nullptr);
        else by_param<float>(t, chunks[c].chunk, a, gs, a.grad_scale != nullptr);
    }
}

}  // namespace

size_t gd_adamw_table(const gd_adamw_tensor* t, uint32_t n, void* out) {
    uint64_t chunks = 0;
    for (uint32_t i = 0; i < n; ++i) chunks += (t[i].n + chunk_of(t[i].state_type == GD_E4M3) - 1) / chunk_of(t[i].state_type == GD_E4M3);
    if (chunks > 0xFFFFFFFFull) return 0;
    const size_t bytes = gd_align256(chunks_at(n) + (size_t)chunks * sizeof(table_chunk));
    if (!out) return bytes;
    uint8_t* b = static_cast<uint8_t*>(out);
    for (size_t i = 0; i < bytes; ++i) b[i] = 0;
    table_head* head = reinterpret_cast<table_head*>(b);
    head->bytes = bytes; head->n_tensors = n; head->n_chunks = (uint32_t)chunks;
    table_tensor* d = reinterpret_cast<table_tensor*>(b + HEAD);
    table_chunk* c = reinterpret_cast<table_chunk*>(b + chunks_at(n));
    for (uint32_t i = 0; i < n; ++i) {
        const gd_adamw_tensor& s = t[i];
        d[i].param = s.d_param; d[i].grad = s.d_grad; d[i].m = s.d_m; d[i].v = s.d_v;
        d[i].m_exp = s.d_m_exp; d[i].v_exp = s.d_v_exp; d[i].copy = s.d_copy;
        d[i].n = s.n; d[i].first_index = s.first_index;
        d[i].lr_scale = s.lr_scale; d[i].weight_decay = s.weight_decay;
        d[i].param_type = (uint8_t)s.param_type; d[i].grad_type = (uint8_t)s.grad_type;
        d[i].copy_type = (uint8_t)s.copy_type; d[i].eight = s.state_type == GD_E4M3;
        for (uint64_t k = 0; k * chunk_of(d[i].eight) < s.n; ++k) { c->tensor = i; c->chunk = (uint32_t)k; ++c; }
    }
    return bytes;
}

hipError_t gd_launch_adamw(const gd_adamw_args& a, hipStream_t s) {
    const uint64_t most = (a.table_bytes - HEAD) / sizeof(table_chunk);
    const uint32_t grid = (uint32_t)(most < (1u << 20) ? most : (1u << 20));
    hipLaunchKernelGGL(adamw_kernel, dim3(grid), dim3(NT), 0, s, a);
    return hipGetLastError();
}
