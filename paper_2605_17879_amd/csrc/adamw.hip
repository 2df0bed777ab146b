// AdamW over many tensors in one launch.
//
// For each element, in fp32, every operation rounded by itself:
//   g = grad * grad_scale;  m = m b1 + g (1 - b1);  v = v b2 + (g (1 - b2)) g;  r = sqrt(v)
//   p = p (1 - lr wd) - (m lr / (1 - b1^t)) / (r / sqrt(1 - b2^t) + eps)
// 8-bit states hold m and r as e4m3 codes under a power of two per block of 256 elements, so that
// decoding and scaling are exact and the only rounding is the one to four significant bits.
//
// The tensors are cut into pieces of CHUNK elements that a table on the device lists; a workgroup
// takes piece after piece.  A wave takes 256 elements at a time, four a lane: 16-byte accesses
// in fp32, and exactly one block of an 8-bit state, whose largest magnitude then takes six exchanges
// between lanes and no LDS.
#include "gd_lanes.h"
#include "gd_operators.h"

namespace {

constexpr uint32_t NT = 256;
constexpr uint32_t CHUNK = 4096;          // elements of a piece: four rounds of a workgroup
constexpr uint32_t ROUNDS = CHUNK / (NT * 4);

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
    uint8_t aligned;        // every array aligned to four of its elements
    uint8_t pad[3];
};
struct table_chunk {
    uint32_t tensor, chunk;
};
constexpr size_t HEAD = 64;

__host__ __device__ inline size_t chunks_at(uint32_t n_tensors) { return HEAD + (size_t)n_tensors * sizeof(table_tensor); }

// Four numbers of an array of type T, those below `n` alone.
template <typename T>
__device__ __forceinline__ void load4(const void* p, uint64_t at, uint32_t n, bool whole, float x[4]) {
    if (whole) {
        const gd_vec<T, 4> q = *reinterpret_cast<const gd_vec<T, 4>*>(static_cast<const T*>(p) + at);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = gd_to_f32(q.v[j]);
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) x[j] = j < n ? gd_to_f32(static_cast<const T*>(p)[at + j]) : 0.0f;
    }
}
template <typename T>
__device__ __forceinline__ void store4(void* p, uint64_t at, uint32_t n, bool whole, const float x[4]) {
    if (whole) {
        gd_vec<T, 4> q;
#pragma unroll
        for (int j = 0; j < 4; ++j) q.v[j] = gd_from_f32<T>(x[j]);
        *reinterpret_cast<gd_vec<T, 4>*>(static_cast<T*>(p) + at) = q;
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j)
            if (j < n) static_cast<T*>(p)[at + j] = gd_from_f32<T>(x[j]);
    }
}

__device__ __forceinline__ uint32_t load_codes(const void* p, uint64_t at, uint32_t n, bool whole) {
    const uint8_t* b = static_cast<const uint8_t*>(p) + at;
    if (whole) return *reinterpret_cast<const uint32_t*>(b);
    uint32_t c = 0;
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j)
        if (j < n) c |= (uint32_t)b[j] << (8 * j);
    return c;
}
__device__ __forceinline__ void store_codes(void* p, uint64_t at, uint32_t n, bool whole, uint32_t c) {
    uint8_t* b = static_cast<uint8_t*>(p) + at;
    if (whole) {
        *reinterpret_cast<uint32_t*>(b) = c;
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j)
            if (j < n) b[j] = (uint8_t)(c >> (8 * j));
    }
}

// Four e4m3 codes times their block's power of two (byte e): exact.
__device__ __forceinline__ void decode4(uint32_t c, uint32_t e, float x[4]) {
    const float two = e == 255 ? __uint_as_float(0x7FC00000u) : __uint_as_float(e << 23);
    x[0] = __builtin_amdgcn_cvt_f32_fp8((int)c, 0) * two;
    x[1] = __builtin_amdgcn_cvt_f32_fp8((int)c, 1) * two;
    x[2] = __builtin_amdgcn_cvt_f32_fp8((int)c, 2) * two;
    x[3] = __builtin_amdgcn_cvt_f32_fp8((int)c, 3) * two;
}

// The largest of a value over the wave.
__device__ __forceinline__ uint32_t wave_max(uint32_t v, uint32_t lane) {
    v = max(v, gd_lane_xor<1>(v, lane));  v = max(v, gd_lane_xor<2>(v, lane));
    v = max(v, gd_lane_xor<4>(v, lane));  v = max(v, gd_lane_xor<8>(v, lane));
    v = max(v, gd_lane_xor<16>(v, lane)); v = max(v, gd_lane_xor<32>(v, lane));
    return v;
}

// The byte of the power of two that brings a magnitude (as bits) into (224, 448], at least 1.
__device__ __forceinline__ uint32_t block_exponent(uint32_t bits) {
    if (bits == 0) return 0;
    if (bits >= 0x7F800000u) return 255;
    const int32_t e = (int32_t)(bits >> 23) - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return e < 1 ? 1u : (uint32_t)e;
}

// One magnitude q <= 448 to a multiple of its e4m3 step, dithered: the digits below the step are dropped
// after a number of 0 to 2^20 - 1 units of 2^-20 of a step was added.  Below 2^-6 the step stays
// 2^-9; adding 2^-6 moves these to numbers of the same step whose bits can be handled alike.
__device__ __forceinline__ float dither_e4m3(float q, uint32_t d) {
    const bool small = q < 0.015625f;
    const float t = small ? q + 0.015625f : q;
    const float y = __uint_as_float((__float_as_uint(t) + d) & 0xFFF00000u);
    return small ? y - 0.015625f : y;
}

// Four numbers to codes under the block's power of two.  d: two 16-bit numbers a word, `high` picks.
template <bool ROOT>
__device__ __forceinline__ uint32_t encode4(const float x[4], uint32_t e, const uint32_t hash[4]) {
    if (e == 255) return 0x7F7F7F7Fu;                        // NaN
    const float up = __uint_as_float(e == 0 ? 0u : (254u - e) << 23);
    float y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float q = fabsf(x[j]) * up;
        const uint32_t d = ((ROOT ? hash[j] >> 16 : hash[j] & 0xFFFFu) << 4) + 8u;
        y[j] = dither_e4m3(q, d);
        if (ROOT) y[j] = y[j] == 0.0f && q > 0.0f ? 0.001953125f : y[j];
        y[j] = copysignf(y[j], x[j]);
    }
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], c, true);
}

// A well-mixed word from an element's index and the seed: a multiplicative start, then two rounds of
// shift, exclusive or and multiplication by odd numbers.
__device__ __forceinline__ uint32_t index_hash(uint64_t i, uint32_t seed) {
    uint32_t x = (uint32_t)i * 0x9E3779B1u + (uint32_t)(i >> 32) * 0x7F4A7C15u + seed * 0x85157AF5u;
    x = (x ^ (x >> 16)) * 0x58F38DEDu;
    x = (x ^ (x >> 15)) * 0x1AC2F6EBu;
    return x ^ (x >> 16);
}

template <typename P, typename G, bool EIGHT>
__device__ __forceinline__ void update_chunk(const table_tensor& t, uint32_t chunk, const gd_adamw_args& a, float gs,
                                             bool scaled) {
    const uint32_t lane = threadIdx.x & 63;
    const float keep = (float)(1.0 - a.lr * t.lr_scale * t.weight_decay);
    const float size = (float)(a.lr * t.lr_scale / a.c1);
    const uint64_t base = (uint64_t)chunk * CHUNK;
    for (uint32_t r = 0; r < ROUNDS; ++r) {
        const uint64_t at = base + (uint64_t)r * (NT * 4) + threadIdx.x * 4;
        // a wave is in or out as a whole for the exchanges of an 8-bit block
        if (base + (uint64_t)r * (NT * 4) + (threadIdx.x & ~63u) * 4 >= t.n) break;
        const uint32_t n = at >= t.n ? 0u : (uint32_t)(t.n - at < 4 ? t.n - at : 4);
        const bool whole = n == 4 && t.aligned;
        float p[4], g[4], m[4], v[4];
        load4<P>(t.param, at, n, whole, p);
        load4<G>(t.grad, at, n, whole, g);
        if (EIGHT) {
            const uint64_t block = at / GD_STATE_BLOCK;
            float q[4];
            decode4(load_codes(t.m, at, n, whole), t.m_exp[block], m);
            decode4(load_codes(t.v, at, n, whole), t.v_exp[block], q);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = q[j] * q[j];
        } else {
            load4<float>(t.m, at, n, whole, m);
            load4<float>(t.v, at, n, whole, v);
        }
        float root[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float gj = scaled ? g[j] * gs : g[j];
            m[j] = m[j] * a.fbeta1 + gj * a.one_beta1;
            v[j] = v[j] * a.fbeta2 + (gj * a.one_beta2) * gj;
            root[j] = sqrtf(v[j]);
            p[j] = p[j] * keep - (m[j] * size) / (root[j] * a.inv_root_c2 + a.eps);
        }
        store4<P>(t.param, at, n, whole, p);
        if (t.copy) {
            if (t.copy_type == GD_BF16) store4<gd_bf16>(t.copy, at, n, whole, p);
            else store4<gd_f16>(t.copy, at, n, whole, p);
        }
        if (EIGHT) {
            // elements behind the end count as zeros
            uint32_t mm = 0, mv = 0, hash[4];
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) {
                if (j >= n) m[j] = root[j] = 0.0f;
                mm = max(mm, __float_as_uint(m[j]) & 0x7FFFFFFFu);
                mv = max(mv, __float_as_uint(root[j]) & 0x7FFFFFFFu);
                hash[j] = index_hash(t.first_index + at + j, a.seed);
            }
            const uint32_t em = block_exponent(wave_max(mm, lane)), ev = block_exponent(wave_max(mv, lane));
            store_codes(t.m, at, n, whole, encode4<false>(m, em, hash));
            store_codes(t.v, at, n, whole, encode4<true>(root, ev, hash));
            if (lane == 0) {
                t.m_exp[at / GD_STATE_BLOCK] = (uint8_t)em;
                t.v_exp[at / GD_STATE_BLOCK] = (uint8_t)ev;
            }
        } else {
            store4<float>(t.m, at, n, whole, m);
            store4<float>(t.v, at, n, whole, v);
        }
    }
}

template <typename P, bool EIGHT>
__device__ __forceinline__ void by_grad(const table_tensor& t, uint32_t chunk, const gd_adamw_args& a, float gs, bool scaled) {
    switch (t.grad_type) {
        case GD_F32: update_chunk<P, float, EIGHT>(t, chunk, a, gs, scaled); break;
        case GD_BF16: update_chunk<P, gd_bf16, EIGHT>(t, chunk, a, gs, scaled); break;
        default: update_chunk<P, gd_f16, EIGHT>(t, chunk, a, gs, scaled); break;
    }
}
template <bool EIGHT>
__device__ __forceinline__ void by_param(const table_tensor& t, uint32_t chunk, const gd_adamw_args& a, float gs, bool scaled) {
    switch (t.param_type) {
        case GD_F32: by_grad<float, EIGHT>(t, chunk, a, gs, scaled); break;
        case GD_BF16: by_grad<gd_bf16, EIGHT>(t, chunk, a, gs, scaled); break;
        default: by_grad<gd_f16, EIGHT>(t, chunk, a, gs, scaled); break;
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
        if (t.eight) by_param<true>(t, chunks[c].chunk, a, gs, a.grad_scale != nullptr);
        else by_param<false>(t, chunks[c].chunk, a, gs, a.grad_scale != nullptr);
    }
}

size_t size_of(uint32_t type) { return type == GD_F32 ? 4 : 2; }

}  // namespace

size_t gd_adamw_table(const gd_adamw_tensor* t, uint32_t n, void* out) {
    uint64_t chunks = 0;
    for (uint32_t i = 0; i < n; ++i) chunks += (t[i].n + CHUNK - 1) / CHUNK;
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
        const size_t state = d[i].eight ? 1 : 4;
        const bool off = ((uintptr_t)s.d_param % (4 * size_of(s.param_type))) || ((uintptr_t)s.d_grad % (4 * size_of(s.grad_type))) ||
                         ((uintptr_t)s.d_m % (4 * state)) || ((uintptr_t)s.d_v % (4 * state)) ||
                         (s.d_copy && (uintptr_t)s.d_copy % 8);
        d[i].aligned = off ? 0 : 1;
        for (uint64_t k = 0; k * CHUNK < s.n; ++k) { c->tensor = i; c->chunk = (uint32_t)k; ++c; }
    }
    return bytes;
}

hipError_t gd_launch_adamw(const gd_adamw_args& a, hipStream_t s) {
    const uint64_t most = (a.table_bytes - HEAD) / sizeof(table_chunk);
    const uint32_t grid = (uint32_t)(most < 2048 ? most : 2048);
    hipLaunchKernelGGL(adamw_kernel, dim3(grid), dim3(NT), 0, s, a);
    return hipGetLastError();
}
