// Internal interface between the host side of the C ABI and the kernels of a sweep's own
// training step (lookup, loss, update).  Nothing here is exported.
#ifndef GD_OPERATORS_H_
#define GD_OPERATORS_H_

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/guard.h"

inline size_t gd_align256(size_t v) { return (v + 255) & ~(size_t)255; }

// A list of tokens or targets as the kernels read it.
struct gd_token_list {
    const void* p;
    uint64_t stride;   // elements between two of them
    uint32_t n;
    uint32_t wide;     // 1: i64, 0: i32
};

struct gd_embed_args {
    const void* weight;  uint64_t weight_stride;
    void* out;           uint64_t out_stride;
    gd_token_list tokens;
    uint32_t vocab, width, dtype;
    float scale;
};

struct gd_embed_grad_args {
    const void* out_grad;  uint64_t out_grad_stride;
    void* weight_grad;     uint64_t weight_grad_stride;
    gd_token_list tokens;
    uint32_t vocab, width, dtype, accumulate;
    float scale;
    uint8_t* work;
};

struct gd_vocab_loss_args {
    const void* hidden;  uint64_t hidden_stride;
    const void* weight;  uint64_t weight_stride;
    gd_token_list targets;
    uint32_t vocab, width, dtype;
    float scale;
    float* loss;  float* lse;  float* mean;
    uint8_t* work;
};

struct gd_vocab_grad_args {
    const void* hidden;  uint64_t hidden_stride;
    const void* weight;  uint64_t weight_stride;
    gd_token_list targets;
    uint32_t vocab, width, dtype;
    float scale;
    const float* lse;  const float* mean;  const float* grad_mean;  const float* grad_rows;
    void* hidden_grad;  uint64_t hidden_grad_stride;   // or null
    void* weight_grad;  uint64_t weight_grad_stride;   // or null
    uint8_t* work;
};

struct gd_adamw_args {
    const uint8_t* table;
    uint64_t table_bytes;
    const float* grad_scale;
    double lr, c1;         // learning rate, 1 - beta1^step
    float fbeta1, fbeta2, one_beta1, one_beta2, inv_root_c2, eps;
    uint32_t seed;
};

// Codes [rows][cols], rows `stride` bytes apart, and the powers of two [blocks of cols][rows].
struct gd_packed_out {
    uint8_t* codes;  uint64_t stride;
    uint8_t* exp;    uint64_t exp_stride;
};

struct gd_pack_args {
    const void* x;  uint64_t stride;
    uint32_t rows, cols, dtype, codes, square;
    gd_packed_out along, across;   // of x, of x transposed; null codes: not asked for
};

struct gd_packed_product_args {
    const void* a;  uint64_t a_stride;  const uint8_t* a_exp;  uint64_t a_exp_stride;
    const void* b;  uint64_t b_stride;  const uint8_t* b_exp;  uint64_t b_exp_stride;
    uint32_t n, m, k, a_codes, b_codes;
    void* out;  uint64_t out_stride;
    uint32_t out_type, accumulate;
    uint32_t short_sums;           // by the 8-bit matrix cores; an out of 16 bits
    uint8_t* work;
};

struct gd_muon_args {
    const void* host_table;
    const uint8_t* table;
    uint8_t* work;
    const float* grad_scale;
    const double* coefficients;   // three a step
    uint32_t steps, nesterov, both;
    float momentum;
    double lr, eps;
};

size_t gd_embed_grad_work(uint64_t n, uint64_t width);
size_t gd_vocab_loss_work(uint64_t n, uint64_t vocab, uint64_t width, bool with_grad);
// Host side of the table: its size, or its bytes where `out` is given.
size_t gd_adamw_table(const gd_adamw_tensor* t, uint32_t n, void* out);

size_t gd_packed_product_work(uint64_t n, uint64_t m, uint64_t k);
// Host side of an update's table, as gd_adamw_table; whether bytes are one; the work area that its matrices need.
size_t gd_muon_table(const gd_muon_tensor* t, uint32_t n, void* out);
bool gd_muon_table_fits(const void* host_table, size_t bytes);
size_t gd_muon_work(const void* host_table, bool both);
bool gd_muon_coefficients_fit(const double* coefficients, uint32_t steps);

hipError_t gd_launch_embed(const gd_embed_args& a, hipStream_t s);
hipError_t gd_launch_embed_grad(const gd_embed_grad_args& a, hipStream_t s);
hipError_t gd_launch_vocab_loss(const gd_vocab_loss_args& a, hipStream_t s);
hipError_t gd_launch_vocab_grad(const gd_vocab_grad_args& a, hipStream_t s);
hipError_t gd_launch_adamw(const gd_adamw_args& a, hipStream_t s);
hipError_t gd_launch_muon(const gd_muon_args& a, hipStream_t s);
hipError_t gd_launch_pack(const gd_pack_args& a, hipStream_t s);
hipError_t gd_launch_packed_product(const gd_packed_product_args& a, hipStream_t s);

#if defined(__HIPCC__)
// ---- what the kernels share ----------------------------------------------------------------

typedef __bf16 gd_bf16;
typedef _Float16 gd_f16;

// Element i of a list, as 64 bits.
__device__ __forceinline__ int64_t gd_token(const gd_token_list& l, uint64_t i) {
    return l.wide ? static_cast<const int64_t*>(l.p)[i * l.stride]
                  : (int64_t)static_cast<const int32_t*>(l.p)[i * l.stride];
}

// Elements from, from + step, ... of a list (the last one where they lie behind its end), all on their way at once: one
// after another behind their own branches, each would be waited for.  The list is not empty.
template <int N>
__device__ __forceinline__ void gd_tokens(const gd_token_list& l, uint32_t from, uint32_t step, int64_t (&t)[N]) {
    if (l.wide) {
#pragma unroll
        for (int b = 0; b < N; ++b) t[b] = static_cast<const int64_t*>(l.p)[min(from + b * step, l.n - 1) * l.stride];
    } else {
        int32_t q[N];
#pragma unroll
        for (int b = 0; b < N; ++b) q[b] = static_cast<const int32_t*>(l.p)[min(from + b * step, l.n - 1) * l.stride];
#pragma unroll
        for (int b = 0; b < N; ++b) t[b] = q[b];
    }
}

// Conversions: to fp32 exactly, from it to nearest even.
template <typename T> __device__ __forceinline__ float gd_to_f32(T v) { return (float)v; }
template <typename T> __device__ __forceinline__ T gd_from_f32(float v) { return (T)v; }

// V elements at once.  Memory is read and written 16 bytes at a time wherever a row begins: such an access needs no more
// alignment than its element has (rows of 4 095 elements in pieces that divide their distance took 2 to 3 times as long).
template <typename T, int V> struct alignas(sizeof(T) * V) gd_vec { T v[V]; };

typedef uint32_t gd_u32x4 __attribute__((ext_vector_type(4)));
typedef gd_u32x4 gd_u32x4_anywhere __attribute__((aligned(2)));

template <typename T, int V>
__device__ __forceinline__ gd_vec<T, V> gd_read(const T* p) {
    if constexpr (sizeof(gd_vec<T, V>) == 16) {
        return __builtin_bit_cast(gd_vec<T, V>, (gd_u32x4)*reinterpret_cast<const gd_u32x4_anywhere*>(p));
    } else {
        gd_vec<T, V> q;
        __builtin_memcpy(&q, p, sizeof(q));
        return q;
    }
}

// A store of data that is not read again soon.
template <typename T, int V>
__device__ __forceinline__ void gd_write_through(T* p, const gd_vec<T, V>& q) {
    if constexpr (sizeof(q) == 16) __builtin_nontemporal_store(__builtin_bit_cast(gd_u32x4, q), reinterpret_cast<gd_u32x4_anywhere*>(p));
    else __builtin_memcpy(p, &q, sizeof(q));
}
#endif

#endif  // GD_OPERATORS_H_
