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

size_t gd_embed_grad_work(uint64_t n, uint64_t width);
size_t gd_vocab_loss_work(uint64_t n, uint64_t vocab, uint64_t width, bool with_grad);
// Host side of the table: its size, or its bytes where `out` is given.
size_t gd_adamw_table(const gd_adamw_tensor* t, uint32_t n, void* out);

hipError_t gd_launch_embed(const gd_embed_args& a, hipStream_t s);
hipError_t gd_launch_embed_grad(const gd_embed_grad_args& a, hipStream_t s);
hipError_t gd_launch_vocab_loss(const gd_vocab_loss_args& a, hipStream_t s);
hipError_t gd_launch_vocab_grad(const gd_vocab_grad_args& a, hipStream_t s);
hipError_t gd_launch_adamw(const gd_adamw_args& a, hipStream_t s);

#if defined(__HIPCC__)
// ---- what the kernels share ----------------------------------------------------------------

typedef __bf16 gd_bf16;
typedef _Float16 gd_f16;

// Element i of a list, as 64 bits.
__device__ __forceinline__ int64_t gd_token(const gd_token_list& l, uint64_t i) {
    return l.wide ? static_cast<const int64_t*>(l.p)[i * l.stride]
                  : (int64_t)static_cast<const int32_t*>(l.p)[i * l.stride];
}

// Conversions: to fp32 exactly, from it to nearest even.
template <typename T> __device__ __forceinline__ float gd_to_f32(T v) { return (float)v; }
template <typename T> __device__ __forceinline__ T gd_from_f32(float v) { return (T)v; }

// V elements at once (V * sizeof(T) = 4, 8 or 16 bytes, aligned to that).
template <typename T, int V> struct alignas(sizeof(T) * V) gd_vec { T v[V]; };

// A store of data that is not read again soon.
template <typename T, int V>
__device__ __forceinline__ void gd_write_through(T* p, const gd_vec<T, V>& q) {
    if constexpr (sizeof(q) == 16) {
        typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
        __builtin_nontemporal_store(*reinterpret_cast<const u32x4*>(&q), reinterpret_cast<u32x4*>(p));
    } else {
        *reinterpret_cast<gd_vec<T, V>*>(p) = q;
    }
}
#endif

#endif  // GD_OPERATORS_H_
