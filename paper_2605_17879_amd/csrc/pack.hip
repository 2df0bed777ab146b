// Packing of a matrix x [n][k] into codes of 8 bits with a power of two for each block of 128: along the rows (a
// block is 128 elements of a row), along the columns (128 of a column; the codes lie transposed), or both in one
// pass over x; or one power of two for each 128 x 128.
//
//   e = the least of 1..254 with max |x| <= MOST 2^(e - 127);  code = the nearest to x 2^(127 - e), ties to even
//
// so that the largest magnitude of a block lies in the upper half of the codes' range (MOST / 2, MOST], unless e is 1.  The
// multiplication by a power of two is exact, so the code's rounding is the only one.
//
// The memory's streams bound it.  A workgroup takes 128 x 128: a lane 4 rows of 8 columns, which lie next to each other along
// both, in registers from the one read to the codes; the row's largest comes from 16 lanes by exchange, the column's
// through the LDS, as do the transposed codes, which are written 16 bytes a lane.  16 384 x 4 096 of bf16 both ways, 271 MB: 50 us, 5.4 TB/s;
// 5 003 x 3 001 of fp32, whose rows begin anywhere, in squares both ways, 90 MB: 17 to 20 us, 4.5 to 5.3 TB/s.  Where there are few of them it is how long one workgroup takes,
// most of that its code's way from memory: 128 x 128 both ways 4.4 us, 6.0 with twice the rows a lane; 1 000 x 1 500 6.2, 8.0, and 10.2 where
// the last numbers of a row were read and written one by one.
#include <type_traits>

#include "gd_operators.h"

namespace {

constexpr uint32_t EDGE = 128, NT = 512, ROWS = 4, WAVES = NT / 64;     // (rows of a lane)

typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef gd_bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef gd_f16 f16x2 __attribute__((ext_vector_type(2)));
constexpr uint32_t NONE = 255, NAN_CODES = 0x7F7F7F7Fu;          // a block that an infinity or a NaN came into

// Two numbers over a power of two as codes, in half HIGH of a word.
template <bool E5M2, bool HIGH>
__device__ __forceinline__ s16x2 two_codes(s16x2 old, bf16x2 x, float two) {
    if constexpr (E5M2) return __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(old, x, two, HIGH);
    else return __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(old, x, two, HIGH);
}
template <bool E5M2, bool HIGH>
__device__ __forceinline__ s16x2 two_codes(s16x2 old, f16x2 x, float two) {
    if constexpr (E5M2) return __builtin_amdgcn_cvt_scalef32_pk_bf8_f16(old, x, two, HIGH);
    else return __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(old, x, two, HIGH);
}
template <bool E5M2, bool HIGH>
__device__ __forceinline__ s16x2 two_codes(s16x2 old, float2 x, float two) {
    if constexpr (E5M2) return __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(old, x.x, x.y, two, HIGH);
    else return __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(old, x.x, x.y, two, HIGH);
}
template <bool E5M2, typename PAIR>
__device__ __forceinline__ uint32_t four_codes(PAIR a, PAIR b, uint32_t e) {
    const float two = __builtin_bit_cast(float, e == 0 ? 0x3F800000u : e << 23);      // (zeros over anything)
    return e == NONE ? NAN_CODES : __builtin_bit_cast(uint32_t, two_codes<E5M2, true>(two_codes<E5M2, false>(s16x2{}, a, two), b, two));
}

// The exponent byte of a block whose largest magnitude has the bits `most`, of fp32.
template <bool E5M2>
__device__ __forceinline__ uint32_t exponent(uint32_t most) {
    constexpr int TOP = E5M2 ? 15 : 8;                           // MOST = 1.75 * 2^TOP
    const int e = (int)(most >> 23) - TOP + ((most & 0x7FFFFFu) > 0x600000u);
    return most == 0 ? 0u : most >= 0x7F800000u ? NONE : (uint32_t)max(e, 1);
}

// The largest of sixteen neighbouring lanes.
template <int CTRL>
__device__ __forceinline__ uint32_t larger_of(uint32_t x) {
    return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ uint32_t most_of_sixteen(uint32_t x) {
    return larger_of<0x121>(larger_of<0x122>(larger_of<0x124>(larger_of<0x128>(x))));     // (rotations by 8, 4, 2 and 1)
}

// Eight neighbouring numbers as they lie in memory, two a pair; magnitudes as numbers that are ordered like them.
template <typename T> struct eight {
    typedef std::conditional_t<std::is_same<T, gd_bf16>::value, bf16x2, f16x2> pair;
    uint32_t w[4];
    __device__ __forceinline__ void load(const T* p) {
        const gd_u32x4 q = *reinterpret_cast<const gd_u32x4_anywhere*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = q[i];
    }
    __device__ __forceinline__ void load_some(const T* p, uint32_t there) {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (i < there) w[i / 2] |= (uint32_t)__builtin_bit_cast(uint16_t, p[i]) << (16 * (i % 2));
    }
    // Number i + gone becomes number i, zeros come from behind.
    __device__ __forceinline__ void move_down(uint32_t gone) {
#pragma unroll
        for (int d = 2; d; d /= 2)
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = gone & (2 * d) ? (i + d < 4 ? w[i + d] : 0) : w[i];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = gone & 1 ? w[i] >> 16 | (i < 3 ? w[i + 1] << 16 : 0) : w[i];
    }
    __device__ __forceinline__ pair at(int i) const { return __builtin_bit_cast(pair, w[i]); }
    // number c of this and of the next row
    static __device__ __forceinline__ pair below(const eight& a, const eight& b, int c) {
        return __builtin_bit_cast(pair, c % 2 ? __builtin_amdgcn_perm(b.w[c / 2], a.w[c / 2], 0x07060302) : __builtin_amdgcn_perm(b.w[c / 2], a.w[c / 2], 0x05040100));
    }
    struct sizes {
        u16x2 w[4];
        __device__ __forceinline__ void take(const eight& x) {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = __builtin_elementwise_max(w[i], __builtin_bit_cast(u16x2, x.w[i] & 0x7FFF7FFFu));
        }
        // of number c, of all, as the bits of fp32
        __device__ __forceinline__ uint32_t of(int c) const { return bits(w[c / 2][c % 2]); }
        __device__ __forceinline__ uint32_t most() const {
            const u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(w[0], w[1]), __builtin_elementwise_max(w[2], w[3]));
            return bits(max(m[0], m[1]));
        }
        static __device__ __forceinline__ uint32_t bits(uint16_t m) { return __builtin_bit_cast(uint32_t, gd_to_f32(__builtin_bit_cast(T, m))); }
    };
};
template <> struct eight<float> {
    typedef float2 pair;
    float x[8];
    __device__ __forceinline__ void load(const float* p) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const gd_vec<float, 4> q = gd_read<float, 4>(p + 4 * h);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[4 * h + i] = q.v[i];
        }
    }
    __device__ __forceinline__ void load_some(const float* p, uint32_t there) {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (i < there) x[i] = p[i];
    }
    __device__ __forceinline__ void move_down(uint32_t gone) {
#pragma unroll
        for (int d = 4; d; d /= 2)
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = gone & d ? (i + d < 8 ? x[i + d] : 0.0f) : x[i];
    }
    __device__ __forceinline__ pair at(int i) const { return make_float2(x[2 * i], x[2 * i + 1]); }
    static __device__ __forceinline__ pair below(const eight& a, const eight& b, int c) { return make_float2(a.x[c], b.x[c]); }
    struct sizes {
        uint32_t w[8];
        __device__ __forceinline__ void take(const eight& x) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = max(w[i], __builtin_bit_cast(uint32_t, x.x[i]) & 0x7FFFFFFFu);
        }
        __device__ __forceinline__ uint32_t of(int c) const { return w[c]; }
        __device__ __forceinline__ uint32_t most() const {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, w[i]);
            return m;
        }
    };
};

// The first `there` bytes, fewer than all, eight, four, two and one at a time.
template <int N>
__device__ __forceinline__ void write_some(uint32_t (&&w)[N], uint8_t* at, uint32_t there) {
    if (N == 4 && (there & 8)) {
        __builtin_memcpy(at, &w[0], 8);
        at += 8;
        w[0] = w[N - 2];
        w[1] = w[N - 1];
    }
    if (there & 4) {
        __builtin_memcpy(at, &w[0], 4);
        at += 4;
        w[0] = w[1];
    }
    if (there & 2) {
        __builtin_memcpy(at, &w[0], 2);
        at += 2;
        w[0] >>= 16;
    }
    if (there & 1) *at = (uint8_t)w[0];
}

template <typename T, bool E5M2>
__global__ __launch_bounds__(NT, 4) void pack_kernel(const gd_pack_args a) {
    __shared__ uint32_t most_of[EDGE][WAVES + 1];                // a column's largest, by wave
    __shared__ uint32_t exp_of[EDGE];
    __shared__ __attribute__((aligned(16))) uint32_t turned[EDGE][EDGE / 4 + 4];   // codes, transposed: column 8 t + c in row 16 c + t
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64, tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const uint32_t tiles_c = (a.cols + EDGE - 1) / EDGE, tile_r = blockIdx.x / tiles_c, tile_c = blockIdx.x % tiles_c;
    const uint32_t row0 = tile_r * EDGE + ty * ROWS, col0 = tile_c * EDGE + tx * 8;
    const T* x = static_cast<const T*>(a.x) + row0 * a.stride + col0;
    const bool whole = col0 + 8 <= a.cols;
    eight<T> v[ROWS] = {};
    // (of a row's last numbers, where they are not eight, the eight that end with them)
    const uint32_t gone = whole ? 0 : col0 + 8 - a.cols;
    if (a.cols >= 8) {
        if (gone < 8) {
#pragma unroll
            for (int j = 0; j < ROWS; ++j)
                if (row0 + j < a.rows) v[j].load(x + j * a.stride - gone);
        }
        if (gone) {
#pragma unroll
            for (int j = 0; j < ROWS; ++j) v[j].move_down(gone);
        }
    } else if (col0 == 0) {
#pragma unroll
        for (int j = 0; j < ROWS; ++j)
            if (row0 + j < a.rows) v[j].load_some(x + j * a.stride, a.cols);
    }
    uint32_t row_most[ROWS];
    typename eight<T>::sizes columns = {};
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        typename eight<T>::sizes row = {};
        row.take(v[j]);
        row_most[j] = row.most();
        columns.take(v[j]);
    }
    uint32_t square_most = 0;
    if (a.square) {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < ROWS; ++j) m = max(m, row_most[j]);
        m = most_of_sixteen(m);
        m = max(m, (uint32_t)__shfl_xor((int)m, 16));
        m = max(m, (uint32_t)__shfl_xor((int)m, 32));
        if (lane == 0) most_of[0][wave] = m;
        __syncthreads();
#pragma unroll
        for (uint32_t w = 0; w < WAVES; ++w) square_most = max(square_most, most_of[0][w]);
    }
    if (a.along.codes) {
#pragma unroll
        for (int j = 0; j < ROWS; ++j) {
            const uint32_t e = exponent<E5M2>(a.square ? square_most : most_of_sixteen(row_most[j])), row = row0 + j;
            const uint2 w = make_uint2(four_codes<E5M2>(v[j].at(0), v[j].at(1), e), four_codes<E5M2>(v[j].at(2), v[j].at(3), e));
            if (row < a.rows) {
                uint8_t* to = a.along.codes + row * a.along.stride + col0;
                if (whole) *reinterpret_cast<uint2*>(to) = w;
                else if (col0 < a.cols) write_some({w.x, w.y}, to, a.cols - col0);
                if (tx == 0) a.along.exp[tile_c * a.along.exp_stride + row] = (uint8_t)e;
            }
        }
    }
    if (!a.across.codes) return;
    if (!a.square) {
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            uint32_t m = columns.of(c);
            m = max(m, (uint32_t)__shfl_xor((int)m, 16));
            m = max(m, (uint32_t)__shfl_xor((int)m, 32));
            if (lane < 16) most_of[tx * 8 + c][wave] = m;
        }
        __syncthreads();
        // (each column's exponent once, by one lane)
        if (threadIdx.x < EDGE) {
            uint32_t m = 0;
#pragma unroll
            for (uint32_t w = 0; w < WAVES; ++w) m = max(m, most_of[threadIdx.x][w]);
            exp_of[threadIdx.x] = exponent<E5M2>(m);
        }
        __syncthreads();
    }
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const uint32_t e = a.square ? exponent<E5M2>(square_most) : exp_of[tx * 8 + c];
        turned[16 * c + tx][ty] = four_codes<E5M2>(eight<T>::below(v[0], v[1], c), eight<T>::below(v[2], v[3], c), e);
    }
    __syncthreads();
    if (threadIdx.x < EDGE && tile_c * EDGE + threadIdx.x < a.cols)
        a.across.exp[tile_r * a.across.exp_stride + tile_c * EDGE + threadIdx.x] = (uint8_t)(a.square ? exponent<E5M2>(square_most) : exp_of[threadIdx.x]);
    const uint32_t from = tile_r * EDGE + (threadIdx.x % 8) * 16;
    for (uint32_t c = threadIdx.x / 8; c < EDGE && tile_c * EDGE + c < a.cols; c += NT / 8) {
        if (from >= a.rows) break;
        const uint4 w = *reinterpret_cast<const uint4*>(&turned[c % 8 * 16 + c / 8][(threadIdx.x % 8) * 4]);
        uint8_t* to = a.across.codes + (tile_c * EDGE + c) * a.across.stride + from;
        if (from + 16 <= a.rows) *reinterpret_cast<uint4*>(to) = w;
        else write_some({w.x, w.y, w.z, w.w}, to, a.rows - from);
    }
}

template <typename T>
void launch(const gd_pack_args& a, hipStream_t s) {
    const uint32_t grid = ((a.rows + EDGE - 1) / EDGE) * ((a.cols + EDGE - 1) / EDGE);
    if (a.codes == GD_E5M2) pack_kernel<T, true><<<grid, NT, 0, s>>>(a);
    else pack_kernel<T, false><<<grid, NT, 0, s>>>(a);
}

}  // namespace

hipError_t gd_launch_pack(const gd_pack_args& a, hipStream_t s) {
    if (a.rows == 0 || a.cols == 0) return hipSuccess;
    if (a.dtype == GD_F32) launch<float>(a, s);
    else if (a.dtype == GD_BF16) launch<gd_bf16>(a, s);
    else launch<gd_f16>(a, s);
    return hipGetLastError();
}
