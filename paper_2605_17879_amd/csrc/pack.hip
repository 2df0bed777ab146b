// Packing of a matrix x [n][k] into codes of 8 bits with a power of two for each block of 128: along the rows (a
// block is 128 elements of a row), along the columns (128 of a column; the codes lie transposed), or both in one
// pass over x; or one power of two for each 128 x 128.
//
//   e = the least of 1..254 with max |x| <= MOST 2^(e - 127);  code = the nearest to x 2^(127 - e), ties to even
//
// so that the largest magnitude of a block lies in the upper half of the codes' range (MOST / 2, MOST], unless e is 1.  The
// multiplication by a power of two is exact, so the code's rounding is the only one.
//
// The memory's streams bound it.  A workgroup takes 128 x 128: a lane 8 rows of 8 columns, which lie next to each other along
// both, in registers from the one read to the codes; the row's largest comes from 16 lanes by exchange, the column's
// through the LDS, as do the transposed codes, which are written 16 bytes a lane.
#include "gd_operators.h"

namespace {

constexpr uint32_t EDGE = 128, NT = 256;

template <bool E5M2> struct format {
    static constexpr uint32_t TOP = E5M2 ? 15 : 8;               // MOST = 1.75 * 2^TOP
    static __device__ __forceinline__ uint32_t four(float a, float b, float c, float d) {
        int w = 0;
        if constexpr (E5M2) {
            w = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, w, false);
            w = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, w, true);
        } else {
            w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, w, false);
            w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
        }
        return (uint32_t)w;
    }
};
constexpr uint32_t NONE = 255, NAN_CODES = 0x7F7F7F7Fu;          // a block that an infinity or a NaN came into

// The exponent byte of a block whose largest magnitude has the bits `most`.
template <bool E5M2>
__device__ __forceinline__ uint32_t exponent(uint32_t most) {
    if (most == 0) return 0;
    if (most >= 0x7F800000u) return NONE;
    const int e = (int)(most >> 23) - (int)format<E5M2>::TOP + ((most & 0x7FFFFFu) > 0x600000u);
    return e < 1 ? 1u : (uint32_t)e;
}
__device__ __forceinline__ float factor(uint32_t e) { return __builtin_bit_cast(float, (254 - min(e, 254u)) << 23); }

__device__ __forceinline__ uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7FFFFFFFu; }

template <bool E5M2>
__device__ __forceinline__ uint2 eight(const float (&x)[8], float f, uint32_t e) {
    if (e == NONE) return make_uint2(NAN_CODES, NAN_CODES);
    return make_uint2(format<E5M2>::four(x[0] * f, x[1] * f, x[2] * f, x[3] * f), format<E5M2>::four(x[4] * f, x[5] * f, x[6] * f, x[7] * f));
}

// The bytes from `at` on of a row that has `there` more.
template <int N>
__device__ __forceinline__ void write_some(const uint32_t (&w)[N], uint8_t* at, uint32_t there) {
#pragma unroll
    for (int b = 0; b < 4 * N; ++b)
        if ((uint32_t)b < there) at[b] = (uint8_t)(w[b / 4] >> (8 * (b % 4)));
}

template <typename T, bool E5M2>
__global__ __launch_bounds__(NT) void pack_kernel(const gd_pack_args a) {
    __shared__ uint32_t most_of[EDGE][5];                        // a column's largest, by wave
    __shared__ uint32_t exp_of[EDGE];
    __shared__ __attribute__((aligned(16))) uint2 turned[EDGE][EDGE / 8 + 2];   // codes, transposed
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64, tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const uint32_t tiles_c = (a.cols + EDGE - 1) / EDGE, tile_r = blockIdx.x / tiles_c, tile_c = blockIdx.x % tiles_c;
    const uint32_t row0 = tile_r * EDGE + ty * 8, col0 = tile_c * EDGE + tx * 8;
    const T* x = static_cast<const T*>(a.x) + col0;
    float v[8][8];
    const bool whole = col0 + 8 <= a.cols;
    constexpr int V = 16 / sizeof(T);
    gd_vec<T, V> raw[8][8 / V];
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int h = 0; h < 8 / V; ++h) {
            raw[j][h] = gd_vec<T, V>{};
            if (row0 + j < a.rows) {
                const T* p = x + (row0 + j) * a.stride + h * V;
                if (whole) {
                    raw[j][h] = gd_read<T, V>(p);
                } else {
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        if (col0 + h * V + e < a.cols) raw[j][h].v[e] = p[e];
                }
            }
        }
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int c = 0; c < 8; ++c) v[j][c] = gd_to_f32(raw[j][c / V].v[c % V]);

    uint32_t row_most[8], col_most[8] = {};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        row_most[j] = 0;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const uint32_t b = magnitude(v[j][c]);
            row_most[j] = max(row_most[j], b);
            col_most[c] = max(col_most[c], b);
        }
    }
    if (a.square) {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max(m, row_most[j]);
#pragma unroll
        for (int d = 1; d < 64; d *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, d));
        if (lane == 0) most_of[0][wave] = m;
        __syncthreads();
        m = max(max(most_of[0][0], most_of[0][1]), max(most_of[0][2], most_of[0][3]));
#pragma unroll
        for (int j = 0; j < 8; ++j) row_most[j] = col_most[j] = m;
    }
    if (a.along.codes) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (!a.square) {
#pragma unroll
                for (int d = 1; d < 16; d *= 2) row_most[j] = max(row_most[j], (uint32_t)__shfl_xor((int)row_most[j], d));
            }
            const uint32_t e = exponent<E5M2>(row_most[j]), row = row0 + j;
            const uint2 w = eight<E5M2>(v[j], factor(e), e);
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
            uint32_t m = col_most[c];
            m = max(m, (uint32_t)__shfl_xor((int)m, 16));
            m = max(m, (uint32_t)__shfl_xor((int)m, 32));
            if (lane < 16) most_of[tx * 8 + c][wave] = m;
        }
        __syncthreads();
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const uint32_t* m = most_of[tx * 8 + c];
            col_most[c] = max(max(m[0], m[1]), max(m[2], m[3]));
        }
    }
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const uint32_t e = exponent<E5M2>(col_most[c]);
        const float column[8] = {v[0][c], v[1][c], v[2][c], v[3][c], v[4][c], v[5][c], v[6][c], v[7][c]};
        turned[tx * 8 + c][ty] = eight<E5M2>(column, factor(e), e);
        if (ty == 0) exp_of[tx * 8 + c] = e;
    }
    __syncthreads();
    if (threadIdx.x < EDGE && tile_c * EDGE + threadIdx.x < a.cols)
        a.across.exp[tile_r * a.across.exp_stride + tile_c * EDGE + threadIdx.x] = (uint8_t)exp_of[threadIdx.x];
    const uint32_t from = tile_r * EDGE + (threadIdx.x % 8) * 16;
    for (uint32_t c = threadIdx.x / 8; c < EDGE && tile_c * EDGE + c < a.cols; c += NT / 8) {
        if (from >= a.rows) break;
        const uint4 w = *reinterpret_cast<const uint4*>(&turned[c][(threadIdx.x % 8) * 2]);
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
