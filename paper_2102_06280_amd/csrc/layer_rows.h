// Device side of the functions of dbw_layers.h: rows in pieces of 16 bytes, and the 8-bit format of checkpoints.
#pragma once

#include "dbw_layers.h"
#include "loss_rows.h"

namespace layer {

using loss::bf16;
using loss::f16;
using loss::Piece;
using loss::u32x4;
using loss::report;

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Rows of T threads each in a workgroup.
template <int T>
constexpr int ROWS_OF = T <= 64 ? 256 / T : 1;

constexpr int BLOCK = 32;                                 // columns that share a power of two
constexpr int64_t padded(int64_t width) { return (width + BLOCK - 1) / BLOCK * BLOCK; }

// Number of a workgroup in a grid of two dimensions.
__device__ __forceinline__ int64_t group_number() { return blockIdx.x + (int64_t)blockIdx.y * gridDim.x; }

template <class E>
struct Bits {
    typedef uint16_t type;
};
template <>
struct Bits<float> {
    typedef uint32_t type;
};

// Columns c ... c + N - 1 of a row, zeros beyond its width.  A row starts where an element may.
template <class E>
__device__ __forceinline__ u32x4 load_piece(const E *row, int c, int width)
{
    typedef const __attribute__((address_space(1))) typename Piece<E>::raw *place;
    typedef const __attribute__((address_space(1))) typename Bits<E>::type *single;
    constexpr int N = Piece<E>::N;
    if (c + N <= width) return *(place)(uint64_t)(row + c);
    u32x4 w = (u32x4)0u;
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (c + j < width) w[j * 4 / N] |= (uint32_t)((single)(uint64_t)row)[c + j] << (N == 8 && j % 2 ? 16 : 0);
    return w;
}
template <class E>
__device__ __forceinline__ void store_piece(E *row, int c, int width, const u32x4 &w)
{
    typedef __attribute__((address_space(1))) typename Piece<E>::raw *place;
    constexpr int N = Piece<E>::N;
    if (c + N <= width) {
        __builtin_nontemporal_store((typename Piece<E>::raw)w, (place)(uint64_t)(row + c));
        return;
    }
    typedef __attribute__((address_space(1))) typename Bits<E>::type *single;
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (c + j < width) ((single)(uint64_t)row)[c + j] = (typename Bits<E>::type)(w[j * 4 / N] >> (N == 8 && j % 2 ? 16 : 0));
}
// The same of fp32 numbers, N of them, at columns c ... of parameters or their gradients, which start on any 4-byte boundary.
template <int N>
__device__ __forceinline__ void load_floats(const float *row, int c, int width, float (&v)[N])
{
#pragma unroll
    for (int q = 0; q < N; q += 4) {
        const u32x4 w = load_piece<float>(row, c + q, width);
        for (int j = 0; j < 4; ++j) v[q + j] = __uint_as_float(w[j]);
    }
}
template <int N>
__device__ __forceinline__ void store_floats(float *row, int c, int width, const float (&v)[N])
{
#pragma unroll
    for (int q = 0; q < N; q += 4) {
        u32x4 w;
        for (int j = 0; j < 4; ++j) w[j] = __float_as_uint(v[q + j]);
        store_piece<float>(row, c + q, width, w);
    }
}

// ---------------------------------------------------------------- 8 bits
//
// A block's exponent e is the smallest with amax <= 448 2^e = 1.75 2^(8 + e), which amax's own exponent and fraction tell.  At
// e >= -117 the smallest step is 2^-9 2^e >= 2^-126: what a code stands for is a normal number of fp32 and of bf16.

__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// bits: of the block's largest finite magnitude
__device__ __forceinline__ int block_exponent(uint32_t bits)
{
    const int e = (int)(bits >> 23) - 135 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e > -117 ? e : -117;
}
__device__ __forceinline__ uint32_t finite_magnitude(float v)
{
    const uint32_t u = __float_as_uint(v) & 0x7fffffffu;
    return u < 0x7f800000u ? u : 0u;
}
// The maximum over the 32 / N neighbouring lanes that hold a block.
template <int N>
__device__ __forceinline__ uint32_t block_max(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, false));     // lanes 1 0 3 2
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, false));     // 2 3 0 1
    if (N == 4) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, false));   // 7 ... 0 within eight
    return v;
}
// Four values of a block as codes.  The conversion rounds to nearest even, and makes NaN of infinities; nothing finite is above 448 but at
// e = 120, where 256 2^e is not finite any more.
__device__ __forceinline__ uint32_t encode4(const float *v, int e)
{
    const float by = power_of_two(-e);
    float q[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        q[j] = v[j] * by;
        if (e == 120 && fabsf(q[j]) > 240.f && fabsf(q[j]) < INFINITY) q[j] = copysignf(240.f, q[j]);
    }
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], w, true);
}
__device__ __forceinline__ void decode4(uint32_t w, float by, float *v)
{
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    v[0] = a[0] * by;
    v[1] = a[1] * by;
    v[2] = b[0] * by;
    v[3] = b[1] * by;
}

// A checkpoint of rows: codes, then a byte a block.
struct Kept {
    uint8_t *codes, *exponents;
    int64_t stride;                                       // of a row's codes
};
__host__ __device__ inline Kept kept_of(void *checkpoint, int64_t rows, int64_t width)
{
    const int64_t stride = padded(width);
    return Kept{(uint8_t *)checkpoint, (uint8_t *)checkpoint + rows * stride, stride};
}

// N columns of row r from c on, c < padded width, by the lanes that hold the block together: all of them call this.
template <int N>
__device__ __forceinline__ void keep_piece(const Kept &k, int64_t r, int c, const float (&v)[N])
{
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) most = max(most, finite_magnitude(v[j]));
    const int e = block_exponent(block_max<N>(most));
    uint8_t *const at = k.codes + r * k.stride + c;
    if (N == 8) *(u32x2 *)at = (u32x2){encode4(v, e), encode4(v + N - 4, e)};
    else *(uint32_t *)at = encode4(v, e);
    if (c % BLOCK == 0) k.exponents[r * (k.stride / BLOCK) + c / BLOCK] = (uint8_t)(e + 127);
}
// Whole pieces: columns beyond the width are zeros.
template <int N>
__device__ __forceinline__ void kept_piece(const Kept &k, int64_t r, int c, float (&v)[N])
{
    const uint8_t *const at = k.codes + r * k.stride + c;
    const float by = power_of_two((int)k.exponents[r * (k.stride / BLOCK) + c / BLOCK] - 127);
    if (N == 8) {
        const u32x2 w = *(const u32x2 *)at;
        decode4(w[0], by, v);
        decode4(w[1], by, v + N - 4);
    } else {
        decode4(*(const uint32_t *)at, by, v);
    }
}

}  // namespace layer
