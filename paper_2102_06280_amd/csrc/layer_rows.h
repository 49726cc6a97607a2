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
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int BLOCK = 32;                                 // columns that share a power of two
constexpr int64_t padded(int64_t width) { return (width + BLOCK - 1) / BLOCK * BLOCK; }

// Number of a workgroup in a grid of two dimensions.
__device__ __forceinline__ int64_t group_number() { return blockIdx.x + (int64_t)blockIdx.y * gridDim.x; }
// Which of a workgroup's rows a thread has, T threads each: in a scalar register where it is a wave's.
template <int T>
__device__ __forceinline__ int slot_of()
{
    const int slot = threadIdx.x / T;
    return T < 64 ? slot : __builtin_amdgcn_readfirstlane(slot);
}
// A worker's rows among `strips` workgroups, which take `step` rows each in turn, so that those that run at a time read and write rows that lie together:
// 8 x 8192 x 2048 bf16 forwards 96.5 us, with a contiguous strip for each 107.
struct Strip {
    int worker, number;
    int64_t first, stride, end;                           // rows of the worker
};
__device__ __forceinline__ Strip strip_of(uint32_t group, uint32_t strips, int step, int per_worker)
{
    const int worker = (int)(group / strips), number = (int)(group % strips);
    return Strip{worker, number, (int64_t)number * step, (int64_t)strips * step, per_worker};
}

template <class E>
struct Bits {
    typedef uint16_t type;
};
template <>
struct Bits<float> {
    typedef uint32_t type;
};

// Columns c ... c + N - 1 of a row, zeros beyond its width, in two steps, so that the loads wait for nothing: the 16 bytes that are
// loaded, the row's last ones where the piece is not whole, and then what they are.  A row starts where an element may.  WIDE: it has N columns at
// least; rows of less are taken one by one.
template <class E, bool WIDE>
__device__ __forceinline__ u32x4 load_raw(const E *row, int c, int width)
{
    typedef const __attribute__((address_space(1))) typename Piece<E>::raw *place;
    typedef const __attribute__((address_space(1))) typename Bits<E>::type *single;
    constexpr int N = Piece<E>::N;
    if (WIDE || width >= N) return *(place)(uint64_t)(row + min(c, width - N));
    u32x4 w = (u32x4)0u;
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (j < width) w[j * 4 / N] |= (uint32_t)((single)(uint64_t)row)[j] << (N == 8 && j % 2 ? 16 : 0);
    return w;
}
template <class E, bool WIDE>
__device__ __forceinline__ u32x4 settled(const u32x4 &w, int c, int width)
{
    constexpr int N = Piece<E>::N;
    if (c + N <= width) return w;
    const int by = (WIDE || width >= N ? c + N - width : c) * (128 / N);       // bits that lie in front of column c
    uint64_t low = (uint64_t)w[1] << 32 | w[0], high = (uint64_t)w[3] << 32 | w[2];
    if (by >= 64) {
        low = by < 128 ? high >> (by - 64) : 0;
        high = 0;
    } else if (by > 0) {
        low = low >> by | high << (64 - by);
        high >>= by;
    }
    return (u32x4){(uint32_t)low, (uint32_t)(low >> 32), (uint32_t)high, (uint32_t)(high >> 32)};
}
template <class E, bool WIDE = false>
__device__ __forceinline__ u32x4 load_piece(const E *row, int c, int width)
{
    return settled<E, WIDE>(load_raw<E, WIDE>(row, c, width), c, width);
}
// And back, past the caches or through them.
template <class E, bool PAST = true>
__device__ __forceinline__ void store_piece(E *row, int c, int width, const u32x4 &w)
{
    typedef __attribute__((address_space(1))) typename Piece<E>::raw *place;
    constexpr int N = Piece<E>::N;
    if (c + N <= width) {
        if constexpr (PAST) __builtin_nontemporal_store((typename Piece<E>::raw)w, (place)(uint64_t)(row + c));
        else *(place)(uint64_t)(row + c) = (typename Piece<E>::raw)w;
        return;
    }
    if (c >= width) return;
    typedef __attribute__((address_space(1))) typename Bits<E>::type *single;
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (c + j < width) ((single)(uint64_t)row)[c + j] = (typename Bits<E>::type)(w[j * 4 / N] >> (N == 8 && j % 2 ? 16 : 0));
}
// The same of fp32 numbers, N of them, at columns c ... of parameters or their gradients, which start on any 4-byte boundary.
template <int N, bool WIDE = false>
__device__ __forceinline__ void load_floats(const float *row, int c, int width, float (&v)[N])
{
#pragma unroll
    for (int q = 0; q < N; q += 4) {
        const u32x4 w = load_piece<float, WIDE>(row, c + q, width);
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
// The maximum over the 32 / N neighbouring lanes that hold a block.
template <int N>
__device__ __forceinline__ uint32_t block_max(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, false));     // lanes 1 0 3 2
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, false));     // 2 3 0 1
    if (N == 4) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, false));   // 7 ... 0 within eight
    return v;
}

// A piece's largest magnitude as fp32 bits (of a type's numbers the larger has the larger bits, whatever lies above the largest finite
// one), or, where that may not be finite, the largest finite one; and the piece's N codes, from the type's own conversion with a scale: to the
// nearest, ties to even, NaN for infinities and NaN.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t finite_magnitude(float v)
{
    const uint32_t u = __float_as_uint(v) & 0x7fffffffu;
    return u < 0x7f800000u ? u : 0u;
}
__device__ __forceinline__ uint32_t pair_max(const u32x4 &w)     // of halves without their signs
{
    u16x2 m = __builtin_bit_cast(u16x2, w[0] & 0x7fff7fffu);
#pragma unroll
    for (int i = 1; i < 4; ++i) {
        const uint32_t next = w[i] & 0x7fff7fffu;
        m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, next));
    }
    return max((uint32_t)m[0], (uint32_t)m[1]);
}
template <class E>
struct Coder;
template <>
struct Coder<float> {
    static __device__ __forceinline__ uint32_t magnitude(const u32x4 &w)
    {
        uint32_t m = w[0] & 0x7fffffffu;
#pragma unroll
        for (int i = 1; i < 4; ++i) m = max(m, w[i] & 0x7fffffffu);
        return m;
    }
    static __device__ __forceinline__ uint32_t code4(const u32x4 &w, int, float scale)
    {
        s16x2 c = {0, 0};
        c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, __uint_as_float(w[0]), __uint_as_float(w[1]), scale, false);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, __uint_as_float(w[2]), __uint_as_float(w[3]), scale, true);
        return __builtin_bit_cast(uint32_t, c);
    }
};
template <>
struct Coder<bf16> {
    static __device__ __forceinline__ uint32_t magnitude(const u32x4 &w) { return pair_max(w) << 16; }
    static __device__ __forceinline__ uint32_t code4(const u32x4 &w, int i, float scale)
    {
        const uint32_t a = w[i], b = w[i + 1];
        s16x2 c = {0, 0};
        c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, a), scale, false);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, b), scale, true);
        return __builtin_bit_cast(uint32_t, c);
    }
};
template <>
struct Coder<f16> {
    static __device__ __forceinline__ uint32_t magnitude(const u32x4 &w)
    {
        return __float_as_uint((float)__builtin_bit_cast(_Float16, (uint16_t)pair_max(w)));
    }
    static __device__ __forceinline__ uint32_t code4(const u32x4 &w, int i, float scale)
    {
        const uint32_t a = w[i], b = w[i + 1];
        s16x2 c = {0, 0};
        c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(c, __builtin_bit_cast(f16x2, a), scale, false);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(c, __builtin_bit_cast(f16x2, b), scale, true);
        return __builtin_bit_cast(uint32_t, c);
    }
};
// Blocks that hold what is not finite, and the topmost one, e = 120, where 256 2^e is not finite any more: one number after the other.
template <class E>
__device__ __forceinline__ uint32_t finite_piece_magnitude(const u32x4 &w)
{
    constexpr int N = Piece<E>::N;
    float v[N];
    Piece<E>::unpack(w, v);
    uint32_t m = 0;
    for (int j = 0; j < N; ++j) m = max(m, finite_magnitude(v[j]));
    return m;
}
template <class E>
__device__ __forceinline__ void code_topmost(const u32x4 &w, uint32_t (&code)[Piece<E>::N / 4])
{
    constexpr int N = Piece<E>::N;
    float v[N];
    Piece<E>::unpack(w, v);
    for (int j = 0; j < N; ++j) {
        v[j] *= 0x1p-120f;
        if (fabsf(v[j]) > 240.f && fabsf(v[j]) < INFINITY) v[j] = copysignf(240.f, v[j]);
    }
    for (int q = 0; q < N / 4; ++q) {
        const int c = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * q], v[4 * q + 1], 0, false);
        code[q] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * q + 2], v[4 * q + 3], c, true);
    }
}
__device__ __forceinline__ void decode4(uint32_t w, float by, float *v)
{
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, by, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, by, true);
    v[0] = a[0];
    v[1] = a[1];
    v[2] = b[0];
    v[3] = b[1];
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

// A piece of row r at column c, c < padded width, zeros beyond the width, by the lanes that hold the block together: all of them call this.
template <class E>
__device__ __forceinline__ void keep_piece(const Kept &k, int64_t r, int c, const u32x4 &w)
{
    constexpr int N = Piece<E>::N;
    typedef __attribute__((address_space(1))) uint8_t *bytes;
    uint32_t most = block_max<N>(Coder<E>::magnitude(w));
    if (most >= 0x7f800000u) most = block_max<N>(finite_piece_magnitude<E>(w));
    const int e = block_exponent(most);
    const float scale = power_of_two(e);
    uint32_t code[N / 4];
#pragma unroll
    for (int q = 0; q < N / 4; ++q) code[q] = Coder<E>::code4(w, 2 * q, scale);
    if (e == 120) code_topmost<E>(w, code);
    const bytes at = (bytes)(uint64_t)(k.codes + r * k.stride + c);
    // (through the caches: past them 4 x 4096 x 4096 bf16 stored and loaded 75 us, so 71)
    if constexpr (N == 8) *(__attribute__((address_space(1))) u32x2 *)at = (u32x2){code[0], code[1]};
    else *(__attribute__((address_space(1))) uint32_t *)at = code[0];
    if (c % BLOCK == 0) ((bytes)(uint64_t)k.exponents)[r * (k.stride / BLOCK) + c / BLOCK] = (uint8_t)(e + 127);
}
// N columns as they are kept, and what they stand for.  Columns beyond the width are zeros.
template <int N>
struct Codes {
    uint32_t w[N / 4];
    uint32_t exponent;                                    // plus 127
};
template <int N>
__device__ __forceinline__ Codes<N> load_codes(const Kept &k, int64_t r, int c)
{
    const __attribute__((address_space(1))) uint8_t *const at = (const __attribute__((address_space(1))) uint8_t *)(uint64_t)(k.codes + r * k.stride + c);
    Codes<N> v;
    if constexpr (N == 8) {
        const u32x2 w = *(const __attribute__((address_space(1))) u32x2 *)at;
        v.w[0] = w[0];
        v.w[1] = w[1];
    } else {
        v.w[0] = *(const __attribute__((address_space(1))) uint32_t *)at;
    }
    v.exponent = *(const __attribute__((address_space(1))) uint8_t *)(uint64_t)(k.exponents + r * (k.stride / BLOCK) + c / BLOCK);
    return v;
}
template <int N>
__device__ __forceinline__ void unpack_codes(const Codes<N> &k, float (&v)[N])
{
    const float by = __uint_as_float(k.exponent << 23);
#pragma unroll
    for (int q = 0; q < N / 4; ++q) decode4(k.w[q], by, v + 4 * q);
}

}  // namespace layer
