// Device side of the losses on rows of logits.
//
// With c = s log2(e), m the largest logit of a row and M = c m (rounded once, the same number everywhere), the row's sum is
// Z = sum_v 2^(c x_v - M), so that log p_y = ln 2 (c x_y - M - log2 Z) and p_v = 2^(c x_v - M) / Z.  Keeping (m, Z) and not L = ln 2 (M + log2 Z)
// keeps the rounding of a large L (2^-24 |L|), and that of M, out of every probability.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dbw.h"
#include "global_access.h"

namespace loss {

constexpr float LOG2E = 1.44269504088896340736f;
constexpr float LN2 = 0.69314718055994530942f;

struct bf16 {
    uint16_t bits;
};
typedef _Float16 f16;

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(f16 v) { return (float)v; }
__device__ __forceinline__ float widen(bf16 v) { return __uint_as_float((uint32_t)v.bits << 16); }

// To the nearest value of the gradient's type, ties to even: the one rounding of a gradient.
template <class E>
__device__ __forceinline__ E narrow(float v);
template <>
__device__ __forceinline__ float narrow<float>(float v) { return v; }
template <>
__device__ __forceinline__ f16 narrow<f16>(float v) { return (f16)v; }
template <>
__device__ __forceinline__ bf16 narrow<bf16>(float v)
{
    const __bf16 b = (__bf16)v;
    return bf16{__builtin_bit_cast(uint16_t, b)};
}

__device__ __forceinline__ float load_as(const void *p, int64_t i, int type)
{
    if (type == 0) return ((const float *)p)[i];
    if (type == 1) return widen(((const bf16 *)p)[i]);
    return widen(((const f16 *)p)[i]);
}

// The rows of a call.
struct Rows {
    const void *x;     // logits
    void *dx;          // their gradient, or null
    int64_t ld, ld_grad;
    int vocab;
    int64_t rows;      // of all workers
    float scale, c;    // s, s log2(e)
    int32_t *status;
};

__device__ __forceinline__ void report(int32_t *status)
{
    if (status) *status = DBW_ERR_INVALID;                // every writer stores the same
}

// A token's column; the caller has seen that it is not negative.
__device__ __forceinline__ int column(const Rows &R, int token)
{
    if (token < R.vocab) return token;
    report(R.status);
    return R.vocab - 1;
}

// What a row's exponentials count from: 2^(c x - M).
//
// The rounding of M moves all of them by 2^(u |M|) and cancels in every ratio, but must not overflow: |M| <= 2^30 keeps it within 2^64.  Beyond,
// the next number below m is at least 64 octaves away, so that nothing but the largest logits counts; then c is a power of two that
// makes c m exact and a step below m 2^9 octaves (also where c m itself overflows, as in a row of the type's lowest value).
// A row of nothing but -inf so far counts from 0: its terms are 2^-inf = 0 and not 2^NaN.
struct Base {
    float c, M;
    bool steep;      // the largest logits only
};
constexpr float STEEP = 1073741824.f;
__device__ __forceinline__ Base base_of(float m, float c)
{
    if (m == -INFINITY) return Base{c, 0.f, false};
    const float M = m * c;
    if (!(fabsf(M) > STEEP) || isinf(m)) return Base{c, M, false};
    const float unit = ldexpf(1.f, 32 - ilogbf(m));
    return Base{unit, m * unit, true};
}
__device__ __forceinline__ float power(float x, const Base &b) { return __builtin_amdgcn_exp2f(fmaf(x, b.c, -b.M)); }

// log2 of a probability, from its logit and the row's (m, Z)
template <class MZ>
__device__ __forceinline__ float log2_p(float x, float c, const MZ &mz)
{
    const Base b = base_of(mz.m, c);
    return (b.steep ? (x - mz.m) * c : fmaf(x, c, -b.M)) - log2f(mz.z);
}

// ---------------------------------------------------------------- reductions

template <int CTRL, int ROWS>
__device__ __forceinline__ float shifted(float v, float identity)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(identity), __float_as_int(v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float uniform(float v) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v))); }
// Over the 64 lanes of a wave, without LDS: shifts by 1, 2, 4 and 8 within 16 lanes, then the rows' last lanes to the next rows.
__device__ __forceinline__ float wave_max(float v)
{
    v = fmaxf(v, shifted<0x111, 0xf>(v, -INFINITY));
    v = fmaxf(v, shifted<0x112, 0xf>(v, -INFINITY));
    v = fmaxf(v, shifted<0x114, 0xf>(v, -INFINITY));
    v = fmaxf(v, shifted<0x118, 0xf>(v, -INFINITY));
    v = fmaxf(v, shifted<0x142, 0xa>(v, -INFINITY));
    v = fmaxf(v, shifted<0x143, 0xc>(v, -INFINITY));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ __forceinline__ float wave_sum(float v)
{
    v += shifted<0x111, 0xf>(v, 0.f);
    v += shifted<0x112, 0xf>(v, 0.f);
    v += shifted<0x114, 0xf>(v, 0.f);
    v += shifted<0x118, 0xf>(v, 0.f);
    v += shifted<0x142, 0xa>(v, 0.f);
    v += shifted<0x143, 0xc>(v, 0.f);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// A maximum and the sum of exponentials that count from it.
struct MaxSum {
    float m, z;
};
// The factor that takes a sum from its own maximum to another, not smaller one.
__device__ __forceinline__ float rescale(float from, float to, float c)
{
    if (from == to) return 1.f;
    if (from == -INFINITY) return 0.f;
    const Base a = base_of(from, c), b = base_of(to, c);
    return a.steep || b.steep ? 0.f : __builtin_amdgcn_exp2f(a.M - b.M);
}
__device__ __forceinline__ MaxSum merged(MaxSum a, MaxSum b, float c)
{
    const float m = fmaxf(a.m, b.m);
    return MaxSum{m, a.z * rescale(a.m, m, c) + b.z * rescale(b.m, m, c)};
}

// What all T threads of a row get from the waves' values, in the waves' order.  lds: T / 64 values that nothing else uses meanwhile; the
// caller's next use of them lies behind a barrier.
template <int T>
__device__ __forceinline__ MaxSum row_merge(MaxSum v, float c, MaxSum *lds)
{
    if (T == 64) return v;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    float m = lds[0].m;
    for (int w = 1; w < T / 64; ++w) m = fmaxf(m, lds[w].m);
    float z = 0.f;
    for (int w = 0; w < T / 64; ++w) z += lds[w].z * rescale(lds[w].m, m, c);
    return MaxSum{uniform(m), uniform(z)};
}
template <int T>
__device__ __forceinline__ float row_sum(float v, float *lds)
{
    v = wave_sum(v);
    if (T == 64) return v;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
    for (int w = 1; w < T / 64; ++w) v += lds[w];
    return uniform(v);
}
template <int T>
__device__ __forceinline__ float row_max(float v, float *lds)
{
    v = wave_max(v);
    if (T == 64) return v;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
    for (int w = 1; w < T / 64; ++w) v = fmaxf(v, lds[w]);
    return uniform(v);
}

// ---------------------------------------------------------------- a row in pieces of 16 bytes

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// 16 bytes that start wherever an element may
template <class E>
struct Piece;
template <>
struct Piece<float> {
    typedef uint32_t raw __attribute__((ext_vector_type(4), aligned(4)));
    static constexpr int N = 4;
    static constexpr uint32_t NOTHING = 0xff800000u;      // -inf, which adds nothing to a sum of exponentials
    static __device__ __forceinline__ void unpack(const u32x4 &w, float (&v)[N])
    {
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
    }
    static __device__ __forceinline__ u32x4 pack(const float (&v)[N])
    {
        u32x4 w;
        for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(v[i]);
        return w;
    }
};
template <>
struct Piece<bf16> {
    typedef uint32_t raw __attribute__((ext_vector_type(4), aligned(2)));
    static constexpr int N = 8;
    static constexpr uint32_t NOTHING = 0xff80ff80u;
    static __device__ __forceinline__ void unpack(const u32x4 &w, float (&v)[N])
    {
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ u32x4 pack(const float (&v)[N])
    {
        typedef float two __attribute__((ext_vector_type(2)));
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        u32x4 w;
        for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((two){v[2 * i], v[2 * i + 1]}, bf16x2));
        return w;
    }
};
template <>
struct Piece<f16> {
    typedef uint32_t raw __attribute__((ext_vector_type(4), aligned(2)));
    typedef f16 pair __attribute__((ext_vector_type(2)));
    static constexpr int N = 8;
    static constexpr uint32_t NOTHING = 0xfc00fc00u;
    static __device__ __forceinline__ void unpack(const u32x4 &w, float (&v)[N])
    {
        for (int i = 0; i < 4; ++i) {
            const uint32_t bits = w[i];                   // (a cast of the vector's element itself gives the first one's bits)
            const pair h = __builtin_bit_cast(pair, bits);
            v[2 * i] = (float)h[0];
            v[2 * i + 1] = (float)h[1];
        }
    }
    static __device__ __forceinline__ u32x4 pack(const float (&v)[N])
    {
        u32x4 w;
        for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, (pair){(f16)v[2 * i], (f16)v[2 * i + 1]});
        return w;
    }
};

// The elements of a row among T threads: pieces of 16 bytes on 16-byte boundaries, thread t's are t, t + T, ...  Of the elements before
// the first boundary thread t has element t, of those behind the last piece thread BEHIND + t: at most one of either a thread.
template <class E, int T>
struct RowOf {
    typedef Piece<E> P;
    typedef const __attribute__((address_space(1))) u32x4 *place;
    static constexpr int BEHIND = 32;
    const E *x;
    int before;          // elements before the first boundary
    int pieces;
    int behind;          // elements behind the last piece
    __device__ __forceinline__ RowOf(const E *row, int vocab) : x(row)
    {
        before = min(vocab, (int)(-(uintptr_t)row & 15) / (int)sizeof(E));
        pieces = (vocab - before) / P::N;
        behind = (vocab - before) % P::N;
    }

    // Pieces first + i T + t, i < C, without a branch: beyond the row's end its last piece again, which clip() takes out when the pieces
    // are looked at.  The row has a piece.  ONCE: they will not be read again, so they need not stay in the caches.
    template <int C, bool ONCE>
    __device__ __forceinline__ void load(int first, u32x4 (&r)[C]) const
    {
        const global_access::bytes base = global_access::uniform_base(x + before);
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const uint32_t p = min(first + i * T + (int)threadIdx.x, pieces - 1);
            r[i] = ONCE ? __builtin_nontemporal_load((place)(base + p * 16u)) : *(place)(base + p * 16u);
        }
    }
    // Piece i of those from `first` on: beyond the row's end it adds nothing.
    __device__ __forceinline__ void clip(int first, int i, u32x4 &r) const
    {
        if (first + (i + 1) * T > pieces) {               // the same for all threads
            const bool in = first + i * T + (int)threadIdx.x < pieces;
#pragma unroll
            for (int j = 0; j < 4; ++j) r[j] = in ? r[j] : P::NOTHING;
        }
    }
    // Takes the columns whose bits are set out of piece i of those from `first` on.
    __device__ __forceinline__ void leave_out(int first, int i, u32x4 &r, const uint8_t *bits) const
    {
        const int p = first + i * T + (int)threadIdx.x;
        uint32_t b = p < pieces ? bits[(p + 1) * P::N >> 3] : 0u;
        if (P::N == 4) b = b >> ((p + 1) & 1) * 4 & 15u;
        if (b) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (P::N == 4) {
                    if (b >> j & 1) r[j] = P::NOTHING;
                } else {
                    const uint32_t m = (b >> 2 * j & 1 ? 0xffffu : 0u) | (b >> 2 * j & 2 ? 0xffff0000u : 0u);
                    r[j] = (r[j] & ~m) | (P::NOTHING & m);
                }
            }
        }
    }
    __device__ __forceinline__ int piece_column(int p) const { return before + p * P::N; }
    __device__ __forceinline__ bool has_single() const
    {
        const int t = threadIdx.x;
        return t < before || (t >= BEHIND && t < BEHIND + behind);
    }
    __device__ __forceinline__ int single_column() const
    {
        const int t = threadIdx.x;
        return t < BEHIND ? t : piece_column(pieces) + t - BEHIND;
    }
    __device__ __forceinline__ float load_single() const { return has_single() ? widen(x[single_column()]) : -INFINITY; }
    // the thread that a column is with
    __device__ __forceinline__ int owner(int v) const
    {
        if (v < before) return v;
        const int p = (v - before) / P::N;
        return p >= pieces ? BEHIND + (v - before) % P::N : p % T;
    }
};

// Keeps the compiler from carrying pieces from one pass to the next unpacked, in twice the registers.
template <int C>
__device__ __forceinline__ void keep_packed(u32x4 (&r)[C])
{
#pragma unroll
    for (int i = 0; i < C; ++i) asm volatile("" : "+v"(r[i]));
}

template <class E>
__device__ __forceinline__ float piece_max(const u32x4 &r, float top)
{
    float v[Piece<E>::N];
    Piece<E>::unpack(r, v);
#pragma unroll
    for (int j = 0; j < Piece<E>::N; ++j) top = fmaxf(top, v[j]);
    return top;
}
template <class E>
__device__ __forceinline__ float piece_sum(const u32x4 &r, const Base &b)
{
    float v[Piece<E>::N], sum = 0.f;
    Piece<E>::unpack(r, v);
#pragma unroll
    for (int j = 0; j < Piece<E>::N; ++j) sum += power(v[j], b);
    return sum;
}

// Adds the pieces from `first` on to a wave's maximum and a lane's sum.  The maximum is the wave's and not the lane's, so that what the exponentials count from is one number in scalar registers.
// left_out: bits of columns that are left out of the sum (LEAVE); column v has bit v - row.before + N, so that a piece's bits are together.
template <bool LEAVE, class E, int T, int C>
__device__ __forceinline__ void add_pieces(const RowOf<E, T> &row, int first, u32x4 (&r)[C], float single, const uint8_t *left_out, float c, float &m, float &z)
{
    float top = single;
#pragma unroll
    for (int i = 0; i < C; ++i) {
        row.clip(first, i, r[i]);
        if (LEAVE) {
            row.leave_out(first, i, r[i], left_out);
            asm volatile("" : "+v"(r[i]));                // one piece after the other
        }
        top = piece_max<E>(r[i], top);
    }
    top = fmaxf(wave_max(top), m);
    z *= rescale(m, top, c);
    m = top;
    const Base base = base_of(m, c);
    const Base b{uniform(base.c), uniform(base.M), false};
    z += power(single, b);
    keep_packed(r);
#pragma unroll
    for (int i = 0; i < C; ++i) z += piece_sum<E>(r[i], b);
}

// Piece i of the gradient of those from `first` on: by 2^(c x - M).
template <class E, int T>
__device__ __forceinline__ void store_piece(global_access::bytes base, int first, int pieces, int i, const u32x4 &r, float by, const Base &b)
{
    typedef Piece<E> P;
    const int p = first + i * T + (int)threadIdx.x;
    if (p < pieces) {
        float v[P::N];
        P::unpack(r, v);
#pragma unroll
        for (int j = 0; j < P::N; ++j) v[j] = by * power(v[j], b);
        __builtin_nontemporal_store((typename P::raw)P::pack(v), (__attribute__((address_space(1))) typename P::raw *)(base + (uint32_t)p * 16u));
    }
}

template <class E, int T, bool NT = false>
__device__ __forceinline__ void zero_row(const Rows &R, int64_t r)
{
    if (!R.dx) return;
    E *dx = (E *)R.dx + r * R.ld_grad;
    const RowOf<E, T> row(dx, R.vocab);
    const global_access::bytes base = global_access::uniform_base(dx + row.before);
    for (int p = threadIdx.x; p < row.pieces; p += T)
        if (NT) __builtin_nontemporal_store((u32x4)(0u), (__attribute__((address_space(1))) u32x4 *)(base + (uint32_t)p * 16u));
        else *(__attribute__((address_space(1))) u32x4 *)(base + (uint32_t)p * 16u) = (u32x4)(0u);
    if (row.has_single()) dx[row.single_column()] = narrow<E>(0.f);
}

// ---------------------------------------------------------------- what a row's loss needs besides its logits

struct Logp {
    const int32_t *tokens;
    float *logp_out, *lse_out;
    struct MaxSum *stats;// (m, Z) of every row, for a gradient in a launch of its own, or null
    const float *weights;// null: no row is left out for its weight
};

struct Policy {
    const int32_t *tokens;
    const float *old_logp, *ref_logp, *advantage, *weights;
    float low, high, kl_coef, weight;     // the bounds of the ratio; the weight of every row where weights is null
    float *logp_out;
    float2 *terms;       // a row's weighted loss and KL term, for the sums over a worker's rows
};

struct Distill {
    const int32_t *index;
    const void *value;
    const float *teacher_lse, *weights;
    float weight;
    int k, value_type;
    float *row_loss_out;
    float2 *terms;
};

// The loss of a row from its token's log-probability, and the derivative.
__device__ __forceinline__ float policy_row(const Policy &P, int64_t r, float w, float logp)
{
    const float a = P.advantage[r], rho = expf(logp - P.old_logp[r]);
    const float free = rho * a, bound = fminf(fmaxf(rho, P.low), P.high) * a;
    float kl = 0.f, dkl = 0.f;
    if (P.ref_logp) {
        const float d = P.ref_logp[r] - logp;
        dkl = -expm1f(d);
        kl = -dkl - d;
    }
    // (rho NaN: the bounded ratio of fminf/fmaxf is not, so the unbounded product comes first)
    const float surrogate = free <= bound || free != free ? free : bound;
    if (P.terms) P.terms[r] = make_float2(w * (P.kl_coef * kl - surrogate), w * kl);
    return w * (P.kl_coef * dkl - (free <= bound || free != free ? free : 0.f));
}

// ---------------------------------------------------------------- kernels

// A grid's threads have to number less than 2^32: many rows make a second dimension.
__device__ __forceinline__ int64_t row_of_block() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// A workgroup of T threads holds the first T C pieces of a row in registers from when they are loaded until the gradient is written: one pass
// over them finds their maximum, one their sum, one the gradient.  The pieces that a longer row has behind them go through other registers,
// T S at a time, and are read again for the gradient, back to front, the latest first.  (S = 0: no row is longer.)
template <class E, int T, int C, int S>
struct Walk {
    static constexpr int REST = T * C;
    RowOf<E, T> row;
    u32x4 r[C];
    float single;
    __device__ __forceinline__ Walk(const E *x, int vocab) : row(x, vocab)
    {
        if (row.pieces > 0) {
            row.template load<C, true>(0, r);
        } else {
#pragma unroll
            for (int i = 0; i < C; ++i) r[i] = (u32x4)(Piece<E>::NOTHING);
        }
        single = row.load_single();
    }
    // (The gradient's pass may find a column that is left out here left out or not.)
    template <bool LEAVE = false>
    __device__ __forceinline__ MaxSum stats(float c, MaxSum *lds, const uint8_t *left_out = nullptr)
    {
        float m = -INFINITY, z = 0.f;
        if (LEAVE) {
            const int bit = row.single_column() - row.before + Piece<E>::N;
            if (row.has_single() && (left_out[bit >> 3] >> (bit & 7) & 1)) single = -INFINITY;
        }
        add_pieces<LEAVE>(row, 0, r, single, left_out, c, m, z);
        if constexpr (S > 0)
            for (int first = REST; first < row.pieces; first += T * S) {
                u32x4 v[S];
                row.template load<S, false>(first, v);
                add_pieces<LEAVE>(row, first, v, -INFINITY, left_out, c, m, z);
            }
        return row_merge<T>(MaxSum{m, wave_sum(z)}, c, lds);
    }
    // dx_v = by 2^(c x - M), and coef more at column y (none if negative)
    __device__ __forceinline__ void gradient(E *dx, float by, const Base &base, int y, float xy, float coef)
    {
        const Base b{uniform(base.c), uniform(base.M), false};
        by = uniform(by);
        const global_access::bytes out = global_access::uniform_base(dx + row.before);
        if constexpr (S > 0)
            if (row.pieces > REST)
                for (int first = REST + (row.pieces - 1 - REST) / (T * S) * (T * S); first >= REST; first -= T * S) {
                    u32x4 v[S];
                    row.template load<S, true>(first, v);
#pragma unroll
                    for (int i = 0; i < S; ++i) store_piece<E, T>(out, first, row.pieces, i, v[i], by, b);
                }
        keep_packed(r);
#pragma unroll
        for (int i = 0; i < C; ++i) store_piece<E, T>(out, 0, row.pieces, i, r[i], by, b);
        if (row.has_single()) dx[row.single_column()] = narrow<E>(by * power(single, b));
        // by the thread that wrote the column before
        if (y >= 0 && (int)threadIdx.x == row.owner(y)) dx[y] = narrow<E>(by * power(xy, b) + coef);
    }
};

// AGAIN: the rows will be read again soon, for their gradient.
template <class E, int T, int C, bool AGAIN>
__global__ __launch_bounds__(T) void logp_kernel(Rows R, Logp P)
{
    __shared__ MaxSum lds[T / 64];
    const int64_t r = row_of_block();
    if (r >= R.rows) return;
    const int token = P.tokens[r];
    if (token < 0 || (P.weights && P.weights[r] == 0.f)) {
        if (threadIdx.x == 0) {
            if (P.logp_out) P.logp_out[r] = 0.f;
            if (P.lse_out) P.lse_out[r] = 0.f;
        }
        return;
    }
    const E *x = (const E *)R.x + r * R.ld;
    const RowOf<E, T> row(x, R.vocab);
    float m = -INFINITY, z = 0.f;
    for (int first = 0; first < row.pieces; first += T * C) {
        u32x4 v[C];
        row.template load<C, !AGAIN>(first, v);
        add_pieces<false>(row, first, v, -INFINITY, nullptr, R.c, m, z);
    }
    const float single = row.load_single(), xy = widen(x[column(R, token)]), top = wave_max(single);
    const MaxSum mz = row_merge<T>(merged(MaxSum{m, wave_sum(z)}, MaxSum{top, wave_sum(power(single, base_of(top, R.c)))}, R.c), R.c, lds);
    if (threadIdx.x == 0) {
        if (P.logp_out) P.logp_out[r] = LN2 * log2_p(xy, R.c, mz);
        if (P.lse_out) P.lse_out[r] = fmaf(R.scale, mz.m, LN2 * log2f(mz.z));
        if (P.stats) P.stats[r] = mz;
    }
}

template <class E, int T, int C, int S>
__global__ __launch_bounds__(T, C == 16 ? 4 : 1) void policy_kernel(Rows R, Policy P)
{
    __shared__ MaxSum lds[T / 64];
    const int64_t r = row_of_block();
    if (r >= R.rows) return;
    const int token = P.tokens[r];
    const float w = P.weights ? P.weights[r] : P.weight;
    if (token < 0 || w == 0.f) {
        if (threadIdx.x == 0) {
            if (P.logp_out) P.logp_out[r] = 0.f;
            P.terms[r] = make_float2(0.f, 0.f);
        }
        zero_row<E, T>(R, r);
        return;
    }
    const E *x = (const E *)R.x + r * R.ld;
    Walk<E, T, C, S> walk(x, R.vocab);
    const int y = column(R, token);
    const float xy = widen(x[y]);
    const MaxSum mz = walk.stats(R.c, lds);
    const float logp = LN2 * log2_p(xy, R.c, mz);
    Policy once = P;
    if (threadIdx.x != 0) once.terms = nullptr;
    const float coef = R.scale * policy_row(once, r, w, logp);
    if (threadIdx.x == 0 && P.logp_out) P.logp_out[r] = logp;
    if (!R.dx) return;
    if (coef == 0.f) zero_row<E, T>(R, r);
    else walk.gradient((E *)R.dx + r * R.ld_grad, -coef / mz.z, base_of(mz.m, R.c), y, xy, coef);
}

// The gradient alone, from (m, Z) or from L: a row's pieces in batches of T C.
template <class E, int T, int C>
__global__ __launch_bounds__(T) void gradient_kernel(Rows R, const int32_t *tokens, const MaxSum *stats, const float *lse,
                                                     const float *coef)
{
    const int64_t r = row_of_block();
    if (r >= R.rows) return;
    const int token = tokens[r];
    const float g = token < 0 || !coef ? 0.f : R.scale * coef[r];
    if (g == 0.f) {
        zero_row<E, T, true>(R, r);
        return;
    }
    const E *x = (const E *)R.x + r * R.ld;
    E *dx = (E *)R.dx + r * R.ld_grad;
    const RowOf<E, T> row(x, R.vocab);
    const int y = column(R, token);
    const float xy = widen(x[y]), single = row.load_single();
    float by = -g;
    Base b;
    if (stats) {
        b = base_of(stats[r].m, R.c);
        by /= stats[r].z;
    } else {                                              // from L: M = L log2(e), Z = 1
        b = base_of(lse[r] / R.scale, R.c);
        if (!b.steep) b.M = lse[r] * LOG2E;
    }
    b = Base{uniform(b.c), uniform(b.M), false};
    by = uniform(by);
    const global_access::bytes out = global_access::uniform_base(dx + row.before);
    for (int first = 0; first < row.pieces; first += T * C) {
        u32x4 v[C];
        row.template load<C, true>(first, v);
#pragma unroll
        for (int i = 0; i < C; ++i) store_piece<E, T>(out, first, row.pieces, i, v[i], by, b);
    }
    if (row.has_single()) dx[row.single_column()] = narrow<E>(by * power(single, b));
    if ((int)threadIdx.x == row.owner(y)) dx[y] = narrow<E>(by * power(xy, b) + g);
}

// The teacher's list of a row is in LDS: columns (-1 where absent), scaled logits, the student's logits, and a bit for every column of the
// vocabulary that is in the list.
template <class E, int T, int C, int S, bool TAIL>
__global__ __launch_bounds__(T, C == 16 ? 4 : 1) void distill_kernel(Rows R, Distill P)
{
    extern __shared__ uint32_t shared[];
    __shared__ MaxSum lds[T / 64], lds_top[T / 64];
    __shared__ float sums[4][T / 64];
    __shared__ int twice;
    int *const at = (int *)shared;
    float *const q = (float *)(shared + P.k);
    float *const xs = (float *)(shared + 2 * P.k);
    uint32_t *const in_top = shared + 3 * P.k;

    const int64_t r = row_of_block();
    if (r >= R.rows) return;
    const int tid = threadIdx.x;
    const float w = P.weights ? P.weights[r] : P.weight;
    if (w == 0.f) {
        if (tid == 0) {
            P.terms[r] = make_float2(0.f, 0.f);
            if (P.row_loss_out) P.row_loss_out[r] = 0.f;
        }
        zero_row<E, T>(R, r);
        return;
    }
    const E *x = (const E *)R.x + r * R.ld;
    Walk<E, T, C, S> walk(x, R.vocab);                       // in flight while the list is looked at

    const int words = (R.vocab + Piece<E>::N + 31) / 32, bit0 = Piece<E>::N - walk.row.before;
    for (int i = tid; i < words; i += T) in_top[i] = 0;
    if (tid == 0) twice = 0;
    __syncthreads();
    for (int j = tid; j < P.k; j += T) {
        int v = P.index[r * P.k + j];
        if (v >= R.vocab) {
            report(R.status);
            v = -1;
        }
        at[j] = v;
        q[j] = R.scale * load_as(P.value, r * P.k + j, P.value_type);
        if (v >= 0) {
            xs[j] = widen(x[v]);
            if (atomicOr(&in_top[v + bit0 >> 5], 1u << (v + bit0 & 31)) >> (v + bit0 & 31) & 1) twice = 1;
        }
    }
    __syncthreads();
    if (twice) {                                          // rare: the first entry of a column counts
        if (tid == 0) {
            report(R.status);
            for (int j = 1; j < P.k; ++j)
                for (int i = 0; i < j; ++i)
                    if (at[i] == at[j]) at[j] = -1;
        }
        __syncthreads();
    }
    float top = -INFINITY, any = 0.f, m_top = -INFINITY;
    for (int j = tid; j < P.k; j += T)
        if (at[j] >= 0) {
            top = fmaxf(top, q[j]);
            any = 1.f;
            m_top = fmaxf(m_top, xs[j]);
        }
    top = row_max<T>(top, sums[0]);
    any = row_max<T>(any, sums[1]);
    float sum = 0.f, z_top = 0.f;
    m_top = wave_max(m_top);
    const Base base_top = base_of(m_top, R.c);
    for (int j = tid; j < P.k; j += T)
        if (at[j] >= 0) {
            sum += expf(q[j] - (top == -INFINITY ? 0.f : top));
            z_top += power(xs[j], base_top);
        }
    sum = row_sum<T>(sum, sums[2]);
    const float norm = TAIL ? P.teacher_lse[r] : top + logf(sum);
    if (any == 0.f || (!TAIL && top == -INFINITY && sum == 0.f)) {
        if (tid == 0) {
            P.terms[r] = make_float2(0.f, 0.f);
            if (P.row_loss_out) P.row_loss_out[r] = 0.f;
        }
        zero_row<E, T>(R, r);
        return;
    }

    // With the tail the student's mass outside the list is summed apart, from a maximum of its own: it may be far below the rest, and as a
    // difference from one it would be lost.
    MaxSum mz;
    float log_out = 0.f;
    if (TAIL) {
        const MaxSum in = row_merge<T>(MaxSum{m_top, wave_sum(z_top)}, R.c, lds_top);
        const MaxSum out = walk.template stats<true>(R.c, lds, (const uint8_t *)in_top);
        mz = merged(out, in, R.c);
        const Base a = base_of(out.m, R.c), b = base_of(mz.m, R.c);
        log_out = LN2 * ((a.steep || b.steep ? (out.m - mz.m) * R.c : a.M - b.M) + (log2f(out.z) - log2f(mz.z)));
    } else {
        mz = walk.stats(R.c, lds);
    }
    const Base base = base_of(mz.m, R.c);
    float part = 0.f, mass = 0.f;
    for (int j = tid; j < P.k; j += T)
        if (at[j] >= 0) {
            const float log_q = q[j] - norm, qj = expf(log_q);
            const float log_p = LN2 * log2_p(xs[j], R.c, mz);
            mass += qj;
            if (!(qj <= 0.f)) part += qj * (log_q - log_p);
            q[j] = expf(log_p) - qj;                      // dl/dx over s
        }
    part = row_sum<T>(part, sums[3]);
    float factor = 1.f;
    if (TAIL) {
        mass = row_sum<T>(mass, sums[0]);                 // (its last use lies two barriers back)
        const float rest = fmaxf(1.f - mass, 0.f);
        if (rest > 0.f) {
            part += rest * (logf(rest) - log_out);
            factor = 1.f - expf(logf(rest) - log_out);
        }
    }
    if (tid == 0) {
        P.terms[r] = make_float2(w * part, 0.f);
        if (P.row_loss_out) P.row_loss_out[r] = part;
    }
    if (!R.dx) return;
    E *dx = (E *)R.dx + r * R.ld_grad;
    walk.gradient(dx, R.scale * w * factor / mz.z, base, -1, 0.f, 0.f);
    __syncthreads();                                      // the list's columns are written over
    for (int j = tid; j < P.k; j += T)
        if (at[j] >= 0) dx[at[j]] = narrow<E>(R.scale * w * q[j]);
}

constexpr int THREADS = 256;
constexpr int WAVES = THREADS / 64;

// loss_out[i], second_out[i] = sums of the terms of worker i's rows, always in the same order.
__global__ __launch_bounds__(THREADS) void sum_kernel(const float2 *terms, int rows, float *loss_out, float *second_out)
{
    __shared__ float lds[2][WAVES];
    const float2 *t = terms + (int64_t)blockIdx.x * rows;
    float a = 0.f, b = 0.f;
    for (int r = threadIdx.x; r < rows; r += THREADS) {
        a += t[r].x;
        b += t[r].y;
    }
    a = row_sum<THREADS>(a, lds[0]);
    b = row_sum<THREADS>(b, lds[1]);
    if (threadIdx.x == 0) {
        loss_out[blockIdx.x] = a;
        if (second_out) second_out[blockIdx.x] = b;
    }
}

struct Preference {
    const int32_t *tokens, *seq_start;
    const float *logp, *ref_logp, *weights;
    float beta, smoothing;
    int pairs;           // of each worker
    int64_t all_rows;
    float *margin_out, *coef;
    int32_t *status;
};

// The margin of a pair and the derivative of its worker's loss with respect to every log-probability of its rows.
__global__ __launch_bounds__(THREADS) void pair_kernel(Preference P)
{
    __shared__ float lds[WAVES];
    const int64_t j = blockIdx.x;
    const int tid = threadIdx.x, n = (int)P.all_rows;
    int a[3];
    for (int i = 0; i < 3; ++i) a[i] = P.seq_start[2 * j + i];
    if (a[0] < 0 || a[1] < a[0] || a[2] < a[1] || a[2] > n) report(P.status);
    a[0] = min(max(a[0], 0), n);
    a[1] = min(max(a[1], a[0]), n);
    a[2] = min(max(a[2], a[1]), n);
    float h = 0.f;
    for (int r = a[0] + tid; r < a[2]; r += THREADS) {
        const float w = P.weights ? P.weights[r] : 1.f;
        const float t = P.tokens[r] < 0 || w == 0.f ? 0.f : w * (P.logp[r] - P.ref_logp[r]);
        h += r < a[1] ? t : -t;
    }
    const float u = P.beta * row_sum<THREADS>(h, lds);
    if (tid == 0) P.margin_out[j] = u;
    const float e = expf(-fabsf(u));                      // sigma(u) = 1 / (1 + e) or e / (1 + e)
    const float sig = (u >= 0.f ? 1.f : e) / (1.f + e), sig_not = (u >= 0.f ? e : 1.f) / (1.f + e);
    const float slope = (u != u ? u : P.smoothing * sig - (1.f - P.smoothing) * sig_not) * P.beta / (float)P.pairs;
    for (int r = a[0] + tid; r < a[2]; r += THREADS) {
        const float w = P.weights ? P.weights[r] : 1.f;
        P.coef[r] = P.tokens[r] < 0 || w == 0.f ? 0.f : (r < a[1] ? slope : -slope) * w;
    }
    if (j == 0)
        for (int r = tid; r < a[0]; r += THREADS) P.coef[r] = 0.f;
    if (j == gridDim.x - 1)
        for (int r = a[2] + tid; r < n; r += THREADS) P.coef[r] = 0.f;
}

// A worker's mean over its pairs, from their margins.
__global__ __launch_bounds__(THREADS) void pair_loss_kernel(const float *margin, int pairs, float smoothing, float *loss_out)
{
    __shared__ float lds[WAVES];
    const float *u = margin + (int64_t)blockIdx.x * pairs;
    float l = 0.f;
    for (int j = threadIdx.x; j < pairs; j += THREADS) {
        const float soft = log1pf(expf(-fabsf(u[j])));
        // -log sigma(u) = max(-u, 0) + soft, -log sigma(-u) = max(u, 0) + soft
        l += u[j] != u[j] ? u[j] : soft + (u[j] >= 0.f ? smoothing * u[j] : (smoothing - 1.f) * u[j]);
    }
    l = row_sum<THREADS>(l, lds);
    if (threadIdx.x == 0) loss_out[blockIdx.x] = pairs ? l / (float)pairs : 0.f;
}

}  // namespace loss
