// Device side of the losses on rows of logits.
//
// With c = s log2(e) and m the largest logit of a row, the row's sum is Z = sum_v 2^(c (x_v - m)), so that log p_y = s (x_y - m) - ln Z and
// p_v = 2^(c (x_v - m)) / Z.  The difference comes first: the largest term is exactly 1, logits may be of any size (masks of a type's lowest value), and
// keeping (m, Z) and not L = s m + ln Z keeps the rounding of a large L (2^-24 |L|) out of every probability.  c is a sum of two numbers: rounded to
// one it would be off by up to 2^-24 of itself, for all terms of all rows in the same direction, which the sum over a sequence's log-probabilities
// does not average out (at s = 0.9 every ln Z was 2.9e-7 too large).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dbw.h"
#include "global_access.h"

namespace loss {

constexpr double LOG2E = 1.44269504088896340736;
constexpr double LN2 = 0.69314718055994530942;

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

// c = s log2(e) as hi + lo.  hi is below c and lo above zero, so that the exponent of a logit of -inf, -inf hi + -inf lo, is -inf.
struct Factor {
    float hi, lo;
    float near;          // the nearest number, for what is not summed
};

// The rows of a call.
struct Rows {
    const void *x;     // logits
    void *dx;          // their gradient, or null
    int64_t ld, ld_grad;
    int vocab;
    int64_t rows;      // of all workers
    float scale;       // s
    Factor c;          // s log2(e)
    int32_t *status;
    bool by_xcd;       // workgroups take rows in the XCDs' order
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

// What a row's exponentials count from: 2^(c (x - m)).  A row of nothing but -inf so far counts from 0: its terms are 2^-inf = 0 and not 2^NaN.
struct Base {
    Factor c;
    float m;
};
__device__ __forceinline__ Base base_of(float m, const Factor &c) { return Base{c, m == -INFINITY ? 0.f : m}; }
__device__ __forceinline__ float times(const Factor &c, float d) { return fmaf(d, c.hi, d * c.lo); }      // rounded once, but for 2^-24 of lo's part
// Of one column, for a gradient: nothing adds these up, and the nearest factor is as good.  An instruction less: 4096 rows of 131072 bf16 distilled in
// 426 us, with power() 439.
__device__ __forceinline__ float power_alone(float x, const Base &b) { return __builtin_amdgcn_exp2f((x - b.m) * b.c.near); }
__device__ __forceinline__ float power(float x, const Base &b) { return __builtin_amdgcn_exp2f(times(b.c, x - b.m)); }

// e^v: log2(e) likewise
__device__ __forceinline__ float exponential(float v)
{
    constexpr float HI = 0x1.715474p0f;
    return __builtin_amdgcn_exp2f(times(Factor{HI, (float)(LOG2E - HI), (float)LOG2E}, v));
}

// A row is T threads' work; a workgroup has T threads, or several rows of 64 or 16 threads each.
template <int T>
__device__ __forceinline__ int tid() { return (int)threadIdx.x & (T - 1); }
// Orders a row's accesses to LDS.
template <int T>
__device__ __forceinline__ void row_barrier()
{
    if (T <= 64) {                                        // a wave's are in order; the compiler's have to be, too
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    } else {
        __syncthreads();
    }
}

// ---------------------------------------------------------------- reductions

template <int CTRL, int ROWS>
__device__ __forceinline__ float shifted(float v, float identity)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(identity), __float_as_int(v), CTRL, ROWS, 0xf, false));
}
// A value that all lanes of a row's waves have, in a scalar register.  (The lanes of one wave have several rows if T < 64.)
template <int T>
__device__ __forceinline__ float uniform(float v)
{
    return T < 64 ? v : __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v)));
}
template <int T>
__device__ __forceinline__ double uniform(double v)
{
    const int64_t b = __double_as_longlong(v);
    if (T < 64) return v;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((int)b), hi = __builtin_amdgcn_readfirstlane((int)(b >> 32));
    return __longlong_as_double((int64_t)((uint64_t)hi << 32 | lo));
}
template <int T>
__device__ __forceinline__ Base uniform(const Base &b) { return Base{{uniform<T>(b.c.hi), uniform<T>(b.c.lo), uniform<T>(b.c.near)}, uniform<T>(b.m)}; }
// Over the 64 lanes of a wave, without LDS: shifts by 1, 2, 4 and 8 within 16 lanes, then the last lanes of 16 to the next ones.  Over 16 lanes:
// rotations, which leave the result in all of them.
template <int T>
__device__ __forceinline__ float lanes_max(float v)
{
    if (T == 16) {
        v = fmaxf(v, shifted<0x121, 0xf>(v, v));
        v = fmaxf(v, shifted<0x122, 0xf>(v, v));
        v = fmaxf(v, shifted<0x124, 0xf>(v, v));
        return fmaxf(v, shifted<0x128, 0xf>(v, v));
    }
    v = fmaxf(v, shifted<0x111, 0xf>(v, -INFINITY));
    v = fmaxf(v, shifted<0x112, 0xf>(v, -INFINITY));
    v = fmaxf(v, shifted<0x114, 0xf>(v, -INFINITY));
    v = fmaxf(v, shifted<0x118, 0xf>(v, -INFINITY));
    v = fmaxf(v, shifted<0x142, 0xa>(v, -INFINITY));
    v = fmaxf(v, shifted<0x143, 0xc>(v, -INFINITY));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
template <int T>
__device__ __forceinline__ float lanes_sum(float v)
{
    if (T == 16) {
        v += shifted<0x121, 0xf>(v, 0.f);
        v += shifted<0x122, 0xf>(v, 0.f);
        v += shifted<0x124, 0xf>(v, 0.f);
        return v + shifted<0x128, 0xf>(v, 0.f);
    }
    v += shifted<0x111, 0xf>(v, 0.f);
    v += shifted<0x112, 0xf>(v, 0.f);
    v += shifted<0x114, 0xf>(v, 0.f);
    v += shifted<0x118, 0xf>(v, 0.f);
    v += shifted<0x142, 0xa>(v, 0.f);
    v += shifted<0x143, 0xc>(v, 0.f);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
// The same in 64 bits.
template <int CTRL, int ROWS>
__device__ __forceinline__ double shifted(double v)
{
    const int64_t b = __double_as_longlong(v);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)b, CTRL, ROWS, 0xf, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, ROWS, 0xf, false);
    return __longlong_as_double((int64_t)((uint64_t)hi << 32 | lo));
}
template <int T>
__device__ __forceinline__ double lanes_sum(double v)
{
    if (T == 16) {
        v += shifted<0x121, 0xf>(v);
        v += shifted<0x122, 0xf>(v);
        v += shifted<0x124, 0xf>(v);
        return v + shifted<0x128, 0xf>(v);
    }
    v += shifted<0x111, 0xf>(v);
    v += shifted<0x112, 0xf>(v);
    v += shifted<0x114, 0xf>(v);
    v += shifted<0x118, 0xf>(v);
    v += shifted<0x142, 0xa>(v);
    v += shifted<0x143, 0xc>(v);
    const int64_t b = __double_as_longlong(v);
    const uint32_t lo = __builtin_amdgcn_readlane((int)b, 63), hi = __builtin_amdgcn_readlane((int)(b >> 32), 63);
    return __longlong_as_double((int64_t)((uint64_t)hi << 32 | lo));
}
__device__ __forceinline__ float wave_max(float v) { return lanes_max<64>(v); }
template <class V>
__device__ __forceinline__ V wave_sum(V v) { return lanes_sum<64>(v); }

// A maximum and the sum of exponentials that count from it.
struct MaxSum {
    float m, z;
};
// ln z to 2^-25, whatever its size: the logarithm in 32 bits is that of a number near one, which is small.
__device__ __forceinline__ double ln(float z)
{
    float f = __builtin_amdgcn_frexp_mantf(z);            // in [1/2, 1)
    int e = __builtin_amdgcn_frexp_expf(z);
    if (f < 0.70710678f) {
        f *= 2.f;
        --e;
    }
    return fma((double)e, LN2, (double)logf(f));
}
// The log of a probability, from its logit and the row's (m, Z), and L.  Where it goes to 32 bits it is rounded once.
__device__ __forceinline__ double log_p(float x, float scale, const MaxSum &mz) { return (double)scale * ((double)x - mz.m) - ln(mz.z); }
__device__ __forceinline__ double log_sum(float scale, const MaxSum &mz) { return fma((double)scale, (double)mz.m, ln(mz.z)); }
// The factor that takes a sum from its own maximum to another, not smaller one.
__device__ __forceinline__ float rescale(float from, float to, const Factor &c)
{
    if (from == to) return 1.f;
    return from == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(times(c, from - to));
}
__device__ __forceinline__ MaxSum merged(MaxSum a, MaxSum b, const Factor &c)
{
    const float m = fmaxf(a.m, b.m);
    return MaxSum{m, a.z * rescale(a.m, m, c) + b.z * rescale(b.m, m, c)};
}

// What all T threads of a row get from the waves' values, in the waves' order.  lds: T / 64 values that nothing else uses meanwhile; the
// caller's next use of them lies behind a barrier.
template <int T>
__device__ __forceinline__ MaxSum row_merge(MaxSum v, const Factor &c, MaxSum *lds)
{
    if (T <= 64) return v;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    float m = lds[0].m;
    for (int w = 1; w < T / 64; ++w) m = fmaxf(m, lds[w].m);
    double z = 0.;
    for (int w = 0; w < T / 64; ++w) z += (double)(lds[w].z * rescale(lds[w].m, m, c));
    return MaxSum{uniform<T>(m), uniform<T>((float)z)};
}
template <int T, class V>
__device__ __forceinline__ V row_sum(V v, V *lds)
{
    v = lanes_sum<T>(v);
    if (T <= 64) return v;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
    for (int w = 1; w < T / 64; ++w) v += lds[w];
    return uniform<T>(v);
}
template <int T>
__device__ __forceinline__ float row_max(float v, float *lds)
{
    v = lanes_max<T>(v);
    if (T <= 64) return v;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
    for (int w = 1; w < T / 64; ++w) v = fmaxf(v, lds[w]);
    return uniform<T>(v);
}

// ---------------------------------------------------------------- a row in pieces of 16 bytes

// The address of a row, in scalar registers where it is a wave's.
template <int T>
__device__ __forceinline__ global_access::bytes base_address(const void *p)
{
    return T < 64 ? (global_access::bytes)(uint64_t)p : global_access::uniform_base(p);
}

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
    static constexpr int BEHIND = 8;      // (either are fewer than 8)
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
        const global_access::bytes base = base_address<T>(x + before);
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const uint32_t p = min(first + i * T + tid<T>(), pieces - 1);
            r[i] = ONCE ? __builtin_nontemporal_load((place)(base + p * 16u)) : *(place)(base + p * 16u);
        }
    }
    // Piece i of those from `first` on: beyond `end` it adds nothing.
    __device__ __forceinline__ void clip(int first, int end, int i, u32x4 &r) const
    {
        if (first + (i + 1) * T > end) {                  // the same for all threads
            const bool in = first + i * T + tid<T>() < end;
#pragma unroll
            for (int j = 0; j < 4; ++j) r[j] = in ? r[j] : P::NOTHING;
        }
    }
    // A piece's bits of `bits`: column v has bit v - before + N, so that a piece's are together.
    __device__ __forceinline__ uint32_t bits_of(int p, const uint8_t *bits) const
    {
        const uint32_t b = p < pieces ? bits[(p + 1) * P::N >> 3] : 0u;
        return P::N == 4 ? b >> ((p + 1) & 1) * 4 & 15u : b;
    }
    // Takes the columns whose bits are set out of piece i of those from `first` on.
    __device__ __forceinline__ void leave_out(int first, int i, u32x4 &r, const uint8_t *bits) const
    {
        const uint32_t b = bits_of(first + i * T + tid<T>(), bits);
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
        const int t = tid<T>();
        return t < before || (t >= BEHIND && t < BEHIND + behind);
    }
    __device__ __forceinline__ int single_column() const
    {
        const int t = tid<T>();
        return t < BEHIND ? t : piece_column(pieces) + t - BEHIND;
    }
    __device__ __forceinline__ float load_single() const { return has_single() ? widen(x[single_column()]) : -INFINITY; }
    // the piece that a column is in, -1 for a single one; and the thread that it is with
    __device__ __forceinline__ int piece_of(int v) const
    {
        const int p = (v - before) / P::N;
        return v < before || p >= pieces ? -1 : p;
    }
    __device__ __forceinline__ int owner(int v) const
    {
        const int p = piece_of(v);
        return p >= 0 ? p % T : v < before ? v : BEHIND + (v - before) % P::N;
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
    float v[Piece<E>::N];
    Piece<E>::unpack(r, v);
#pragma unroll
    for (int j = 0; j < Piece<E>::N; ++j) v[j] = power(v[j], b);
#pragma unroll
    for (int d = 1; d < Piece<E>::N; d *= 2)
#pragma unroll
        for (int j = 0; j < Piece<E>::N; j += 2 * d) v[j] += v[j + d];
    return v[0];
}

// Adds the pieces from `first` on to a wave's maximum and a lane's sum, which is held in 64 bits: where one token is almost certain the sum is little more
// than one, and each addition in 32 bits would cost the log-probability another 2^-25.  The maximum is the wave's and not the lane's, so that what the
// exponentials count from is one number in scalar registers.
// left_out: bits of columns that are left out of the sum (LEAVE); column v has bit v - row.before + N, so that a piece's bits are together.
template <bool LEAVE, class E, int T, int C>
__device__ __forceinline__ void add_pieces(const RowOf<E, T> &row, int first, int end, u32x4 (&r)[C], float single, const uint8_t *left_out, const Factor &c,
                                           float &m, double &z)
{
    float top = single;
#pragma unroll
    for (int i = 0; i < C; ++i) {
        row.clip(first, end, i, r[i]);
        if (LEAVE) {
            row.leave_out(first, i, r[i], left_out);
            asm volatile("" : "+v"(r[i]));                // one piece after the other
        }
        top = piece_max<E>(r[i], top);
    }
    top = fmaxf(lanes_max<T>(top), m);
    z *= rescale(m, top, c);
    m = top;
    const Base b = uniform<T>(base_of(m, c));
    z += power(single, b);
    keep_packed(r);
#pragma unroll
    for (int i = 0; i < C; ++i) z += (double)piece_sum<E>(r[i], b);
}

// Piece i of the gradient of those from `first` on: by 2^(c (x - m)).
// LATER: parts of the row are going to be written over, so it stays in the L2 for a while.
template <class E, int T, bool LATER = false>
__device__ __forceinline__ void store_piece(global_access::bytes base, int first, int end, int i, const u32x4 &r, float by, const Base &b)
{
    typedef Piece<E> P;
    typedef __attribute__((address_space(1))) typename P::raw *place;
    const int p = first + i * T + tid<T>();
    if (p < end) {
        float v[P::N];
        P::unpack(r, v);
#pragma unroll
        for (int j = 0; j < P::N; ++j) v[j] = by * power_alone(v[j], b);
        if (LATER) *(place)(base + (uint32_t)p * 16u) = P::pack(v);
        else __builtin_nontemporal_store((typename P::raw)P::pack(v), (place)(base + (uint32_t)p * 16u));
    }
}

// Zeros into pieces first ... end - 1 of a row, and with the first ones into the single elements.
template <class E, int T, bool NT = false>
__device__ __forceinline__ void zero_pieces(const Rows &R, int64_t r, int first, int end)
{
    if (!R.dx) return;
    E *dx = (E *)R.dx + r * R.ld_grad;
    const RowOf<E, T> row(dx, R.vocab);
    const global_access::bytes base = base_address<T>(dx + row.before);
    end = min(end, row.pieces);
    for (int p = first + tid<T>(); p < end; p += T) {
        __attribute__((address_space(1))) u32x4 *at = (__attribute__((address_space(1))) u32x4 *)(base + (uint32_t)p * 16u);
        if (NT) __builtin_nontemporal_store((u32x4)(0u), at);
        else *at = (u32x4)(0u);
    }
    if (first == 0 && row.has_single()) dx[row.single_column()] = narrow<E>(0.f);
}
template <class E, int T>
__device__ __forceinline__ void zero_row(const Rows &R, int64_t r) { zero_pieces<E, T>(R, r, 0, INT32_MAX); }

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
    __device__ __forceinline__ MaxSum stats(const Factor &c, MaxSum *lds, const uint8_t *left_out = nullptr)
    {
        float m = -INFINITY;
        double z = 0.;
        if (LEAVE) {
            const int bit = row.single_column() - row.before + Piece<E>::N;
            if (row.has_single() && (left_out[bit >> 3] >> (bit & 7) & 1)) single = -INFINITY;
        }
        add_pieces<LEAVE>(row, 0, row.pieces, r, single, left_out, c, m, z);
        if constexpr (S > 0)
            for (int first = REST; first < row.pieces; first += T * S) {
                u32x4 v[S];
                row.template load<S, false>(first, v);
                add_pieces<LEAVE>(row, first, row.pieces, v, -INFINITY, left_out, c, m, z);
            }
        return row_merge<T>(MaxSum{m, (float)lanes_sum<T>(z)}, c, lds);
    }
    // dx_v = by 2^(c (x - m)), and coef more at column y (none if negative)
    template <bool LATER = false>
    __device__ __forceinline__ void gradient(E *dx, float by, const Base &base, int y, float xy, float coef)
    {
        const Base b = uniform<T>(base);
        by = uniform<T>(by);
        const global_access::bytes out = base_address<T>(dx + row.before);
        if constexpr (S > 0)
            if (row.pieces > REST)
                for (int first = REST + (row.pieces - 1 - REST) / (T * S) * (T * S); first >= REST; first -= T * S) {
                    u32x4 v[S];
                    row.template load<S, true>(first, v);
#pragma unroll
                    for (int i = 0; i < S; ++i) store_piece<E, T, LATER>(out, first, row.pieces, i, v[i], by, b);
                }
        keep_packed(r);
#pragma unroll
        for (int i = 0; i < C; ++i) store_piece<E, T, LATER>(out, 0, row.pieces, i, r[i], by, b);
        if (row.has_single()) dx[row.single_column()] = narrow<E>(by * power_alone(single, b));
        // by the thread that wrote the column before
        if (y >= 0 && tid<T>() == row.owner(y)) dx[y] = narrow<E>(by * power_alone(xy, b) + coef);
    }
};

}  // namespace loss
