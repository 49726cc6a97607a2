// Layer norm with every worker's own weights, its backward pass, and rows kept in 8 bits (dbw_layers.h).
#pragma once

#include "layer_rows.h"

namespace layer {

struct Norm {
    const void *x;
    const uint8_t *mask;
    const float *params;
    int64_t ld, ld_out, ld_params, weight_at, bias_at;
    int64_t rows;                                         // of all workers
    int per_worker, width, workers;
    int strips;                                           // workgroups of a worker
    float eps;
    void *y;
    float *stats;
    Kept kept;                                            // codes null: not wanted
};

// What the first of 16 lanes has.
__device__ __forceinline__ float of_lane_0(float v) { return loss::shifted<0x150, 0xf>(v, 0.f); }

// Sums of K numbers over a row's T threads, the same in all of them (16 lanes add in as many orders: the first one's).  lds: T / 64 times K floats of the row's
// that nothing else uses until the next barrier but one.
template <int T, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], float (*lds)[K])
{
#pragma unroll
    for (int k = 0; k < K; ++k) {
        v[k] = loss::lanes_sum<T>(v[k]);
        if (T == 16) v[k] = of_lane_0(v[k]);
    }
    if (T <= 64) return;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int k = 0; k < K; ++k) lds[(threadIdx.x & (T - 1)) >> 6][k] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        v[k] = lds[0][k];
#pragma unroll
        for (int w = 1; w < T / 64; ++w) v[k] += lds[w][k];
    }
}

// Which of a group's next rows take part, looked up a turn before their loads, which would wait for it otherwise.
template <int R, int SLOTS>
struct Ahead {
    const uint8_t *mask;                                  // of the group's first row
    int64_t end;
    uint8_t rows[R];
    __device__ __forceinline__ Ahead(const uint8_t *all, int64_t first, int64_t rows_left) : mask(all ? all + first : nullptr), end(rows_left) {}
    __device__ __forceinline__ void look(int64_t at)
    {
#pragma unroll
        for (int q = 0; q < R; ++q) {
            rows[q] = 1;
            if (mask && at + q * SLOTS < end) rows[q] = ((const __attribute__((address_space(1))) uint8_t *)(uint64_t)mask)[at + q * SLOTS];
        }
    }
    __device__ __forceinline__ bool on(int64_t at, int q) const { return at + q * SLOTS < end && rows[q]; }
};

// The row's first number, which its mean counts from: of lane 0 where a row is a wave's or 16 lanes', or as it was loaded.
template <class E, int T>
__device__ __forceinline__ float first_of(float lane_0, float loaded)
{
    if (T == 16) return of_lane_0(lane_0);
    if (T == 64) return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(lane_0)));
    return loaded;
}

// A piece's numbers added up in pairs: of equal numbers exactly.
template <int N>
__device__ __forceinline__ float piece_sum(const float (&v)[N])
{
    if constexpr (N == 4) return (v[0] + v[1]) + (v[2] + v[3]);
    else return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
}

// Piece i of C, all of which but the last are whole: in two steps as load_raw and settled.
template <class E, bool WIDE, int C>
__device__ __forceinline__ u32x4 load_turn(const E *row, int i, int c, int width)
{
    typedef const __attribute__((address_space(1))) typename Piece<E>::raw *place;
    if (i < C - 1) return *(place)(uint64_t)(row + c);
    return load_raw<E, WIDE>(row, c, width);
}
template <class E, bool WIDE, int C>
__device__ __forceinline__ u32x4 settled_turn(const u32x4 &w, int i, int c, int width)
{
    return i < C - 1 ? w : settled<E, WIDE>(w, c, width);
}

// A row in the registers of T threads, C pieces each.  A workgroup has SLOTS such groups of threads and walks over a strip of a worker's rows, a row a
// group at a time, with the weights in registers and the next row on its way.  The mean comes first, then the
// sums of the differences from it and of their squares: the first of these is what the rounding of the mean left, which counts where a row's mean is
// large beside its spread.  Means are sums of shares x / D and not quotients of sums: a product that a difference follows may be contracted with it for
// some of a row's pieces and not for others, and differences from two centres, half a step of the mean apart, have no such rest.
//
// The mean counts from the row's first number x_0: mu = x_0 + mean of (x - x_0), a piece's N numbers added up before N x_0 goes off them.  Equal numbers add up
// exactly in pairs, so that a row of them has differences of zero, and the mean of other rows is off by a step or two of mu and by what is small beside
// the spread.  Sums of x over a row leave many steps of mu, and where the spread is less, the squares' mean without the rest's square is rounding, of either
// sign: rho of NaN, or of a spread that is not there.  As it is, the two differ: numbers that are not all equal lie steps of their own apart.
//
// Memory bounds it: 8 x 2048 x 2048 bf16 23.0 us, keeping 8 bits too 32.0 (134 and 168 MB, 5.8 and 5.2 TB/s), one row of 4096 3.3 us.
template <class E, int T, int C, int SLOTS>
__global__ __launch_bounds__(T * SLOTS, T == 64 ? 3 : 1) void norm_kernel(Norm P)
{
    constexpr int N = Piece<E>::N, WAVES = (T + 63) / 64;
    constexpr bool WIDE = T * C > 16;
    __shared__ float totals[SLOTS][WAVES][1], sums[SLOTS][WAVES][2];
    const int64_t group = group_number();
    if (group >= (int64_t)P.workers * P.strips) return;
    const Strip strip = strip_of((uint32_t)group, P.strips, SLOTS, P.per_worker);
    const int t = loss::tid<T>(), slot = slot_of<T>();
    const int64_t base = (int64_t)strip.worker * P.per_worker;
    const float inverse = 1.f / (float)P.width;
    u32x4 next[C];
    typename Bits<E>::type next_first;
    bool next_on;
    Ahead<1, SLOTS> ahead(P.mask, base + slot, strip.end - slot);
    ahead.look(strip.first);
    const auto load = [&](int64_t at) {
        const int64_t r = base + at + slot;
        next_on = ahead.on(at, 0);
        if (next_on) {
            if (T > 64) next_first = *(const __attribute__((address_space(1))) typename Bits<E>::type *)(uint64_t)((const E *)P.x + r * P.ld);
#pragma unroll
            for (int i = 0; i < C; ++i) next[i] = load_turn<E, WIDE, C>((const E *)P.x + r * P.ld, i, (i * T + t) * N, P.width);
        }
        ahead.look(at + strip.stride);
    };
    load(strip.first);
    float w[C][N], b[C][N];
    const float *const params = P.params + strip.worker * P.ld_params;
#pragma unroll
    for (int i = 0; i < C; ++i) {
        for (int j = 0; j < N; ++j) w[i][j] = 1.f, b[i][j] = 0.f;
        if (P.weight_at >= 0) load_floats<N, WIDE>(params + P.weight_at, (i * T + t) * N, P.width, w[i]);
        if (P.bias_at >= 0) load_floats<N, WIDE>(params + P.bias_at, (i * T + t) * N, P.width, b[i]);
    }
    // Rows are written a turn later, in front of the loads of the rows behind the next: waiting for loads is waiting for all that was asked for before
    // them, and nothing then waits for stores that have just begun.  (Backwards from 8 bits with a mask, 8 x 2048 x 2048 bf16: 48 us -> 37.)
    u32x4 out[C];
    int64_t last = -1;
    const auto store = [&](int64_t at) {
        const int64_t row = at + slot;
        if (row < strip.end)
#pragma unroll
            for (int i = 0; i < C; ++i) store_piece<E>((E *)P.y + (base + row) * P.ld_out, (i * T + t) * N, P.width, out[i]);
    };
    for (int64_t at = strip.first; at < strip.end; at += strip.stride) {
        const bool on = next_on;
        const int64_t row = at + slot;
        float v[C][N], first, total[1] = {0.f}, s[2] = {0.f, 0.f};
        u32x4 raw[C];
#pragma unroll
        for (int i = 0; i < C; ++i) raw[i] = on ? settled_turn<E, WIDE, C>(next[i], i, (i * T + t) * N, P.width) : (u32x4)0u;
        if (last >= 0) store(last);
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int c = (i * T + t) * N;
            if (P.kept.codes && row < strip.end && c < (int)P.kept.stride) keep_piece<E>(P.kept, base + row, c, raw[i]);
            Piece<E>::unpack(raw[i], v[i]);
            if (i == 0) first = first_of<E, T>(v[0][0], on ? loss::widen(__builtin_bit_cast(E, next_first)) : 0.f);
            if (i == C - 1 && c + N > P.width)
#pragma unroll
                for (int j = 0; j < N; ++j) v[i][j] = c + j < P.width ? v[i][j] : first;
            total[0] = fmaf(piece_sum(v[i]) - N * first, inverse, total[0]);
        }
        load(at + strip.stride);
        row_sums<T>(total, totals[slot]);
        const float mean = total[0] + first;
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int c = (i * T + t) * N;
#pragma unroll
            for (int j = 0; j < N; ++j) v[i][j] -= mean;
            if (i == C - 1 && c + N > P.width)
#pragma unroll
                for (int j = 0; j < N; ++j) v[i][j] = c + j < P.width ? v[i][j] : 0.f;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                s[0] = fmaf(v[i][j], inverse, s[0]);
                s[1] = fmaf(v[i][j], v[i][j], s[1]);
            }
        }
        row_sums<T>(s, sums[slot]);
        const float rest = s[0];
        const float rstd = 1.f / sqrtf(fmaf(-rest, rest, s[1] * inverse) + P.eps);
        if (P.stats && t == 0 && row < strip.end)
            *(__attribute__((address_space(1))) f32x2 *)(uint64_t)(P.stats + 2 * (base + row)) = on ? (f32x2){mean + rest, rstd} : (f32x2)0.f;
        const float less = -rest * rstd;
#pragma unroll
        for (int i = 0; i < C; ++i) {
#pragma unroll
            for (int j = 0; j < N; ++j) v[i][j] = fmaf(fmaf(v[i][j], rstd, less), w[i][j], b[i][j]);
            const u32x4 packed = Piece<E>::pack(v[i]);
            out[i] = on ? packed : (u32x4)0u;
        }
        last = at;
    }
    if (last >= 0) store(last);
}

// Rows that registers do not hold: read three times, by one workgroup.
template <class E, int T>
__global__ __launch_bounds__(T) void norm_long_kernel(Norm P)
{
    constexpr int N = Piece<E>::N;
    __shared__ float totals[T / 64][1], sums[T / 64][2];
    const int64_t r = group_number();
    const int t = threadIdx.x;
    if (r >= P.rows) return;
    const bool on = !P.mask || P.mask[r];
    const E *const x = (const E *)P.x + r * P.ld;
    E *const y = (E *)P.y + r * P.ld_out;
    const float inverse = 1.f / (float)P.width;
    u32x4 next = on ? load_raw<E, true>(x, t * N, P.width) : (u32x4)0u;
    const float first = on ? loss::widen(*x) : 0.f;       // (asked for beside the first pieces)
    float v[N], total[1] = {0.f};
    if (on)
        for (int c = t * N; c < P.width; c += T * N) {
            Piece<E>::unpack(settled<E, true>(next, c, P.width), v);
            next = load_raw<E, true>(x, c + T * N, P.width);
            if (c + N > P.width)
                for (int j = 0; j < N; ++j) v[j] = c + j < P.width ? v[j] : first;
            total[0] = fmaf(piece_sum(v) - N * first, inverse, total[0]);
        }
    row_sums<T>(total, totals);
    const float mean = first + total[0];
    float s[2] = {0.f, 0.f};
    if (on)
        for (int c = t * N; c < P.width; c += T * N) {
            Piece<E>::unpack(load_piece<E, true>(x, c, P.width), v);
            float part[2] = {0.f, 0.f};
            for (int j = 0; j < N; ++j) {
                const float d = c + j < P.width ? v[j] - mean : 0.f;
                part[0] = fmaf(d, inverse, part[0]);
                part[1] = fmaf(d, d, part[1]);
            }
            s[0] += part[0];
            s[1] += part[1];
        }
    row_sums<T>(s, sums);
    const float rest = s[0];
    const float rstd = 1.f / sqrtf(fmaf(-rest, rest, s[1] * inverse) + P.eps);
    if (P.stats && t == 0) {
        P.stats[2 * r] = on ? mean + rest : 0.f;
        P.stats[2 * r + 1] = on ? rstd : 0.f;
    }
    const float *const params = P.params + r / P.per_worker * P.ld_params;
    for (int c = t * N; c < (int)padded(P.width); c += T * N) {
        const u32x4 raw = on ? load_piece<E, true>(x, c, P.width) : (u32x4)0u;
        if (P.kept.codes) keep_piece<E>(P.kept, r, c, raw);
        Piece<E>::unpack(raw, v);
        if (c >= P.width) continue;
        float w[N], b[N];
        for (int j = 0; j < N; ++j) w[j] = 1.f, b[j] = 0.f;
        if (P.weight_at >= 0) load_floats<N, true>(params + P.weight_at, c, P.width, w);
        if (P.bias_at >= 0) load_floats<N, true>(params + P.bias_at, c, P.width, b);
        for (int j = 0; j < N; ++j) v[j] = on ? fmaf((v[j] - mean - rest) * rstd, w[j], b[j]) : 0.f;
        store_piece<E>(y, c, P.width, Piece<E>::pack(v));
    }
}

// ---------------------------------------------------------------- backward

struct NormGrad {
    const void *dy, *x;                                   // x null: from what was kept
    Kept kept;
    const uint8_t *mask;
    const float *stats, *params;
    int64_t ld, ld_out, ld_params, ld_grads, weight_at, bias_at;
    int64_t rows;
    int per_worker, width, workers;
    int strips;                                           // workgroups of a worker
    void *dx;
    float *grads;                                         // null: not wanted
    float *parts;                                         // [worker][strip][2][part_ld]: dw and db of the strips; null: one strip, straight into grads
    int64_t part_ld;
    f32x2 *means;                                         // of long rows: mean of g and of g u
};

// Piece i of C of the input as it is read, and its numbers.
template <class E, bool KEPT>
struct Input {
    u32x4 raw;
    template <bool WIDE, int C>
    __device__ __forceinline__ void load(const NormGrad &P, int64_t r, int i, int c) { raw = load_turn<E, WIDE, C>((const E *)P.x + r * P.ld, i, c, P.width); }
    template <bool WIDE, int C>
    __device__ __forceinline__ void unpack(bool on, int i, int c, int width, float (&v)[Piece<E>::N]) const
    {
        Piece<E>::unpack(on ? settled_turn<E, WIDE, C>(raw, i, c, width) : (u32x4)0u, v);
    }
};
template <class E>
struct Input<E, true> {
    Codes<Piece<E>::N> raw;
    template <bool, int C>
    __device__ __forceinline__ void load(const NormGrad &P, int64_t r, int i, int c)
    {
        raw = load_codes<Piece<E>::N>(P.kept, r, i < C - 1 || c < P.width ? c : 0);
    }
    template <bool, int>
    __device__ __forceinline__ void unpack(bool on, int, int, int, float (&v)[Piece<E>::N]) const
    {
        Codes<Piece<E>::N> codes = raw;
        for (uint32_t &w : codes.w) w = on ? w : 0u;
        codes.exponent = on ? codes.exponent : 127u;
        unpack_codes<Piece<E>::N>(codes, v);
    }
};
template <class E, bool KEPT>
__device__ __forceinline__ void input_piece(const NormGrad &P, int64_t r, int c, float (&v)[Piece<E>::N])
{
    Input<E, KEPT> in;
    in.template load<true, 1>(P, r, 0, c);
    in.template unpack<true, 1>(true, 0, c, P.width, v);
}
// Where a workgroup's share of dw (which = 0) or db goes, or null.
__device__ __forceinline__ float *part_of(const NormGrad &P, int worker, int strip, int which)
{
    const int64_t at = which ? P.bias_at : P.weight_at;
    if (!P.grads || at < 0) return nullptr;
    if (P.parts) return P.parts + (((int64_t)worker * P.strips + strip) * 2 + which) * P.part_ld;
    return P.grads + worker * P.ld_grads + at;
}

// As norm_kernel, R rows a group at a time, whose sums share their barriers; every thread's columns are the same in all rows, so that it sums dw and db in
// registers.  Rows that take no part are zeros with a mean and a scale of zero.  Memory bounds long batches (8 x 8192 x 2048 bf16 from 8 bits 133 us,
// 5.0 TB/s); shorter ones pay some 8 us for the first rows' way and for adding up (8 x 2048 x 2048 37 us).
template <class E, int T, int C, int SLOTS, int R, bool KEPT>
__global__ __launch_bounds__(T * SLOTS) void norm_grad_kernel(NormGrad P)
{
    constexpr int N = Piece<E>::N, WAVES = (T + 63) / 64;
    constexpr bool WIDE = T * C > 16;
    __shared__ float sums[2][SLOTS][WAVES][2 * R];
    extern __shared__ float joined[];                     // [SLOTS][C * N][T], one of dw and db after the other
    const int64_t group = group_number();
    if (group >= (int64_t)P.workers * P.strips) return;
    const Strip strip = strip_of((uint32_t)group, P.strips, R * SLOTS, P.per_worker);
    const int t = loss::tid<T>(), slot = slot_of<T>();
    const int64_t base = (int64_t)strip.worker * P.per_worker;
    const float inverse = 1.f / (float)P.width;
    u32x4 next_dy[R][C];
    Input<E, KEPT> next[R][C];
    f32x2 next_stats[R];
    bool next_on[R];
    Ahead<R, SLOTS> ahead(P.mask, base + slot, strip.end - slot);
    ahead.look(strip.first);
    const auto load = [&](int64_t at) {
#pragma unroll
        for (int q = 0; q < R; ++q) {
            const int64_t r = base + at + q * SLOTS + slot;
            next_on[q] = ahead.on(at, q);
            next_stats[q] = (f32x2)0.f;
            if (next_on[q]) {
                next_stats[q] = *(const __attribute__((address_space(1))) f32x2 *)(uint64_t)(P.stats + 2 * r);
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    next_dy[q][i] = load_turn<E, WIDE, C>((const E *)P.dy + r * P.ld_out, i, (i * T + t) * N, P.width);
                    next[q][i].template load<WIDE, C>(P, r, i, (i * T + t) * N);
                }
            }
        }
        ahead.look(at + strip.stride);
    };
    load(strip.first);
    float w[C][N], dw[C][N], db[C][N];
#pragma unroll
    for (int i = 0; i < C; ++i) {
        for (int j = 0; j < N; ++j) w[i][j] = 1.f, dw[i][j] = db[i][j] = 0.f;
        if (P.weight_at >= 0) load_floats<N, WIDE>(P.params + strip.worker * P.ld_params + P.weight_at, (i * T + t) * N, P.width, w[i]);
    }
    u32x4 out[R][C];
    int64_t last = -1;
    const auto store = [&](int64_t at) {
#pragma unroll
        for (int q = 0; q < R; ++q) {
            const int64_t row = at + q * SLOTS + slot;
            if (row < strip.end)
#pragma unroll
                for (int i = 0; i < C; ++i) store_piece<E>((E *)P.dx + (base + row) * P.ld, (i * T + t) * N, P.width, out[q][i]);
        }
    };
    int turn = 0;
    for (int64_t at = strip.first; at < strip.end; at += strip.stride, turn ^= 1) {
        float g[R][C][N], u[R][C][N], s[2 * R], rstd[R];
#pragma unroll
        for (int q = 0; q < R; ++q) {
            const float mean = next_stats[q][0];
            rstd[q] = next_stats[q][1];
            s[2 * q] = s[2 * q + 1] = 0.f;
#pragma unroll
            for (int i = 0; i < C; ++i) {
                const int c = (i * T + t) * N;
                Piece<E>::unpack(next_on[q] ? settled_turn<E, WIDE, C>(next_dy[q][i], i, c, P.width) : (u32x4)0u, g[q][i]);
                next[q][i].template unpack<WIDE, C>(next_on[q], i, c, P.width, u[q][i]);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    u[q][i][j] = (u[q][i][j] - mean) * rstd[q];
                    // Of columns beyond the width dy is zero, and with it all sums, but (0 - mu) rho may be infinite.  (Without a branch: in one, of rows where that
                    // is so or of pieces that are not whole, 16 x 1779 x 2983 from 8 bits 97 us, so 92.4.)
                    if (i == C - 1) u[q][i][j] = c + j < P.width ? u[q][i][j] : 0.f;
                }
            }
        }
        if (last >= 0) store(last);
        load(at + strip.stride);
#pragma unroll
        for (int q = 0; q < R; ++q)
#pragma unroll
            for (int i = 0; i < C; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    dw[i][j] = fmaf(g[q][i][j], u[q][i][j], dw[i][j]);
                    db[i][j] += g[q][i][j];
                    g[q][i][j] *= w[i][j];
                    s[2 * q] += g[q][i][j];
                    s[2 * q + 1] = fmaf(g[q][i][j], u[q][i][j], s[2 * q + 1]);
                }
        row_sums<T>(s, sums[turn][slot]);
#pragma unroll
        for (int q = 0; q < R; ++q) {
            const float mean_g = s[2 * q] * inverse, mean_gu = s[2 * q + 1] * inverse;
#pragma unroll
            for (int i = 0; i < C; ++i) {
#pragma unroll
                for (int j = 0; j < N; ++j) g[q][i][j] = rstd[q] * fmaf(-mean_gu, u[q][i][j], g[q][i][j] - mean_g);
                out[q][i] = Piece<E>::pack(g[q][i]);
            }
        }
        last = at;
    }
    if (last >= 0) store(last);
    // the groups' sums, piece i of all of them by group i mod SLOTS
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float *const to = part_of(P, strip.worker, strip.number, which);
        if (!to) continue;
        float (&mine)[C][N] = which ? db : dw;
        if (SLOTS > 1) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < C; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j) joined[((slot * C + i) * N + j) * T + t] = mine[i][j];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < C; ++i)
                if (i % SLOTS == slot)
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        mine[i][j] = joined[(i * N + j) * T + t];
                        for (int q = 1; q < SLOTS; ++q) mine[i][j] += joined[((q * C + i) * N + j) * T + t];
                    }
        }
#pragma unroll
        for (int i = 0; i < C; ++i)
            if (i % SLOTS == slot && (i * T + t) * N < P.width) store_floats<N>(to, (i * T + t) * N, P.width, mine[i]);
    }
}

// Long rows, first their two means ...
template <class E, int T, bool KEPT>
__global__ __launch_bounds__(T) void norm_means_kernel(NormGrad P)
{
    constexpr int N = Piece<E>::N;
    __shared__ float sums[T / 64][2];
    const int64_t r = group_number();
    if (r >= P.rows || (P.mask && !P.mask[r])) return;
    const int worker = (int)(r / P.per_worker);
    const float mean = P.stats[2 * r], rstd = P.stats[2 * r + 1];
    float s[2] = {0.f, 0.f};
    for (int c = threadIdx.x * N; c < P.width; c += T * N) {
        float g[N], u[N], w[N];
        for (int j = 0; j < N; ++j) w[j] = 1.f;
        if (P.weight_at >= 0) load_floats<N, true>(P.params + worker * P.ld_params + P.weight_at, c, P.width, w);
        Piece<E>::unpack(load_piece<E, true>((const E *)P.dy + r * P.ld_out, c, P.width), g);
        input_piece<E, KEPT>(P, r, c, u);
        float part[2] = {0.f, 0.f};
        for (int j = 0; j < N; ++j) {
            const float d = g[j] * w[j];
            part[0] += d;
            part[1] = c + j < P.width ? fmaf(d, (u[j] - mean) * rstd, part[1]) : part[1];
        }
        s[0] += part[0];
        s[1] += part[1];
    }
    row_sums<T>(s, sums);
    const float inverse = 1.f / (float)P.width;
    if (threadIdx.x == 0) P.means[r] = (f32x2){s[0] * inverse, s[1] * inverse};
}
// ... then, a slice of the columns at a time, the rest.
template <class E, int T, bool KEPT>
__global__ __launch_bounds__(T) void norm_grad_long_kernel(NormGrad P, int slices)
{
    constexpr int N = Piece<E>::N;
    const int64_t group = group_number();
    if (group >= (int64_t)P.workers * P.strips * slices) return;
    const int64_t which_strip = group / slices;
    const int worker = (int)(which_strip / P.strips), strip = (int)(which_strip % P.strips);
    const int c = ((int)(group % slices) * T + threadIdx.x) * N;
    if (c >= P.width) return;
    float w[N], dw[N], db[N];
    for (int j = 0; j < N; ++j) w[j] = 1.f, dw[j] = db[j] = 0.f;
    if (P.weight_at >= 0) load_floats<N, true>(P.params + worker * P.ld_params + P.weight_at, c, P.width, w);
    for (int64_t at = strip; at < P.per_worker; at += P.strips) {
        const int64_t r = (int64_t)worker * P.per_worker + at;
        float g[N], u[N];
        for (int j = 0; j < N; ++j) g[j] = 0.f;
        if (!P.mask || P.mask[r]) {
            const float mean = P.stats[2 * r], rstd = P.stats[2 * r + 1];
            const f32x2 s = P.means[r];
            Piece<E>::unpack(load_piece<E, true>((const E *)P.dy + r * P.ld_out, c, P.width), g);
            input_piece<E, KEPT>(P, r, c, u);
            for (int j = 0; j < N; ++j) {
                u[j] = (u[j] - mean) * rstd;
                dw[j] = fmaf(g[j], u[j], dw[j]);
                db[j] += g[j];
                g[j] = rstd * (g[j] * w[j] - s[0] - u[j] * s[1]);
            }
        }
        store_piece<E>((E *)P.dx + r * P.ld, c, P.width, Piece<E>::pack(g));
    }
    for (int which = 0; which < 2; ++which) {
        float *const to = part_of(P, worker, strip, which);
        if (to) store_floats<N>(to, c, P.width, which ? db : dw);
    }
}
// The strips' shares: 64 columns a workgroup, four a thread, its 16 rows of threads every sixteenth strip, eight loads on their way at a time.  One worker
// of 4096 x 2048 in 512 strips with 32 columns a workgroup, 8 rows of threads and one load after the other: 25 us.
constexpr int SUM_COLUMNS = 64, SUM_ROWS = 16;
__global__ __launch_bounds__(SUM_COLUMNS / 4 * SUM_ROWS) void norm_sum_kernel(NormGrad P, int slices)
{
    __shared__ f32x4 lds[SUM_ROWS][SUM_COLUMNS / 4];
    const int64_t group = group_number();
    const int which = (int)(group % 2);
    const int slice = (int)(group / 2 % slices);
    const int64_t worker = group / 2 / slices;
    const int64_t at = which ? P.bias_at : P.weight_at;
    if (worker >= P.workers || at < 0) return;
    const int q = threadIdx.x / (SUM_COLUMNS / 4), k = threadIdx.x % (SUM_COLUMNS / 4), c = slice * SUM_COLUMNS + 4 * k;
    f32x4 v = (f32x4)0.f;
    if (c < P.width) {
        const float *const part = P.parts + (worker * P.strips * 2 + which) * P.part_ld + c;
        const int64_t stride = 2 * P.part_ld;
        for (int s = q; s < P.strips; s += 8 * SUM_ROWS) {
            f32x4 w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = s + i * SUM_ROWS < P.strips ? *(const f32x4 *)(part + (s + i * SUM_ROWS) * stride) : (f32x4)0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) v += w[i];
        }
    }
    lds[q][k] = v;
    __syncthreads();
    if (q == 0 && c < P.width) {
        for (int s = 1; s < SUM_ROWS; ++s) v += lds[s][k];
        float to[4] = {v[0], v[1], v[2], v[3]};
        store_floats<4>(P.grads + worker * P.ld_grads + at, c, P.width, to);
    }
}
// Workers without rows.
__global__ __launch_bounds__(256) void norm_zero_kernel(NormGrad P, int slices)
{
    const int64_t group = group_number();
    const int c = (int)(group % slices) * 256 + threadIdx.x;
    const int64_t worker = group / slices;
    if (worker >= P.workers || c >= P.width) return;
    if (P.weight_at >= 0) P.grads[worker * P.ld_grads + P.weight_at + c] = 0.f;
    if (P.bias_at >= 0) P.grads[worker * P.ld_grads + P.bias_at + c] = 0.f;
}

// ---------------------------------------------------------------- checkpoints

struct Store {
    const void *x;
    const uint8_t *mask;
    void *out;
    int64_t ld, rows;
    int width;
    Kept kept;
};
// Memory bounds both: 4 x 4096 x 4096 bf16 36.7 and 29.2 us (203 MB each, 5.5 and 7.0 TB/s, the codes still in the last-level cache for the second).
//
// A workgroup has STORE_PIECES x STORE_THREADS pieces that follow one another, a thread every STORE_THREADS-th; a row is a multiple of the pieces of a
// block.  4 x 4096 x 4096 bf16 stored and loaded with one, two and four pieces a thread 73, 67.6 and 71 us.
constexpr int STORE_THREADS = 256, STORE_PIECES = 2;
struct Spot {
    int64_t r;
    int c;
};
// Where a workgroup's pieces lie: the first one's row and place in it, and, to divide by, one over a row's pieces (at most 2^18, so that what is divided
// is below 2^19 and a quotient in fp32 is off by one at most).
template <int N>
struct Pieces {
    int64_t row;
    int in_row, pieces;
    float inverse;
    __device__ __forceinline__ Pieces(const Store &P)
    {
        pieces = (int)(P.kept.stride / N);
        const int64_t first = group_number() * (STORE_THREADS * STORE_PIECES);
        row = first / pieces;
        in_row = (int)(first % pieces);
        inverse = 1.f / (float)pieces;
    }
    __device__ __forceinline__ Spot spot(int i) const
    {
        const int at = in_row + i * STORE_THREADS + (int)threadIdx.x;
        int q = (int)((float)at * inverse), rest = at - q * pieces;
        if (rest < 0) --q, rest += pieces;
        if (rest >= pieces) ++q, rest -= pieces;
        return Spot{row + q, rest * N};
    }
};
template <class E>
__global__ __launch_bounds__(STORE_THREADS) void store_kernel(Store P)
{
    const Pieces<Piece<E>::N> pieces(P);
    u32x4 w[STORE_PIECES];
#pragma unroll
    for (int i = 0; i < STORE_PIECES; ++i) {
        const Spot s = pieces.spot(i);
        w[i] = (u32x4)0u;
        if (s.r < P.rows && (!P.mask || P.mask[s.r])) w[i] = load_piece<E>((const E *)P.x + s.r * P.ld, s.c, P.width);
    }
#pragma unroll
    for (int i = 0; i < STORE_PIECES; ++i) {
        const Spot s = pieces.spot(i);
        if (s.r < P.rows) keep_piece<E>(P.kept, s.r, s.c, w[i]);
    }
}
template <class E>
__global__ __launch_bounds__(STORE_THREADS) void load_kernel(Store P)
{
    constexpr int N = Piece<E>::N;
    const Pieces<N> pieces(P);
    Codes<N> w[STORE_PIECES];
#pragma unroll
    for (int i = 0; i < STORE_PIECES; ++i) {
        const Spot s = pieces.spot(i);
        if (s.r < P.rows) w[i] = load_codes<N>(P.kept, s.r, s.c);
    }
#pragma unroll
    for (int i = 0; i < STORE_PIECES; ++i) {
        const Spot s = pieces.spot(i);
        float v[N];
        unpack_codes<N>(w[i], v);
        if (s.r < P.rows) store_piece<E>((E *)P.out + s.r * P.ld, s.c, P.width, Piece<E>::pack(v));
    }
}

}  // namespace layer
