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
    int strips, strip_rows;                               // of a worker
    float eps;
    void *y;
    float *stats;
    Kept kept;                                            // codes null: not wanted
};

// Sums of two numbers over a row's T threads.  lds: 2 T / 64 floats of the row's that nothing else uses until the next barrier.
template <int T>
__device__ __forceinline__ f32x2 row_sums(f32x2 v, f32x2 *lds)
{
    v = (f32x2){loss::lanes_sum<T>(v[0]), loss::lanes_sum<T>(v[1])};
    if (T <= 64) return v;
    if ((threadIdx.x & 63) == 0) lds[(threadIdx.x & (T - 1)) >> 6] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < T / 64; ++w) v += lds[w];
    return v;
}

// A row in the registers of T threads, C pieces each; a workgroup walks over a strip of a worker's rows, ROWS at a time, with the weights in registers and
// the next row on its way.  The mean comes first, then the sums of the differences from it and of their squares: the first of these is what the
// rounding of the mean left, which counts where a row's mean is large beside its spread.
template <class E, int T, int C, int ROWS>
__global__ __launch_bounds__(T * ROWS) void norm_kernel(Norm P)
{
    constexpr int N = Piece<E>::N;
    constexpr bool WIDE = T * C > 16;
    __shared__ f32x2 sums[2][ROWS][(T + 63) / 64];
    const int64_t group = group_number();
    if (group >= (int64_t)P.workers * P.strips) return;
    const Strip strip = strip_of((uint32_t)group, P.strips, P.strip_rows, P.per_worker);
    const int t = loss::tid<T>(), slot = slot_of<T>();
    const int64_t base = (int64_t)strip.worker * P.per_worker;
    const float inverse = 1.f / (float)P.width;
    u32x4 next[C];
    bool next_on = false;
    const auto load = [&](int at) {
        const int64_t r = base + at + slot;
        next_on = at + slot < strip.end && (!P.mask || P.mask[r]);
        if (next_on)
#pragma unroll
            for (int i = 0; i < C; ++i) next[i] = load_raw<E, WIDE>((const E *)P.x + r * P.ld, (i * T + t) * N, P.width);
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
    for (int at = strip.first; at < strip.end; at += ROWS) {
        const bool on = next_on, there = at + slot < strip.end;
        const int64_t r = base + at + slot;
        float v[C][N];
        f32x2 s = (f32x2)0.f;
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const u32x4 raw = on ? settled<E, WIDE>(next[i], (i * T + t) * N, P.width) : (u32x4)0u;
            if (P.kept.codes && there && (i * T + t) * N < (int)P.kept.stride) keep_piece<E>(P.kept, r, (i * T + t) * N, raw);
            Piece<E>::unpack(raw, v[i]);
        }
        load(at + ROWS);
        if (!on) {                                        // (T > 64: a row is the workgroup's)
            if (there) {
                if (P.stats && t == 0) *(__attribute__((address_space(1))) f32x2 *)(uint64_t)(P.stats + 2 * r) = s;
#pragma unroll
                for (int i = 0; i < C; ++i) store_piece<E>((E *)P.y + r * P.ld_out, (i * T + t) * N, P.width, (u32x4)0u);
            }
            continue;
        }
#pragma unroll
        for (int i = 0; i < C; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) s[j & 1] += v[i][j];
        const float mean = row_sums<T>((f32x2){s[0] + s[1], 0.f}, sums[0][slot])[0] * inverse;
        s = (f32x2)0.f;
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int c = (i * T + t) * N;
#pragma unroll
            for (int j = 0; j < N; ++j) v[i][j] -= mean;
            if (c + N > P.width)
#pragma unroll
                for (int j = 0; j < N; ++j) v[i][j] = c + j < P.width ? v[i][j] : 0.f;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                s[0] += v[i][j];
                s[1] = fmaf(v[i][j], v[i][j], s[1]);
            }
        }
        s = row_sums<T>(s, sums[1][slot]);
        const float rest = s[0] * inverse;
        const float rstd = 1.f / sqrtf(fmaf(-rest, rest, s[1] * inverse) + P.eps);
        if (P.stats && t == 0) *(__attribute__((address_space(1))) f32x2 *)(uint64_t)(P.stats + 2 * r) = (f32x2){mean + rest, rstd};
        const float less = -rest * rstd;
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int c = (i * T + t) * N;
#pragma unroll
            for (int j = 0; j < N; ++j) v[i][j] = fmaf(fmaf(v[i][j], rstd, less), w[i][j], b[i][j]);
            store_piece<E>((E *)P.y + r * P.ld_out, c, P.width, Piece<E>::pack(v[i]));
        }
    }
}

// Rows that registers do not hold: read three times, by one workgroup.
template <class E, int T>
__global__ __launch_bounds__(T) void norm_long_kernel(Norm P)
{
    constexpr int N = Piece<E>::N;
    __shared__ f32x2 sums[2][T / 64];
    const int64_t r = group_number();
    const int t = threadIdx.x;
    if (r >= P.rows) return;
    const bool on = !P.mask || P.mask[r];
    const E *const x = (const E *)P.x + r * P.ld;
    E *const y = (E *)P.y + r * P.ld_out;
    float v[N];
    float total = 0.f;
    if (on)
        for (int c = t * N; c < P.width; c += T * N) {
            Piece<E>::unpack(load_piece<E, true>(x, c, P.width), v);
            float part = 0.f;
            for (int j = 0; j < N; ++j) part += v[j];
            total += part;
        }
    const float inverse = 1.f / (float)P.width;
    const float mean = row_sums<T>((f32x2){total, 0.f}, sums[0])[0] * inverse;
    f32x2 s = (f32x2)0.f;
    if (on)
        for (int c = t * N; c < P.width; c += T * N) {
            Piece<E>::unpack(load_piece<E, true>(x, c, P.width), v);
            f32x2 part = (f32x2)0.f;
            for (int j = 0; j < N; ++j) {
                const float d = c + j < P.width ? v[j] - mean : 0.f;
                part[0] += d;
                part[1] = fmaf(d, d, part[1]);
            }
            s += part;
        }
    s = row_sums<T>(s, sums[1]);
    const float rest = s[0] * inverse;
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
    int strips, strip_rows;                               // a worker's rows are cut into strips, a workgroup each
    void *dx;
    float *grads;                                         // null: not wanted
    float *parts;                                         // [worker][strip][2][part_ld]: dw and db of the strips; null: one strip, straight into grads
    int64_t part_ld;
    f32x2 *means;                                         // of long rows: mean of g and of g u
};

// A piece of the input as it is read, and its numbers.
template <class E, bool KEPT>
struct Input {
    u32x4 raw;
    template <bool WIDE>
    __device__ __forceinline__ void load(const NormGrad &P, int64_t r, int c) { raw = load_raw<E, WIDE>((const E *)P.x + r * P.ld, c, P.width); }
    template <bool WIDE>
    __device__ __forceinline__ void unpack(int c, int width, float (&v)[Piece<E>::N]) const { Piece<E>::unpack(settled<E, WIDE>(raw, c, width), v); }
};
template <class E>
struct Input<E, true> {
    Codes<Piece<E>::N> raw;
    template <bool>
    __device__ __forceinline__ void load(const NormGrad &P, int64_t r, int c) { raw = load_codes<Piece<E>::N>(P.kept, r, c < P.width ? c : 0); }
    template <bool>
    __device__ __forceinline__ void unpack(int, int, float (&v)[Piece<E>::N]) const { unpack_codes<Piece<E>::N>(raw, v); }
};
template <class E, bool KEPT>
__device__ __forceinline__ void input_piece(const NormGrad &P, int64_t r, int c, float (&v)[Piece<E>::N])
{
    Input<E, KEPT> in;
    in.template load<true>(P, r, c);
    in.template unpack<true>(c, P.width, v);
}
// Where a workgroup's share of dw (which = 0) or db goes, or null.
__device__ __forceinline__ float *part_of(const NormGrad &P, int worker, int strip, int which)
{
    const int64_t at = which ? P.bias_at : P.weight_at;
    if (!P.grads || at < 0) return nullptr;
    if (P.parts) return P.parts + (((int64_t)worker * P.strips + strip) * 2 + which) * P.part_ld;
    return P.grads + worker * P.ld_grads + at;
}

// A workgroup walks over its strip, T threads a row and ROWS rows at a time; every thread's columns are the same in all rows, so that it sums
// dw and db in registers.
template <class E, int T, int C, int ROWS, bool KEPT>
__global__ __launch_bounds__(T * ROWS) void norm_grad_kernel(NormGrad P)
{
    constexpr int N = Piece<E>::N;
    constexpr bool WIDE = T * C > 16;
    __shared__ f32x2 sums[2][ROWS][(T + 63) / 64];
    extern __shared__ float joined[];                     // [ROWS - 1][T][C * N], one of dw and db after the other
    const int64_t group = group_number();
    if (group >= (int64_t)P.workers * P.strips) return;
    const Strip cut = strip_of((uint32_t)group, P.strips, P.strip_rows, P.per_worker);
    const int worker = cut.worker, strip = cut.number;
    const int t = loss::tid<T>(), slot = slot_of<T>();
    const int64_t base = (int64_t)worker * P.per_worker;
    const float inverse = 1.f / (float)P.width;
    u32x4 next_dy[C];
    Input<E, KEPT> next[C];
    f32x2 next_stats = (f32x2)0.f;
    bool next_on = false;
    const auto load = [&](int at) {
        const int64_t r = base + at + slot;
        next_on = at + slot < cut.end && (!P.mask || P.mask[r]);
        if (next_on) {
            next_stats = *(const __attribute__((address_space(1))) f32x2 *)(uint64_t)(P.stats + 2 * r);
#pragma unroll
            for (int i = 0; i < C; ++i) {
                const int c = (i * T + t) * N;
                next_dy[i] = load_raw<E, WIDE>((const E *)P.dy + r * P.ld_out, c, P.width);
                next[i].template load<WIDE>(P, r, c);
            }
        }
    };
    load(cut.first);
    float w[C][N], dw[C][N], db[C][N];
#pragma unroll
    for (int i = 0; i < C; ++i) {
        for (int j = 0; j < N; ++j) w[i][j] = 1.f, dw[i][j] = db[i][j] = 0.f;
        if (P.weight_at >= 0) load_floats<N, WIDE>(P.params + worker * P.ld_params + P.weight_at, (i * T + t) * N, P.width, w[i]);
    }
    int turn = 0;
    for (int at = cut.first; at < cut.end; at += ROWS) {
        const bool there = at + slot < cut.end, on = next_on;
        const int64_t r = base + at + slot;
        float g[C][N], u[C][N];
        const float mean = next_stats[0], rstd = next_stats[1];
        f32x2 s = (f32x2)0.f;
#pragma unroll
        for (int i = 0; i < C; ++i) {
            Piece<E>::unpack(settled<E, WIDE>(next_dy[i], (i * T + t) * N, P.width), g[i]);
            next[i].template unpack<WIDE>((i * T + t) * N, P.width, u[i]);
        }
        load(at + ROWS);
        if (!on) {                                        // (T > 64: a row is the workgroup's)
            if (there)
#pragma unroll
                for (int i = 0; i < C; ++i) store_piece<E>((E *)P.dx + r * P.ld, (i * T + t) * N, P.width, (u32x4)0u);
            continue;
        }
        // (columns beyond the width: dy, and with it all sums, is zero there)
#pragma unroll
        for (int i = 0; i < C; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                u[i][j] = (u[i][j] - mean) * rstd;
                dw[i][j] = fmaf(g[i][j], u[i][j], dw[i][j]);
                db[i][j] += g[i][j];
                g[i][j] *= w[i][j];
                s[0] += g[i][j];
                s[1] = fmaf(g[i][j], u[i][j], s[1]);
            }
        s = row_sums<T>(s, sums[turn][slot]) * inverse;
        turn ^= 1;
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int c = (i * T + t) * N;
#pragma unroll
            for (int j = 0; j < N; ++j) g[i][j] = rstd * fmaf(-s[1], u[i][j], g[i][j] - s[0]);
            store_piece<E>((E *)P.dx + r * P.ld, c, P.width, Piece<E>::pack(g[i]));
        }
    }
    for (int which = 0; which < 2; ++which) {
        float *const to = part_of(P, worker, strip, which);
        if (!to) continue;
        if (ROWS > 1) {
            __syncthreads();
            if (slot)
                for (int i = 0; i < C; ++i)
                    for (int j = 0; j < N; ++j) joined[((slot - 1) * C * N + i * N + j) * T + t] = which ? db[i][j] : dw[i][j];
            __syncthreads();
            if (slot == 0)
                for (int i = 0; i < C; ++i)
                    for (int j = 0; j < N; ++j)
                        for (int q = 0; q < ROWS - 1; ++q) (which ? db : dw)[i][j] += joined[(q * C * N + i * N + j) * T + t];
        }
        if (slot == 0)
#pragma unroll
            for (int i = 0; i < C; ++i)
                if ((i * T + t) * N < P.width) store_floats<N>(to, (i * T + t) * N, P.width, which ? db[i] : dw[i]);
    }
}

// Long rows, first their two means ...
template <class E, int T, bool KEPT>
__global__ __launch_bounds__(T) void norm_means_kernel(NormGrad P)
{
    constexpr int N = Piece<E>::N;
    __shared__ f32x2 sums[T / 64];
    const int64_t r = group_number();
    if (r >= P.rows || (P.mask && !P.mask[r])) return;
    const int worker = (int)(r / P.per_worker);
    const float mean = P.stats[2 * r], rstd = P.stats[2 * r + 1];
    f32x2 s = (f32x2)0.f;
    for (int c = threadIdx.x * N; c < P.width; c += T * N) {
        float g[N], u[N], w[N];
        for (int j = 0; j < N; ++j) w[j] = 1.f;
        if (P.weight_at >= 0) load_floats<N, true>(P.params + worker * P.ld_params + P.weight_at, c, P.width, w);
        Piece<E>::unpack(load_piece<E, true>((const E *)P.dy + r * P.ld_out, c, P.width), g);
        input_piece<E, KEPT>(P, r, c, u);
        f32x2 part = (f32x2)0.f;
        for (int j = 0; j < N; ++j) {
            const float d = g[j] * w[j];
            part[0] += d;
            part[1] = c + j < P.width ? fmaf(d, (u[j] - mean) * rstd, part[1]) : part[1];
        }
        s += part;
    }
    s = row_sums<T>(s, sums) * (1.f / (float)P.width);
    if (threadIdx.x == 0) P.means[r] = s;
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
    const int first = strip * P.strip_rows, end = min(first + P.strip_rows, P.per_worker);
    float w[N], dw[N], db[N];
    for (int j = 0; j < N; ++j) w[j] = 1.f, dw[j] = db[j] = 0.f;
    if (P.weight_at >= 0) load_floats<N, true>(P.params + worker * P.ld_params + P.weight_at, c, P.width, w);
    for (int at = first; at < end; ++at) {
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
// The strips' shares, added in the strips' order: 32 columns a workgroup, its 8 rows of threads every eighth strip.
constexpr int SUM_COLUMNS = 32, SUM_ROWS = 8;
__global__ __launch_bounds__(SUM_COLUMNS * SUM_ROWS) void norm_sum_kernel(NormGrad P, int slices)
{
    __shared__ float lds[SUM_ROWS][SUM_COLUMNS];
    const int64_t group = group_number();
    const int which = (int)(group % 2);
    const int slice = (int)(group / 2 % slices);
    const int64_t worker = group / 2 / slices;
    const int64_t at = which ? P.bias_at : P.weight_at;
    if (worker >= P.workers || at < 0) return;
    const int q = threadIdx.x / SUM_COLUMNS, c = slice * SUM_COLUMNS + threadIdx.x % SUM_COLUMNS;
    float v = 0.f;
    if (c < P.width)
        for (int s = q; s < P.strips; s += SUM_ROWS) v += P.parts[((worker * P.strips + s) * 2 + which) * P.part_ld + c];
    lds[q][threadIdx.x % SUM_COLUMNS] = v;
    __syncthreads();
    if (q == 0 && c < P.width) {
        for (int s = 1; s < SUM_ROWS; ++s) v += lds[s][threadIdx.x];
        P.grads[worker * P.ld_grads + at + c] = v;
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
// A workgroup has STORE_PIECES x STORE_THREADS pieces that follow one another, a thread every STORE_THREADS-th; a row is a multiple of the pieces of a
// block.
constexpr int STORE_THREADS = 256, STORE_PIECES = 4;
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
