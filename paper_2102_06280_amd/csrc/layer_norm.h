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
    int per_worker, width;
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

// A row in the registers of T threads, C pieces each.  The mean comes first, then the sums of the differences from it and of their squares:
// the first of these is what the rounding of the mean left, which counts where a row's mean is large beside its spread.
template <class E, int T, int C>
__global__ __launch_bounds__(ROWS_OF<T> * T) void norm_kernel(Norm P)
{
    constexpr int N = Piece<E>::N, ROWS = ROWS_OF<T>;
    __shared__ f32x2 sums[2][(T + 63) / 64];
    const int64_t r = group_number() * ROWS + threadIdx.x / T;
    const int t = loss::tid<T>();
    if (r >= P.rows) return;                              // (whole waves' worth of lanes that share a row; T > 64: one row a workgroup)
    const bool on = !P.mask || P.mask[r];
    const E *const x = (const E *)P.x + r * P.ld;
    E *const y = (E *)P.y + r * P.ld_out;
    float v[C][N];
    float total = 0.f;
#pragma unroll
    for (int i = 0; i < C; ++i) {
        u32x4 w = (u32x4)0u;
        if (on) w = load_piece<E>(x, (i * T + t) * N, P.width);
        Piece<E>::unpack(w, v[i]);
#pragma unroll
        for (int j = 0; j < N; ++j) total += v[i][j];
    }
    const float inverse = 1.f / (float)P.width;
    const float mean = row_sums<T>((f32x2){total, 0.f}, sums[0])[0] * inverse;
    f32x2 s = (f32x2)0.f;
#pragma unroll
    for (int i = 0; i < C; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float d = (i * T + t) * N + j < P.width ? v[i][j] - mean : 0.f;
            s[0] += d;
            s[1] = fmaf(d, d, s[1]);
        }
    s = row_sums<T>(s, sums[1]);
    const float rest = s[0] * inverse;
    const float rstd = 1.f / sqrtf(fmaf(-rest, rest, s[1] * inverse) + P.eps);
    if (P.stats && t == 0) {
        P.stats[2 * r] = on ? mean + rest : 0.f;
        P.stats[2 * r + 1] = on ? rstd : 0.f;
    }
    const float *const params = P.params + r / P.per_worker * P.ld_params;
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const int c = (i * T + t) * N;
        if (P.kept.codes && c < (int)P.kept.stride) keep_piece<N>(P.kept, r, c, v[i]);
        if (c >= P.width) continue;
        float w[N], b[N];
        for (int j = 0; j < N; ++j) w[j] = 1.f, b[j] = 0.f;
        if (P.weight_at >= 0) load_floats<N>(params + P.weight_at, c, P.width, w);
        if (P.bias_at >= 0) load_floats<N>(params + P.bias_at, c, P.width, b);
#pragma unroll
        for (int j = 0; j < N; ++j) v[i][j] = on ? fmaf((v[i][j] - mean - rest) * rstd, w[j], b[j]) : 0.f;
        store_piece<E>(y, c, P.width, Piece<E>::pack(v[i]));
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
            Piece<E>::unpack(load_piece<E>(x, c, P.width), v);
            float part = 0.f;
            for (int j = 0; j < N; ++j) part += v[j];
            total += part;
        }
    const float inverse = 1.f / (float)P.width;
    const float mean = row_sums<T>((f32x2){total, 0.f}, sums[0])[0] * inverse;
    f32x2 s = (f32x2)0.f;
    if (on)
        for (int c = t * N; c < P.width; c += T * N) {
            Piece<E>::unpack(load_piece<E>(x, c, P.width), v);
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
        for (int j = 0; j < N; ++j) v[j] = 0.f;
        if (on) Piece<E>::unpack(load_piece<E>(x, c, P.width), v);
        if (P.kept.codes) keep_piece<N>(P.kept, r, c, v);
        if (c >= P.width) continue;
        float w[N], b[N];
        for (int j = 0; j < N; ++j) w[j] = 1.f, b[j] = 0.f;
        if (P.weight_at >= 0) load_floats<N>(params + P.weight_at, c, P.width, w);
        if (P.bias_at >= 0) load_floats<N>(params + P.bias_at, c, P.width, b);
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

template <class E, bool KEPT>
__device__ __forceinline__ void input_piece(const NormGrad &P, int64_t r, int c, float (&v)[Piece<E>::N])
{
    if (KEPT) kept_piece<Piece<E>::N>(P.kept, r, c, v);
    else Piece<E>::unpack(load_piece<E>((const E *)P.x + r * P.ld, c, P.width), v);
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
    __shared__ f32x2 sums[2][ROWS][(T + 63) / 64];
    extern __shared__ float joined[];                     // [ROWS - 1][T][C * N], one of dw and db after the other
    const int64_t group = group_number();
    if (group >= (int64_t)P.workers * P.strips) return;
    const int worker = (int)(group / P.strips), strip = (int)(group % P.strips);
    const int t = loss::tid<T>(), slot = threadIdx.x / T;
    const int first = strip * P.strip_rows, end = min(first + P.strip_rows, P.per_worker);
    const float inverse = 1.f / (float)P.width;
    float w[C][N], dw[C][N], db[C][N];
#pragma unroll
    for (int i = 0; i < C; ++i) {
        for (int j = 0; j < N; ++j) w[i][j] = 1.f, dw[i][j] = db[i][j] = 0.f;
        if (P.weight_at >= 0 && P.params) load_floats<N>(P.params + worker * P.ld_params + P.weight_at, (i * T + t) * N, P.width, w[i]);
    }
    int turn = 0;
    for (int at = first; at < end; at += ROWS, turn ^= 1) {
        const bool there = at + slot < end;
        const int64_t r = (int64_t)worker * P.per_worker + at + slot;
        const bool on = there && (!P.mask || P.mask[r]);
        float g[C][N], u[C][N];
        const float mean = on ? P.stats[2 * r] : 0.f, rstd = on ? P.stats[2 * r + 1] : 0.f;
        f32x2 s = (f32x2)0.f;
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int c = (i * T + t) * N;
            for (int j = 0; j < N; ++j) g[i][j] = u[i][j] = 0.f;
            if (on && c < P.width) {
                Piece<E>::unpack(load_piece<E>((const E *)P.dy + r * P.ld_out, c, P.width), g[i]);
                input_piece<E, KEPT>(P, r, c, u[i]);
            }
#pragma unroll
            for (int j = 0; j < N; ++j) {
                u[i][j] = on && c + j < P.width ? (u[i][j] - mean) * rstd : 0.f;
                dw[i][j] = fmaf(g[i][j], u[i][j], dw[i][j]);
                db[i][j] += g[i][j];
                g[i][j] *= w[i][j];
                s[0] += g[i][j];
                s[1] = fmaf(g[i][j], u[i][j], s[1]);
            }
        }
        s = row_sums<T>(s, sums[turn][slot]) * inverse;
        if (there)
#pragma unroll
            for (int i = 0; i < C; ++i) {
                const int c = (i * T + t) * N;
                if (c >= P.width) continue;
                for (int j = 0; j < N; ++j) g[i][j] = on ? rstd * (g[i][j] - s[0] - u[i][j] * s[1]) : 0.f;
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
        if (P.weight_at >= 0 && P.params) load_floats<N>(P.params + worker * P.ld_params + P.weight_at, c, P.width, w);
        Piece<E>::unpack(load_piece<E>((const E *)P.dy + r * P.ld_out, c, P.width), g);
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
    if (P.weight_at >= 0 && P.params) load_floats<N>(P.params + worker * P.ld_params + P.weight_at, c, P.width, w);
    for (int at = first; at < end; ++at) {
        const int64_t r = (int64_t)worker * P.per_worker + at;
        float g[N], u[N];
        for (int j = 0; j < N; ++j) g[j] = 0.f;
        if (!P.mask || P.mask[r]) {
            const float mean = P.stats[2 * r], rstd = P.stats[2 * r + 1];
            const f32x2 s = P.means[r];
            Piece<E>::unpack(load_piece<E>((const E *)P.dy + r * P.ld_out, c, P.width), g);
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
constexpr int STORE_THREADS = 256;
// A thread has a piece of a row; a row is `pieces` threads'.
template <class E>
__global__ __launch_bounds__(STORE_THREADS) void store_kernel(Store P)
{
    constexpr int N = Piece<E>::N;
    const int64_t pieces = P.kept.stride / N, piece = group_number() * STORE_THREADS + threadIdx.x;
    const int64_t r = piece / pieces;
    const int c = (int)(piece % pieces) * N;
    if (r >= P.rows) return;                              // (a block's lanes together)
    float v[N];
    for (int j = 0; j < N; ++j) v[j] = 0.f;
    if (!P.mask || P.mask[r]) Piece<E>::unpack(load_piece<E>((const E *)P.x + r * P.ld, c, P.width), v);
    keep_piece<N>(P.kept, r, c, v);
}
template <class E>
__global__ __launch_bounds__(STORE_THREADS) void load_kernel(Store P)
{
    constexpr int N = Piece<E>::N;
    const int64_t pieces = P.kept.stride / N, piece = group_number() * STORE_THREADS + threadIdx.x;
    const int64_t r = piece / pieces;
    const int c = (int)(piece % pieces) * N;
    if (r >= P.rows || c >= P.width) return;
    float v[N];
    kept_piece<N>(P.kept, r, c, v);
    store_piece<E>((E *)P.out + r * P.ld, c, P.width, Piece<E>::pack(v));
}

}  // namespace layer
