// Device side of the losses on rows of logits.
//
// With c = s log2(e), m the largest logit of a row and M = c m (rounded once, the same number everywhere), the row's sum is
// Z = sum_v 2^(c x_v - M), so that log p_y = ln 2 (c x_y - M - log2 Z) and p_v = 2^(c x_v - M) / Z.  Keeping (m, Z) and not L = ln 2 (M + log2 Z)
// keeps the rounding of a large L (2^-24 |L|), and that of M, out of every probability.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dbw.h"

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
__device__ __forceinline__ float log2_p(float x, float c, float2 mz)
{
    const Base b = base_of(mz.x, c);
    return (b.steep ? (x - mz.x) * c : fmaf(x, c, -b.M)) - log2f(mz.y);
}

template <int WAVES>
__device__ __forceinline__ float block_max(float v, float *lds)
{
    for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
    for (int w = 1; w < WAVES; ++w) v = fmaxf(v, lds[w]);
    return v;
}
template <int WAVES, class T>
__device__ __forceinline__ T block_sum(T v, T *lds)
{
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
    for (int w = 1; w < WAVES; ++w) v += lds[w];
    return v;
}

// ---------------------------------------------------------------- what a row's loss needs besides its logits

struct Logp {
    const int32_t *tokens;
    float *logp_out, *lse_out;
    float2 *stats;       // (m, Z) of every row, for a gradient in a launch of its own, or null
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

constexpr int THREADS = 256;
constexpr int WAVES = THREADS / 64;

// A grid's threads have to number less than 2^32: many rows make a second dimension.
__device__ __forceinline__ int64_t row_of_block() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

template <class E>
__device__ __forceinline__ void zero_row(const Rows &R, int64_t r)
{
    if (!R.dx) return;
    E *dx = (E *)R.dx + r * R.ld_grad;
    for (int v = threadIdx.x; v < R.vocab; v += THREADS) dx[v] = narrow<E>(0.f);
}

// (m, Z) of a row
template <class E>
__device__ __forceinline__ float2 row_stats(const Rows &R, const E *x, float *lds)
{
    float m = -INFINITY;
    for (int v = threadIdx.x; v < R.vocab; v += THREADS) m = fmaxf(m, widen(x[v]));
    m = block_max<WAVES>(m, lds);
    const Base base = base_of(m, R.c);
    float z = 0.f;
    for (int v = threadIdx.x; v < R.vocab; v += THREADS) z += power(widen(x[v]), base);
    return make_float2(m, block_sum<WAVES>(z, lds));
}

// dx_v = coef ([v = y] - p_v)
template <class E>
__device__ __forceinline__ void row_gradient(const Rows &R, const E *x, int64_t r, int y, const Base &base, float z, float coef)
{
    E *dx = (E *)R.dx + r * R.ld_grad;
    const float by = -coef / z;
    for (int v = threadIdx.x; v < R.vocab; v += THREADS) {
        const float e = by * power(widen(x[v]), base);
        dx[v] = narrow<E>(v == y ? e + coef : e);
    }
}

template <class E>
__global__ __launch_bounds__(THREADS) void logp_kernel(Rows R, Logp P)
{
    __shared__ float lds[WAVES];
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
    const float2 mz = row_stats<E>(R, x, lds);
    if (threadIdx.x == 0) {
        if (P.logp_out) P.logp_out[r] = LN2 * log2_p(widen(x[column(R, token)]), R.c, mz);
        if (P.lse_out) P.lse_out[r] = fmaf(R.scale, mz.x, LN2 * log2f(mz.y));
        if (P.stats) P.stats[r] = mz;
    }
}

template <class E>
__global__ __launch_bounds__(THREADS) void policy_kernel(Rows R, Policy P)
{
    __shared__ float lds[WAVES];
    const int64_t r = row_of_block();
    if (r >= R.rows) return;
    const int token = P.tokens[r];
    const float w = P.weights ? P.weights[r] : P.weight;
    if (token < 0 || w == 0.f) {
        if (threadIdx.x == 0) {
            if (P.logp_out) P.logp_out[r] = 0.f;
            P.terms[r] = make_float2(0.f, 0.f);
        }
        zero_row<E>(R, r);
        return;
    }
    const E *x = (const E *)R.x + r * R.ld;
    const int y = column(R, token);
    const float xy = widen(x[y]);
    const float2 mz = row_stats<E>(R, x, lds);
    const float logp = LN2 * log2_p(xy, R.c, mz);
    Policy once = P;
    if (threadIdx.x != 0) once.terms = nullptr;
    const float coef = policy_row(once, r, w, logp);
    if (threadIdx.x == 0 && P.logp_out) P.logp_out[r] = logp;
    if (!R.dx) return;
    if (coef == 0.f) zero_row<E>(R, r);
    else row_gradient<E>(R, x, r, y, base_of(mz.x, R.c), mz.y, R.scale * coef);
}

// The gradient alone, from (m, Z) or from L.
template <class E>
__global__ __launch_bounds__(THREADS) void gradient_kernel(Rows R, const int32_t *tokens, const float2 *stats, const float *lse,
                                                           const float *coef)
{
    const int64_t r = row_of_block();
    if (r >= R.rows) return;
    const int token = tokens[r];
    const float g = token < 0 || !coef ? 0.f : coef[r];
    if (g == 0.f) {
        zero_row<E>(R, r);
        return;
    }
    const E *x = (const E *)R.x + r * R.ld;
    float z = 1.f;
    Base base;
    if (stats) {
        base = base_of(stats[r].x, R.c);
        z = stats[r].y;
    } else {                                              // from L: M = L log2(e), Z = 1
        base = base_of(lse[r] / R.scale, R.c);
        if (!base.steep) base.M = lse[r] * LOG2E;
    }
    row_gradient<E>(R, x, r, column(R, token), base, z, R.scale * g);
}

template <class E>
__global__ __launch_bounds__(THREADS) void distill_kernel(Rows R, Distill P)
{
    extern __shared__ uint32_t shared[];
    __shared__ float lds[WAVES];
    __shared__ int twice;
    const int words = (R.vocab + 31) / 32;
    int *const at = (int *)shared;                        // the teacher's columns, -1 where absent
    float *const q = (float *)(shared + P.k);             // its probabilities
    uint32_t *const in_top = shared + 2 * P.k;            // a bit per column: is it one of the teacher's

    const int64_t r = row_of_block();
    if (r >= R.rows) return;
    const int tid = threadIdx.x;
    const float w = P.weights ? P.weights[r] : P.weight;
    bool out = w == 0.f;
    float norm = 0.f;
    if (!out) {
        for (int i = tid; i < words; i += THREADS) in_top[i] = 0;
        if (tid == 0) twice = 0;
        __syncthreads();
        for (int j = tid; j < P.k; j += THREADS) {
            int v = P.index[r * P.k + j];
            if (v >= R.vocab) {
                report(R.status);
                v = -1;
            }
            at[j] = v;
            q[j] = R.scale * load_as(P.value, r * P.k + j, P.value_type);
            if (v >= 0 && (atomicOr(&in_top[v >> 5], 1u << (v & 31)) >> (v & 31) & 1)) twice = 1;
        }
        __syncthreads();
        if (twice) {                                      // rare: the first entry of a column counts
            if (tid == 0) {
                report(R.status);
                for (int j = 1; j < P.k; ++j)
                    for (int i = 0; i < j; ++i)
                        if (at[i] == at[j]) at[j] = -1;
            }
            __syncthreads();
        }
        float top = -INFINITY, any = 0.f;
        for (int j = tid; j < P.k; j += THREADS)
            if (at[j] >= 0) {
                top = fmaxf(top, q[j]);
                any = 1.f;
            }
        top = block_max<WAVES>(top, lds);
        any = block_max<WAVES>(any, lds);
        float sum = 0.f;
        for (int j = tid; j < P.k; j += THREADS)
            if (at[j] >= 0) sum += expf(q[j] - (top == -INFINITY ? 0.f : top));
        sum = block_sum<WAVES>(sum, lds);
        norm = P.teacher_lse ? P.teacher_lse[r] : top + logf(sum);
        out = any == 0.f || (!P.teacher_lse && top == -INFINITY && sum == 0.f);
    }
    if (out) {
        if (tid == 0) {
            P.terms[r] = make_float2(0.f, 0.f);
            if (P.row_loss_out) P.row_loss_out[r] = 0.f;
        }
        zero_row<E>(R, r);
        return;
    }

    const E *x = (const E *)R.x + r * R.ld;
    const float2 mz = row_stats<E>(R, x, lds);
    // the student's mass outside the teacher's tokens, from a maximum of its own: it may be far below the rest
    float rest = 0.f, log_out = 0.f;
    if (P.teacher_lse) {
        float m = -INFINITY, z = 0.f;
        for (int v = tid; v < R.vocab; v += THREADS)
            if (!(in_top[v >> 5] >> (v & 31) & 1)) m = fmaxf(m, widen(x[v]));
        m = block_max<WAVES>(m, lds);
        const Base base = base_of(m, R.c), all = base_of(mz.x, R.c);
        for (int v = tid; v < R.vocab; v += THREADS)
            if (!(in_top[v >> 5] >> (v & 31) & 1)) z += power(widen(x[v]), base);
        z = block_sum<WAVES>(z, lds);
        log_out = LN2 * ((base.steep || all.steep ? (m - mz.x) * R.c : base.M - all.M) + (log2f(z) - log2f(mz.y)));
    }
    float part = 0.f, mass = 0.f;
    for (int j = tid; j < P.k; j += THREADS)
        if (at[j] >= 0) {
            const float log_q = q[j] - norm, qj = expf(log_q);
            const float log_p = LN2 * log2_p(widen(x[at[j]]), R.c, mz);
            mass += qj;
            if (!(qj <= 0.f)) part += qj * (log_q - log_p);
            q[j] = expf(log_p) - qj;                      // dl/dx over s
        }
    part = block_sum<WAVES>(part, lds);
    mass = block_sum<WAVES>(mass, lds);
    float factor = 1.f;
    if (P.teacher_lse) {
        rest = fmaxf(1.f - mass, 0.f);
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
    const Base base = base_of(mz.x, R.c);
    const float by = R.scale * w * factor / mz.y;
    for (int v = tid; v < R.vocab; v += THREADS)
        if (!(in_top[v >> 5] >> (v & 31) & 1))
            dx[v] = narrow<E>(by * power(widen(x[v]), base));
    for (int j = tid; j < P.k; j += THREADS)
        if (at[j] >= 0) dx[at[j]] = narrow<E>(R.scale * w * q[j]);
}

// loss_out[i], second_out[i] = sums of the terms of worker i's rows, always in the same order.
__global__ __launch_bounds__(THREADS) void sum_kernel(const float2 *terms, int rows, float *loss_out, float *second_out)
{
    __shared__ float lds[WAVES];
    const float2 *t = terms + (int64_t)blockIdx.x * rows;
    float a = 0.f, b = 0.f;
    for (int r = threadIdx.x; r < rows; r += THREADS) {
        a += t[r].x;
        b += t[r].y;
    }
    a = block_sum<WAVES>(a, lds);
    b = block_sum<WAVES>(b, lds);
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
    const float u = P.beta * block_sum<WAVES>(h, lds);
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
    l = block_sum<WAVES>(l, lds);
    if (threadIdx.x == 0) loss_out[blockIdx.x] = pairs ? l / (float)pairs : 0.f;
}

}  // namespace loss
