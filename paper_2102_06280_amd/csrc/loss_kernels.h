// Kernels of the losses on rows of logits.
//
// Where rows are many and long, those that write gradients are bound by memory (vector units busy 33 to 73 % of the time), those that only read by their
// instructions as much (86 %): a bf16 logit is two bytes to read for an exponential, at a quarter of the rate of other instructions, and six or seven of
// those.  Pieces beyond a row's end are computed as well, so short rows, and rows a little longer than a whole number of a workgroup's passes, are
// bound by instructions.  The rows are independent, so a
// row belongs to one workgroup, or its part of one, from its first byte to its gradient, and only the sums over a worker's rows cross workgroups:
// through memory and a second, small launch, in a fixed order (no atomics on floating point).  Figures: us on MI355X, logits read and gradients
// written at the rate named; a plain copy with streaming accesses reaches 6.5 TB/s here.
#pragma once

#include "loss_rows.h"

namespace loss {

constexpr int THREADS = 256;              // of workgroups that do not walk along a row
constexpr int WAVES = THREADS / 64;

// A grid's threads have to number less than 2^32: many workgroups make a second dimension (2^22 pairs or workers of 1024 threads would be as many).
__device__ __forceinline__ int64_t group() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }

// Rows of 64 or 16 threads share a workgroup of 256.
template <int T>
constexpr int ROWS_OF = T <= 64 ? 256 / T : 1;
template <int T>
__device__ __forceinline__ int row_in_group() { return T == 64 ? wave_id() : T < 64 ? (int)threadIdx.x / T : 0; }
template <int T>
__device__ __forceinline__ int64_t row_of_group(int64_t g) { return ROWS_OF<T> * g + row_in_group<T>(); }

// Workgroups go to the eight XCDs in turn: this gives each XCD rows that lie together.
__device__ __forceinline__ int64_t row_by_xcd(int64_t g, int64_t rows)
{
    const int64_t each = rows / 8;
    return g < each * 8 ? g % 8 * each + g / 8 : g;
}

// Few and long rows are cut into slices, a workgroup each, to fill the chip; what a slice finds goes through memory to a second launch.
struct Slices {
    int count;           // of a row; 1: rows are whole
    int pieces;          // of a slice (the last may have fewer)
};
// Slice s = first ... end - 1 of a row's pieces; slice 0 has the single elements, too.
__device__ __forceinline__ void slice_of(const Slices &S, int s, int pieces, int &first, int &end)
{
    first = S.count == 1 ? 0 : s * S.pieces;
    end = S.count == 1 ? pieces : min(first + S.pieces, pieces);
}
// A row's (m, Z) from its slices', on every one of T = 1, 16 or 64 lanes.
template <int T>
__device__ __forceinline__ MaxSum joined(const MaxSum *slices, int count, const Factor &c)
{
    MaxSum own{-INFINITY, 0.f};
    for (int s = tid<T>(); s < count; s += T) own = merged(own, slices[s], c);
    if (T == 1) return own;
    const float m = lanes_max<T>(own.m);
    return MaxSum{m, (float)lanes_sum<T>((double)(own.z * rescale(own.m, m, c)))};
}
constexpr int MAX_SLICES = 32;

// Sums over a workgroup's waves, in their order.  A worker's sums are held in 64 bits: of thousands of terms that are alike, roundings to 32 bits have
// one sign.
__device__ __forceinline__ void store_sums(double a, double b, double2 *lds, float *first_out, float *second_out)
{
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = make_double2(a, b);
    __syncthreads();
    if (threadIdx.x != 0) return;
    a = b = 0.;
    for (unsigned w = 0; w < blockDim.x / 64; ++w) {
        a += lds[w].x;
        b += lds[w].y;
    }
    *first_out = (float)a;
    if (second_out) *second_out = (float)b;
}

// ---------------------------------------------------------------- log-probabilities

struct Logp {
    const int32_t *tokens;
    const float *weights;// null: no row is left out for its weight
    float *logp_out, *lse_out;
    float *low;          // what rounding to 32 bits took off every log-probability, or null
    MaxSum *stats;       // (m, Z) of every slice, or null
    float *token_logit;  // of every row where there are slices
    Slices slices;
};

// A log-probability in 32 bits, and what that leaves of it
__device__ __forceinline__ void store_logp(double l, float *logp, float *low)
{
    const float rounded = (float)l;
    *logp = rounded;
    if (low) *low = isinf(rounded) ? 0.f : (float)(l - rounded);
}
__device__ __forceinline__ bool takes_part(const Logp &P, int64_t r) { return P.tokens[r] >= 0 && !(P.weights && P.weights[r] == 0.f); }

// (m, Z) of a wave's part of pieces first ... end - 1 of a row, and of its single elements if those are asked for.  ONCE: the pieces will not be read again.
template <bool ONCE, class E, int T, int C>
__device__ __forceinline__ MaxSum sums_of(const RowOf<E, T> &row, int first, int end, bool singles, const Factor &c)
{
    float m = -INFINITY;
    double sum = 0.;
    for (; first < end; first += T * C) {
        u32x4 v[C];
        row.template load<C, ONCE>(first, v);
        add_pieces<false>(row, first, end, v, -INFINITY, nullptr, c, m, sum);
    }
    MaxSum mz{m, (float)lanes_sum<T>(sum)};
    if (singles) {
        const float single = row.load_single(), top = lanes_max<T>(single);
        mz = merged(mz, MaxSum{top, lanes_sum<T>(power(single, base_of(top, c)))}, c);
    }
    return mz;
}

// A workgroup a row, or a slice: one pass, the maximum and the sum of a batch after the other.  4096 x 65536 bf16, a tenth of the rows without
// a part, 0.48 GB in 83 us, 5.8 TB/s, bound by memory and instructions; a single row by latency.  AGAIN: the rows will be read again soon, for their gradient.
template <class E, int T, int C, bool AGAIN>
__global__ __launch_bounds__(T * ROWS_OF<T>) void logp_kernel(Rows R, Logp P)
{
    __shared__ MaxSum lds[T > 64 ? T / 64 : 1];
    const int64_t r = T <= 64 ? row_of_group<T>(group()) : group() / P.slices.count;
    const int s = T <= 64 ? 0 : (int)(group() % P.slices.count);
    if (r >= R.rows) return;
    if (!takes_part(P, r)) {
        if (tid<T>() == 0 && P.slices.count == 1) {
            if (P.logp_out) P.logp_out[r] = 0.f;
            if (P.lse_out) P.lse_out[r] = 0.f;
        }
        return;
    }
    const E *x = (const E *)R.x + r * R.ld;
    const RowOf<E, T> row(x, R.vocab);
    int first, end;
    slice_of(P.slices, s, row.pieces, first, end);
    const MaxSum part = sums_of<!AGAIN, E, T, C>(row, first, end, s == 0, R.c);
    const float xy = widen(x[column(R, P.tokens[r])]);
    const MaxSum mz = row_merge<T>(part, R.c, lds);
    if (tid<T>() != 0) return;
    if (P.slices.count > 1) {
        P.stats[r * P.slices.count + s] = mz;
        if (s == 0) P.token_logit[r] = xy;
        return;
    }
    if (P.logp_out) store_logp(log_p(xy, R.scale, mz), P.logp_out + r, P.low ? P.low + r : nullptr);
    if (P.lse_out) P.lse_out[r] = (float)log_sum(R.scale, mz);
    if (P.stats) P.stats[r] = mz;
}

// A wave a row: its log-probability from its slices.
__global__ __launch_bounds__(64) void join_kernel(Rows R, Logp P)
{
    const int64_t r = blockIdx.x;
    float logp = 0.f, lse = 0.f;
    if (takes_part(P, r)) {
        const MaxSum mz = joined<64>(P.stats + r * P.slices.count, P.slices.count, R.c);
        logp = (float)log_p(P.token_logit[r], R.scale, mz);
        lse = (float)log_sum(R.scale, mz);
    }
    if (threadIdx.x != 0) return;
    if (P.logp_out) P.logp_out[r] = logp;
    if (P.lse_out) P.lse_out[r] = lse;
}

// dx_v = by 2^(c (x - m)) over pieces first ... end - 1, T C at a time, and coef more at column y if that is among them.
template <class E, int T, int C>
__device__ __forceinline__ void slice_gradient(const Rows &R, const RowOf<E, T> &row, int64_t r, int first, int end, float by, Base b, int y,
                                               float coef)
{
    E *dx = (E *)R.dx + r * R.ld_grad;
    const bool singles = first == 0;
    const int yp = row.piece_of(y);
    const bool mine = tid<T>() == row.owner(y) && (yp < 0 ? singles : yp >= first && yp < end);
    const float xy = mine ? widen(row.x[y]) : 0.f, single = singles ? row.load_single() : 0.f;
    b = uniform<T>(b);
    by = uniform<T>(by);
    const global_access::bytes out = base_address<T>(dx + row.before);
    for (; first < end; first += T * C) {
        u32x4 v[C];
        row.template load<C, true>(first, v);
#pragma unroll
        for (int i = 0; i < C; ++i) store_piece<E, T>(out, first, end, i, v[i], by, b);
    }
    if (singles && row.has_single()) dx[row.single_column()] = narrow<E>(by * power_alone(single, b));
    if (mine) dx[y] = narrow<E>(by * power_alone(xy, b) + coef);
}

// ---------------------------------------------------------------- pairs of sequences

struct Preference {
    const int32_t *tokens, *seq_start;
    const float *ref_logp, *weights;
    float beta, smoothing, scale;
    Factor c;
    int pairs;           // of each worker
    int64_t all_pairs, all_rows;
    float *logp, *margin_out, *coef;
    float *low;          // what log-probabilities have lost to 32 bits: of a sum over a sequence it is the larger part of the error.  The same memory as
                         // coef, which a pair needs when its sums are known
    MaxSum *stats;       // of every slice, and where rows have several
    MaxSum *joined;      // of every row
    const float *token_logit;
    int slices;
    int32_t *status;
};

__device__ __forceinline__ bool takes_part(const Preference &P, int64_t r) { return P.tokens[r] >= 0 && !(P.weights && P.weights[r] == 0.f); }

// (Numbers of rows go up to 2^31 - 2: those that count on in steps of a workgroup's threads need 64 bits.)
// Rows a[0] ... a[1] - 1 and a[1] ... a[2] - 1 of pair j, within the rows there are whatever the offsets say.
__device__ __forceinline__ void rows_of_pair(const Preference &P, int64_t j, int (&a)[3])
{
    const int n = (int)P.all_rows;
    for (int i = 0; i < 3; ++i) a[i] = P.seq_start[2 * j + i];
    if (a[0] < 0 || a[1] < a[0] || a[2] < a[1] || a[2] > n) report(P.status);
    a[0] = min(max(a[0], 0), n);
    a[1] = min(max(a[1], a[0]), n);
    a[2] = min(max(a[2], a[1]), n);
}
// A thread's part, one of `threads`, of the difference between the pair's summed log ratios.
__device__ __forceinline__ double part_of_pair(const Preference &P, const int (&a)[3], int thread, int threads)
{
    double h = 0.;
    for (int64_t r = (int64_t)a[0] + thread; r < a[2]; r += threads)
        if (takes_part(P, r)) {
            const double term = (P.weights ? P.weights[r] : 1.f) * ((double)P.logp[r] - P.ref_logp[r] + P.low[r]);
            h += r < a[1] ? term : -term;
        }
    return h;
}
// The derivative of a worker's loss with respect to the difference of a pair, times beta; from the pair's margin.
__device__ __forceinline__ float slope_of(const Preference &P, float u)
{
    const float e = expf(-fabsf(u));                      // sigma(u) = 1 / (1 + e) or e / (1 + e)
    const float sig = (u >= 0.f ? 1.f : e) / (1.f + e), sig_not = (u >= 0.f ? e : 1.f) / (1.f + e);
    return (u != u ? u : P.smoothing * sig - (1.f - P.smoothing) * sig_not) * P.beta / (float)P.pairs;
}

constexpr int PAIR_THREADS = 1024;       // 64 rows at a time where their slices have to be joined

// Log-probabilities of rows from their slices, T lanes a row.
template <int T>
__device__ __forceinline__ void join_rows(const Preference &P, int from, int to)
{
    const bool first = threadIdx.x % T == 0;
    for (int64_t r = (int64_t)from + threadIdx.x / T; r < to; r += PAIR_THREADS / T) {
        double logp = 0.;
        if (takes_part(P, r)) {
            const MaxSum mz = joined<T>(P.stats + r * P.slices, P.slices, P.c);
            logp = log_p(P.token_logit[r], P.scale, mz);
            if (first) P.joined[r] = mz;
        }
        if (first) store_logp(logp, P.logp + r, P.low + r);
    }
}

// (Short and bound by latency, 4 to 6 us: it stands between two passes over the logits because a coefficient needs the sums of all its pair's rows.)
// The margin of a pair and the derivative of its worker's loss with respect to every log-probability of its rows.  Rows in no sequence are
// the first and the last pair's.
__global__ __launch_bounds__(PAIR_THREADS) void pair_kernel(Preference P)
{
    __shared__ double lds[PAIR_THREADS / 64];
    const int64_t j = group();
    if (j >= P.all_pairs) return;
    const int t = threadIdx.x, n = (int)P.all_rows;
    int a[3];
    rows_of_pair(P, j, a);
    const int from = j == 0 ? 0 : a[0], to = j == P.all_pairs - 1 ? n : a[2];
    if (P.slices > 1) {
        if (P.slices > 8) join_rows<16>(P, from, to);     // few rows
        else join_rows<1>(P, from, to);
        __syncthreads();
    }
    const float u = (float)(P.beta * row_sum<PAIR_THREADS>(part_of_pair(P, a, t, PAIR_THREADS), lds));
    if (t == 0) P.margin_out[j] = u;
    const float slope = slope_of(P, u);
    for (int64_t r = (int64_t)from + t; r < to; r += PAIR_THREADS)
        P.coef[r] = takes_part(P, r) && r >= a[0] && r < a[2] ? (r < a[1] ? slope : -slope) * (P.weights ? P.weights[r] : 1.f) : 0.f;
}

// A worker's mean over its pairs, from their margins.
struct PairLoss {
    const float *margin;
    int workers, pairs;
    float smoothing;
    float *loss_out;     // null: not asked for
};
__device__ __forceinline__ float loss_of(const PairLoss &P, float u)
{
    // -log sigma(u) = max(-u, 0) + soft, -log sigma(-u) = max(u, 0) + soft
    const float soft = log1pf(expf(-fabsf(u)));
    return u != u ? u : soft + (u >= 0.f ? P.smoothing * u : (P.smoothing - 1.f) * u);
}
template <int T>
__device__ __forceinline__ void pair_loss(const PairLoss &P, int64_t worker, double *lds)
{
    double l = 0.;
    for (int j = threadIdx.x; j < P.pairs; j += T) l += loss_of(P, P.margin[worker * P.pairs + j]);
    l = row_sum<T>(l, lds);
    if (threadIdx.x == 0) P.loss_out[worker] = P.pairs ? (float)(l / P.pairs) : 0.f;
}
__global__ __launch_bounds__(THREADS) void pair_loss_kernel(PairLoss P)
{
    __shared__ double lds[WAVES];
    pair_loss<THREADS>(P, blockIdx.x, lds);
}

// ---------------------------------------------------------------- a gradient alone

struct Gradient {
    const int32_t *tokens;
    const float *coef;   // null: none
    const MaxSum *stats; // (m, Z) of every row, or (FROM_L)
    const float *lse;    // L
    Slices slices;
    PairLoss pairs;      // workgroups behind the rows' give every worker's loss
};

// Largest |L| that is taken as it is: in 32 bits it is off by up to 2^-17, and so is every probability, of itself.  Larger ones have lost too much of ln Z
// (all of it in a row of equal logits of 1e30), or are infinite where their row is not.
constexpr float MOST_L = 256.f;

// FROM_L: a row whose L is larger than that is summed again, whole and by the workgroup of its first slice, which then also writes it all: in place, nobody
// else may write what is still to be read.
template <class E, int T, int C, bool FROM_L>
__device__ __forceinline__ void gradient_of_slice(const Rows &R, const Gradient &P, int64_t r, int s, int token, float g, MaxSum *lds)
{
    const RowOf<E, T> row((const E *)R.x + r * R.ld, R.vocab);
    if (g == 0.f) {
        // (the pieces of the gradient's row may be one more than those of the logits')
        zero_pieces<E, T, true>(R, r, s * P.slices.pieces, s == P.slices.count - 1 ? INT32_MAX : (s + 1) * P.slices.pieces);
        return;
    }
    int first, end;
    slice_of(P.slices, s, row.pieces, first, end);
    float by;
    MaxSum mz;
    bool summed = !FROM_L;
    if (FROM_L) {
        const float L = P.lse[r], m = L / R.scale;
        summed = !(fabsf(L) <= MOST_L && fabsf(m) < INFINITY);
        if (summed) {
            if (s != 0) return;
            first = 0;
            end = row.pieces;
            mz = row_merge<T>(sums_of<false, E, T, C>(row, first, end, true, R.c), R.c, lds);
        } else {
            // p = exp(s (x - m) - d) with d = L - s m, what the division's rounding has left
            mz.m = m;
            by = fmaf(g, fmaf(-R.scale, m, L), -g);
        }
    } else {
        mz = P.stats[r];
    }
    if (summed) by = -g / mz.z;
    const Base b = base_of(mz.m, R.c);
    slice_gradient<E, T, C>(R, row, r, first, end, by, b, column(R, token), g);
}

// A workgroup a slice of 16 KB: the row's (m, Z) are known, so every piece is by itself.  Bound by memory: 8192 x 32768 bf16, 15 % of the rows without a part,
// 0.99 GB in 148 us, 6.7 TB/s with what is left of the rows in the last-level cache.
template <class E, int T, int C, bool FROM_L>
__global__ __launch_bounds__(T * ROWS_OF<T>) void gradient_kernel(Rows R, Gradient P)
{
    __shared__ double lds[T * ROWS_OF<T> / 64];
    __shared__ MaxSum lds_row[T > 64 ? T / 64 : 1];
    const int64_t groups = T <= 64 ? (R.rows + ROWS_OF<T> - 1) / ROWS_OF<T> : R.rows * P.slices.count;
    if (group() >= groups) {
        const int64_t worker = group() - groups;
        if (P.pairs.loss_out && worker < P.pairs.workers) pair_loss<T * ROWS_OF<T>>(P.pairs, worker, lds);
        return;
    }
    const int64_t r = T <= 64 ? row_of_group<T>(group()) : group() / P.slices.count;
    const int s = T <= 64 ? 0 : (int)(group() % P.slices.count);
    if (r >= R.rows) return;
    const int token = P.tokens[r];
    gradient_of_slice<E, T, C, FROM_L>(R, P, r, s, token, token < 0 || !P.coef ? 0.f : R.scale * P.coef[r], lds_row);
}

// Margins and loss of a worker with few rows and short pairs, a wave a pair, by a workgroup of THREADS.
__device__ __forceinline__ void sums_of_pairs(const PairLoss &P, const Preference &Q, int64_t worker, double2 *lds)
{
    int a[3];
    double loss = 0.;
    for (int j = wave_id(); j < Q.pairs; j += WAVES) {
        rows_of_pair(Q, worker * Q.pairs + j, a);
        const float u = (float)(Q.beta * wave_sum(part_of_pair(Q, a, threadIdx.x & 63, 64)));
        if ((threadIdx.x & 63) == 0) Q.margin_out[worker * Q.pairs + j] = u;
        loss += loss_of(P, u);
    }
    store_sums(loss / Q.pairs, 0., lds, P.loss_out + worker, nullptr);
}
__global__ __launch_bounds__(THREADS) void pair_sums_kernel(PairLoss P, Preference Q)
{
    __shared__ double2 lds[WAVES];
    sums_of_pairs(P, Q, blockIdx.x, lds);
}

// The gradient for few rows in short pairs, with every coefficient from the log-probabilities of its pair, which the threads of a row sum up again
// for each row; workgroups behind the rows' give margins and losses.
template <class E, int T, int C>
__global__ __launch_bounds__(T * ROWS_OF<T>) void pair_gradient_kernel(Rows R, Gradient P, Preference Q)
{
    static_assert(T * ROWS_OF<T> == THREADS, "the workgroups behind the rows' have as many threads as pair_sums_kernel's");
    __shared__ double2 lds[WAVES];
    constexpr int LANES = T < 64 ? T : 64;
    const int64_t groups = T <= 64 ? (R.rows + ROWS_OF<T> - 1) / ROWS_OF<T> : R.rows * P.slices.count;
    int a[3];
    if (group() >= groups) {
        const int64_t worker = group() - groups;
        if (worker >= P.pairs.workers) return;
        sums_of_pairs(P.pairs, Q, worker, lds);
        return;
    }
    const int64_t r = T <= 64 ? row_of_group<T>(group()) : group() / P.slices.count;
    const int s = T <= 64 ? 0 : (int)(group() % P.slices.count);
    if (r >= R.rows) return;
    const int token = P.tokens[r];
    float g = 0.f;
    if (takes_part(Q, r)) {
        // the last sequence that starts at the row or before it
        const int lane = threadIdx.x & (LANES - 1), sequences = 2 * P.pairs.workers * Q.pairs;
        float starts = 0.f;
        for (int q = lane; q < sequences; q += LANES) starts += Q.seq_start[q] <= r ? 1.f : 0.f;
        const int q = (int)lanes_sum<LANES>(starts) - 1;
        if (q >= 0) {
            rows_of_pair(Q, q / 2, a);
            const float slope = slope_of(Q, (float)(Q.beta * lanes_sum<LANES>(part_of_pair(Q, a, lane, LANES))));
            if (r >= a[0] && r < a[2]) g = R.scale * (r < a[1] ? slope : -slope) * (Q.weights ? Q.weights[r] : 1.f);
        }
    }
    gradient_of_slice<E, T, C, false>(R, P, r, s, token, g, nullptr);
}

// ---------------------------------------------------------------- policy

struct Policy {
    const int32_t *tokens;
    const float *old_logp, *ref_logp, *advantage, *weights;
    float low, high, kl_coef, weight;     // the bounds of the ratio; the weight of every row where weights is null
    float *logp_out;
    float2 *terms;       // a row's weighted loss and KL term, for the sums over a worker's rows
    // where rows are cut
    const MaxSum *stats;
    const float *token_logit;
    int parts;           // slices that a row's stats are of
    Slices slices;       // of the gradient
    int rows;            // of each worker
    float *loss_out, *kl_out;
};

// A row's figures besides its logits, all asked for at once, before the logits.
struct PolicyFigures {
    float w, a, old, ref;
};
__device__ __forceinline__ PolicyFigures figures_of(const Policy &P, int64_t r, float w)
{
    return PolicyFigures{w, P.advantage[r], P.old_logp[r], P.ref_logp ? P.ref_logp[r] : 0.f};
}
// What a row adds to its worker's sums, and the derivative with respect to its log-probability.
struct PolicyRow {
    float loss, kl, slope;
};
__device__ __forceinline__ PolicyRow policy_of(const Policy &P, const PolicyFigures &F, float logp)
{
    const float w = F.w, a = F.a, rho = expf(logp - F.old);
    // A factor of zero takes its term out also where the other one is beyond 32 bits (a ratio that is NaN stays so).
    const bool no_ratio = a == 0.f && rho == rho;
    const float product = no_ratio ? 0.f : rho * a, bounded = no_ratio ? 0.f : fminf(fmaxf(rho, P.low), P.high) * a;
    const bool free = product <= bounded || product != product;     // (fminf and fmaxf would take a ratio that is NaN for a bound)
    float kl = 0.f, dkl = 0.f;
    if (P.ref_logp) {
        const float d = F.ref - logp;
        dkl = -expm1f(d);
        kl = -dkl - d;
    }
    const bool no_kl = P.kl_coef == 0.f && dkl == dkl;
    const float kl_term = no_kl ? 0.f : P.kl_coef * kl, kl_slope = no_kl ? 0.f : P.kl_coef * dkl;
    return PolicyRow{w * (kl_term - (free ? product : bounded)), w * kl, w * (kl_slope - (free ? product : 0.f))};
}
__device__ __forceinline__ float weight_of(const Policy &P, int64_t r)
{
    return P.tokens[r] < 0 ? 0.f : P.weights ? P.weights[r] : P.weight;
}

// A row's terms and its gradient, by T threads.
template <class E, int T, int C, int S>
__device__ __forceinline__ float2 policy_whole_row(const Rows &R, const Policy &P, int64_t r, MaxSum *lds)
{
    const float w = weight_of(P, r);
    if (w == 0.f) {
        if (tid<T>() == 0 && P.logp_out) P.logp_out[r] = 0.f;
        zero_row<E, T>(R, r);
        return make_float2(0.f, 0.f);
    }
    const E *x = (const E *)R.x + r * R.ld;
    Walk<E, T, C, S> walk(x, R.vocab);
    const PolicyFigures figures = figures_of(P, r, w);
    const int y = column(R, P.tokens[r]);
    const float xy = widen(x[y]);
    const MaxSum mz = walk.stats(R.c, lds);
    const float logp = (float)log_p(xy, R.scale, mz);
    const PolicyRow p = policy_of(P, figures, logp);
    if (tid<T>() == 0 && P.logp_out) P.logp_out[r] = logp;
    if (R.dx) {
        const float coef = R.scale * p.slope;
        if (coef == 0.f) zero_row<E, T>(R, r);
        else walk.gradient((E *)R.dx + r * R.ld_grad, -coef / mz.z, base_of(mz.m, R.c), y, xy, coef);
    }
    return make_float2(p.loss, p.kl);
}

// A workgroup a row, which is read once and stays in registers until its gradient is written: the coefficient needs nothing but the row's own sum.
// Bound by memory: 4096 x 32768 bf16, 15 % of the rows without a part, 0.5 GB in 88 us, 5.7 TB/s.
template <class E, int T, int C, int S>
__global__ __launch_bounds__(T * ROWS_OF<T>, C == 16 ? 4 : 1) void policy_kernel(Rows R, Policy P)
{
    __shared__ MaxSum lds[T > 64 ? T / 64 : 1];
    const int64_t r = row_of_group<T>(R.by_xcd ? row_by_xcd(group(), R.rows) : group());
    if (r >= R.rows) return;
    const float2 terms = policy_whole_row<E, T, C, S>(R, P, r, lds);
    if (tid<T>() == 0) P.terms[r] = terms;
}

// All of a worker's rows in one workgroup, T threads each, and their sums: one launch.
template <class E, int T, int C>
__global__ __launch_bounds__(1024) void policy_worker_kernel(Rows R, Policy P)
{
    __shared__ double2 lds[16];
    const int64_t worker = group();
    if (worker * P.rows >= R.rows) return;
    double a = 0., b = 0.;
    for (int t = row_in_group<T>(); t < P.rows; t += blockDim.x / T) {
        const float2 terms = policy_whole_row<E, T, C, 0>(R, P, worker * P.rows + t, nullptr);
        if (tid<T>() == 0) {
            a += terms.x;
            b += terms.y;
        }
    }
    store_sums(wave_sum(a), wave_sum(b), lds, P.loss_out + worker, P.kl_out ? P.kl_out + worker : nullptr);
}

// The second launch for rows in slices: the slices' gradients, and behind them a workgroup for every worker's sums.
template <class E, int T, int C>
__global__ __launch_bounds__(T) void policy_slices_kernel(Rows R, Policy P)
{
    __shared__ double2 lds[T / 64];
    const int64_t b = blockIdx.x, cut = R.dx ? R.rows * P.slices.count : 0;
    const int n = P.slices.count;
    if (b >= cut) {
        const int64_t worker = b - cut;
        double loss = 0., kl = 0.;
        for (int t = threadIdx.x / 16; t < P.rows; t += T / 16) {
            const int64_t r = worker * P.rows + t;
            const float w = weight_of(P, r);
            float logp = 0.f;
            if (w != 0.f) {
                logp = (float)log_p(P.token_logit[r], R.scale, joined<16>(P.stats + r * P.parts, P.parts, R.c));
                const PolicyRow p = policy_of(P, figures_of(P, r, w), logp);
                if (threadIdx.x % 16 == 0) {
                    loss += p.loss;
                    kl += p.kl;
                }
            }
            if (P.logp_out && threadIdx.x % 16 == 0) P.logp_out[r] = logp;
        }
        store_sums(wave_sum(loss), wave_sum(kl), lds, P.loss_out + worker, P.kl_out ? P.kl_out + worker : nullptr);
        return;
    }
    const int64_t r = b / n;
    const int s = (int)(b % n);
    const float w = weight_of(P, r);
    float coef = 0.f;
    MaxSum mz;
    if (w != 0.f) {
        mz = joined<64>(P.stats + r * P.parts, P.parts, R.c);
        coef = R.scale * policy_of(P, figures_of(P, r, w), (float)log_p(P.token_logit[r], R.scale, mz)).slope;
    }
    if (coef == 0.f) {
        zero_pieces<E, T>(R, r, s * P.slices.pieces, s == n - 1 ? INT32_MAX : (s + 1) * P.slices.pieces);
        return;
    }
    const RowOf<E, T> row((const E *)R.x + r * R.ld, R.vocab);
    int first, end;
    slice_of(P.slices, s, row.pieces, first, end);
    slice_gradient<E, T, C>(R, row, r, first, end, -coef / mz.z, base_of(mz.m, R.c), column(R, P.tokens[r]), coef);
}

// ---------------------------------------------------------------- distillation

struct Distill {
    const int32_t *index;
    const void *value;
    const float *teacher_lse, *weights;
    float weight;
    int k, value_type;
    float *row_loss_out;
    float2 *terms;
    int rows;            // of each worker
    float *loss_out;
};

// LDS words of a row: the teacher's columns (-1 where absent), its logits, the student's logits, and a bit for every column of the
// vocabulary that is in the list, which begin with Piece::N - row.before <= 8 unused ones.
__host__ __device__ __forceinline__ int distill_words(int k, int vocab) { return 3 * k + (vocab + 8 + 31) / 32; }

// A row's weighted loss, and its gradient, by T threads.
template <class E, int T, int C, int S, bool TAIL>
__device__ __forceinline__ float distill_whole_row(const Rows &R, const Distill &P, int64_t r, uint32_t *shared, MaxSum *lds, MaxSum *lds_top,
                                                   float (*sums)[T > 64 ? T / 64 : 1], double *masses)
{
    const int t = tid<T>();
    const float w = P.weights ? P.weights[r] : P.weight;
    if (w == 0.f) {
        if (t == 0 && P.row_loss_out) P.row_loss_out[r] = 0.f;
        zero_row<E, T>(R, r);
        return 0.f;
    }
    const E *x = (const E *)R.x + r * R.ld;
    Walk<E, T, C, S> walk(x, R.vocab);                    // in flight while the list is looked at

    int *const at = (int *)shared;
    float *const q = (float *)(shared + P.k);
    float *const xs = (float *)(shared + 2 * P.k);
    uint32_t *const in_top = shared + 3 * P.k;
    const int bit0 = Piece<E>::N - walk.row.before;
    for (int i = t; i < distill_words(P.k, R.vocab) - 3 * P.k; i += T) in_top[i] = 0;
    row_barrier<T>();
    float seen = 0.f, top = -INFINITY, m_top = -INFINITY;           // seen: 1 an entry, 2 a column twice
    for (int first = t; first < P.k; first += 4 * T) {    // four entries of a thread at a time: two round trips to memory for all of them
        int v[4];
        float value[4], xv[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = P.index[r * P.k + min(first + u * T, P.k - 1)];
        if (P.value_type == 0) {
#pragma unroll
            for (int u = 0; u < 4; ++u) value[u] = ((const float *)P.value)[r * P.k + min(first + u * T, P.k - 1)];
        } else {
            uint16_t bits[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) bits[u] = ((const uint16_t *)P.value)[r * P.k + min(first + u * T, P.k - 1)];
#pragma unroll
            for (int u = 0; u < 4; ++u) value[u] = P.value_type == 1 ? widen(bf16{bits[u]}) : widen(__builtin_bit_cast(f16, bits[u]));
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (v[u] >= R.vocab) {
                report(R.status);
                v[u] = -1;
            }
            xv[u] = widen(x[max(v[u], 0)]);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int j = first + u * T;
            if (j >= P.k) break;
            at[j] = v[u];
            q[j] = value[u];
            xs[j] = xv[u];
            if (v[u] >= 0) {
                const int bit = v[u] + bit0;
                seen = fmaxf(seen, atomicOr(&in_top[bit >> 5], 1u << (bit & 31)) >> (bit & 31) & 1 ? 2.f : 1.f);
            }
        }
    }
    row_barrier<T>();
    seen = row_max<T>(seen, sums[0]);
    if (seen == 2.f) {                                    // the first entry of a column counts
        if (t == 0) report(R.status);
        // An entry looks for its column among those before it.  One that has found it says so beside its column, which later ones still compare
        // with, and goes when all have looked.  3 rows of 33001 f16 with 1024 entries, half of them the first again: 61 us; 25 ms by one thread.
        constexpr int AGAIN = 1 << 30;                    // columns are below 2^20
        for (int j = t; j < P.k; j += T) {
            const int v = at[j];
            if (v < 0) continue;
            for (int i = 0; i < j; ++i)
                if ((at[i] & ~AGAIN) == v) {
                    at[j] = v | AGAIN;
                    break;
                }
        }
        row_barrier<T>();
        for (int j = t; j < P.k; j += T)
            if (at[j] >= AGAIN) at[j] = -1;
        row_barrier<T>();
    }
    for (int j = t; j < P.k; j += T)
        if (at[j] >= 0) {
            top = fmaxf(top, q[j]);
            m_top = fmaxf(m_top, xs[j]);
        }
    top = row_max<T>(top, sums[1]);
    m_top = lanes_max<T>(m_top);
    const Base base_top = base_of(m_top, R.c);
    float sum = 0.f, z_top = 0.f;
    const float from = top == -INFINITY ? 0.f : top;      // differences of logits first: they may be of any size
    for (int j = t; j < P.k; j += T)
        if (at[j] >= 0) {
            sum += power(q[j], Base{R.c, from});
            z_top += power(xs[j], base_top);
        }
    sum = row_sum<T>(sum, sums[2]);
    if (seen == 0.f || (!TAIL && top == -INFINITY && sum == 0.f)) {
        if (t == 0 && P.row_loss_out) P.row_loss_out[r] = 0.f;
        zero_row<E, T>(R, r);
        return 0.f;
    }

    // With the tail the student's mass outside the list is summed apart, from a maximum of its own: it may be far below the rest, and as a
    // difference from one it would be lost.
    MaxSum mz, out;                                       // of the row; of what is not in the list, or of the row
    float log_out = 0.f;
    if (TAIL) {
        const MaxSum in = row_merge<T>(MaxSum{m_top, lanes_sum<T>(z_top)}, R.c, lds_top);
        out = walk.template stats<true>(R.c, lds, (const uint8_t *)in_top);
        mz = merged(out, in, R.c);
        log_out = (float)(log_p(out.m, R.scale, mz) + ln(out.z));
    } else {
        mz = out = walk.stats(R.c, lds);
    }
    // With the tail the list's mass is taken from one: s t - L is rounded once, as a difference, and not its terms, which may be large.
    const float norm = TAIL ? P.teacher_lse[r] : (float)ln(sum), ln_z = (float)ln(mz.z);
    float part = 0.f;
    double mass = 0.;
    for (int j = t; j < P.k; j += T)
        if (at[j] >= 0) {
            const float log_q = fmaf(R.scale, TAIL ? q[j] : q[j] - from, -norm), qj = exponential(log_q);
            const float log_pj = fmaf(R.scale, xs[j] - mz.m, -ln_z);
            mass += qj;
            if (!(qj <= 0.f)) part += qj * (log_q - log_pj);
            q[j] = exponential(log_pj) - qj;              // dl/dx over s
        }
    part = row_sum<T>(part, sums[3]);
    float mass_out = 1.f;                                 // s times this is the sum of the gradient's columns that are not in the list
    if (TAIL) {
        mass = row_sum<T>(mass, masses);
        float rest = mass > 1. ? 0.f : (float)(1. - mass);
        // Nothing outside: the list's mass is one but for the rounding of L (2^-24 |L|) and of k <= 1024 entries (2^-24 (ln k + 4)); either four times.
        if (out.z == 0.f && rest <= 0x1p-22f * (fabsf(norm) + 12.f)) rest = 0.f;
        if (rest > 0.f) part += rest * (logf(rest) - log_out);
        // p_v (1 - R / S) = (S - R) p_v / S: p_v alone may be too small for 32 bits, p_v / S is not
        mass_out = expf(log_out) - rest;
    }
    if (t == 0 && P.row_loss_out) P.row_loss_out[r] = part;
    if (R.dx) {
        E *dx = (E *)R.dx + r * R.ld_grad;
        // Single elements written over in lines that have left the L2 cost more than the streaming stores gain where they are many: 14664
        // rows of 3920 bf16, k = 152: 75 us and 106 with streaming stores; 8192 rows of 8000, k = 64: 70 and 67.  (Kernels of longer rows have no
        // registers left for both kinds.)
        // Where nothing is outside, by is finite all the same: what it writes is a token's that cannot occur, or written over.
        const float by = TAIL && out.z == 0.f && mz.z > 0.f ? 0.f : R.scale * w * mass_out / out.z;
        const Base base = base_of(out.m, R.c);
        if (T <= 64 && P.k >= R.vocab / 64) walk.template gradient<true>(dx, by, base, -1, 0.f, 0.f);
        else walk.template gradient<false>(dx, by, base, -1, 0.f, 0.f);
        if (T > 64) __syncthreads();                      // the list's columns are written over
        for (int j = t; j < P.k; j += T)
            if (at[j] >= 0) dx[at[j]] = narrow<E>(R.scale * w * q[j]);
    }
    return w * part;
}

// As policy_kernel, with the list in LDS beside it.  Bound by memory, and by what the list costs a row (five short loops over it with barriers between):
// 2048 x 32000 bf16, 64 entries, 0.25 GB in 57 us, 4.4 TB/s; 4096 x 131072, 128 entries, 2.15 GB in 420 us, 5.1 TB/s.
template <class E, int T, int C, int S, bool TAIL>
__global__ __launch_bounds__(T * ROWS_OF<T>, C == 16 ? 4 : 1) void distill_kernel(Rows R, Distill P)
{
    extern __shared__ uint32_t shared[];
    __shared__ MaxSum lds[T > 64 ? T / 64 : 1], lds_top[T > 64 ? T / 64 : 1];
    __shared__ float sums[4][T > 64 ? T / 64 : 1];
    __shared__ double masses[T > 64 ? T / 64 : 1];
    const int64_t r = row_of_group<T>(R.by_xcd ? row_by_xcd(group(), R.rows) : group());
    if (r >= R.rows) return;
    const float term = distill_whole_row<E, T, C, S, TAIL>(R, P, r, shared + row_in_group<T>() * distill_words(P.k, R.vocab), lds, lds_top, sums, masses);
    if (tid<T>() == 0) P.terms[r] = make_float2(term, 0.f);
}

// All of a worker's rows in one workgroup, T threads each, and their sum.
template <class E, int T, int C, bool TAIL>
__global__ __launch_bounds__(1024) void distill_worker_kernel(Rows R, Distill P)
{
    extern __shared__ uint32_t shared[];
    __shared__ double2 lds[16];
    const int64_t worker = group();
    if (worker * P.rows >= R.rows) return;
    double a = 0.;
    for (int t = row_in_group<T>(); t < P.rows; t += blockDim.x / T) {
        const float term = distill_whole_row<E, T, C, 0, TAIL>(R, P, worker * P.rows + t,
                                                               shared + row_in_group<T>() * distill_words(P.k, R.vocab), nullptr, nullptr, nullptr, nullptr);
        if (tid<T>() == 0) a += term;
        row_barrier<T>();                                 // the next row's list takes this one's place
    }
    store_sums(wave_sum(a), 0., lds, P.loss_out + worker, nullptr);
}

// ---------------------------------------------------------------- sums

// loss_out[i], second_out[i] = sums of the terms of worker i's rows, always in the same order.
__global__ __launch_bounds__(THREADS) void sum_kernel(const float2 *terms, int rows, float *loss_out, float *second_out)
{
    __shared__ double2 lds[WAVES];
    const float2 *t = terms + (int64_t)blockIdx.x * rows;
    double a = 0., b = 0.;
    for (int64_t r = threadIdx.x; r < rows; r += THREADS) {
        a += t[r].x;
        b += t[r].y;
    }
    store_sums(wave_sum(a), wave_sum(b), lds, loss_out + blockIdx.x, second_out ? second_out + blockIdx.x : nullptr);
}

}  // namespace loss
