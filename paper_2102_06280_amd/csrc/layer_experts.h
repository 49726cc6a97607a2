// Tokens sorted by expert and back (dbw_layers.h).
#pragma once

#include "layer_rows.h"

namespace layer {

struct Sort {
    const int32_t *expert;
    int32_t *start, *place, *source, *status;
    int32_t *counts;                                      // [worker][chunk][E], where a worker's slots are several workgroups'
    int64_t workers;
    int slots, experts;                                   // of a worker
    int chunk, chunks;                                    // slots of a workgroup, workgroups of a worker
};
constexpr int SORT_WAVES = 8, SORT_THREADS = 64 * SORT_WAVES;

__device__ __forceinline__ int expert_of(const Sort &P, int64_t slot)
{
    const int e = P.expert[slot];
    if (e < P.experts) return e < 0 ? -1 : e;
    report(P.status);
    return -1;
}

// How many slots of a chunk name each expert.
__global__ __launch_bounds__(SORT_THREADS) void sort_count_kernel(Sort P)
{
    extern __shared__ int32_t count[];                    // [E]
    const int64_t group = group_number();
    const int64_t worker = group / P.chunks;
    const int chunk = (int)(group % P.chunks);
    if (worker >= P.workers) return;
    for (int e = threadIdx.x; e < P.experts; e += SORT_THREADS) count[e] = 0;
    __syncthreads();
    const int64_t base = worker * P.slots + (int64_t)chunk * P.chunk;
    const int length = min(P.chunk, P.slots - chunk * P.chunk);
    for (int s = threadIdx.x; s < length; s += SORT_THREADS) {
        const int e = expert_of(P, base + s);
        if (e >= 0) atomicAdd(&count[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < P.experts; e += SORT_THREADS) P.counts[group * P.experts + e] = count[e];
}

// A chunk's slots to their rows.  A wave has a contiguous part of the chunk and counts its experts; an expert's rows begin behind those of
// smaller ones, within them a chunk's behind earlier chunks', a wave's behind earlier waves', and a lane's behind the lower lanes that name
// the same expert.  Counts are integers: nothing depends on the order of the atomics.  The latency of two launches bounds it (4 x 8192 slots 4.6 and 5.1 us), or
// of one (a chunk's slots or fewer, 3.9).
__global__ __launch_bounds__(SORT_THREADS) void sort_kernel(Sort P)
{
    extern __shared__ int32_t count[];                    // [waves][E], and a number a wave
    const int64_t group = group_number();
    const int64_t worker = group / P.chunks;
    const int chunk = (int)(group % P.chunks);
    if (worker >= P.workers) return;
    const int E = P.experts, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    int32_t *const mine = count + wave * E, *const totals = count + SORT_WAVES * E;
    const int begin = chunk * P.chunk, length = min(P.chunk, P.slots - begin);
    const int part = ((length + SORT_WAVES - 1) / SORT_WAVES + 63) / 64 * 64;
    const int first = min(wave * part, length), last = min(first + part, length);
    const int64_t base = worker * P.slots, mid = base + begin;     // the worker's and the chunk's first slot
    for (int e = threadIdx.x; e < SORT_WAVES * E; e += SORT_THREADS) count[e] = 0;
    __syncthreads();
    for (int s = first + lane; s < last; s += 64) {
        const int e = expert_of(P, mid + s);
        if (e >= 0) atomicAdd(&mine[e], 1);
    }
    __syncthreads();
    // SORT_THREADS experts at a time: rows of all slots, and those before this chunk's
    int before = 0;                                       // rows of the experts of earlier turns
    for (int e0 = 0; e0 < E; e0 += SORT_THREADS) {
        const int e = e0 + (int)threadIdx.x;
        int all = 0, earlier = 0;
        if (e < E) {
            if (P.chunks == 1)
                for (int w = 0; w < SORT_WAVES; ++w) all += count[w * E + e];
            else
#pragma unroll 8
                for (int c = 0; c < P.chunks; ++c) {
                    const int n = P.counts[(worker * P.chunks + c) * E + e];
                    all += n;
                    if (c < chunk) earlier += n;
                }
        }
        int upto = all;                                   // the sum over lanes up to this one
        for (int d = 1; d < 64; d <<= 1) {
            const int v = __shfl_up(upto, d);
            if (lane >= d) upto += v;
        }
        if (lane == 63) totals[wave] = upto;
        __syncthreads();
        int here = before + upto - all;
        for (int w = 0; w < SORT_WAVES; ++w) {
            if (w < wave) here += totals[w];
            before += totals[w];
        }
        if (e < E) {
            if (chunk == 0) P.start[worker * (E + 1) + e] = (int32_t)(base + here);
            here += earlier;
            for (int w = 0; w < SORT_WAVES; ++w) {
                const int n = count[w * E + e];
                count[w * E + e] = here;
                here += n;
            }
        }
        __syncthreads();
    }
    if (chunk == 0 && threadIdx.x == 0) P.start[worker * (E + 1) + E] = (int32_t)(base + before);
    for (int s = threadIdx.x; s < length; s += SORT_THREADS)
        if (begin + s >= before) P.source[mid + s] = -1;
    for (int s0 = first; s0 < last; s0 += 64) {
        const int s = s0 + lane;
        const int e = s < last ? expert_of(P, mid + s) : -1;
        uint64_t same = __ballot(e >= 0);
        for (int bit = 1; bit < E; bit <<= 1) {
            const uint64_t set = __ballot(e >= 0 && (e & bit));
            same &= e >= 0 && (e & bit) ? set : ~set;
        }
        const int rank = __popcll(same & (((uint64_t)1 << lane) - 1));
        int row = -1;
        if (e >= 0) row = mine[e] + rank;
        loss::row_barrier<64>();
        if (e >= 0 && rank == 0) mine[e] += __popcll(same);
        loss::row_barrier<64>();
        if (s < last) P.place[mid + s] = e >= 0 ? (int32_t)(base + row) : -1;
        if (e >= 0) P.source[base + row] = (int32_t)(mid + s);
    }
}

// ---------------------------------------------------------------- rows of tokens and sorted rows

struct Move {
    const void *tokens;                                   // x, or dy
    void *out;                                            // y
    const void *sorted_in;
    void *sorted_out;
    const int32_t *place;
    const float *weights;
    float *dweights;
    int32_t *status;
    int64_t ld, ld_sorted, rows;                          // rows: tokens of all workers
    int64_t slots;                                        // of a worker
    int per_worker, width, k;
};

// Memory bounds all of these: 4 x 4096 x 2048 bf16, two of 16 experts, gathered in 36 us (201 MB, 5.6 TB/s), combined in 36 (5.6), gradient 60 (336 MB, 5.6).
//
// A wave has a token, or some of its columns, C pieces a lane at a time.  Of up to 64 slots of the token each lane has one: its sorted row, or -1, and its
// weight, which go to the whole wave when they are used.
constexpr int MOVE_WAVES = 4, MOVE_THREADS = 64 * MOVE_WAVES;
struct Token {
    int64_t row;
    int chunk;                                            // of its columns
};
__device__ __forceinline__ Token token_of(uint32_t chunks)
{
    const int64_t wave = group_number() * MOVE_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (chunks == 1) return Token{wave, 0};
    return Token{wave / chunks, (int)(wave % chunks)};
}
struct Slots {
    int place;
    float weight;
    __device__ __forceinline__ Slots(const Move &P, int64_t row, int first_slot)
    {
        const int j = first_slot + (threadIdx.x & 63);
        const int64_t slot = row * P.k + j, first = (uint32_t)row / (uint32_t)P.per_worker * P.slots;
        place = -1;
        weight = 0.f;
        if (j >= P.k) return;
        const int32_t p = ((const __attribute__((address_space(1))) int32_t *)(uint64_t)P.place)[slot];
        weight = P.weights ? ((const __attribute__((address_space(1))) float *)(uint64_t)P.weights)[slot] : 1.f;
        if (p >= first && p < first + P.slots) place = p;
        else if (p >= 0) report(P.status);
    }
    __device__ __forceinline__ int place_of(int j) const { return __builtin_amdgcn_readlane(place, j); }
    __device__ __forceinline__ float weight_of(int j) const { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(weight), j)); }
};

template <class E, int C>
__global__ __launch_bounds__(MOVE_THREADS) void gather_kernel(Move P, int chunks)
{
    constexpr int N = Piece<E>::N;
    const Token token = token_of(chunks);
    if (token.row >= P.rows) return;
    const int c0 = (token.chunk * C * 64 + (threadIdx.x & 63)) * N;
    u32x4 w[C];
#pragma unroll
    for (int i = 0; i < C; ++i) w[i] = load_raw<E, false>((const E *)P.tokens + token.row * P.ld, c0 + i * 64 * N, P.width);
    for (int j0 = 0; j0 < P.k; j0 += 64) {
        const Slots slots(P, token.row, j0);
        if (j0 == 0)
#pragma unroll
            for (int i = 0; i < C; ++i) w[i] = settled<E, false>(w[i], c0 + i * 64 * N, P.width);
        const int count = min(64, P.k - j0);
        for (int j = 0; j < count; ++j) {
            const int p = slots.place_of(j);
            if (p < 0) continue;
            E *const to = (E *)P.sorted_out + p * P.ld_sorted;
#pragma unroll
            for (int i = 0; i < C; ++i) store_piece<E>(to, c0 + i * 64 * N, P.width, w[i]);
        }
    }
}

constexpr int TOGETHER = 2;                               // slots whose rows are asked for before the first is used
template <class E, int C>
__global__ __launch_bounds__(MOVE_THREADS) void combine_kernel(Move P, int chunks)
{
    constexpr int N = Piece<E>::N;
    const Token token = token_of(chunks);
    if (token.row >= P.rows) return;
    const int c0 = (token.chunk * C * 64 + (threadIdx.x & 63)) * N;
    float v[C][N] = {};
    for (int j0 = 0; j0 < P.k; j0 += 64) {
        const Slots slots(P, token.row, j0);
        const int count = min(64, P.k - j0);
        for (int j = 0; j < count; j += TOGETHER) {
            u32x4 z[TOGETHER][C];
#pragma unroll
            for (int q = 0; q < TOGETHER; ++q) {
                const int p = j + q < count ? slots.place_of(j + q) : -1;
#pragma unroll
                for (int i = 0; i < C; ++i) z[q][i] = (u32x4)0u;
                if (p >= 0)
#pragma unroll
                    for (int i = 0; i < C; ++i) z[q][i] = load_raw<E, false>((const E *)P.sorted_in + p * P.ld_sorted, c0 + i * 64 * N, P.width);
            }
#pragma unroll
            for (int q = 0; q < TOGETHER; ++q) {
                if (j + q >= count || slots.place_of(j + q) < 0) continue;
                const float by = slots.weight_of(j + q);
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    float x[N];
                    Piece<E>::unpack(settled<E, false>(z[q][i], c0 + i * 64 * N, P.width), x);
#pragma unroll
                    for (int n = 0; n < N; ++n) v[i][n] = fmaf(by, x[n], v[i][n]);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < C; ++i) store_piece<E>((E *)P.out + token.row * P.ld, c0 + i * 64 * N, P.width, Piece<E>::pack(v[i]));
}

// Here a wave has the whole token, or, where there are few, a workgroup (WAVES of them); as many columns at a time as the lanes hold.  What they have of a few
// slots' products is summed in the end.
template <class E, int C, int WAVES>
__global__ __launch_bounds__(MOVE_THREADS) void combine_grad_kernel(Move P)
{
    constexpr int N = Piece<E>::N, Q = 2, T = 64 * WAVES;  // Q: slots at a time
    __shared__ float sums[2][WAVES][Q];
    const int64_t row = WAVES == 1 ? token_of(1).row : group_number();
    if (row >= P.rows) return;
    const int t = threadIdx.x % T;
    const E *const dy = (const E *)P.tokens + row * P.ld;
    int turn = 0;
    for (int j0 = 0; j0 < P.k; j0 += 64) {
        const Slots slots(P, row, j0);
        const int count = min(64, P.k - j0);
        float mine = 0.f;                                 // of the slot that is the lane's
        for (int j = 0; j < count; j += Q) {
            int p[Q];
            float dot[Q] = {};
            for (int q = 0; q < Q; ++q) p[q] = j + q < count ? slots.place_of(j + q) : -1;
            for (int c0 = t * N; c0 < P.width; c0 += C * T * N) {
                u32x4 d[C], z[Q][C];
#pragma unroll
                for (int i = 0; i < C; ++i) d[i] = load_raw<E, false>(dy, c0 + i * T * N, P.width);
                if (P.dweights)
#pragma unroll
                    for (int q = 0; q < Q; ++q)
                        if (p[q] >= 0)
#pragma unroll
                            for (int i = 0; i < C; ++i)
                                z[q][i] = load_raw<E, false>((const E *)P.sorted_in + p[q] * P.ld_sorted, c0 + i * T * N, P.width);
                float g[C][N];
#pragma unroll
                for (int i = 0; i < C; ++i) Piece<E>::unpack(settled<E, false>(d[i], c0 + i * T * N, P.width), g[i]);
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    if (p[q] < 0) continue;
                    const float by = slots.weight_of(j + q);
                    float part = 0.f;
#pragma unroll
                    for (int i = 0; i < C; ++i) {
                        const int c = c0 + i * T * N;
                        float x[N];
                        if (P.dweights) {
                            Piece<E>::unpack(settled<E, false>(z[q][i], c, P.width), x);
#pragma unroll
                            for (int n = 0; n < N; ++n) part = fmaf(g[i][n], x[n], part);
                        }
#pragma unroll
                        for (int n = 0; n < N; ++n) x[n] = by * g[i][n];
                        store_piece<E>((E *)P.sorted_out + p[q] * P.ld_sorted, c, P.width, Piece<E>::pack(x));
                    }
                    dot[q] += part;
                }
            }
            if (!P.dweights) continue;
#pragma unroll
            for (int q = 0; q < Q; ++q) dot[q] = loss::lanes_sum<64>(dot[q]);
            if (WAVES > 1) {
                if ((threadIdx.x & 63) == 0)
#pragma unroll
                    for (int q = 0; q < Q; ++q) sums[turn][threadIdx.x >> 6][q] = dot[q];
                __syncthreads();
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    dot[q] = sums[turn][0][q];
                    for (int w = 1; w < WAVES; ++w) dot[q] += sums[turn][w][q];
                }
                turn ^= 1;
            }
#pragma unroll
            for (int q = 0; q < Q; ++q)
                if (t == j + q) mine = dot[q];
        }
        if (P.dweights && t < count) ((__attribute__((address_space(1))) float *)(uint64_t)P.dweights)[row * P.k + j0 + t] = mine;
    }
}

// Rows of up to 256 bytes: 16 lanes a token, a piece each, and a few slots at a time.  24 x 2351 x 16 fp16
// with four slots there and back 24.6 us, by a wave a token 50.4.
constexpr int NARROW_BYTES = 256, NARROW_TOKENS = MOVE_THREADS / 16, NARROW_SLOTS = 4;
struct NarrowSlots {
    int64_t place[NARROW_SLOTS];
    float weight[NARROW_SLOTS];
    __device__ __forceinline__ NarrowSlots(const Move &P, int64_t row, int j0)
    {
        const int64_t first = (uint32_t)row / (uint32_t)P.per_worker * P.slots;
#pragma unroll
        for (int q = 0; q < NARROW_SLOTS; ++q) {
            const int64_t slot = row * P.k + min(j0 + q, P.k - 1);
            place[q] = ((const __attribute__((address_space(1))) int32_t *)(uint64_t)P.place)[slot];
            weight[q] = P.weights ? ((const __attribute__((address_space(1))) float *)(uint64_t)P.weights)[slot] : 1.f;
        }
#pragma unroll
        for (int q = 0; q < NARROW_SLOTS; ++q) {
            const bool there = place[q] >= first && place[q] < first + P.slots;
            if (place[q] >= 0 && !there) report(P.status);
            if (!there || j0 + q >= P.k) place[q] = -1;
        }
    }
};
enum { GATHER, COMBINE, COMBINE_GRAD };
template <class E, int WHAT>
__global__ __launch_bounds__(MOVE_THREADS) void narrow_kernel(Move P)
{
    constexpr int N = Piece<E>::N;
    const int64_t row = group_number() * NARROW_TOKENS + (threadIdx.x >> 4);
    if (row >= P.rows) return;
    const int c = (threadIdx.x & 15) * N;
    u32x4 raw = (u32x4)0u;
    if (WHAT != COMBINE) raw = load_piece<E>((const E *)P.tokens + row * P.ld, c, P.width);
    float g[N], v[N] = {};
    Piece<E>::unpack(raw, g);
    for (int j0 = 0; j0 < P.k; j0 += NARROW_SLOTS) {
        const NarrowSlots slots(P, row, j0);
        u32x4 z[NARROW_SLOTS];
        const bool reads = WHAT == COMBINE || (WHAT == COMBINE_GRAD && P.dweights);
#pragma unroll
        for (int q = 0; q < NARROW_SLOTS; ++q) {
            z[q] = (u32x4)0u;
            if (reads && slots.place[q] >= 0) z[q] = load_raw<E, false>((const E *)P.sorted_in + slots.place[q] * P.ld_sorted, c, P.width);
        }
#pragma unroll
        for (int q = 0; q < NARROW_SLOTS; ++q) {
            const bool there = slots.place[q] >= 0;
            float x[N];
            Piece<E>::unpack(settled<E, false>(z[q], c, P.width), x);
            if (WHAT == COMBINE && there)
#pragma unroll
                for (int n = 0; n < N; ++n) v[n] = fmaf(slots.weight[q], x[n], v[n]);
            if (WHAT == COMBINE_GRAD && P.dweights) {
                float dot = 0.f;
#pragma unroll
                for (int n = 0; n < N; ++n) dot = fmaf(g[n], x[n], dot);
                dot = loss::lanes_sum<16>(dot);
                if ((threadIdx.x & 15) == 0 && j0 + q < P.k)
                    ((__attribute__((address_space(1))) float *)(uint64_t)P.dweights)[row * P.k + j0 + q] = there ? dot : 0.f;
            }
            if (WHAT != COMBINE && there) {
                if (WHAT == COMBINE_GRAD)
#pragma unroll
                    for (int n = 0; n < N; ++n) x[n] = slots.weight[q] * g[n];
                store_piece<E>((E *)P.sorted_out + slots.place[q] * P.ld_sorted, c, P.width, WHAT == GATHER ? raw : Piece<E>::pack(x));
            }
        }
    }
    if (WHAT == COMBINE) store_piece<E>((E *)P.out + row * P.ld, c, P.width, Piece<E>::pack(v));
}

}  // namespace layer
