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
// the same expert.  Counts are integers: nothing depends on the order of the atomics.
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
// The sorted row of a token's slot, or -1.
__device__ __forceinline__ int64_t place_of(const Move &P, int64_t slot, int64_t first)
{
    const int32_t p = P.place[slot];
    if (p < 0) return -1;
    if (p >= first && p < first + P.slots) return p;
    report(P.status);
    return -1;
}

constexpr int MOVE_THREADS = 256;
// A wave has a token.
template <class E>
__global__ __launch_bounds__(MOVE_THREADS) void gather_kernel(Move P)
{
    constexpr int N = Piece<E>::N;
    const int64_t r = group_number() * (MOVE_THREADS / 64) + (threadIdx.x >> 6);
    if (r >= P.rows) return;
    const int64_t first = r / P.per_worker * P.slots;
    for (int c = (threadIdx.x & 63) * N; c < P.width; c += 64 * N) {
        const u32x4 w = load_piece<E>((const E *)P.tokens + r * P.ld, c, P.width);
        for (int j = 0; j < P.k; ++j) {
            const int64_t p = place_of(P, r * P.k + j, first);
            if (p >= 0) store_piece<E>((E *)P.sorted_out + p * P.ld_sorted, c, P.width, w);
        }
    }
}
template <class E>
__global__ __launch_bounds__(MOVE_THREADS) void combine_kernel(Move P)
{
    constexpr int N = Piece<E>::N;
    const int64_t r = group_number() * (MOVE_THREADS / 64) + (threadIdx.x >> 6);
    if (r >= P.rows) return;
    const int64_t first = r / P.per_worker * P.slots;
    for (int c = (threadIdx.x & 63) * N; c < P.width; c += 64 * N) {
        float v[N], z[N];
        for (int i = 0; i < N; ++i) v[i] = 0.f;
        for (int j = 0; j < P.k; ++j) {
            const int64_t p = place_of(P, r * P.k + j, first);
            if (p < 0) continue;
            const float w = P.weights ? P.weights[r * P.k + j] : 1.f;
            Piece<E>::unpack(load_piece<E>((const E *)P.sorted_in + p * P.ld_sorted, c, P.width), z);
            for (int i = 0; i < N; ++i) v[i] = fmaf(w, z[i], v[i]);
        }
        store_piece<E>((E *)P.out + r * P.ld, c, P.width, Piece<E>::pack(v));
    }
}
template <class E>
__global__ __launch_bounds__(MOVE_THREADS) void combine_grad_kernel(Move P)
{
    constexpr int N = Piece<E>::N;
    const int64_t r = group_number() * (MOVE_THREADS / 64) + (threadIdx.x >> 6);
    if (r >= P.rows) return;
    const int64_t first = r / P.per_worker * P.slots;
    for (int j = 0; j < P.k; ++j) {
        const int64_t slot = r * P.k + j, p = place_of(P, slot, first);
        float dot = 0.f;
        if (p >= 0) {
            const float w = P.weights ? P.weights[slot] : 1.f;
            for (int c = (threadIdx.x & 63) * N; c < P.width; c += 64 * N) {
                float d[N], z[N];
                Piece<E>::unpack(load_piece<E>((const E *)P.tokens + r * P.ld, c, P.width), d);
                if (P.dweights) {
                    Piece<E>::unpack(load_piece<E>((const E *)P.sorted_in + p * P.ld_sorted, c, P.width), z);
                    float part = 0.f;
                    for (int i = 0; i < N; ++i) part = fmaf(d[i], z[i], part);
                    dot += part;
                }
                for (int i = 0; i < N; ++i) d[i] *= w;
                store_piece<E>((E *)P.sorted_out + p * P.ld_sorted, c, P.width, Piece<E>::pack(d));
            }
        }
        if (P.dweights) {
            dot = loss::lanes_sum<64>(dot);
            if ((threadIdx.x & 63) == 0) P.dweights[slot] = dot;
        }
    }
}

}  // namespace layer
