// The weight gradient of a linear layer whose input was kept in 8 bits (dbw_layers.h).
#pragma once

#include "layer_rows.h"

namespace layer {

struct Linear {
    const void *dy;
    Kept kept;
    const int32_t *start, *source;
    int32_t *status;
    float *grads;
    int64_t ld, ld_grads, weight_at, bias_at;
    int64_t workers;
    int rows, in, out, experts, tokens, k;                // rows, tokens: of a worker
};
// The rows of dy of a worker's layer.
struct Range {
    int64_t first, end;
};
__device__ __forceinline__ Range range_of(const Linear &P, int64_t worker, int expert)
{
    const int64_t low = worker * P.rows, high = low + P.rows;
    if (!P.start) return Range{low, high};
    const int64_t at = worker * (P.experts + 1) + expert, a = P.start[at], b = P.start[at + 1];
    if (a >= low && b <= high && a <= b) return Range{a, b};
    report(P.status);
    return Range{low, low};
}
// The checkpoint's row of a row of dy, or -1.
__device__ __forceinline__ int64_t input_row(const Linear &P, int64_t worker, int64_t row)
{
    if (!P.source) return row;
    const int64_t low = worker * P.tokens;
    const int32_t slot = P.source[row];
    const int64_t r = slot < 0 ? -1 : slot / P.k;
    if (r >= low && r < low + P.tokens) return r;
    report(P.status);
    return -1;
}

constexpr int TILE = 64, STEP = 16;
template <class E>
__global__ __launch_bounds__(256) void weight_grad_kernel(Linear P, int tiles_out, int tiles_in)
{
    __shared__ float d[STEP][TILE], x[STEP][TILE];
    const int64_t group = group_number();
    const int64_t layer = group / ((int64_t)tiles_out * tiles_in);
    const int tile = (int)(group % ((int64_t)tiles_out * tiles_in));
    const int64_t worker = layer / P.experts;
    const int expert = (int)(layer % P.experts);
    if (worker >= P.workers) return;
    const int o0 = tile / tiles_in * TILE, i0 = tile % tiles_in * TILE;
    const Range range = range_of(P, worker, expert);
    const int column = threadIdx.x % TILE, q = threadIdx.x / TILE, to = threadIdx.x / 16 * 4, ti = threadIdx.x % 16 * 4;
    float acc[4][4] = {}, bias[4] = {};
    for (int64_t r0 = range.first; r0 < range.end; r0 += STEP) {
        __syncthreads();
        for (int s = q; s < STEP; s += 256 / TILE) {
            const int64_t r = r0 + s;
            const int64_t in = r < range.end ? input_row(P, worker, r) : -1;
            d[s][column] = in >= 0 && o0 + column < P.out ? loss::widen(((const E *)P.dy)[r * P.ld + o0 + column]) : 0.f;
            float v[4] = {0.f, 0.f, 0.f, 0.f};
            if (in >= 0 && i0 + column < P.in) {
                const int c = i0 + column;
                const float by = power_of_two((int)P.kept.exponents[in * (P.kept.stride / BLOCK) + c / BLOCK] - 127);
                decode4(P.kept.codes[in * P.kept.stride + c], by, v);
            }
            x[s][column] = v[0];
        }
        __syncthreads();
        for (int s = 0; s < STEP; ++s)
            for (int a = 0; a < 4; ++a) {
                const float g = d[s][to + a];
                bias[a] += g;
                for (int b = 0; b < 4; ++b) acc[a][b] = fmaf(g, x[s][ti + b], acc[a][b]);
            }
    }
    float *const grads = P.grads + worker * P.ld_grads;
    for (int a = 0; a < 4; ++a) {
        const int o = o0 + to + a;
        if (o >= P.out) continue;
        for (int b = 0; b < 4; ++b)
            if (i0 + ti + b < P.in) grads[P.weight_at + ((int64_t)expert * P.out + o) * P.in + i0 + ti + b] = acc[a][b];
        if (i0 == 0 && ti == 0 && P.bias_at >= 0) grads[P.bias_at + (int64_t)expert * P.out + o] = bias[a];
    }
}

}  // namespace layer
