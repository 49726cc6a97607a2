// The weight gradient of a linear layer whose input was kept in 8 bits (dbw_layers.h): dW = sum over rows of dy x'.
//
// What a code stands for is exact in bf16, and so is dy as one (bf16), two (fp16) or three (fp32) bf16 numbers: every product on the bf16
// matrix instruction is exact, and fp32 sums are all that rounds.
//
// 4 x 4096 x 2048 x 2048 bf16 135 us (1.02 PFLOP/s; the library's bf16 product of these sizes, without the decoding, takes 105), matrix cores busy 41 %, LDS
// 31 %, vector units 29 % of the time under a profiler: what is left are waits, with two waves a SIMD and a barrier every 32 rows.  fp16 and fp32 take two and three
// products for one: 2 x 4096 x 2048 x 2048 125 and 178 us.  Short batches are bound by writing dW, workgroup after workgroup (1 x 300 x 4096 x 4096 24 us,
// 67 MB).  Tried without gain: wave priorities, four waves of 128 x 128 (spilled), tiles of 128 x 128 with two workgroups a compute unit (216), the
// next rows put into LDS at a step's beginning or end (within 2 %).
#pragma once

#include <algorithm>
#include <type_traits>

#include "layer_rows.h"

namespace layer {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char *lds_bytes;

struct Linear {
    const void *dy;
    Kept kept;
    const int32_t *start, *source;
    int32_t *status;
    float *grads;
    int64_t ld, ld_grads, weight_at, bias_at;
    int64_t workers;
    int rows, in, out, experts, tokens, k;                // rows, tokens: of a worker
    int tiles_out, tiles_in, splits;
    float *parts;                                         // [split][weights of all layers, then their biases], where the rows are split
};
// The rows of dy of a worker's layer.
struct Range {
    int64_t first, end;
};
__device__ __forceinline__ Range range_of(const Linear &P, int64_t worker, int expert)
{
    const int64_t low = worker * P.rows, high = low + P.rows;
    if (!P.start) return Range{low, high};
    const auto start = (const __attribute__((address_space(1))) int32_t *)(uint64_t)P.start;
    const int64_t at = worker * (P.experts + 1) + expert, a = start[at], b = start[at + 1];
    if (a >= low && b <= high && a <= b) return Range{a, b};
    report(P.status);
    return Range{low, low};
}
// The checkpoint's row that belongs to a slot, or -1.
__device__ __forceinline__ int input_row(const Linear &P, int64_t worker, int32_t slot)
{
    const int64_t low = worker * P.tokens;
    const int r = slot < 0 ? -1 : slot / P.k;
    if (r >= low && r < low + P.tokens) return r;
    report(P.status);
    return -1;
}

// A workgroup's tile.  Workgroups go to the XCDs in turn, each with an L2 of its own: an XCD gets tiles that follow one another, which read the same rows
// (4 x 4096 x 2048 x 2048 bf16 145 us, tiles to the XCDs in turn 153).  With experts the work of a workgroup is what its expert has of rows; so
// every layer's tiles are shared out to all XCDs, and the workers' longest layers come first (2 x 4096 x 1024 x 2048, two of eight experts, the most popular
// four times as popular as the least: 140 us, in the experts' own order 174), which a wave finds by counting, up to 64 experts.
constexpr int XCDS = 8, SORTED_EXPERTS = 64;
struct Share {
    int64_t worker;
    int expert, split, tile;
    Range range;
};
__device__ __forceinline__ int64_t from_lane(int64_t v, int lane)
{
    const uint32_t low = __builtin_amdgcn_readlane((int)v, lane), high = __builtin_amdgcn_readlane((int)(v >> 32), lane);
    return (int64_t)((uint64_t)high << 32 | low);
}
__device__ __forceinline__ bool share_of(const Linear &P, Share &s)
{
    // (as many workgroups as there are tiles to write: far below 2^32)
    const uint32_t per_layer = (uint32_t)P.tiles_out * (uint32_t)P.tiles_in, workers = (uint32_t)P.workers, splits = (uint32_t)P.splits;
    const uint32_t groups = per_layer * splits * workers * (uint32_t)P.experts;
    uint32_t group = (uint32_t)group_number();
    if (group >= groups) return false;
    if (!P.start) {
        const uint32_t xcd = group % XCDS;
        group = xcd * (groups / XCDS) + min(xcd, groups % XCDS) + group / XCDS;
    }
    s.tile = (int)(group % per_layer);
    group /= per_layer;
    s.split = (int)(group % splits);
    group /= splits;
    s.worker = group % workers;
    s.expert = (int)(group / workers);
    if (P.start && per_layer % XCDS == 0) s.tile = s.tile % XCDS * (int)(per_layer / XCDS) + s.tile / XCDS;
    if (!P.start || P.experts == 1 || P.experts > SORTED_EXPERTS) {
        s.range = range_of(P, s.worker, s.expert);
        return true;
    }
    // the layer that has as many longer ones before it as `expert` says
    const int lane = threadIdx.x & 63;
    Range mine{0, -1};
    if (lane < P.experts) mine = range_of(P, s.worker, lane);
    const int length = (int)(mine.end - mine.first);
    int longer = 0;
    for (int e = 0; e < P.experts; ++e) {
        const int other = __builtin_amdgcn_readlane(length, e);
        longer += other > length || (other == length && e < lane);
    }
    s.expert = __builtin_ctzll(__ballot(lane < P.experts && longer == s.expert));
    s.range = Range{from_lane(mine.first, s.expert), from_lane(mine.end, s.expert)};
    return true;
}

// A piece of dy as bf16 planes, the large parts first.
template <class E>
struct Planes;
template <>
struct Planes<bf16> {
    static constexpr int COUNT = 1;
    static __device__ __forceinline__ void split(const u32x4 &w, u32x4 (&p)[1]) { p[0] = w; }
};
__device__ __forceinline__ uint32_t nearest(float a, float b)
{
    const bf16x2 r = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ float low_half(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_half(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// What is left of v without its larger part; nothing of an infinity, and of NaN NaN (whose upper half may be that of an infinity).
__device__ __forceinline__ float rest_of(float v, float part) { return fabsf(v) == INFINITY ? 0.f : v - part; }
template <>
struct Planes<f16> {                                      // 11 bits: the nearest eight and what is left
    static constexpr int COUNT = 2;
    static __device__ __forceinline__ void split(const u32x4 &w, u32x4 (&p)[2])
    {
        float v[8];
        Piece<f16>::unpack(w, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[0][i] = nearest(v[2 * i], v[2 * i + 1]);
            p[1][i] = nearest(rest_of(v[2 * i], low_half(p[0][i])), rest_of(v[2 * i + 1], high_half(p[0][i])));
        }
    }
};
template <>
struct Planes<float> {                                    // 24 bits: the upper eight towards zero, so that they stay finite, the nearest eight of the rest,
                                                          // and what is left
    static constexpr int COUNT = 3;
    static __device__ __forceinline__ void split(const u32x4 &w, u32x2 (&p)[3])
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float a = __uint_as_float(w[2 * i]), b = __uint_as_float(w[2 * i + 1]);
            p[0][i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x07060302u);
            const float c = rest_of(a, high_half(w[2 * i])), d = rest_of(b, high_half(w[2 * i + 1]));
            p[1][i] = nearest(c, d);
            p[2][i] = nearest(c - low_half(p[1][i]), d - high_half(p[1][i]));
        }
    }
};

// Tiles in LDS: rows of COLUMNS bf16, in units of 16 columns.  The transposing read takes of 16 lanes four rows' 32 bytes each, a
// matrix instruction's operand four such blocks, of four rows by two units and of another four rows.  Units of neighbouring rows are
// exchanged so that those of half a wave lie on different banks.
template <int COLUMNS>
__device__ __forceinline__ int unit_place(int row, int unit)
{
    static_assert(COLUMNS >= 64, "four units at least");
    return unit ^ (COLUMNS >= 128 ? 2 * (row & 3) : 2 * ((row >> 1) & 1));
}
template <int COLUMNS>
__device__ __forceinline__ int lds_offset(int row, int column)     // column: a multiple of 4
{
    return row * (COLUMNS * 2) + unit_place<COLUMNS>(row, column >> 4) * 32 + (column & 15) * 2;
}
// An operand of v_mfma_f32_32x32x16_bf16 from 16 rows: a lane has column l % 32, and of its eight numbers the first four are those of rows 4 (l / 32)
// and on, the others of rows 8 + 4 (l / 32) and on.  (Both operands take the rows in this order.)  Where in a tile a lane reads for the columns from
// `column` on, of rows 0 to 15; other sixteens lie 16 rows further.
template <int COLUMNS>
__device__ __forceinline__ int operand_place(int column)
{
    const int l = threadIdx.x & 63, i = l & 15;
    return lds_offset<COLUMNS>(4 * (l >> 5) + (i >> 2), column + 16 * ((l >> 4) & 1) + 4 * (i & 3));
}
template <int COLUMNS>
__device__ __forceinline__ bf16x8 operand(lds_bytes at)
{
    typedef __attribute__((address_space(3))) s16x4 *place;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((place)at);
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((place)(at + 8 * COLUMNS * 2));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// A workgroup's tile: OUT x IN of a layer's weights, by WO x WI waves, STEP rows at a time.
template <int OUT_, int IN_, int WO_, int WI_, int STEP_>
struct Tile {
    static constexpr int OUT = OUT_, IN = IN_, WO = WO_, WI = WI_, STEP = STEP_;
    static constexpr int THREADS = 64 * WO * WI;
};
constexpr int BUFFERS = 3, LINE = 128;                    // LINE: bytes of a cache line
template <class E, class T>
constexpr int tile_lds() { return BUFFERS * T::STEP * 2 * (Planes<E>::COUNT * T::OUT + T::IN) + 4 * T::STEP * 4; }

template <class E, class T, bool SOURCED>
__global__ __launch_bounds__(T::THREADS) void weight_grad_kernel(Linear P)
{
    constexpr int N = Piece<E>::N, PLANES = Planes<E>::COUNT;
    constexpr int A_PIECES = T::OUT / N, A_ROWS = T::THREADS / A_PIECES, A_COUNT = T::STEP / A_ROWS;
    constexpr int B_PIECES = T::IN / 16, B_ROWS = std::min(T::THREADS / B_PIECES, T::STEP), B_COUNT = T::STEP / B_ROWS;
    constexpr bool B_ALL = B_PIECES * B_ROWS == T::THREADS;          // or the first threads only
    static_assert(A_COUNT * A_ROWS == T::STEP && B_COUNT * B_ROWS == T::STEP, "whole turns");
    constexpr int MI = T::OUT / T::WO / 32, NI = T::IN / T::WI / 32;
    constexpr int A_BYTES = T::STEP * T::OUT * 2, B_BYTES = T::STEP * T::IN * 2, BUFFER = PLANES * A_BYTES + B_BYTES;
    extern __shared__ char shared[];
    const lds_bytes lds = (lds_bytes)shared;
    int32_t *const rows_of = (int32_t *)(shared + BUFFERS * BUFFER);       // [4][STEP]: the checkpoint's rows

    Share mine;
    if (!share_of(P, mine)) return;
    const int tile = mine.tile, split = mine.split, expert = mine.expert;
    const int64_t worker = mine.worker;
    const int o0 = tile / P.tiles_in * T::OUT, i0 = tile % P.tiles_in * T::IN;
    Range range = mine.range;
    if (P.tokens == 0 && range.end > range.first) {       // (no row of the checkpoint is any of these rows')
        range.end = range.first;
        report(P.status);
    }
    if (P.splits > 1) {
        const int64_t part = ((range.end - range.first + P.splits - 1) / P.splits + T::STEP - 1) / T::STEP * T::STEP;
        range.first = min(range.first + split * part, range.end);
        range.end = min(range.first + part, range.end);
    }
    const uint32_t length = (uint32_t)(range.end - range.first), steps = (length + T::STEP - 1) / T::STEP;    // (rows beyond it: below 2^32)

    const int t = threadIdx.x;
    const int ac = t % A_PIECES * N, ar = t / A_PIECES, bc = t % B_PIECES * 16, br = B_ALL ? t / B_PIECES : min(t / B_PIECES, B_ROWS - 1);
    const bool a_in = o0 + ac < P.out, b_in = i0 + bc < P.kept.stride;
    const int64_t exponents_stride = P.kept.stride / BLOCK;
    const int b_column = min(i0 + bc, (int)P.kept.stride - 16);
    // A step's rows on their way to LDS, and what of them counts.
    struct Staged {
        u32x4 a[A_COUNT], b[B_COUNT];
        uint32_t e[B_COUNT];
        bool a_on[A_COUNT], b_on[B_COUNT];
    };
    const bool with_bias = P.bias_at >= 0 && i0 == 0;
    float bias[N] = {};

    // The checkpoint's rows of a step, which a load goes by: read a step ahead.
    int a_row[A_COUNT], b_row[B_COUNT];
    const auto take = [&](uint32_t step) {
        if (!SOURCED) return;
#pragma unroll
        for (int i = 0; i < A_COUNT; ++i) a_row[i] = rows_of[(step & 3) * T::STEP + ar + i * A_ROWS];
#pragma unroll
        for (int i = 0; i < B_COUNT; ++i) b_row[i] = rows_of[(step & 3) * T::STEP + br + i * B_ROWS];
    };
    // Loads without a condition, of rows and columns that are there.
    const auto load = [&](Staged &to, uint32_t step) {
#pragma unroll
        for (int i = 0; i < A_COUNT; ++i) {
            const int s = ar + i * A_ROWS;
            const uint32_t at = step * T::STEP + s;
            to.a_on[i] = a_in && at < length && (!SOURCED || a_row[i] >= 0);
            to.a[i] = load_raw<E, false>((const E *)P.dy + (range.first + min(at, length - 1)) * P.ld, o0 + ac, P.out);
        }
#pragma unroll
        for (int i = 0; i < B_COUNT; ++i) {
            const int s = br + i * B_ROWS;
            const uint32_t at = step * T::STEP + s;
            const int64_t r = SOURCED ? max(b_row[i], 0) : range.first + min(at, length - 1);
            to.b_on[i] = b_in && at < length && (!SOURCED || b_row[i] >= 0);
            to.b[i] = *(const __attribute__((address_space(1))) u32x4 *)(uint64_t)(P.kept.codes + r * P.kept.stride + b_column);
            to.e[i] = *(const __attribute__((address_space(1))) uint8_t *)(uint64_t)(P.kept.exponents + r * exponents_stride + b_column / BLOCK);
        }
    };
    int a_to[A_COUNT], b_to[B_COUNT];
#pragma unroll
    for (int i = 0; i < A_COUNT; ++i) a_to[i] = lds_offset<T::OUT>(ar + i * A_ROWS, ac);
#pragma unroll
    for (int i = 0; i < B_COUNT; ++i) b_to[i] = lds_offset<T::IN>(br + i * B_ROWS, bc);
    const auto put = [&](const Staged &from, auto buffer) {
        const lds_bytes at = lds + decltype(buffer)::value * BUFFER;
#pragma unroll
        for (int i = 0; i < A_COUNT; ++i) {
            const u32x4 w = from.a_on[i] ? settled<E, false>(from.a[i], o0 + ac, P.out) : (u32x4)0u;
            if constexpr (N == 8) {
                u32x4 p[PLANES];
                Planes<E>::split(w, p);
#pragma unroll
                for (int q = 0; q < PLANES; ++q) *(__attribute__((address_space(3))) u32x4 *)(at + q * A_BYTES + a_to[i]) = p[q];
            } else {
                u32x2 p[PLANES];
                Planes<E>::split(w, p);
#pragma unroll
                for (int q = 0; q < PLANES; ++q) *(__attribute__((address_space(3))) u32x2 *)(at + q * A_BYTES + a_to[i]) = p[q];
            }
            if (with_bias) {
                float v[N];
                Piece<E>::unpack(w, v);
#pragma unroll
                for (int j = 0; j < N; ++j) bias[j] += v[j];
            }
        }
#pragma unroll
        for (int i = 0; i < B_COUNT; ++i) {
            const float by = __uint_as_float(from.e[i] << 23);
            u32x4 w[2];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t code = from.b_on[i] ? from.b[i][q] : 0u;
                w[q / 2][q % 2 * 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code, by, false));
                w[q / 2][q % 2 * 2 + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code, by, true));
            }
            const lds_bytes to = at + PLANES * A_BYTES + b_to[i];
            if (B_ALL || t < B_PIECES * B_ROWS) {
                *(__attribute__((address_space(3))) u32x4 *)to = w[0];
                *(__attribute__((address_space(3))) u32x4 *)(to + 16) = w[1];
            }
        }
    };
    // The checkpoint's rows of a step, looked up by the first threads; the next step's slots are asked for a step ahead.
    int32_t next_slot = -1;
    const auto ask = [&](uint32_t step, int threads) {
        const uint32_t s = step * T::STEP + t;
        if (t < threads && s < length) next_slot = ((const __attribute__((address_space(1))) int32_t *)(uint64_t)P.source)[range.first + s];
    };
    const auto look_up = [&](uint32_t step) {
        if (!SOURCED) return;
        if (t < T::STEP) rows_of[(step & 3) * T::STEP + t] = step * T::STEP + t < length ? input_row(P, worker, next_slot) : -1;
        ask(step + 1, T::STEP);
    };
    static_assert(4 * T::STEP <= T::THREADS, "four steps' rows at once");
    if (SOURCED) {
        ask(0, 4 * T::STEP);
        if (t < 4 * T::STEP) rows_of[t] = (uint32_t)t < length ? input_row(P, worker, next_slot) : -1;
        ask(4, T::STEP);
        __syncthreads();
    }

    f32x16 acc[MI][NI] = {};
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6), wo = wave / T::WI * (T::OUT / T::WO), wi = wave % T::WI * (T::IN / T::WI);
    int d_at[MI], x_at[NI];
#pragma unroll
    for (int i = 0; i < MI; ++i) d_at[i] = operand_place<T::OUT>(wo + 32 * i);
#pragma unroll
    for (int j = 0; j < NI; ++j) x_at[j] = operand_place<T::IN>(wi + 32 * j);
    // 16 rows' operands, and their products.
    struct Operands {
        bf16x8 x[NI], d[PLANES][MI];
    };
    const auto fetch = [&](Operands &f, auto buffer, auto row) {
        const lds_bytes at = lds + decltype(buffer)::value * BUFFER;
        constexpr int s = decltype(row)::value;
#pragma unroll
        for (int j = 0; j < NI; ++j) f.x[j] = operand<T::IN>(at + (PLANES * A_BYTES + s * T::IN * 2) + x_at[j]);
#pragma unroll
        for (int q = PLANES - 1; q >= 0; --q)
#pragma unroll
            for (int i = 0; i < MI; ++i) f.d[q][i] = operand<T::OUT>(at + (q * A_BYTES + s * T::OUT * 2) + d_at[i]);
    };
    const auto multiply = [&](const Operands &f) {
#pragma unroll
        for (int q = PLANES - 1; q >= 0; --q)
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.d[q][i], f.x[j], acc[i][j], 0, 0, 0);
    };
    // A step's rows go through three buffers: step s is multiplied, step s + 1 lies ready, so that its first operands are fetched in front of the barrier,
    // and step s + 2, which has come meanwhile, is put into the third, where step s - 1 was; step s + 3 is asked for.  Operands are fetched while the ones
    // before them are multiplied.  The rows that step s + 4 takes of the checkpoint are read from LDS and those of step s + 5 looked up, into the place that
    // step s + 3 had, read in front of the last barrier.
    Operands even, odd;
    Staged coming;
    const auto turn = [&](uint32_t step, auto buffer) {
        constexpr int B = decltype(buffer)::value;
        typedef std::integral_constant<int, (B + 1) % BUFFERS> Next;
        typedef std::integral_constant<int, (B + 2) % BUFFERS> Third;
        if constexpr (T::STEP == 32) {
            fetch(odd, buffer, std::integral_constant<int, 16>());
            multiply(even);
        } else {
            fetch(odd, buffer, std::integral_constant<int, 16>());
            multiply(even);
            fetch(even, buffer, std::integral_constant<int, 32>());
            multiply(odd);
            fetch(odd, buffer, std::integral_constant<int, 48>());
            multiply(even);
        }
        put(coming, Third());
        load(coming, step + 3);
        take(step + 4);
        look_up(step + 5);
        fetch(even, Next(), std::integral_constant<int, 0>());
        multiply(odd);
        __syncthreads();
    };
    if (steps > 0) {
        typedef std::integral_constant<int, 0> First;
        typedef std::integral_constant<int, 1> Second;
        typedef std::integral_constant<int, 2> Third;
        // (the sums' registers are free as yet)
        Staged first, second;
        take(0);
        load(first, 0);
        take(1);
        load(second, 1);
        take(2);
        load(coming, 2);
        take(3);
        put(first, First());
        put(second, Second());
        if (SOURCED) __syncthreads();                     // rows 0 have been read: rows 4 go there
        look_up(4);
        __syncthreads();
        fetch(even, First(), std::integral_constant<int, 0>());
        for (uint32_t step = 0; step < steps; step += BUFFERS) {
            turn(step, First());
            if (step + 1 < steps) turn(step + 1, Second());
            if (step + 2 < steps) turn(step + 2, Third());
        }
    }

    const int64_t layer = worker * P.experts + expert, weights = (int64_t)P.out * P.in;
    const int64_t all = P.workers * P.experts;
    float *const to = P.splits > 1 ? P.parts + split * all * (weights + P.out) + layer * weights
                                   : P.grads + worker * P.ld_grads + P.weight_at + expert * weights;
    // Sums go through LDS, 32 rows of every wave row at a time, and from there to memory as whole rows of the tile.  (From the registers, 32 columns
    // of two rows at a time, 12 x 1 x 279 x 2960 with 22 experts 448 us instead of 269: the lines that rows share were written in parts.)  Rows of whole lines go past
    // the caches, others through them, where lines that tiles share are put together: bf16, past and through, 12 x 22 layers of 4 x 512 x 2960 270 and
    // 348 us, with weights that begin 4 or 32 bytes behind a line 512 and 367; of 4 x 279 x 2960 312 and 269; 2 x 8 of 1024 x 1024 x 2048 4 bytes behind one 115 and 102;
    // 4 x 512 x 2048 x 2048 33.1 and 29.1.  (The other way round 8 x 16 of 64 x 1000 x 1000, whose rows begin on 32 bytes: 141 and 164.)
    constexpr int PITCH = T::IN + 8;                      // floats: the two rows that a wave writes at a time lie on different banks
    static_assert(T::WO * 32 * PITCH * 4 <= BUFFERS * BUFFER, "room for them");
    float *const held = (float *)shared;                  // [WO * 32][PITCH]
    const int l = t & 63;
    const bool lines = (uintptr_t)to % LINE == 0 && P.in % (LINE / 4) == 0;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        if (i > 0) __syncthreads();
#pragma unroll
        for (int v = 0; v < 16; ++v)
#pragma unroll
            for (int j = 0; j < NI; ++j)
                held[(wave / T::WI * 32 + 8 * (v / 4) + 4 * (l >> 5) + v % 4) * PITCH + wi + 32 * j + (l & 31)] = acc[i][j][v];
        __syncthreads();
        constexpr int EACH = T::IN / 4, AT_ONCE = T::THREADS / EACH;
#pragma unroll
        for (int r0 = 0; r0 < T::WO * 32; r0 += AT_ONCE) {
            const int r = r0 + t / EACH, c = t % EACH * 4, o = o0 + r / 32 * (T::OUT / T::WO) + 32 * i + r % 32;
            if (o >= P.out) continue;
            const u32x4 w = *(const u32x4 *)(held + r * PITCH + c);
            if (lines) {
                asm volatile("");                         // (around it: or both stores become one, through the caches)
                store_piece<float>(to + (int64_t)o * P.in + i0, c, P.in - i0, w);
                asm volatile("");
            } else {
                store_piece<float, false>(to + (int64_t)o * P.in + i0, c, P.in - i0, w);
            }
        }
    }
    if (with_bias) {
        // the sums of the threads that have the same columns, in their order
        float *const sums = (float *)shared;              // [A_ROWS][OUT]
        __syncthreads();
#pragma unroll
        for (int j = 0; j < N; ++j) sums[ar * T::OUT + ac + j] = bias[j];
        __syncthreads();
        float *const biases = P.splits > 1 ? P.parts + split * all * (weights + P.out) + all * weights + layer * P.out
                                           : P.grads + worker * P.ld_grads + P.bias_at + (int64_t)expert * P.out;
        for (int c = t; c < T::OUT; c += T::THREADS) {
            float v = 0.f;
            for (int r = 0; r < A_ROWS; ++r) v += sums[r * T::OUT + c];
            if (o0 + c < P.out) biases[o0 + c] = v;
        }
    }
}

// The splits' shares, in their order.
constexpr int SUM_THREADS = 256;
__global__ __launch_bounds__(SUM_THREADS) void weight_grad_sum_kernel(Linear P)
{
    const int64_t weights = (int64_t)P.experts * P.out * P.in, biases = (int64_t)P.experts * P.out, each = weights + (P.bias_at >= 0 ? biases : 0);
    const int64_t i = group_number() * SUM_THREADS + threadIdx.x;
    const int64_t worker = i / each, c = i % each;
    if (worker >= P.workers) return;
    const int64_t at = c < weights ? worker * weights + c : P.workers * weights + worker * biases + c - weights;
    float v = 0.f;
    for (int s = 0; s < P.splits; ++s) v += P.parts[s * P.workers * (weights + biases) + at];
    P.grads[worker * P.ld_grads + (c < weights ? P.weight_at + c : P.bias_at + c - weights)] = v;
}

}  // namespace layer
