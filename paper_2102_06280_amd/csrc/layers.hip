// Entry points of what lies between the products of a language model (dbw_layers.h): argument checks and launches.  No context and no
// allocation: what the kernels need beyond inputs and outputs is the caller's scratch memory.
#include <math.h>

#include <type_traits>

#include "dbw_internal.h"
#include "dbw_layers.h"
#include "layer_experts.h"
#include "layer_norm.h"
#include "layer_wgrad.h"

namespace {

constexpr int64_t MAX_GROUPS = 1 << 22;                   // workers

size_t size_of(int type) { return type == DBW_TYPE_F32 ? 4 : 2; }
bool no_type(int type) { return type < DBW_TYPE_F32 || type > DBW_TYPE_F16; }
bool off(const void *p, size_t boundary) { return (uintptr_t)p % boundary != 0; }
// A stride of which so many rows' offsets in bytes fit 64 bits.
bool too_long(int64_t ld, int64_t rows) { return ld > INT64_MAX / 8 / (rows + 1); }

template <class F>
void by_type(int type, F f)
{
    if (type == DBW_TYPE_F32) f(float());
    else if (type == DBW_TYPE_BF16) f(loss::bf16());
    else f(loss::f16());
}
dim3 grid_of(int64_t groups)
{
    const int64_t x = groups < (1 << 20) ? groups : 1 << 20;
    return dim3((uint32_t)x, (uint32_t)((groups + x - 1) / x));
}

struct Shape {
    int64_t rows, ld, ld_out;
    size_t e;                                             // bytes of an element
};
int check_shape(const dbw_rows *l, Shape *S)
{
    if (!l) return DBW_ERR_NULL;
    if (l->workers < 1 || l->rows < 0 || l->width < 1 || no_type(l->type)) return DBW_ERR_INVALID;
    S->ld = l->ld ? l->ld : l->width;
    S->ld_out = l->ld_out ? l->ld_out : S->ld;
    if (S->ld < l->width || S->ld_out < l->width) return DBW_ERR_INVALID;
    S->rows = (int64_t)l->workers * l->rows;
    S->e = size_of(l->type);
    if (l->width > DBW_LAYER_MAX_WIDTH || l->workers > MAX_GROUPS || S->rows > INT32_MAX || too_long(S->ld, S->rows) || too_long(S->ld_out, S->rows))
        return DBW_ERR_UNSUPPORTED;
    return DBW_OK;
}
// Whether arrays of rows share memory.
bool overlap(const void *a, int64_t rows_a, int64_t ld_a, const void *b, int64_t rows_b, int64_t ld_b, int64_t width, size_t e)
{
    if (!a || !b || rows_a < 1 || rows_b < 1) return false;
    const uintptr_t p = (uintptr_t)a, q = (uintptr_t)b;
    const size_t na = e * (size_t)((rows_a - 1) * ld_a + width), nb = e * (size_t)((rows_b - 1) * ld_b + width);
    return p < q + nb && q < p + na;
}
// Columns of the parameters' rows: `count` from `at` on, or none (at < 0).
bool outside(int64_t at, int64_t count, int64_t ld) { return at >= 0 && (count > ld || at > ld - count); }

layer::Kept kept_of(const void *checkpoint, const Shape &S, const dbw_rows *l) { return layer::kept_of((void *)checkpoint, S.rows, l->width); }
int64_t checkpoint_bytes(int64_t rows, int64_t width) { return rows * (layer::padded(width) + layer::padded(width) / layer::BLOCK); }

// Which kernel takes a row of a norm: T threads, C pieces each, SLOTS such groups of threads in a workgroup, R rows of a group at a time backwards (forwards one).  A wave a row as long
// as its registers hold it: no barriers.  Microseconds when the plans were chosen, workers x rows x width, bf16 unless said otherwise: forwards
// 8 x 2048 x 2048 by a wave 23.5, by 256 threads, four rows between two barriers, 24.8; 4 x 2048 x 4096 by 256 threads 23.3, by 128 28.5, by 512 28.0; backwards from 8 bits
// 8 x 2048 x 4096 by 128 threads, two rows at a time, 75.8, by 256 one row at a time 78.7, by 512 79.9.  16 x 64 x 16 fp32 by 16 threads a row, four rows
// each, 7.9, one each 11.4.  4 x 2048 x 12288 backwards by 512 threads 143, by 1024 threads, whose registers do not hold it all, 274.
// Three pieces a thread where they hold the row: forwards, and backwards from 8 bits, 8 x 2048 x 1536 19.1 and 26.5, with four pieces 23.4 and 29.3; 16 x 1779 x
// 2983 by 128 threads 75 and 91, by 256 with two pieces 79 and by 128 with four 147; 8 x 2048 x 5296 by 256 threads 73 and 98, by 512 with two 77 and 126;
// 4 x 2048 x 12288 by 512 87 and 118, with four 105 and 176.
// Since whole pieces are loaded without a look at the width: forwards 8 x 2048 x 2048 23.0, 4 x 2048 x 4096 21.8, 8 x 2048 x 1536 16.8, 16 x 1779 x 2983 75, 8 x 2048 x 5296 72,
// 4 x 2048 x 12288 83; backwards from 8 bits 8 x 2048 x 4096 73.8, the others as they were.  Four pieces by 512 threads are more than the registers of 16-bit
// rows backwards hold, 34 of them go to scratch memory from x and 38 from 8 bits: 4 x 2048 x 16000 190 and 165 us, of 121 and 101 by their bytes.
template <int T_, int C_, int SLOTS_, int R_>
struct Plan {
    static constexpr int T = T_, C = C_, SLOTS = SLOTS_, R = R_;
};
template <bool BACK, class F>
constexpr bool by_row(int64_t bytes, F f)
{
    if (bytes <= 16 * 16) f(std::conditional_t<BACK, Plan<16, 1, 16, 4>, Plan<16, 1, 16, 1>>());
    else if (bytes <= 64 * 16) f(Plan<64, 1, 4, 1>());
    else if (bytes <= 2 * 64 * 16) f(Plan<64, 2, 4, 1>());
    else if (bytes <= 3 * 64 * 16) f(Plan<64, 3, 4, 1>());
    else if (bytes <= 4 * 64 * 16) f(Plan<64, 4, 4, 1>());
    else if (bytes <= 3 * 128 * 16) f(Plan<128, 3, 2, 1>());
    else if (bytes <= 2 * 256 * 16) f(std::conditional_t<BACK, Plan<128, 4, 2, 1>, Plan<256, 2, 1, 1>>());
    else if (bytes <= 3 * 256 * 16) f(Plan<256, 3, 1, 1>());
    else if (bytes <= 2 * 512 * 16) f(Plan<512, 2, 1, 1>());
    else if (bytes <= 3 * 512 * 16) f(Plan<512, 3, 1, 1>());
    else if (bytes <= 4 * 512 * 16) f(Plan<512, 4, 1, 1>());
    else return false;
    return true;
}
// The kernels count on it: all of a plan's pieces but the last are whole.  (A row's last 16 bytes may be 2 or 4 of its own.)
template <bool BACK>
constexpr bool pieces_are_whole()
{
    bool whole = true;
    for (int64_t piece = 0; piece < 2048; ++piece)
        by_row<BACK>(16 * piece + 2, [&](auto p) { whole = whole && 16 * piece + 2 > (p.C - 1) * p.T * 16 && piece < p.C * p.T; });
    return whole;
}
static_assert(pieces_are_whole<false>() && pieces_are_whole<true>(), "rows are longer than all of a plan's pieces but the last");
constexpr int LONG_THREADS = 1024, LONG_GRAD_THREADS = 256;

// Workgroups of a worker, which take rows_at_once rows each in turn: `groups` for all workers, if there are so many rows for at least `turns` turns.
int strips_of(const dbw_rows *l, int rows_at_once, int64_t groups, int turns)
{
    const int64_t most = (groups + l->workers - 1) / l->workers, each = (int64_t)turns * rows_at_once;
    const int64_t count = (l->rows + each - 1) / each;
    return (int)(count < 1 ? 1 : count < most ? count : most);
}
template <bool BACK>
int rows_at_once(const dbw_rows *l, const Shape &S)
{
    int n = 1;
    by_row<BACK>(S.e * l->width, [&](auto p) { n = p.SLOTS * p.R; });
    return n;
}
// Forwards, 8 x 2048 x 2048: 1024 workgroups 23.1, 4096 32.  Backwards every workgroup has 8 bytes a column to add up in the end: 512 of them, or as
// many as have 64 rows each, up to 1024.  From 8 bits 8 x 2048 x 2048 with 512 and 1024 37.8 and 42.8, 8 x 8192 x 2048 145 and 133, 4 x 2048 x 4096
// 42.0 and 54.2.
constexpr int NORM_GROUPS = 2048, GRAD_GROUPS = 512;
int grad_strips_of(const dbw_rows *l, const Shape &S)
{
    const int64_t groups = S.rows / 64;
    return strips_of(l, rows_at_once<true>(l, S), groups < GRAD_GROUPS ? GRAD_GROUPS : groups < 2 * GRAD_GROUPS ? groups : 2 * GRAD_GROUPS, 2);
}
dim3 store_grid(int64_t pieces)
{
    constexpr int each = layer::STORE_THREADS * layer::STORE_PIECES;
    return grid_of((pieces + each - 1) / each);
}
int64_t part_ld(const dbw_rows *l) { return (l->width + 3) / 4 * 4; }

}  // namespace

extern "C" int64_t dbw_checkpoint_bytes(const dbw_rows *shape)
{
    Shape S;
    const int rc = check_shape(shape, &S);
    return rc == DBW_OK ? checkpoint_bytes(S.rows, shape->width) : rc;
}

extern "C" int dbw_checkpoint_store(const dbw_rows *shape, const void *x, const uint8_t *mask, void *checkpoint, void *stream)
{
    Shape S;
    const int rc = check_shape(shape, &S);
    if (rc != DBW_OK) return rc;
    if (S.rows > 0 && (!x || !checkpoint)) return DBW_ERR_NULL;
    if (off(x, S.e) || off(checkpoint, 16)) return DBW_ERR_INVALID;
    if (S.rows == 0) return DBW_OK;
    const layer::Store P{x, mask, nullptr, S.ld, S.rows, shape->width, kept_of(checkpoint, S, shape)};
    by_type(shape->type, [&](auto e) {
        typedef decltype(e) E;
        const int64_t pieces = S.rows * (P.kept.stride / layer::Piece<E>::N);
        hipLaunchKernelGGL(layer::store_kernel<E>, store_grid(pieces), dim3(layer::STORE_THREADS), 0,
                           (hipStream_t)stream, P);
    });
    DBW_HIP(hipGetLastError());
    return DBW_OK;
}

extern "C" int dbw_checkpoint_load(const dbw_rows *shape, const void *checkpoint, void *x_out, void *stream)
{
    Shape S;
    const int rc = check_shape(shape, &S);
    if (rc != DBW_OK) return rc;
    if (S.rows > 0 && (!x_out || !checkpoint)) return DBW_ERR_NULL;
    if (off(x_out, S.e) || off(checkpoint, 16)) return DBW_ERR_INVALID;
    if (S.rows == 0) return DBW_OK;
    const layer::Store P{nullptr, nullptr, x_out, S.ld_out, S.rows, shape->width, kept_of(checkpoint, S, shape)};
    by_type(shape->type, [&](auto e) {
        typedef decltype(e) E;
        const int64_t pieces = S.rows * (P.kept.stride / layer::Piece<E>::N);
        hipLaunchKernelGGL(layer::load_kernel<E>, store_grid(pieces), dim3(layer::STORE_THREADS), 0,
                           (hipStream_t)stream, P);
    });
    DBW_HIP(hipGetLastError());
    return DBW_OK;
}

extern "C" int dbw_layer_norm(const dbw_rows *shape, const void *x, const uint8_t *mask, const float *params, int64_t ld_params,
                              int64_t weight_at, int64_t bias_at, float eps, void *y, float *stats_out, void *checkpoint, void *stream)
{
    Shape S;
    const int rc = check_shape(shape, &S);
    if (rc != DBW_OK) return rc;
    if ((S.rows > 0 && (!x || !y)) || ((weight_at >= 0 || bias_at >= 0) && !params)) return DBW_ERR_NULL;
    if (off(x, S.e) || off(y, S.e) || off(checkpoint, 16) || off(params, 4) || !(eps > 0.f) || !isfinite(eps)) return DBW_ERR_INVALID;
    if (outside(weight_at, shape->width, ld_params) || outside(bias_at, shape->width, ld_params)) return DBW_ERR_INVALID;
    if ((weight_at >= 0 || bias_at >= 0) && too_long(ld_params, shape->workers)) return DBW_ERR_UNSUPPORTED;
    if (!(x == y && S.ld == S.ld_out) && overlap(x, S.rows, S.ld, y, S.rows, S.ld_out, shape->width, S.e)) return DBW_ERR_ALIAS;
    if (S.rows == 0) return DBW_OK;
    const int strips = strips_of(shape, rows_at_once<false>(shape, S), NORM_GROUPS, 1);
    layer::Norm P{x, mask, params, S.ld, S.ld_out, ld_params, weight_at, bias_at, S.rows, shape->rows, shape->width, shape->workers, strips, eps, y,
                  stats_out, kept_of(checkpoint, S, shape)};
    if (!checkpoint) P.kept.codes = nullptr;
    hipStream_t s = (hipStream_t)stream;
    by_type(shape->type, [&](auto e) {
        typedef decltype(e) E;
        if (!by_row<false>(S.e * shape->width, [&](auto p) {
                hipLaunchKernelGGL((layer::norm_kernel<E, p.T, p.C, p.SLOTS>), grid_of((int64_t)shape->workers * strips), dim3(p.T * p.SLOTS), 0, s, P);
            }))
            hipLaunchKernelGGL((layer::norm_long_kernel<E, LONG_THREADS>), grid_of(S.rows), dim3(LONG_THREADS), 0, s, P);
    });
    DBW_HIP(hipGetLastError());
    return DBW_OK;
}

extern "C" int64_t dbw_layer_norm_work_bytes(const dbw_rows *shape)
{
    Shape S;
    const int rc = check_shape(shape, &S);
    if (rc != DBW_OK) return rc;
    const int strips = grad_strips_of(shape, S);
    int64_t bytes = strips > 1 ? (int64_t)shape->workers * strips * 2 * part_ld(shape) * 4 : 0;
    if (!by_row<true>(S.e * shape->width, [](auto) {})) bytes += 8 * S.rows;
    return bytes + 16;
}

extern "C" int dbw_layer_norm_grad(const dbw_rows *shape, const void *dy, const void *x, const void *checkpoint, const uint8_t *mask,
                                   const float *stats, const float *params, int64_t ld_params, int64_t weight_at, int64_t bias_at, void *dx,
                                   float *grads, int64_t ld_grads, void *work, void *stream)
{
    Shape S;
    const int rc = check_shape(shape, &S);
    if (rc != DBW_OK) return rc;
    if (!work || (S.rows > 0 && (!dy || !dx || !stats || (!x && !checkpoint))) || (weight_at >= 0 && !params)) return DBW_ERR_NULL;
    if (x && checkpoint) return DBW_ERR_INVALID;
    if (off(dy, S.e) || off(x, S.e) || off(dx, S.e) || off(checkpoint, 16) || off(work, 16) || off(params, 4) || off(grads, 4)) return DBW_ERR_INVALID;
    if (outside(weight_at, shape->width, ld_params)) return DBW_ERR_INVALID;
    if (grads && (outside(weight_at, shape->width, ld_grads) || outside(bias_at, shape->width, ld_grads))) return DBW_ERR_INVALID;
    if (grads && weight_at >= 0 && bias_at >= 0 && weight_at < bias_at + shape->width && bias_at < weight_at + shape->width) return DBW_ERR_ALIAS;
    if ((weight_at >= 0 && too_long(ld_params, shape->workers)) || (grads && too_long(ld_grads, shape->workers))) return DBW_ERR_UNSUPPORTED;
    if (dx != x && overlap(x, S.rows, S.ld, dx, S.rows, S.ld, shape->width, S.e)) return DBW_ERR_ALIAS;
    if (!(dx == dy && S.ld == S.ld_out) && overlap(dy, S.rows, S.ld_out, dx, S.rows, S.ld, shape->width, S.e)) return DBW_ERR_ALIAS;
    if (weight_at < 0 && bias_at < 0) grads = nullptr;
    const int strips = grad_strips_of(shape, S);
    layer::NormGrad P{dy, x, kept_of(checkpoint, S, shape), mask, stats, params, S.ld, S.ld_out, ld_params, ld_grads, weight_at, bias_at, S.rows,
                      shape->rows, shape->width, shape->workers, strips, dx, grads, nullptr, part_ld(shape), nullptr};
    hipStream_t s = (hipStream_t)stream;
    if (S.rows == 0) {
        const int slices = (shape->width + 255) / 256;
        if (grads) hipLaunchKernelGGL(layer::norm_zero_kernel, grid_of((int64_t)slices * shape->workers), dim3(256), 0, s, P, slices);
        DBW_HIP(hipGetLastError());
        return DBW_OK;
    }
    const int64_t groups = (int64_t)shape->workers * strips;
    if (strips > 1) P.parts = (float *)work;
    P.means = (layer::f32x2 *)((float *)work + (strips > 1 ? groups * 2 * P.part_ld : 0));
    by_type(shape->type, [&](auto e) {
        typedef decltype(e) E;
        const auto rows = [&](auto p) {
            const size_t lds = (size_t)(p.SLOTS > 1 ? p.SLOTS : 0) * p.T * p.C * layer::Piece<E>::N * 4;
            if (x) hipLaunchKernelGGL((layer::norm_grad_kernel<E, p.T, p.C, p.SLOTS, p.R, false>), grid_of(groups), dim3(p.T * p.SLOTS), lds, s, P);
            else hipLaunchKernelGGL((layer::norm_grad_kernel<E, p.T, p.C, p.SLOTS, p.R, true>), grid_of(groups), dim3(p.T * p.SLOTS), lds, s, P);
        };
        if (!by_row<true>(S.e * shape->width, rows)) {
            constexpr int T = LONG_GRAD_THREADS, COLUMNS = T * layer::Piece<E>::N;
            const int slices = (shape->width + COLUMNS - 1) / COLUMNS;
            if (x) {
                hipLaunchKernelGGL((layer::norm_means_kernel<E, LONG_THREADS, false>), grid_of(S.rows), dim3(LONG_THREADS), 0, s, P);
                hipLaunchKernelGGL((layer::norm_grad_long_kernel<E, T, false>), grid_of(groups * slices), dim3(T), 0, s, P, slices);
            } else {
                hipLaunchKernelGGL((layer::norm_means_kernel<E, LONG_THREADS, true>), grid_of(S.rows), dim3(LONG_THREADS), 0, s, P);
                hipLaunchKernelGGL((layer::norm_grad_long_kernel<E, T, true>), grid_of(groups * slices), dim3(T), 0, s, P, slices);
            }
        }
    });
    if (grads && strips > 1) {
        const int slices = (shape->width + layer::SUM_COLUMNS - 1) / layer::SUM_COLUMNS;
        hipLaunchKernelGGL(layer::norm_sum_kernel, grid_of((int64_t)shape->workers * slices * 2), dim3(layer::SUM_COLUMNS / 4 * layer::SUM_ROWS), 0, s, P, slices);
    }
    DBW_HIP(hipGetLastError());
    return DBW_OK;
}

// ---------------------------------------------------------------- experts

namespace {

// Slots of a workgroup, of which a worker has 256 at most: each of them adds up what all of them counted.
constexpr int SORT_CHUNK = 1024, SORT_CHUNKS = 256;
int chunk_of(const dbw_routing *l)
{
    const int64_t each = ((int64_t)l->tokens * l->k + SORT_CHUNKS - 1) / SORT_CHUNKS;
    return each > SORT_CHUNK ? (int)each : SORT_CHUNK;
}
int chunks_of(const dbw_routing *l) { return (int)(((int64_t)l->tokens * l->k + chunk_of(l) - 1) / chunk_of(l)); }

int check_routing(const dbw_routing *l)
{
    if (!l) return DBW_ERR_NULL;
    if (l->workers < 1 || l->tokens < 0 || l->k < 1 || l->experts < 1) return DBW_ERR_INVALID;
    const int64_t slots = (int64_t)l->tokens * l->k;
    if (l->workers > MAX_GROUPS || slots > INT32_MAX || slots * l->workers > INT32_MAX || l->experts > DBW_EXPERTS_MAX ||
        (int64_t)l->workers * (l->experts + 1) > INT32_MAX)
        return DBW_ERR_UNSUPPORTED;
    return DBW_OK;
}
// Checks that the calls on rows have in common, and the kernels' view of them.
int check_move(const dbw_routing *routing, const dbw_rows *shape, const void *tokens, const void *sorted, const int32_t *place,
               const float *weights, int32_t *status, Shape *S, layer::Move *P)
{
    int rc = check_routing(routing);
    if (rc == DBW_OK) rc = check_shape(shape, S);
    if (rc != DBW_OK) return rc;
    if (shape->workers != routing->workers || shape->rows != routing->tokens) return DBW_ERR_INVALID;
    const int64_t slots = (int64_t)routing->tokens * routing->k, all = slots * routing->workers;
    if (too_long(S->ld_out, all)) return DBW_ERR_UNSUPPORTED;
    if (S->rows > 0 && (!tokens || !sorted || !place)) return DBW_ERR_NULL;
    if (off(tokens, S->e) || off(sorted, S->e)) return DBW_ERR_INVALID;
    if (overlap(tokens, S->rows, S->ld, sorted, all, S->ld_out, shape->width, S->e)) return DBW_ERR_ALIAS;
    *P = layer::Move{nullptr, nullptr, nullptr, nullptr, place, weights, nullptr, status, S->ld, S->ld_out, S->rows, slots, shape->rows, shape->width,
                     routing->k};
    return DBW_OK;
}
dim3 move_grid(int64_t waves) { return grid_of((waves + layer::MOVE_WAVES - 1) / layer::MOVE_WAVES); }
// Pieces of a lane: rows in chunks of 64 C pieces, a wave each, four pieces a lane where that leaves waves enough.
constexpr int64_t MOVE_ENOUGH = 4096, MOVE_FEW = 1024;
template <class E, int WHAT>
bool launch_narrow(int64_t row_bytes, const layer::Move &P, hipStream_t s)
{
    if (row_bytes > layer::NARROW_BYTES) return false;
    hipLaunchKernelGGL((layer::narrow_kernel<E, WHAT>), grid_of((P.rows + layer::NARROW_TOKENS - 1) / layer::NARROW_TOKENS), dim3(layer::MOVE_THREADS), 0, s, P);
    return true;
}
template <class F>
void by_chunk(int64_t rows, int64_t row_bytes, F f)
{
    const auto chunks = [&](int c) { return (int)((row_bytes + 1024 * c - 1) / (1024 * c)); };
    if (row_bytes > 2048 && rows * chunks(4) >= MOVE_ENOUGH) f(std::integral_constant<int, 4>(), chunks(4));
    else if (row_bytes > 1024 && rows * chunks(2) >= MOVE_ENOUGH) f(std::integral_constant<int, 2>(), chunks(2));
    else f(std::integral_constant<int, 1>(), chunks(1));
}

}  // namespace

extern "C" int64_t dbw_expert_work_bytes(const dbw_routing *routing)
{
    const int rc = check_routing(routing);
    if (rc != DBW_OK) return rc;
    const int64_t chunks = routing->tokens > 0 ? chunks_of(routing) : 1;
    return 16 + (chunks > 1 ? routing->workers * chunks * routing->experts * 4 : 0);
}

extern "C" int dbw_expert_sort(const dbw_routing *routing, const int32_t *expert, int32_t *start_out, int32_t *place_out, int32_t *source_out,
                               int32_t *status_out, void *work, void *stream)
{
    const int rc = check_routing(routing);
    if (rc != DBW_OK) return rc;
    const int64_t slots = (int64_t)routing->tokens * routing->k;
    if (!start_out || !work || (slots > 0 && (!expert || !place_out || !source_out))) return DBW_ERR_NULL;
    if (off(work, 16)) return DBW_ERR_INVALID;
    const int chunks = slots > 0 ? chunks_of(routing) : 1;
    const layer::Sort P{expert, start_out, place_out, source_out, status_out, (int32_t *)work, routing->workers, (int)slots, routing->experts, chunk_of(routing),
                        chunks};
    hipStream_t s = (hipStream_t)stream;
    const dim3 grid = grid_of((int64_t)routing->workers * chunks), block(layer::SORT_THREADS);
    if (chunks > 1) hipLaunchKernelGGL(layer::sort_count_kernel, grid, block, routing->experts * 4, s, P);
    hipLaunchKernelGGL(layer::sort_kernel, grid, block, (layer::SORT_WAVES * routing->experts + layer::SORT_WAVES) * 4, s, P);
    DBW_HIP(hipGetLastError());
    return DBW_OK;
}

extern "C" int dbw_expert_gather(const dbw_routing *routing, const dbw_rows *shape, const void *x, const int32_t *place, void *sorted,
                                 int32_t *status_out, void *stream)
{
    Shape S;
    layer::Move P;
    const int rc = check_move(routing, shape, x, sorted, place, nullptr, status_out, &S, &P);
    if (rc != DBW_OK) return rc;
    if (S.rows == 0) return DBW_OK;
    P.tokens = x;
    P.sorted_out = sorted;
    by_type(shape->type, [&](auto e) {
        if (launch_narrow<decltype(e), layer::GATHER>(S.e * shape->width, P, (hipStream_t)stream)) return;
        by_chunk(S.rows, S.e * shape->width, [&](auto c, int chunks) {
            hipLaunchKernelGGL((layer::gather_kernel<decltype(e), c.value>), move_grid(S.rows * chunks), dim3(layer::MOVE_THREADS), 0, (hipStream_t)stream, P,
                               chunks);
        });
    });
    DBW_HIP(hipGetLastError());
    return DBW_OK;
}

extern "C" int dbw_expert_combine(const dbw_routing *routing, const dbw_rows *shape, const void *sorted, const int32_t *place, const float *weights,
                                  void *y, int32_t *status_out, void *stream)
{
    Shape S;
    layer::Move P;
    const int rc = check_move(routing, shape, y, sorted, place, weights, status_out, &S, &P);
    if (rc != DBW_OK) return rc;
    if (S.rows == 0) return DBW_OK;
    P.sorted_in = sorted;
    P.out = y;
    by_type(shape->type, [&](auto e) {
        if (launch_narrow<decltype(e), layer::COMBINE>(S.e * shape->width, P, (hipStream_t)stream)) return;
        by_chunk(S.rows, S.e * shape->width, [&](auto c, int chunks) {
            hipLaunchKernelGGL((layer::combine_kernel<decltype(e), c.value>), move_grid(S.rows * chunks), dim3(layer::MOVE_THREADS), 0, (hipStream_t)stream, P,
                               chunks);
        });
    });
    DBW_HIP(hipGetLastError());
    return DBW_OK;
}

extern "C" int dbw_expert_combine_grad(const dbw_routing *routing, const dbw_rows *shape, const void *dy, const void *sorted, const int32_t *place,
                                       const float *weights, void *dsorted, float *dweights, int32_t *status_out, void *stream)
{
    Shape S;
    layer::Move P;
    const int rc = check_move(routing, shape, dy, dsorted, place, weights, status_out, &S, &P);
    if (rc != DBW_OK) return rc;
    const int64_t all = S.rows * routing->k;
    if (S.rows > 0 && dweights && !sorted) return DBW_ERR_NULL;
    if (off(sorted, S.e)) return DBW_ERR_INVALID;
    if (dweights && sorted != dsorted && overlap(sorted, all, S.ld_out, dsorted, all, S.ld_out, shape->width, S.e)) return DBW_ERR_ALIAS;
    if (S.rows == 0) return DBW_OK;
    P.tokens = dy;
    P.sorted_in = sorted;
    P.sorted_out = dsorted;
    P.dweights = dweights;
    by_type(shape->type, [&](auto e) {
        typedef decltype(e) E;
        const int64_t bytes = S.e * shape->width;
        if (launch_narrow<E, layer::COMBINE_GRAD>(bytes, P, (hipStream_t)stream)) return;
        const auto launch = [&](auto kernel, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(layer::MOVE_THREADS), 0, (hipStream_t)stream, P); };
        if (bytes > 2048 && S.rows <= MOVE_FEW) launch(layer::combine_grad_kernel<E, 2, layer::MOVE_WAVES>, grid_of(S.rows));
        else if (bytes > 2048) launch(layer::combine_grad_kernel<E, 4, 1>, move_grid(S.rows));
        else if (bytes > 1024) launch(layer::combine_grad_kernel<E, 2, 1>, move_grid(S.rows));
        else launch(layer::combine_grad_kernel<E, 1, 1>, move_grid(S.rows));
    });
    DBW_HIP(hipGetLastError());
    return DBW_OK;
}

// ---------------------------------------------------------------- weight gradient

namespace {

int check_linear(const dbw_linear *l, int64_t *ld)
{
    if (!l) return DBW_ERR_NULL;
    if (l->workers < 1 || l->rows < 0 || l->inputs < 1 || l->outputs < 1 || no_type(l->type) || l->experts < 1 || l->tokens < 0 || l->k < 1) return DBW_ERR_INVALID;
    *ld = l->ld ? l->ld : l->outputs;
    if (*ld < l->outputs) return DBW_ERR_INVALID;
    const int64_t rows = (int64_t)l->workers * l->rows;
    if (l->workers > MAX_GROUPS || rows > INT32_MAX || (int64_t)l->workers * l->tokens > INT32_MAX || l->inputs > DBW_LAYER_MAX_WIDTH ||
        l->outputs > DBW_LAYER_MAX_WIDTH || l->experts > DBW_EXPERTS_MAX || (int64_t)l->workers * (l->experts + 1) > INT32_MAX || too_long(*ld, rows))
        return DBW_ERR_UNSUPPORTED;
    return DBW_OK;
}

// Tiles of the weights, a workgroup each, and into how many parts a layer's rows are split.
typedef layer::Tile<256, 256, 2, 4, 32> Large;
typedef layer::Tile<128, 256, 2, 4, 32> LargeSplit;       // of operands in parts
typedef layer::Tile<128, 128, 2, 2, 32> Middle;
typedef layer::Tile<64, 128, 2, 2, 32> MiddleSplit;
typedef layer::Tile<64, 64, 2, 2, 64> Small;
typedef layer::Tile<64, 64, 2, 2, 32> SmallSplit;         // in three
struct Cut {
    int tile;                                             // 0: small, 1: middle, 2: large
    int64_t tiles_out, tiles_in, layers;
    int splits;
};
// Of the tiles that fill the chip, the one whose tiles take least time for all of the weights, in the time that a large one takes for its area, a hundredth as
// the unit: 4 x 1024 rows a layer, 16 layers of 1024 x 1024, large, middle and small tiles bf16 200, 228 and 397 us, fp16 340, 399 and 721, fp32 477, 697
// and 881.  Layers of few rows are bound by a tile's latency, which middle tiles hide better, two and more to a compute unit: 8 x 16 layers bf16 of 64 rows 119 and
// 106, of 128 137 and 129, of 256 176 and 174 (fp16 of 64 146 and 151).
//
// Large tiles fill the chip with one for each compute unit; middle ones with two, or where there is so much to do that splitting the rows pays: 1 x 4096 x
// 2048 x 2048 bf16 67.7 us (small tiles 82, large ones 71.9), 1 x 8192 x 1024 x 1024 40.9 (50, 53), but 8 x 1024 x 512 x 512 29 and small ones
// 15.3, 2 x 1024 x 768 x 2304 34 and 25.4.  Small ones are taken where neither does.  Parts have 512 rows at least: 2 x 512 x 500 x 700 fp32 whole 15.8, in halves 26.6.
constexpr int64_t CHIP = 256, MUCH = 400000, PART = 512, FEW_ROWS = 128;
Cut cut_of(const dbw_linear *l)
{
    const bool whole = l->type == DBW_TYPE_BF16, thirds = l->type == DBW_TYPE_F32;
    const int64_t rows = l->rows / l->experts, layers = (int64_t)l->workers * l->experts;
    const int outs[3] = {Small::OUT, whole ? Middle::OUT : MiddleSplit::OUT, whole ? Large::OUT : LargeSplit::OUT}, ins[3] = {Small::IN, Middle::IN, Large::IN};
    const int price[3] = {thirds ? 185 : 200, thirds ? 145 : whole && rows <= FEW_ROWS ? 90 : 115, 100};
    Cut c;
    c.tile = -1;
    c.layers = layers;
    c.splits = 1;
    double least = 0;
    int64_t groups = 0;
    for (int tile = 2; tile >= 0; --tile) {
        const int64_t out = (l->outputs + outs[tile] - 1) / outs[tile], in = (l->inputs + ins[tile] - 1) / ins[tile], n = out * in * layers;
        const bool fills = tile == 2 ? n >= CHIP : tile == 1 ? n >= 2 * CHIP || n * rows >= MUCH : n >= CHIP || c.tile < 0;
        const double cost = (double)price[tile] * outs[tile] * ins[tile] * n;
        if (!fills || (c.tile >= 0 && cost >= least)) continue;
        c.tile = tile;
        c.tiles_out = out;
        c.tiles_in = in;
        groups = n;
        least = cost;
    }
    if (groups < (c.tile == 1 ? 2 * CHIP : CHIP)) {
        int64_t splits = 2 * CHIP / groups;
        if (splits > rows / PART) splits = rows / PART;
        if (splits > 1) c.splits = (int)splits;
    }
    return c;
}

}  // namespace

extern "C" int64_t dbw_checkpoint_weight_grad_work_bytes(const dbw_linear *shape)
{
    int64_t ld;
    const int rc = check_linear(shape, &ld);
    if (rc != DBW_OK) return rc;
    const Cut cut = cut_of(shape);
    return 16 + (cut.splits > 1 ? 4 * cut.splits * shape->workers * shape->experts * (int64_t)shape->outputs * (shape->inputs + 1) : 0);
}

extern "C" int dbw_checkpoint_weight_grad(const dbw_linear *shape, const void *dy, const void *checkpoint, const int32_t *start,
                                          const int32_t *source, float *grads, int64_t ld_grads, int64_t weight_at, int64_t bias_at,
                                          int32_t *status_out, void *work, void *stream)
{
    int64_t ld;
    const int rc = check_linear(shape, &ld);
    if (rc != DBW_OK) return rc;
    if (!work || !grads || (shape->rows > 0 && !dy) || (shape->rows > 0 && shape->tokens > 0 && !checkpoint) || (!start && shape->experts > 1))
        return DBW_ERR_NULL;
    const size_t e = size_of(shape->type);
    const int64_t count = (int64_t)shape->experts * shape->outputs, weights = count * shape->inputs;   // at most 2^50
    if (off(dy, e) || off(checkpoint, 16) || off(work, 16) || off(grads, 4) || (!source && shape->rows != shape->tokens)) return DBW_ERR_INVALID;
    if (weight_at < 0 || outside(weight_at, weights, ld_grads) || outside(bias_at, count, ld_grads)) return DBW_ERR_INVALID;
    if (bias_at >= 0 && bias_at < weight_at + weights && weight_at < bias_at + count) return DBW_ERR_ALIAS;
    if (too_long(ld_grads, shape->workers)) return DBW_ERR_UNSUPPORTED;
    const int64_t tokens = (int64_t)shape->workers * shape->tokens;
    const Cut cut = cut_of(shape);
    const int64_t groups = cut.tiles_out * cut.tiles_in * cut.layers * cut.splits;
    const layer::Linear P{dy, layer::kept_of((void *)checkpoint, tokens, shape->inputs), start, source, status_out, grads, ld, ld_grads, weight_at,
                          bias_at, shape->workers, shape->rows, shape->inputs, shape->outputs, shape->experts, shape->tokens, shape->k, (int)cut.tiles_out,
                          (int)cut.tiles_in, cut.splits, (float *)work};
    hipStream_t s = (hipStream_t)stream;
    bool fits = true;
    by_type(shape->type, [&](auto v) {
        typedef decltype(v) E;
        const auto launch = [&](auto tile) {
            typedef decltype(tile) T;
            constexpr int lds = layer::tile_lds<E, T>();
            const auto run = [&](auto kernel) {
                // more than 64 KB have to be asked for
                if (lds > 65536) fits = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds) == hipSuccess;
                if (fits) hipLaunchKernelGGL(kernel, grid_of(groups), dim3(T::THREADS), lds, s, P);
            };
            if (source) run(layer::weight_grad_kernel<E, T, true>);
            else run(layer::weight_grad_kernel<E, T, false>);
        };
        if (cut.tile == 0) launch(std::conditional_t<layer::Planes<E>::COUNT == 3, SmallSplit, Small>());
        else if constexpr (layer::Planes<E>::COUNT == 1) {
            if (cut.tile == 1) launch(Middle());
            else launch(Large());
        } else {
            if (cut.tile == 1) launch(MiddleSplit());
            else launch(LargeSplit());
        }
    });
    if (!fits) return DBW_ERR_HIP;
    if (cut.splits > 1) {
        const int64_t all = (int64_t)shape->workers * (weights + (bias_at >= 0 ? count : 0));
        hipLaunchKernelGGL(layer::weight_grad_sum_kernel, grid_of((all + layer::SUM_THREADS - 1) / layer::SUM_THREADS), dim3(layer::SUM_THREADS), 0, s, P);
    }
    DBW_HIP(hipGetLastError());
    return DBW_OK;
}
