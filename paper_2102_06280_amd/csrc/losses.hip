// Entry points of the losses on logits (dbw_losses.h): argument checks and launches.  No context and no allocation: what the
// kernels need beyond inputs and outputs is the caller's scratch memory.
#include <math.h>

#include "dbw_internal.h"
#include "dbw_losses.h"
#include "loss_kernels.h"

namespace {

size_t size_of(int type) { return type == DBW_TYPE_F32 ? 4 : 2; }

constexpr int64_t MAX_GROUPS = 1 << 22;   // of workers, and of pairs

struct Shape {
    int64_t rows;        // of all workers
    int64_t ld, ld_grad, row_bytes;
    loss::Rows R;
};

int check_shape(const dbw_logits *l, Shape *out)
{
    if (!l) return DBW_ERR_NULL;
    if (l->workers < 1 || l->rows < 0 || l->vocab < 1 || l->type < DBW_TYPE_F32 || l->type > DBW_TYPE_F16) return DBW_ERR_INVALID;
    out->ld = l->ld ? l->ld : l->vocab;
    out->ld_grad = l->ld_grad ? l->ld_grad : out->ld;
    if (out->ld < l->vocab || out->ld_grad < l->vocab) return DBW_ERR_INVALID;
    if (!(l->scale > 0.f) || !isfinite(l->scale * (float)loss::LOG2E)) return DBW_ERR_INVALID;
    out->rows = (int64_t)l->workers * l->rows;
    const int64_t most = INT64_MAX / 8 / (out->rows + 1);  // of a stride: offsets in bytes fit 64 bits
    if (l->vocab > DBW_LOSS_MAX_VOCAB || l->workers > MAX_GROUPS || out->rows > INT32_MAX || out->ld > most || out->ld_grad > most)
        return DBW_ERR_UNSUPPORTED;
    return DBW_OK;
}

// Scratch memory: a row's maximum and sum, and the two terms of its loss or its coefficient and its log-probability; what slices of few rows found.
struct Work {
    loss::MaxSum *stats;
    float2 *terms;
    float *coef, *logp;
    loss::MaxSum *slices;
    float *token_logit;
};
constexpr int64_t WORK_PER_ROW = 16;
constexpr int SLICED_ROWS = 1024, SLICE_GROUPS = 2048;    // rows that may be cut, and workgroups that they are cut for
constexpr int POLICY_ROWS = 64, POLICY_GROUPS = 512;     // the same where a row would be read once if it were whole: policy 64 x 100000
                                                          // 15.4, whole 20.2; 128 x 100000 24.2 and 21.1
constexpr int64_t WORK_FIXED = 8 * SLICE_GROUPS + 4 * SLICED_ROWS;

Work split_work(void *work, int64_t rows)
{
    Work w;
    w.slices = (loss::MaxSum *)work;
    w.token_logit = (float *)(w.slices + SLICE_GROUPS);
    w.stats = (loss::MaxSum *)(w.token_logit + SLICED_ROWS);
    w.terms = (float2 *)(w.stats + rows);
    w.coef = (float *)w.terms;
    w.logp = w.coef + rows;
    return w;
}

// Bytes of a row from which every XCD gets rows that lie together, of kernels that hold a row: policy 6144 x 32768 (64 KB) 147 us, with rows to the XCDs
// in turn 156; 12288 x 16384 148 and 140.
constexpr int64_t XCD_ROW = 65536;

loss::Factor factor_of(float scale)
{
    const double c = scale * loss::LOG2E;
    float hi = (float)c;
    if (hi >= c) hi = nextafterf(hi, 0.f);
    const float lo = (float)(c - hi), least = 0x1p-149f;
    return loss::Factor{fmaxf(hi, least), fmaxf(lo, least), (float)c};
}

// Checks that all calls have in common, and the kernels' view of the rows.
int prepare(const dbw_logits *l, const void *logits, void *dlogits, int32_t *status, const void *work, Shape *S)
{
    const int rc = check_shape(l, S);
    if (rc != DBW_OK) return rc;
    const size_t e = size_of(l->type);
    if (S->rows > 0 && !logits) return DBW_ERR_NULL;
    if ((uintptr_t)logits % e || (uintptr_t)dlogits % e || (uintptr_t)work % 8) return DBW_ERR_INVALID;
    if (dlogits && S->rows > 0 && !(dlogits == logits && S->ld == S->ld_grad)) {
        const uintptr_t a = (uintptr_t)logits, b = (uintptr_t)dlogits;
        const size_t na = e * (size_t)((S->rows - 1) * S->ld + l->vocab), nb = e * (size_t)((S->rows - 1) * S->ld_grad + l->vocab);
        if (a < b + nb && b < a + na) return DBW_ERR_ALIAS;
    }
    S->row_bytes = (int64_t)e * l->vocab;
    S->R = loss::Rows{logits, dlogits, S->ld, S->ld_grad, l->vocab, S->rows, l->scale, factor_of(l->scale), status, S->row_bytes >= XCD_ROW};
    return DBW_OK;
}

dim3 grid_of(int64_t groups)
{
    const int64_t x = groups < (1 << 20) ? groups : 1 << 20;
    return dim3((uint32_t)x, (uint32_t)((groups + x - 1) / x));
}

// Which kernel takes a row, by its length in bytes: T threads, C pieces a thread at a time (Walk: and S at a time of what lies behind them).
// Times below in us, bf16 unless said otherwise, rows x vocabulary.  (Those of one plan or rule against another were taken when a term of a sum took an
// instruction less: kernels that only read a row take 4 % more now, those of many short rows 4 to 12 %, on either side.)
template <int T_, int C_, int S_ = 0>
struct Plan {
    static constexpr int T = T_, C = C_, S = S_;
    static constexpr int ROWS = loss::ROWS_OF<T>, THREADS = T * ROWS;      // of a workgroup
    static dim3 grid(int64_t rows) { return grid_of((rows + ROWS - 1) / ROWS); }
};
constexpr int SHORT_ROW = 2048;                           // bytes of a row that 16 threads take: a wave's instructions then serve four rows.  Policy
                                                          // 671088 x 100: 302, by a wave each 526; log-probabilities 65536 x 1024: 24.2 and 32.8
template <class F>
void by_short_row(int64_t bytes, F f)
{
    if (bytes <= 4 * 16 * 16) f(Plan<16, 4>());
    else f(Plan<16, 8>());
}
// For the kernels that hold a row.  Policy 4096 x 32768 (64 KB): <512, 8> 91, <256, 16> 93 to 105, <1024, 4> 95.  4096 x 65536 (128 KB): <512, 16> 193,
// half of the row held 198.  2048 x 131072 (256 KB): <512, 16, 8>, which holds half, 205; all of it in the registers of <1024, 16> 223, in registers and
// LDS of <512, 22> 217; a quarter held 214.  One workgroup a compute unit, as a whole row of 256 KB takes, leaves the memory idle while it
// computes.
template <class F>
void by_row(int64_t bytes, F f)
{
    if (bytes <= SHORT_ROW) by_short_row(bytes, f);
    else if (bytes <= 8 * 64 * 16) f(Plan<64, 8>());
    else if (bytes <= 4 * 256 * 16) f(Plan<256, 4>());
    else if (bytes <= 8 * 256 * 16) f(Plan<256, 8>());
    else if (bytes <= 8 * 512 * 16) f(Plan<512, 8>());
    else if (bytes <= 16 * 512 * 16) f(Plan<512, 16>());
    else f(Plan<512, 16, 8>());
}
// For those that only read it: 4096 x 65536, a tenth of the rows without a part, in 83, 5.8 TB/s.
template <class F>
void by_length(int64_t bytes, F f)
{
    if (bytes <= SHORT_ROW) by_short_row(bytes, f);
    else if (bytes <= 8 * 64 * 16) f(Plan<64, 2>());
    else if (bytes <= 128 << 10) f(Plan<256, 8>());
    else f(Plan<1024, 8>());
}
int pieces_of(const dbw_logits *l) { return l->vocab / (16 / (int)size_of(l->type)); }

// Few long rows are read in slices: 1 x 131072 9.2, by one workgroup 11.6 (its exponentials alone take 6); 200 x 80000 11.8 and 13.2, 700 x 80000 26.7
// and 32.3.  Shorter ones are not, where a launch has to join the slices: 1 x 50000 9.4, whole 7.4; 200 x 5000 9.4 and 5.8.
constexpr int64_t LONG_ROW = 128 << 10;
constexpr int SLICE_LONG = 2048;                          // pieces of a slice from which threads take eight at a time
loss::Slices slices_of(const dbw_logits *l, int64_t rows, int most_rows, int groups)
{
    loss::Slices S{1, 0};
    const int pieces = pieces_of(l);
    if (rows < 1 || rows > most_rows) return S;
    int count = groups / (int)rows;
    if (count > loss::MAX_SLICES) count = loss::MAX_SLICES;
    const int unit = pieces / count >= SLICE_LONG ? SLICE_LONG : 512;
    const int units = (pieces + unit - 1) / unit;         // of whole plans
    if (units < 2) return S;
    S.pieces = (units + count - 1) / count * unit;
    S.count = (pieces + S.pieces - 1) / S.pieces;
    return S;
}
template <class F>
void by_slice(const loss::Slices &slices, F f)
{
    if (slices.pieces % SLICE_LONG == 0) f(Plan<256, 8>());
    else f(Plan<256, 2>());
}

// A gradient that is written from what is known of its row is so in slices of 16 KB, or of 8 KB where those would leave compute units idle.
// Log-probabilities and gradient 2048 x 100000: whole rows 233, slices of 8, 16 and 32 KB 217, 212, 217; preference 128 x 32001 fp32 with slices of 8 KB
// 18.2, of 16 KB 21.0.
constexpr int GRADIENT_GROUPS = 1536;
loss::Slices gradient_slices_of(const dbw_logits *l, int64_t rows)
{
    const int pieces = pieces_of(l);
    if (pieces <= 8 * 64) return loss::Slices{1, 0};
    const int each = rows * ((pieces + 1023) / 1024) >= GRADIENT_GROUPS ? 1024 : 512;
    return loss::Slices{(pieces + each - 1) / each, each};
}
template <class F>
void by_gradient_slice(const loss::Slices &slices, int64_t row_bytes, F f)
{
    if (row_bytes <= SHORT_ROW) by_short_row(row_bytes, f);
    else if (slices.pieces == 0) f(Plan<64, 2>());
    else if (slices.pieces == 512) f(Plan<256, 2>());
    else f(Plan<256, 4>());
}

// All rows of a worker in one workgroup: its threads (0: rather not) for rows of T threads each, few enough that `turns` of them one after the
// other take no longer than a second launch.  Policy 16 x 32 x 259 fp32 8.2, with a launch for the sums 11.2; 64 x 64 x 500 8.3 and 11.4, by a wave a row,
// four one after the other, 15.2.  Distillation 8 x 16 x 1000 fp32 7.8 and 10.1; 64 x 60 x 500 by a wave a row 20.0, with a second launch 10.6.
int one_group_threads(const dbw_logits *l, int64_t row_bytes, int turns)
{
    const int T = row_bytes <= SHORT_ROW ? 16 : 64;
    const int64_t threads = ((int64_t)l->rows * T + 63) / 64 * 64;
    if (l->rows < 1 || row_bytes > 8 * 64 * 16 || threads > turns * 1024 || l->rows * row_bytes > 64 << 10) return 0;
    return threads < 1024 ? (int)threads : 1024;
}
template <class F>
void by_group_row(int64_t bytes, F f)
{
    if (bytes <= SHORT_ROW) by_short_row(bytes, f);
    else f(Plan<64, 8>());
}

// Calls f with a value of the logits' type.
template <class F>
void by_type(int type, F f)
{
    if (type == DBW_TYPE_F32) f(float());
    else if (type == DBW_TYPE_BF16) f(loss::bf16());
    else f(loss::f16());
}

// (m, Z) of every row or slice; log-probabilities where rows are whole.  again: the rows will be read again soon.
void launch_logp(const dbw_logits *l, const Shape &S, const loss::Logp &P, bool again, hipStream_t s)
{
    by_type(l->type, [&](auto e) {
        const auto launch = [&](auto p) {
            const dim3 grid = p.grid(S.rows * P.slices.count), block(p.THREADS);
            if (again) hipLaunchKernelGGL((loss::logp_kernel<decltype(e), p.T, p.C, true>), grid, block, 0, s, S.R, P);
            else hipLaunchKernelGGL((loss::logp_kernel<decltype(e), p.T, p.C, false>), grid, block, 0, s, S.R, P);
        };
        if (P.slices.count > 1) by_slice(P.slices, launch);
        else by_length(S.row_bytes, launch);
    });
}
// pairs: what the kernel sums pairs up from by itself, or null
void launch_gradient(const dbw_logits *l, const Shape &S, const loss::Gradient &P, const loss::Preference *pairs, hipStream_t s)
{
    by_type(l->type, [&](auto e) {
        typedef decltype(e) E;
        by_gradient_slice(P.slices, S.row_bytes, [&](auto p) {
            const dim3 grid = grid_of((S.rows * P.slices.count + p.ROWS - 1) / p.ROWS + (P.pairs.loss_out ? P.pairs.workers : 0)), block(p.THREADS);
            if (pairs) hipLaunchKernelGGL((loss::pair_gradient_kernel<E, p.T, p.C>), grid, block, 0, s, S.R, P, *pairs);
            else if (P.stats) hipLaunchKernelGGL((loss::gradient_kernel<E, p.T, p.C, false>), grid, block, 0, s, S.R, P);
            else hipLaunchKernelGGL((loss::gradient_kernel<E, p.T, p.C, true>), grid, block, 0, s, S.R, P);
        });
    });
}

}  // namespace

extern "C" int64_t dbw_loss_work_bytes(const dbw_logits *shape)
{
    Shape S;
    const int rc = check_shape(shape, &S);
    return rc == DBW_OK ? WORK_FIXED + WORK_PER_ROW * S.rows : rc;
}

extern "C" int dbw_token_logp(const dbw_logits *shape, const void *logits, const int32_t *tokens, float *logp_out, float *lse_out,
                              int32_t *status_out, void *work, void *stream)
{
    Shape S;
    const int rc = prepare(shape, logits, nullptr, status_out, work, &S);
    if (rc != DBW_OK) return rc;
    if (!work || (S.rows > 0 && (!tokens || !logp_out))) return DBW_ERR_NULL;
    if (S.rows == 0) return DBW_OK;
    const Work W = split_work(work, S.rows);
    hipStream_t s = (hipStream_t)stream;
    const loss::Slices slices = S.row_bytes > LONG_ROW ? slices_of(shape, S.rows, SLICED_ROWS, SLICE_GROUPS) : loss::Slices{1, 0};
    const loss::Logp P{tokens, nullptr, logp_out, lse_out, nullptr, slices.count > 1 ? W.slices : nullptr, W.token_logit, slices};
    launch_logp(shape, S, P, lse_out != nullptr, s);      // L is asked for where a gradient follows
    if (slices.count > 1) hipLaunchKernelGGL(loss::join_kernel, dim3((uint32_t)S.rows), dim3(64), 0, s, S.R, P);
    DBW_HIP(hipGetLastError());
    return DBW_OK;
}

extern "C" int dbw_token_logp_grad(const dbw_logits *shape, const void *logits, const int32_t *tokens, const float *lse,
                                   const float *coef, void *dlogits, int32_t *status_out, void *stream)
{
    Shape S;
    const int rc = prepare(shape, logits, dlogits, status_out, nullptr, &S);
    if (rc != DBW_OK) return rc;
    if (S.rows > 0 && (!tokens || !lse || !coef || !dlogits)) return DBW_ERR_NULL;
    if (S.rows == 0) return DBW_OK;
    const loss::Gradient P{tokens, coef, nullptr, lse, gradient_slices_of(shape, S.rows), loss::PairLoss{}};
    launch_gradient(shape, S, P, nullptr, (hipStream_t)stream);
    DBW_HIP(hipGetLastError());
    return DBW_OK;
}

extern "C" int dbw_distill_loss(const dbw_logits *shape, int32_t k, const void *logits, const int32_t *teacher_index,
                                int32_t teacher_type, const void *teacher_logits, const float *teacher_lse, const float *weights,
                                float *loss_out, float *row_loss_out, void *dlogits, int32_t *status_out, void *work, void *stream)
{
    Shape S;
    const int rc = prepare(shape, logits, dlogits, status_out, work, &S);
    if (rc != DBW_OK) return rc;
    if (!work || !loss_out || (S.rows > 0 && (!teacher_index || !teacher_logits))) return DBW_ERR_NULL;
    if (k < 1 || teacher_type < DBW_TYPE_F32 || teacher_type > DBW_TYPE_F16 || (uintptr_t)teacher_logits % size_of(teacher_type))
        return DBW_ERR_INVALID;
    if (k > DBW_TEACHER_MAX || shape->vocab > DBW_DISTILL_MAX_VOCAB) return DBW_ERR_UNSUPPORTED;
    const Work W = split_work(work, S.rows);
    hipStream_t s = (hipStream_t)stream;
    if (S.rows > 0) {
        const loss::Distill P{teacher_index, teacher_logits, teacher_lse, weights, 1.f / (float)shape->rows, k, teacher_type, row_loss_out, W.terms,
                              shape->rows, loss_out};
        const size_t lds = 4 * (size_t)loss::distill_words(k, shape->vocab);
        bool fits = true;
        const auto launch = [&](auto kernel, dim3 grid, int threads, size_t bytes) {
            // more than 64 KB have to be asked for
            if (bytes > 65536) fits = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == hipSuccess;
            if (fits) hipLaunchKernelGGL(kernel, grid, dim3((uint32_t)threads), bytes, s, S.R, P);
        };
        const int row_threads = S.row_bytes <= SHORT_ROW ? 16 : 64;
        int group_threads = one_group_threads(shape, S.row_bytes, 1);
        if (group_threads / row_threads * lds > 65536) group_threads = 0;
        by_type(shape->type, [&](auto e) {
            typedef decltype(e) E;
            if (group_threads)
                by_group_row(S.row_bytes, [&](auto p) {
                    const dim3 grid = grid_of(shape->workers);
                    const size_t bytes = group_threads / p.T * lds;
                    if (teacher_lse) launch(loss::distill_worker_kernel<E, p.T, p.C, true>, grid, group_threads, bytes);
                    else launch(loss::distill_worker_kernel<E, p.T, p.C, false>, grid, group_threads, bytes);
                });
            else {
                const auto rows = [&](auto p) {
                    if (teacher_lse) launch(loss::distill_kernel<E, p.T, p.C, p.S, true>, p.grid(S.rows), p.THREADS, p.ROWS * lds);
                    else launch(loss::distill_kernel<E, p.T, p.C, p.S, false>, p.grid(S.rows), p.THREADS, p.ROWS * lds);
                };
                // Lists that 64 KB do not hold for 16 rows: a wave a row.  40000 x 700 bf16 with 350 entries 110 us,
                // with registers for 8 KB 147; 4096 x 1000 with 700 24.6 and 27.5.
                if (S.row_bytes <= SHORT_ROW && 16 * lds > 65536) rows(Plan<64, 2>());
                else by_row(S.row_bytes, rows);
            }
        });
        if (!fits) return DBW_ERR_HIP;
        DBW_HIP(hipGetLastError());
        if (group_threads) return DBW_OK;
    }
    hipLaunchKernelGGL(loss::sum_kernel, dim3((uint32_t)shape->workers), dim3(loss::THREADS), 0, s, W.terms, shape->rows, loss_out,
                       (float *)nullptr);
    DBW_HIP(hipGetLastError());
    return DBW_OK;
}

extern "C" int dbw_preference_loss(const dbw_logits *shape, int32_t pairs, const void *logits, const int32_t *tokens,
                                   const int32_t *seq_start, const float *ref_logp, const float *weights, float beta,
                                   float smoothing, float *loss_out, float *margin_out, float *logp_out, void *dlogits,
                                   int32_t *status_out, void *work, void *stream)
{
    Shape S;
    const int rc = prepare(shape, logits, dlogits, status_out, work, &S);
    if (rc != DBW_OK) return rc;
    if (!work || !loss_out || !seq_start || (pairs > 0 && !margin_out) || (S.rows > 0 && (!tokens || !ref_logp))) return DBW_ERR_NULL;
    if (pairs < 0 || !isfinite(beta) || !(smoothing >= 0.f && smoothing <= 1.f)) return DBW_ERR_INVALID;
    const int64_t all_pairs = (int64_t)shape->workers * pairs;
    if (all_pairs > MAX_GROUPS) return DBW_ERR_UNSUPPORTED;
    const Work W = split_work(work, S.rows);
    hipStream_t s = (hipStream_t)stream;
    float *const logp = logp_out ? logp_out : W.logp;
    // Few rows in few and short pairs: the gradient's workgroups sum their pairs up themselves, which costs less than a launch in between.  Two to four
    // pairs of 10 to 250 rows x 80 to 3840 bf16 11.4 us, with the launch 14.7; 128 x 20000 (40 KB) 11.8 and 14.8, but 128 x 60000 20.2 and 15.8:
    // longer rows are better read in slices, which only the launch joins.  A worker's pairs are one workgroup's, four at a time: of 1000 x 500 16 pairs
    // 13.7 and 14.2, 64 23 and 14.2, 500 116 and 14.2; and every row looks for its sequence among all: 128 pairs of 16 workers 11.1 and 14.2,
    // 512 of 64 or more workers 14.5 and 14.2.
    const bool few = pairs > 0 && pairs <= 16 && all_pairs <= 256 && S.rows > 0 && S.rows <= 1024 && S.row_bytes <= 48 << 10 && S.rows <= 64 * all_pairs;
    loss::Slices slices{1, 0};
    if (S.rows > 0) {
        if (pairs > 0 && !few) slices = slices_of(shape, S.rows, SLICED_ROWS, SLICE_GROUPS);  // (whose parts the pairs' kernel joins)
        const bool cut = slices.count > 1;
        launch_logp(shape, S, loss::Logp{tokens, weights, logp, nullptr, W.coef, cut ? W.slices : W.stats, W.token_logit, slices}, dlogits != nullptr, s);
        DBW_HIP(hipGetLastError());
    }
    const loss::PairLoss mean{margin_out, shape->workers, pairs, smoothing, loss_out};
    if (pairs > 0) {
        const loss::Preference P{tokens, seq_start, ref_logp, weights, beta, smoothing, S.R.scale, S.R.c, pairs, all_pairs, S.rows, logp, margin_out, W.coef,
                                 W.coef, W.slices, W.stats, W.token_logit, slices.count, status_out};
        if (few) {
            if (dlogits) launch_gradient(shape, S, loss::Gradient{tokens, nullptr, W.stats, nullptr, gradient_slices_of(shape, S.rows), mean}, &P, s);
            else hipLaunchKernelGGL(loss::pair_sums_kernel, dim3((uint32_t)shape->workers), dim3(loss::THREADS), 0, s, mean, P);
            DBW_HIP(hipGetLastError());
            return DBW_OK;
        }
        hipLaunchKernelGGL(loss::pair_kernel, grid_of(P.all_pairs), dim3(loss::PAIR_THREADS), 0, s, P);
        DBW_HIP(hipGetLastError());
    }
    if (dlogits && S.rows > 0)
        launch_gradient(shape, S, loss::Gradient{tokens, pairs > 0 ? W.coef : nullptr, W.stats, nullptr, gradient_slices_of(shape, S.rows), mean}, nullptr, s);
    else
        hipLaunchKernelGGL(loss::pair_loss_kernel, dim3((uint32_t)shape->workers), dim3(loss::THREADS), 0, s, mean);
    DBW_HIP(hipGetLastError());
    return DBW_OK;
}

extern "C" int dbw_policy_loss(const dbw_logits *shape, const void *logits, const int32_t *tokens, const float *old_logp,
                               const float *ref_logp, const float *advantage, const float *weights, float clip_low, float clip_high,
                               float kl_coef, float *loss_out, float *kl_out, float *logp_out, void *dlogits, int32_t *status_out,
                               void *work, void *stream)
{
    Shape S;
    const int rc = prepare(shape, logits, dlogits, status_out, work, &S);
    if (rc != DBW_OK) return rc;
    if (!work || !loss_out || (S.rows > 0 && (!tokens || !old_logp || !advantage))) return DBW_ERR_NULL;
    if (!(clip_low >= 0.f && clip_low <= 1.f) || !(clip_high >= 0.f) || !isfinite(kl_coef)) return DBW_ERR_INVALID;
    const Work W = split_work(work, S.rows);
    hipStream_t s = (hipStream_t)stream;
    if (S.rows > 0) {
        const loss::Slices slices = slices_of(shape, S.rows, POLICY_ROWS, POLICY_GROUPS);
        const bool cut = slices.count > 1;
        const int group_threads = one_group_threads(shape, S.row_bytes, 2);
        const loss::Policy P{tokens, old_logp, ref_logp, advantage, weights, 1.f - clip_low, 1.f + clip_high, kl_coef,
                             1.f / (float)shape->rows, logp_out, W.terms, W.slices, W.token_logit, slices.count, gradient_slices_of(shape, S.rows),
                             shape->rows, loss_out, kl_out};
        if (cut) launch_logp(shape, S, loss::Logp{tokens, weights, nullptr, nullptr, nullptr, W.slices, W.token_logit, slices}, dlogits != nullptr, s);
        by_type(shape->type, [&](auto e) {
            typedef decltype(e) E;
            if (cut)
                by_gradient_slice(P.slices, S.row_bytes, [&](auto p) {
                    if constexpr (p.T > 64) {             // (rows that are cut are longer)
                        const int64_t groups = (dlogits ? S.rows * P.slices.count : 0) + shape->workers;
                        hipLaunchKernelGGL((loss::policy_slices_kernel<E, p.T, p.C>), dim3((uint32_t)groups), dim3(p.T), 0, s, S.R, P);
                    }
                });
            else if (group_threads)
                by_group_row(S.row_bytes, [&](auto p) {
                    hipLaunchKernelGGL((loss::policy_worker_kernel<E, p.T, p.C>), grid_of(shape->workers), dim3(group_threads), 0, s, S.R, P);
                });
            else
                by_row(S.row_bytes, [&](auto p) {
                    hipLaunchKernelGGL((loss::policy_kernel<E, p.T, p.C, p.S>), p.grid(S.rows), dim3(p.THREADS), 0, s, S.R, P);
                });
        });
        DBW_HIP(hipGetLastError());
        if (cut || group_threads) return DBW_OK;
    }
    hipLaunchKernelGGL(loss::sum_kernel, dim3((uint32_t)shape->workers), dim3(loss::THREADS), 0, s, W.terms, shape->rows, loss_out, kl_out);
    DBW_HIP(hipGetLastError());
    return DBW_OK;
}
