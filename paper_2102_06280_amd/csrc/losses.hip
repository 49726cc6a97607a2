// Entry points of the losses on logits (dbw_losses.h): argument checks and launches.  No context and no allocation: what the
// kernels need beyond inputs and outputs is the caller's scratch memory.
#include <math.h>

#include "dbw_internal.h"
#include "dbw_losses.h"
#include "loss_rows.h"

namespace {

size_t size_of(int type) { return type == DBW_TYPE_F32 ? 4 : 2; }

constexpr int64_t MAX_GROUPS = 1 << 22;   // of kernels that take a workgroup per worker or pair

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
    if (!(l->scale > 0.f) || !isfinite(l->scale * loss::LOG2E)) return DBW_ERR_INVALID;
    out->rows = (int64_t)l->workers * l->rows;
    if (l->vocab > DBW_LOSS_MAX_VOCAB || l->workers > MAX_GROUPS || out->rows > INT32_MAX || out->ld > INT64_MAX / 8 / (out->rows + 1) || out->ld_grad > INT64_MAX / 8 / (out->rows + 1))
        return DBW_ERR_UNSUPPORTED;
    return DBW_OK;
}

// Scratch memory: per row the maximum and the sum, and two terms of a loss (or its coefficient and its log-probability).
struct Work {
    loss::MaxSum *stats;
    float2 *terms;
    float *coef, *logp;
};
constexpr int64_t WORK_PER_ROW = 16;

Work split_work(void *work, int64_t rows)
{
    Work w;
    w.stats = (loss::MaxSum *)work;
    w.terms = (float2 *)(w.stats + rows);
    w.coef = (float *)w.terms;
    w.logp = w.coef + rows;
    return w;
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
    S->R = loss::Rows{logits, dlogits, S->ld, S->ld_grad, l->vocab, S->rows, l->scale, l->scale * loss::LOG2E, status};
    return DBW_OK;
}

dim3 grid_of(int64_t rows)
{
    const int64_t x = rows < (1 << 20) ? rows : 1 << 20;
    return dim3((uint32_t)x, (uint32_t)((rows + x - 1) / x));
}

// Threads and pieces a thread for rows of that many bytes.  A row of up to 16 KB a wave, or 256 KB a workgroup, stays in registers; longer ones are walked in batches.
template <int T_, int C_, int S_ = 0>
struct Plan {
    static constexpr int T = T_, C = C_, S = S_;
};
template <class F>
void by_row(int64_t bytes, F f)
{
    if (bytes <= 2 * 64 * 16) f(Plan<64, 2>());
    else if (bytes <= 8 * 64 * 16) f(Plan<64, 8>());
    else if (bytes <= 4 * 256 * 16) f(Plan<256, 4>());
    else if (bytes <= 8 * 256 * 16) f(Plan<256, 8>());
    else if (bytes <= 16 * 256 * 16) f(Plan<512, 8>());
    else if (bytes <= 16 * 512 * 16) f(Plan<512, 16>());
    else f(Plan<512, 16, 8>());
}
// Calls f with a value of the logits' type.
template <class F>
void by_type(int type, F f)
{
    if (type == DBW_TYPE_F32) f(float());
    else if (type == DBW_TYPE_BF16) f(loss::bf16());
    else f(loss::f16());
}
// The kernels that only read a row, or only write one from what is known of it, need not hold it.
template <class F>
void by_length(int64_t bytes, F f)
{
    if (bytes <= 8 * 64 * 16) f(Plan<64, 2>());
    else if (bytes <= 128 << 10) f(Plan<256, 8>());
    else f(Plan<1024, 8>());
}

}  // namespace

extern "C" int64_t dbw_loss_work_bytes(const dbw_logits *shape)
{
    Shape S;
    const int rc = check_shape(shape, &S);
    return rc == DBW_OK ? WORK_PER_ROW * (S.rows + 1) : rc;
}

extern "C" int dbw_token_logp(const dbw_logits *shape, const void *logits, const int32_t *tokens, float *logp_out, float *lse_out,
                              int32_t *status_out, void *work, void *stream)
{
    Shape S;
    const int rc = prepare(shape, logits, nullptr, status_out, work, &S);
    if (rc != DBW_OK) return rc;
    if (!work || (S.rows > 0 && (!tokens || !logp_out))) return DBW_ERR_NULL;
    if (S.rows == 0) return DBW_OK;
    const loss::Logp P{tokens, logp_out, lse_out, nullptr, nullptr};
    by_type(shape->type, [&](auto e) {
        by_length(S.row_bytes, [&](auto p) {
            const dim3 grid = grid_of(S.rows), block(p.T);
            // L is asked for where a gradient follows
            if (lse_out) hipLaunchKernelGGL((loss::logp_kernel<decltype(e), p.T, p.C, true>), grid, block, 0, (hipStream_t)stream, S.R, P);
            else hipLaunchKernelGGL((loss::logp_kernel<decltype(e), p.T, p.C, false>), grid, block, 0, (hipStream_t)stream, S.R, P);
        });
    });
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
    by_type(shape->type, [&](auto e) {
        by_length(S.row_bytes, [&](auto p) {
            hipLaunchKernelGGL((loss::gradient_kernel<decltype(e), p.T, p.C>), grid_of(S.rows), dim3(p.T), 0, (hipStream_t)stream, S.R,
                               tokens, (const loss::MaxSum *)nullptr, lse, coef);
        });
    });
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
        const loss::Distill P{teacher_index, teacher_logits, teacher_lse, weights, 1.f / (float)shape->rows, k, teacher_type, row_loss_out, W.terms};
        const size_t lds = 4 * ((size_t)3 * k + ((size_t)shape->vocab + 8 + 31) / 32);
        bool fits = true;
        const auto launch = [&](auto kernel, int threads) {
            // more than 64 KB have to be asked for
            if (lds > 65536) fits = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) == hipSuccess;
            if (fits) hipLaunchKernelGGL(kernel, grid_of(S.rows), dim3((uint32_t)threads), lds, s, S.R, P);
        };
        by_type(shape->type, [&](auto e) {
            by_row(S.row_bytes, [&](auto p) {
                if (teacher_lse) launch(loss::distill_kernel<decltype(e), p.T, p.C, p.S, true>, p.T);
                else launch(loss::distill_kernel<decltype(e), p.T, p.C, p.S, false>, p.T);
            });
        });
        if (!fits) return DBW_ERR_HIP;
        DBW_HIP(hipGetLastError());
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
    if ((int64_t)shape->workers * pairs > MAX_GROUPS) return DBW_ERR_UNSUPPORTED;
    const Work W = split_work(work, S.rows);
    hipStream_t s = (hipStream_t)stream;
    float *const logp = logp_out ? logp_out : W.logp;
    if (S.rows > 0) {
        const loss::Logp P{tokens, logp, nullptr, W.stats, weights};
        by_type(shape->type, [&](auto e) {
            by_length(S.row_bytes, [&](auto p) {
                hipLaunchKernelGGL((loss::logp_kernel<decltype(e), p.T, p.C, true>), grid_of(S.rows), dim3(p.T), 0, s, S.R, P);
            });
        });
        DBW_HIP(hipGetLastError());
    }
    if (pairs > 0) {
        const loss::Preference P{tokens, seq_start, logp, ref_logp, weights, beta, smoothing, pairs, S.rows, margin_out, W.coef, status_out};
        hipLaunchKernelGGL(loss::pair_kernel, dim3((uint32_t)(shape->workers * pairs)), dim3(loss::THREADS), 0, s, P);
        DBW_HIP(hipGetLastError());
    }
    hipLaunchKernelGGL(loss::pair_loss_kernel, dim3((uint32_t)shape->workers), dim3(loss::THREADS), 0, s, margin_out, pairs, smoothing,
                       loss_out);
    DBW_HIP(hipGetLastError());
    if (dlogits && S.rows > 0) {
        by_type(shape->type, [&](auto e) {
            by_length(S.row_bytes, [&](auto p) {
                hipLaunchKernelGGL((loss::gradient_kernel<decltype(e), p.T, p.C>), grid_of(S.rows), dim3(p.T), 0, s, S.R, tokens,
                                   (const loss::MaxSum *)W.stats, (const float *)nullptr, (const float *)(pairs > 0 ? W.coef : nullptr));
            });
        });
        DBW_HIP(hipGetLastError());
    }
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
        const loss::Policy P{tokens, old_logp, ref_logp, advantage, weights, 1.f - clip_low, 1.f + clip_high, kl_coef,
                             1.f / (float)shape->rows, logp_out, W.terms};
        by_type(shape->type, [&](auto e) {
            by_row(S.row_bytes, [&](auto p) {
                hipLaunchKernelGGL((loss::policy_kernel<decltype(e), p.T, p.C, p.S>), grid_of(S.rows), dim3(p.T), 0, s, S.R, P);
            });
        });
        DBW_HIP(hipGetLastError());
    }
    hipLaunchKernelGGL(loss::sum_kernel, dim3((uint32_t)shape->workers), dim3(loss::THREADS), 0, s, W.terms, shape->rows, loss_out, kl_out);
    DBW_HIP(hipGetLastError());
    return DBW_OK;
}
