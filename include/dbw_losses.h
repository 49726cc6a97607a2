/*
 * dbw_losses.h - losses on the logits of language models, for all N simulated workers at once, with the logits' gradients.
 *
 * The models themselves are the caller's: a round takes their gradients as ext_grads (dbw_round, dbw.h).  These functions
 * are the end of such a model: rows of V logits, one for every token position of every worker, go in; every worker's loss
 * and the gradient with respect to the logits come out.  Conventions (pointers, streams, error codes, padding) as in
 * dbw.h; no context: nothing is allocated, nothing synchronises, no memset is recorded, so the calls may be captured into
 * a graph.  Everything asynchronous on `stream`.
 *
 * Rows.  Worker i's token positions are the rows i * T + t, 0 <= t < T; row r starts at element r * ld.  Logits and
 * gradients are fp32, bf16 or fp16 and need no alignment beyond an element's; V and ld may be odd.  With s = `scale` (one
 * over the temperature) the model's distribution in a row x is p_v = exp(s x_v - L), L = log sum_v exp(s x_v).
 *
 * Precision.  Exponentials, losses and gradients are computed in fp32, sums in fp32 or more; a gradient is rounded once to the type of the
 * logits.  A log-probability is off by about 2^-24 before it is rounded to fp32, to either side alike, and enters a preference loss's sums before
 * that rounding: they are held in 64 bits.  No sum depends on the order in which workgroups run: the same call gives the same bits.
 *
 * Rows that take no part.  A row whose token is negative or whose weight is 0 is not read: whatever its logits and its
 * other inputs hold (infinities, NaN), it adds nothing to any sum, its log-probability is given as 0 and its gradient
 * as zeros.  In the other rows a logit of -inf is a token that cannot occur (p_v = 0, gradient 0), and +inf, NaN
 * or a row of nothing but -inf gives NaN, as the formulas do.
 *
 * In place.  dlogits may be the same array as logits (same pointer and stride); any other overlap of the two is
 * DBW_ERR_ALIAS.  The other arrays must not overlap what the call writes.
 *
 * status_out [dev, 1] int32 or NULL is set to DBW_ERR_INVALID if the data are (a token beyond the vocabulary, a teacher's
 * index beyond it or twice in a row, offsets of sequences out of order) and otherwise left as it is: clear it before
 * the first call and look when convenient.
 *
 * work [dev, dbw_loss_work_bytes(shape) bytes, on an 8-byte boundary] is scratch memory of the call's; what it holds before and after means
 * nothing.  Calls that may overlap in time need one each.
 */
#ifndef DBW_LOSSES_H
#define DBW_LOSSES_H

#include "dbw.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { DBW_TYPE_F32 = 0, DBW_TYPE_BF16 = 1, DBW_TYPE_F16 = 2 };

#define DBW_LOSS_MAX_VOCAB (1 << 28)

/* Logits of all workers, and their gradient. */
typedef struct {
    int32_t workers; /* N >= 1, at most 2^22 */
    int32_t rows;    /* T >= 0 token positions of each worker; N * T < 2^31 (DBW_ERR_UNSUPPORTED beyond) */
    int32_t vocab;   /* V >= 1 columns, at most DBW_LOSS_MAX_VOCAB (DBW_ERR_UNSUPPORTED beyond) */
    int32_t type;    /* DBW_TYPE_* of logits and dlogits */
    int64_t ld;      /* stride of the logits' rows in elements, >= V; 0 means V */
    int64_t ld_grad; /* stride of dlogits' rows, >= V; 0 means ld.  Columns [V, ld_grad) are not written */
    float scale;     /* s > 0, s log2(e) finite */
} dbw_logits;

/* Bytes of scratch memory for any call on this shape, or a negative DBW_ERR_* code. */
int64_t dbw_loss_work_bytes(const dbw_logits *shape);

/* Log-probabilities of given tokens: logp_out[r] = s x_y - L with y = tokens[r].
 *   tokens   [dev, N*T] int32; negative: the row takes no part; >= V is taken as V - 1 and reported
 *   logp_out [dev, N*T] float
 *   lse_out  [dev, N*T] float L of every row (0 where it takes no part), for dbw_token_logp_grad, or NULL */
int dbw_token_logp(const dbw_logits *shape, const void *logits, const int32_t *tokens, float *logp_out, float *lse_out,
                   int32_t *status_out, void *work, void *stream);

/* Gradient of a function of the log-probabilities: with c_r its derivative with respect to logp_out[r] (coef [dev, N*T]),
 * dlogits[r][v] = s c_r ([v = y] - p_v).  lse as dbw_token_logp gave it for these logits.  A row with c_r = 0 takes no part.
 * The rounding of L enters every p_v, by up to 2^-17 of it where |L| <= 256; a row with a larger L, of which too little of the
 * logarithm would be left, is summed again (one workgroup takes the whole row, so many such rows cost little and a few long ones latency). */
int dbw_token_logp_grad(const dbw_logits *shape, const void *logits, const int32_t *tokens, const float *lse,
                        const float *coef, void *dlogits, int32_t *status_out, void *stream);

/* Distillation from a teacher's top logits: a row's loss is the divergence of p from the teacher's distribution q,
 * given by the logits t_j of k tokens K of the teacher's choice (the best k, say) at the same scale s.
 * Without teacher_lse, q is normalised over K: q_j = exp(s t_j) / sum_K exp(s t),
 *     l = sum_K q_j log(q_j / p_j),     dl/dx_v = s (p_v - q_v).
 * With teacher_lse [dev, N*T] (the teacher's own L over its whole vocabulary) q_j = exp(s t_j - teacher_lse), and everything
 * outside K is one more class with the rest of either mass, R = max(0, 1 - sum_K q) and S = sum of p_v outside K:
 *     l = sum_K q_j log(q_j / p_j) + R log(R / S),     dl/dx_v = s (p_v - q_v) in K, s p_v (1 - R / S) outside.
 * Where nothing can lie outside K (S = 0: K is the whole vocabulary, or all other logits are -inf) an R of up to 2^-22 (|teacher_lse| + 12) is
 * taken for the rounding of teacher_lse and for no rest; a larger one makes the loss infinite.
 * loss_out[i] = sum over worker i's rows of weights[r] l_r; the gradient carries the weights too.  (A factor of 1 / s^2 that keeps
 * gradients comparable between temperatures goes into the weights.)
 *   k               1 <= k <= DBW_TEACHER_MAX
 *   teacher_index   [dev, N*T*k] int32; negative: absent (a shorter list); beyond the vocabulary, or a second time in its
 *                   row: reported, and absent
 *   teacher_logits  [dev, N*T*k] of teacher_type (DBW_TYPE_*); -inf is a token of K with q = 0.  A row whose list leaves nothing
 *                   (no entry, or without teacher_lse none above -inf) takes no part
 *   weights         [dev, N*T] float or NULL (1 / T each); 0: the row takes no part
 *   loss_out        [dev, N] float;  row_loss_out [dev, N*T] float l_r or NULL;  dlogits as logits, or NULL
 * V <= DBW_DISTILL_MAX_VOCAB (DBW_ERR_UNSUPPORTED beyond). */
#define DBW_TEACHER_MAX 1024
#define DBW_DISTILL_MAX_VOCAB (1 << 20)
int dbw_distill_loss(const dbw_logits *shape, int32_t k, const void *logits, const int32_t *teacher_index,
                     int32_t teacher_type, const void *teacher_logits, const float *teacher_lse, const float *weights,
                     float *loss_out, float *row_loss_out, void *dlogits, int32_t *status_out, void *work, void *stream);

/* Preference loss on paired log ratios.  Sequence q is the rows [seq_start[q], seq_start[q + 1]) (any length, also none);
 * pair j = sequences 2j (preferred) and 2j + 1, and worker i has the pairs i * pairs ... (i + 1) * pairs - 1.  With the summed log ratios
 * h_q = sum over the sequence of weights[r] (logp_r - ref_logp[r]):
 *     u_j = beta (h_2j - h_2j+1),   l_j = -(1 - a) log sigma(u_j) - a log sigma(-u_j),   a = smoothing,
 * loss_out[i] = mean of worker i's l_j (0 without pairs).
 *   seq_start  [dev, 2*N*pairs + 1] int32, ascending within [0, N*T] (otherwise reported, and the results mean nothing)
 *   tokens     as dbw_token_logp;  ref_logp [dev, N*T] float, not read where a row takes no part
 *   weights    [dev, N*T] float or NULL (1 each; 1 / length gives mean ratios); 0: the row takes no part
 *   beta       finite;  smoothing in [0, 1]
 *   margin_out [dev, N*pairs] float u_j;  logp_out [dev, N*T] float or NULL;  dlogits as logits, or NULL
 * Rows in no sequence have a zero gradient.  N * pairs <= 2^22 (DBW_ERR_UNSUPPORTED beyond). */
int dbw_preference_loss(const dbw_logits *shape, int32_t pairs, const void *logits, const int32_t *tokens,
                        const int32_t *seq_start, const float *ref_logp, const float *weights, float beta,
                        float smoothing, float *loss_out, float *margin_out, float *logp_out, void *dlogits,
                        int32_t *status_out, void *work, void *stream);

/* Clipped policy loss with a KL term.  With rho = exp(logp_r - old_logp[r]), A = advantage[r], d = ref_logp[r] - logp_r:
 *     kl_r = exp(d) - d - 1,   l_r = -min(rho A, clip(rho, 1 - clip_low, 1 + clip_high) A) + kl_coef kl_r,
 *     dl/dlogp = -(rho A where rho A <= clip(rho) A, else 0) + kl_coef (1 - exp(d)),
 * loss_out[i] = sum over worker i's rows of weights[r] l_r; kl_out[i] likewise of kl_r.
 *   tokens     as dbw_token_logp;  old_logp, ref_logp, advantage [dev, N*T] float, not read where a row takes no part;
 *              ref_logp may be NULL (no KL term: kl_r = 0)
 *   weights    [dev, N*T] float or NULL (1 / T each); 0: the row takes no part
 *   clip_low in [0, 1], clip_high >= 0, kl_coef finite
 *   loss_out, kl_out [dev, N] float, logp_out [dev, N*T] float, dlogits as logits; all but loss_out may be NULL */
int dbw_policy_loss(const dbw_logits *shape, const void *logits, const int32_t *tokens, const float *old_logp,
                    const float *ref_logp, const float *advantage, const float *weights, float clip_low, float clip_high,
                    float kl_coef, float *loss_out, float *kl_out, float *logp_out, void *dlogits, int32_t *status_out,
                    void *work, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* DBW_LOSSES_H */
