/*
 * dbw_layers.h - what lies between the dense products of a language model, for all N simulated workers at once, with its gradients.
 *
 * The models themselves are the caller's: a round takes their gradients as ext_grads (dbw_round, dbw.h), which begin with a loss on
 * logits (dbw_losses.h).  These functions are what such a model has between its matrix products, forwards and backwards: layer norm
 * with every worker's own weights, activations that are kept in 8 bits until the backward pass needs them, and tokens that are sorted
 * by expert and brought back.  Parameters are read from, and their gradients written to, rows of [N][ld] floats as dbw_round takes them, at
 * column numbers that the caller gives.  Conventions (pointers, streams, error codes, padding) as in dbw.h; no context: nothing
 * is allocated, nothing synchronises, no memset is recorded, so the calls may be captured into a graph.  Everything asynchronous
 * on `stream`.
 *
 * Rows.  Worker i's token positions are the rows i * T + t, 0 <= t < T.  Activations and their gradients are fp32, bf16 or fp16 and
 * need no alignment beyond an element's; widths and strides may be odd.  Columns between a row's width and its stride are neither
 * read nor written.  What is computed is computed and summed in fp32 and rounded once to the type of its array.  No
 * sum depends on the order in which workgroups run: the same call gives the same bits.  Squares that pass the largest fp32 number make a norm's rho 0,
 * and a row with numbers of magnitude 2^124 and more, unless all are equal, may be NaN.  In the weight gradient from 8 bits fp32 values of
 * magnitude below 2^-110 enter to within 2^-133 each.
 *
 * Rows that take no part.  mask [dev, N*T] uint8 or NULL: a row whose entry is 0 is not read, whatever it holds (infinities, NaN); its outputs
 * are given as zeros and it adds nothing to any sum.  In the other rows infinities and NaN go through the formulas.
 *
 * In place only where an entry point says so: any other overlap of what a call writes with what it reads or writes is DBW_ERR_ALIAS where
 * both are rows of activations (also of rows that lie between one another's), and the caller's to avoid elsewhere.
 *
 * work is scratch memory of the call's, on a 16-byte boundary, of the size that the function next to the entry point gives; what it holds before and
 * after means nothing.  Calls that may overlap in time need one each.
 */
#ifndef DBW_LAYERS_H
#define DBW_LAYERS_H

#include "dbw.h"
#include "dbw_losses.h" /* DBW_TYPE_* */

#ifdef __cplusplus
extern "C" {
#endif

#define DBW_LAYER_MAX_WIDTH (1 << 20)

/* Rows of all workers, and the rows that a call makes of them. */
typedef struct {
    int32_t workers; /* N >= 1, at most 2^22 (DBW_ERR_UNSUPPORTED beyond) */
    int32_t rows;    /* T >= 0 token positions of each worker; N * T < 2^31 (DBW_ERR_UNSUPPORTED beyond) */
    int32_t width;   /* D >= 1 columns, at most DBW_LAYER_MAX_WIDTH (DBW_ERR_UNSUPPORTED beyond) */
    int32_t type;    /* DBW_TYPE_* of all arrays of rows */
    int64_t ld;      /* stride of the rows that go in, in elements, >= D; 0 means D.  An array's gradient has the array's stride */
    int64_t ld_out;  /* stride of the rows that come out, >= D; 0 means ld */
} dbw_rows;

/* ---- activations in 8 bits -------------------------------------------------------------------------------------------------
 *
 * 32 columns of a row share a power of two 2^e; each of them is one byte, a number of 4 significant bits (sign, 4 bits of exponent, 3 of
 * fraction; the format e4m3, whose largest value is 448 and smallest 2^-9).  e is the smallest integer with which the block's largest finite
 * magnitude is at most 448 2^e, at least -117; values are rounded to the nearest, ties to even.  So a value is off by at most 2^-4 of
 * itself or 2^-10 2^e, whichever is more; magnitudes of 1.875 2^127 and more are kept as that, infinities and NaN as NaN, which leave
 * the block's other columns as they are.  What a code stands for is exact in bf16 and fp32.
 *
 * A checkpoint [dev, dbw_checkpoint_bytes(shape) bytes, on a 16-byte boundary] holds the codes of all rows, each padded with zeros to a
 * multiple of 32, one row behind the other, and behind them a byte e + 127 for every block of every row.  It is the same for
 * all three types, and goes by the shape's workers, rows and width alone. */

/* Bytes of a checkpoint of rows of this shape, or a negative DBW_ERR_* code. */
int64_t dbw_checkpoint_bytes(const dbw_rows *shape);

/* Puts rows x [dev, stride ld] into a checkpoint.  Rows that take no part are kept as zeros. */
int dbw_checkpoint_store(const dbw_rows *shape, const void *x, const uint8_t *mask, void *checkpoint, void *stream);

/* What the checkpoint's rows stand for, rounded to the shape's type (exact but for fp16): x_out [dev, stride ld_out]. */
int dbw_checkpoint_load(const dbw_rows *shape, const void *checkpoint, void *x_out, void *stream);

/* ---- layer norm ------------------------------------------------------------------------------------------------------------
 *
 * Of a row x of worker i, with that worker's weight w and bias b,
 *     mu = mean of x,  rho = 1 / sqrt(mean of (x - mu)^2 + eps),  y_c = w_c rho (x_c - mu) + b_c.
 *   params     [dev, N * ld_params] float: worker i's weight is the D columns from weight_at on of row i, its bias those from bias_at on;
 *              weight_at or bias_at negative: none (w = 1, b = 0); both: params is not read and may be NULL
 *   eps        > 0, finite
 *   y          [dev, stride ld_out]; may be x itself (same pointer and stride)
 *   stats_out  [dev, N*T*2] float mu and rho of every row (0 where it takes no part), for the backward pass, or NULL
 *   checkpoint as dbw_checkpoint_store makes it of x, or NULL */
int dbw_layer_norm(const dbw_rows *shape, const void *x, const uint8_t *mask, const float *params, int64_t ld_params,
                   int64_t weight_at, int64_t bias_at, float eps, void *y, float *stats_out, void *checkpoint, void *stream);

int64_t dbw_layer_norm_work_bytes(const dbw_rows *shape);

/* Its backward pass, from dy [dev, stride ld_out].  With u_c = rho (x_c - mu) and g_c = w_c dy_c,
 *     dx_c = rho (g_c - mean of g - u_c mean of (g u)),  dw_c = sum over the worker's rows of dy_c u_c,  db_c = sum of dy_c.
 *   x          [dev, stride ld], or NULL: what `checkpoint` stands for is taken for x (one of the two is given).  That is off by 2^-4 of x at most, and so
 *              u by 2^-4 of |x| rho: where a row's mean is large beside its spread, u is lost by |mu| rho 2^-4, whatever the spread
 *   stats      mu and rho as dbw_layer_norm gave them; u takes mu's own rounding, 2^-24 |mu| rho, where the forward pass does not
 *   dx         [dev, stride ld]; may be x itself, or dy if the strides are equal
 *   grads      [dev, N * ld_grads] float: dw goes to the columns from weight_at on of every worker's row, db to those from
 *              bias_at on; the other columns are left as they are.  A part whose column number is negative is not wanted; NULL: neither is
 *   params     as above, read for the weight alone */
int dbw_layer_norm_grad(const dbw_rows *shape, const void *dy, const void *x, const void *checkpoint, const uint8_t *mask,
                        const float *stats, const float *params, int64_t ld_params, int64_t weight_at, int64_t bias_at, void *dx,
                        float *grads, int64_t ld_grads, void *work, void *stream);

/* ---- tokens by expert ------------------------------------------------------------------------------------------------------
 *
 * Every token t of a worker has k slots, t * k + j, each of which names one of the worker's E experts or none.  Sorted rows are the
 * slots in the order of their experts, those of one expert in their own order: worker i's are rows i * T * k and on, as many as
 * its slots name experts; the rows behind them up to (i + 1) * T * k are nobody's, and are neither read nor written. */
#define DBW_EXPERTS_MAX 1024
typedef struct {
    int32_t workers; /* N >= 1, at most 2^22 (DBW_ERR_UNSUPPORTED beyond) */
    int32_t tokens;  /* T >= 0 of each worker */
    int32_t k;       /* slots of a token, >= 1; N * T * k < 2^31 (DBW_ERR_UNSUPPORTED beyond) */
    int32_t experts; /* E >= 1 of each worker, at most DBW_EXPERTS_MAX; N * (E + 1) < 2^31 (DBW_ERR_UNSUPPORTED beyond) */
} dbw_routing;

int64_t dbw_expert_work_bytes(const dbw_routing *routing);

/* The order of the slots.
 *   expert     [dev, N*T*k] int32; negative: the slot names none.  >= E: reported, and taken as none.  A token may name an expert twice
 *   start_out  [dev, N*(E+1)] int32: expert e of worker i has the sorted rows start[i (E+1) + e] ... start[i (E+1) + e + 1] - 1
 *   place_out  [dev, N*T*k] int32: the sorted row of each slot, -1 where it names none
 *   source_out [dev, N*T*k] int32: the slot of each sorted row, -1 for rows that are nobody's
 *   status_out [dev, 1] int32 or NULL, as in dbw_losses.h, also in the functions below */
int dbw_expert_sort(const dbw_routing *routing, const int32_t *expert, int32_t *start_out, int32_t *place_out, int32_t *source_out,
                    int32_t *status_out, void *work, void *stream);

/* Tokens' rows x [dev, stride ld] into the sorted rows `sorted` [dev, stride ld_out]: row place[t k + j] becomes row t.
 * place as dbw_expert_sort gave it, no row twice; an entry that is none of its worker's sorted rows is reported, and taken as -1.
 * In this and the following functions the shape's workers and rows are the routing's N and T. */
int dbw_expert_gather(const dbw_routing *routing, const dbw_rows *shape, const void *x, const int32_t *place, void *sorted,
                      int32_t *status_out, void *stream);

/* Sorted rows added up for each token: y_t = sum over j of weights[t k + j] times sorted row place[t k + j], slots that name none left out
 * whatever their weight; a token without any gets zeros.  Without weights (NULL, 1 each) this is the gradient of dbw_expert_gather.
 *   sorted [dev, stride ld_out], weights [dev, N*T*k] float or NULL, y [dev, stride ld] */
int dbw_expert_combine(const dbw_routing *routing, const dbw_rows *shape, const void *sorted, const int32_t *place, const float *weights,
                       void *y, int32_t *status_out, void *stream);

/* The gradient of that, from dy [dev, stride ld]: dsorted row place[t k + j] = weights[t k + j] dy_t, and dweights[t k + j] = the sum over the columns of
 * dy_t times sorted row place[t k + j] (0 where the slot names none).
 *   dsorted [dev, stride ld_out]; may be `sorted` itself;  dweights [dev, N*T*k] float, or NULL, and then `sorted` is not read and may be NULL */
int dbw_expert_combine_grad(const dbw_routing *routing, const dbw_rows *shape, const void *dy, const void *sorted, const int32_t *place,
                            const float *weights, void *dsorted, float *dweights, int32_t *status_out, void *stream);

/* ---- the weight gradient of a linear layer whose input was kept in 8 bits --------------------------------------------------
 *
 * Of y = W x + b with W [outputs][inputs]: dW = sum over rows of dy x', db = sum of dy, x being what the checkpoint stands for.  Every worker
 * has E layers (experts; 1: an ordinary layer), one behind the other: worker i's dW of layer e goes to the outputs * inputs columns from
 * weight_at + e outputs inputs on of row i of grads, its db to those from bias_at + e outputs on. */
typedef struct {
    int32_t workers; /* N >= 1, at most 2^22 */
    int32_t rows;    /* R >= 0 rows of dy of each worker; N * R < 2^31 */
    int32_t inputs, outputs; /* widths >= 1, at most DBW_LAYER_MAX_WIDTH */
    int32_t type;    /* DBW_TYPE_* of dy */
    int32_t experts; /* E >= 1, at most DBW_EXPERTS_MAX; N * (E + 1) < 2^31 */
    int32_t tokens;  /* T >= 0 rows of the checkpoint of each worker; N * T < 2^31.  (DBW_ERR_UNSUPPORTED beyond any of these) */
    int32_t k;       /* slots of a token, >= 1 */
    int64_t ld;      /* stride of dy's rows, >= outputs; 0 means outputs */
} dbw_linear;

int64_t dbw_checkpoint_weight_grad_work_bytes(const dbw_linear *shape);

/*   dy         [dev, N*R rows]
 *   checkpoint of N*T rows of `inputs` columns
 *   start      [dev, N*(E+1)] int32 as dbw_expert_sort gave it, or NULL with E = 1: all R rows of a worker.  Rows in no layer are not read.
 *              Numbers out of order or beyond the worker's rows are reported, and the results mean nothing
 *   source     [dev, N*R] int32 as dbw_expert_sort gave it: row p of dy belongs to row source[p] / k of the checkpoint, which is the tokens'
 *              before sorting (one that is none of the worker's is reported, and its row left out).  NULL: to row p; R = T then
 *   grads      [dev, N * ld_grads] float; bias_at negative: db is not wanted.  The gradient of a layer without rows is zeros */
int dbw_checkpoint_weight_grad(const dbw_linear *shape, const void *dy, const void *checkpoint, const int32_t *start,
                               const int32_t *source, float *grads, int64_t ld_grads, int64_t weight_at, int64_t bias_at,
                               int32_t *status_out, void *work, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* DBW_LAYERS_H */
