/*
 * dtree_scores.h -- C ABI of libdscores: operators on rows of class scores (gfx950).
 *
 * dtree.h answers a record with one class, or (DT_OUT_VOTES_U8) with every class's number of
 * votes.  The operators here work on such answers, or on any classifier's scores:
 *   - ds_top_scores: the k best classes of each row and the row's log-sum-exp, the form in
 *     which a teacher's answers are kept.
 *   - ds_sample: one class drawn from each row by temperature, top-k, top-p and min-p, from
 *     random numbers that the caller gives.
 *   - ds_distill, ds_distill_backward: the loss of a student's scores against a teacher's
 *     top scores, and its gradient.
 *
 * Scores: n rows of n_classes elements, row r at d_x + r*ld elements, of type DT_F32, DT_F16,
 * DT_BF16 or DT_U8.  A uint8 element v is a number of votes; its score is ln(v), -inf for
 * none.  Pointers to scores need the alignment of their element, nothing more; no byte outside
 * the rows' elements is read.
 *
 * ds_top_scores and ds_sample never choose a class whose score is -inf or NaN: a row that has
 * no other is empty.  Classes of equal score count from the lowest index, -0 equals +0.
 *
 * Calls are asynchronous on `stream` (a hipStream_t; NULL = the null stream) of the current
 * device, which the buffers must belong to.  A call puts kernel launches on the stream and
 * nothing else (no allocation, copy, memset or synchronisation), so it may be captured in a
 * HIP graph.  Buffers are the caller's and must stay valid until the work completes; outputs
 * overlap neither each other nor an input; calls that may run at the same time need workspaces of
 * their own, calls that follow each other on a stream may share one.  n == 0 launches nothing.
 * Nothing is written on an error return.  All calls are noexcept; ds_last_error() has the last
 * error's message of the calling thread.
 */
#ifndef DTREE_SCORES_H
#define DTREE_SCORES_H

#include "dtree.h"

#ifdef __cplusplus
extern "C" {
#endif

#define DS_MAX_CLASSES (1 << 20)   /* classes of a row */
#define DS_MAX_TOP 256             /* k of ds_top_scores and of a teacher */
#define DS_MAX_TEMPERATURE 1152921504606846976.0f   /* of ds_distill: 2^60 */

/* Detailed message of the calling thread's last failed ds_* call ("" if none). */
const char *ds_last_error(void);

/*
 * The k best classes of each row, best first.
 *   k         1 .. min(n_classes, DS_MAX_TOP)
 *   d_values  n rows of k floats: the scores, exactly; -inf behind the row's last class with
 *             a score
 *   d_index   n rows of k int32: their classes; -1 where the value is -inf
 *   d_lse     n floats: ln(sum over the row of e^score); -inf for an empty row
 * A score of +inf is a score like any other; the row's d_lse is then +inf.
 * Errors: DT_ERR_INVALID_ARG (null pointers with n > 0, n < 0, n_classes < 1, ld < n_classes
 * with n > 1, k out of range, unknown type, misaligned pointer), DT_ERR_UNSUPPORTED
 * (n_classes > DS_MAX_CLASSES, n > 2^31 - 1), DT_ERR_HIP (launch failure).
 */
dt_status ds_top_scores(const void *d_x, dt_dtype type, int64_t n, int32_t n_classes, int64_t ld,
                        int32_t k, float *d_values, int32_t *d_index, float *d_lse, void *stream);

/*
 * How ds_sample chooses.  Each setting is a number for all rows, or, where its pointer is not
 * NULL, a device array of n of them.  With w_c = e^((score_c - best score) / temperature):
 *   temperature  > 0.  0: the best class.
 *   top_k        only the top_k best classes stay; < 1: all
 *   top_p        of these, best first, only as many stay as are needed for a share of top_p of
 *                their weight; at least the best; >= 1: all
 *   min_p        of these, only classes with w_c >= min_p stay (the best has 1); 0: all
 * Numbers outside these ranges are refused.  In arrays, which the call cannot see, they mean:
 * a temperature below 0 or NaN is 0, one of +inf makes all classes equal in weight whose score is
 * finite (if the best one's is), a top_p that is NaN is 1 and one below 0 is 0, a min_p
 * that is NaN or below 0 is 0 and one above 1 is 1.
 */
typedef struct {
    const float *d_temperature;
    const int32_t *d_top_k;
    const float *d_top_p;
    const float *d_min_p;
    float temperature;
    int32_t top_k;
    float top_p;
    float min_p;
} ds_sampling;

/*
 * One class for each row: the first, in the order of the classes, up to which the weights of
 * the classes that stay add up to more than u times their sum.
 *   d_u       n floats, each in [0, 1): uniform random numbers (below 0 or NaN counts as 0, 1
 *             and above as the largest number below 1)
 *   d_labels  n int32: the class; -1 for an empty row
 * Weights are computed in 64 bits and added as whole multiples of 2^-42 of the best class's,
 * so the result does not depend on any order of summation; a class more than 30 nats (times
 * the temperature) below the best is never drawn.  Of scores of +inf, all have weight 1 and
 * no finite score has any.  Votes at temperature 1 have their exact number as weight.
 * Errors: as ds_top_scores; DT_ERR_INVALID_ARG also for settings out of range.
 */
dt_status ds_sample(const void *d_x, dt_dtype type, int64_t n, int32_t n_classes, int64_t ld,
                    const float *d_u, const ds_sampling *settings, int32_t *d_labels,
                    void *stream);

/*
 * Distillation from a teacher's top scores.  With temperature t, the teacher's k entries
 * (value v_j, class i_j) of a row and the student's scores x of that row,
 *   p = softmax(v / t) over the entries,  q = softmax(x / t) over all classes,
 *   loss = t^2 * sum_j p_j (ln p_j - ln q_{i_j}),
 *   gradient = g * t * (q_c - sum of p_j over the entries of class c)
 * for a weight g of the row's loss.  An entry whose class is outside 0 .. n_classes - 1
 * (padding) or whose value is -inf is left out.  A row without entries, or without a student's
 * score above -inf, has loss 0 and gradient 0.  A NaN or +inf among the student's scores makes
 * the row's loss and gradient NaN; one among the teacher's remaining values makes the loss, and
 * the gradient at the teacher's classes, NaN.  A teacher's class of some weight whose student's
 * score is -inf makes the loss +inf.  The loss, a difference
 * of logarithms, is off by about 2^-22 t^2 however small it is, and more where scores are far
 * apart.
 *   type       of the student's scores and of the gradient: DT_F32, DT_F16 or DT_BF16
 *   d_values, d_index   the teacher's entries, n rows of k, 1 <= k <= DS_MAX_TOP
 *   temperature  positive: 4.5e-39 (1.5 / t is a number) .. DS_MAX_TEMPERATURE (t^2 is one)
 *   d_g        n floats; NULL: no gradient is computed (d_grad is then NULL as well)
 *   d_loss     n floats
 *   d_stats    n pairs of floats, aligned to 8, which ds_distill_backward takes: the row's
 *              largest score m and the sum of e^((x - m) / t)
 *   d_grad     n rows of n_classes, row stride ld_grad elements; must not overlap the scores
 *   d_work     workspace of at least ds_distill_work_bytes() bytes, aligned to 8 (NULL if 0)
 * Errors: as ds_top_scores; DT_ERR_INVALID_ARG also for a temperature out of range, a workspace
 * that is too small, or ld_grad < n_classes with n > 1.
 */
dt_status ds_distill(const void *d_x, dt_dtype type, int64_t n, int32_t n_classes, int64_t ld,
                     const float *d_values, const int32_t *d_index, int32_t k, float temperature,
                     const float *d_g, float *d_loss, float *d_stats, void *d_grad,
                     int64_t ld_grad, void *d_work, int64_t work_bytes, void *stream);

/* The gradient alone, from the d_stats that ds_distill wrote for the same arguments. */
dt_status ds_distill_backward(const void *d_x, dt_dtype type, int64_t n, int32_t n_classes,
                              int64_t ld, const float *d_values, const int32_t *d_index,
                              int32_t k, float temperature, const float *d_stats, const float *d_g,
                              void *d_grad, int64_t ld_grad, void *stream);

/* Bytes of workspace that ds_distill takes for n rows of n_classes; 0 for many. */
int64_t ds_distill_work_bytes(int64_t n, int32_t n_classes);

#ifdef __cplusplus
}
#endif

#endif /* DTREE_SCORES_H */
