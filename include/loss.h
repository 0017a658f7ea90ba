/*
 * loss.h -- C ABI of the MI355X (gfx950) losses over a layer's outputs: softmax
 * cross entropy over many classes (a vocabulary) and distillation from a teacher's
 * largest logits, each with its gradients, without the logits in memory.
 *
 * The layer is linear.h's: F is kn x ci (kn classes of ci features), X is ci x t (one
 * column per token) and Z = F X + bias 1^T (kn x t).  Column n of Z gives
 *        lse_n = log sum_m exp(Z_mn / T),        p_mn = exp(Z_mn / T - lse_n).
 *
 * Cross entropy (T = 1), y_n the label of column n:
 *        loss_n = lse_n - Z_{y_n n},             dZ_mn = g_n (p_mn - [m = y_n]).
 * Where y_n is `ignore`, loss_n is 0 and column n adds nothing to any gradient; a label
 * outside 0 .. kn - 1 that is not `ignore` gives a NaN loss and NaN gradients.
 *
 * Distillation, i_jn and v_jn (j < k) the teacher's largest logits of column n:
 *        q_jn = exp(v_jn / T) / sum_j exp(v_jn / T),
 *        loss_n = T^2 sum_j q_jn (log q_jn - (Z_{i_jn n} / T - lse_n)),
 *        dZ_mn = g_n T (p_mn - sum_{j: i_jn = m} q_jn).
 * Entries with a negative index or the logit -infinity do not count (columns may have
 * fewer than k); a column without any has loss 0 and adds nothing to any gradient.
 * The same class may come several times, each entry counts.  An index from kn on gives
 * a NaN loss and NaN gradients.
 *
 * g_n = dL/dloss_n; gradients: dX = F^T dZ, dF = dZ X^T, dbias = dZ 1.  A column with
 * g_n = 0, or one that does not count, adds nothing to dF and dbias even where X or Z
 * are infinite or NaN there or its target is invalid; its dX is zero where F is finite
 * (a product with zeros, so that an infinity or a NaN of F makes it NaN).
 *
 * Classes can be masked by a bias of -infinity: p is 0 there.  A column in which every
 * class is masked has lse = -infinity and NaN gradients.
 *
 * Types: F, X, bias, dX, dF and dbias are LINEAR_F32, LINEAR_BF16 or LINEAR_F16
 * (linear.h); losses, lse and g are fp32.  Z is summed in fp32, and everything up to
 * the loss is computed in fp32; exponentials of 16-bit layers' Z are the hardware's, off by
 * up to about 2^-22, also in the fp32 loss.  The gradients compute Z again, a piece of the
 * classes at a time (at most 8192 of them, or 256 MB of dZ where that is more; several pieces have
 * about as many each); a piece's dZ is held in the layer's type, one rounding
 * (16-bit types: times a factor that puts the largest finite |g| T at 2^15, so that
 * neither large nor small g leave fp16's range), dX is added up over the pieces in fp32,
 * and each result is rounded once: a 16-bit dX or dF is off by up to about 1.4 roundings
 * in its norm.  dbias is summed before that rounding.  Every result is reproducible.
 *
 * Storage and rules are linear.h's: X and dX have their first index fastest and a
 * leading dimension; F and dF have either index fastest (f_order); any address and
 * leading dimension that the type allows are taken; pointers are DEVICE pointers of
 * the current HIP device; calls are stream-ordered, nothing is retained, the caller
 * owns the workspace (at least the bytes that the query names, 16-byte aligned, or NULL
 * where that is 0; calls on different streams or in different captured graphs need one
 * each).  Outputs may not overlap inputs or one another.  Return value: 0, or -i when
 * argument i (1-based) is invalid, with nothing enqueued, or LINEAR_ERR_HIP_BASE - e.
 */
#ifndef LOSS_H
#define LOSS_H

#include <stdint.h>
#include <hip/hip_runtime_api.h>

#include "linear.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Types of labels and indices. */
#define LOSS_I32 1
#define LOSS_I64 2

/* Most entries of a column's teacher. */
#define LOSS_MAX_K 1024

/* Bytes of workspace of the two forward calls (host only; k = 0 for labels), or -i
 * when argument i is invalid.  aligned = 1 says that F and X have 16-byte aligned
 * addresses and leading dimensions of whole 16 bytes, below 2^22 bytes; what 0 gives
 * is enough for any. */
int64_t convgemm_linear_loss_workspace(int dtype, int64_t kn, int64_t ci, int64_t t, int f_order, int k, int aligned);

/* loss_n and lse_n (t values each) from labels.
 *   dtype .. bias     : as in convgemm_linear;
 *   labels, itype     : t values of type LOSS_I32 or LOSS_I64;
 *   ignore            : the label of columns that do not count. */
int convgemm_linear_cross_entropy(int dtype, int64_t kn, int64_t ci, int64_t t, const void* F, int f_order, int64_t ldf,
                                  const void* X, int64_t ldx, const void* bias, const void* labels, int itype, int64_t ignore,
                                  float* loss, float* lse, void* workspace, int64_t workspace_bytes, hipStream_t stream);

/* loss_n and lse_n (of Z / T) from a teacher's logits.
 *   top, ttype, ldtop : k x t logits, first index fastest, of type LINEAR_*;
 *   index, itype, ldi : their classes, k x t, first index fastest;
 *   k                 : 1 .. LOSS_MAX_K;
 *   temperature       : T > 0. */
int convgemm_linear_distill(int dtype, int64_t kn, int64_t ci, int64_t t, const void* F, int f_order, int64_t ldf,
                            const void* X, int64_t ldx, const void* bias, int k, const void* top, int ttype, int64_t ldtop,
                            const void* index, int itype, int64_t ldi, double temperature, float* loss, float* lse,
                            void* workspace, int64_t workspace_bytes, hipStream_t stream);

/* Bytes of workspace of the two backward calls (host only; k = 0 for labels). */
int64_t convgemm_linear_loss_backward_workspace(int dtype, int64_t kn, int64_t ci, int64_t t, int f_order, int k, int aligned);

/* dX, dF (F's order) and dbias; each may be NULL and is then not computed (the
 * bytes that the query names are enough all the same).
 *   lse               : what the forward call gave;
 *   g, ginc           : dL/dloss_n at g[n ginc]; ginc = 0: one value for all columns. */
int convgemm_linear_cross_entropy_backward(int dtype, int64_t kn, int64_t ci, int64_t t, const void* F, int f_order,
                                           int64_t ldf, const void* X, int64_t ldx, const void* bias, const void* labels,
                                           int itype, int64_t ignore, const float* lse, const float* g, int ginc, void* dX,
                                           int64_t lddx, void* dF, int64_t lddf, void* dbias, void* workspace,
                                           int64_t workspace_bytes, hipStream_t stream);

int convgemm_linear_distill_backward(int dtype, int64_t kn, int64_t ci, int64_t t, const void* F, int f_order, int64_t ldf,
                                     const void* X, int64_t ldx, const void* bias, int k, const void* top, int ttype,
                                     int64_t ldtop, const void* index, int itype, int64_t ldi, double temperature,
                                     const float* lse, const float* g, int ginc, void* dX, int64_t lddx, void* dF,
                                     int64_t lddf, void* dbias, void* workspace, int64_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* LOSS_H */
