/*
 * group_norm.h -- C ABI of the MI355X (gfx950) group norm with an activation, for maps
 * stored with the channels fastest, as a convolution leaves them, and its gradients.
 *
 * I has c channels, s positions and b images.  The channels are dealt into `groups` runs
 * of c / groups; over the n = (c / groups) s values of a group in one image
 *        mean = sum I / n,   var = sum (I - mean)^2 / n,   rstd = 1 / sqrt(var + eps),
 *        xhat = (I - mean) rstd,    Z = weight xhat + bias (by channel),    O = act(Z)
 * with linear.h's activations.  groups = 1 with s = 1 is the norm of each token's
 * features, groups = c that of each channel's map.
 *
 * Gradients, for dO = dL/dO, with avg over the same n values:
 *        dZ = dO act'(Z),    d = weight dZ,
 *        dI = rstd (d - avg d - xhat avg(d xhat)),
 *        dweight = sum dZ xhat,    dbias = sum dZ    over positions and images.
 *
 * Types: I, O, weight, bias and the gradients are LINEAR_F32, LINEAR_BF16 or LINEAR_F16;
 * mean and rstd are fp32.  Everything is computed in fp32: the mean first and the squares
 * around it (or four values at a time around the mean of those before, parts then joined by
 * their means), never as a difference of two large sums; each result is rounded once.
 * relu's slope jumps where Z = 0: it goes by Z as computed from the fp32 mean and rstd, and
 * a Z within their roundings of 0 may fall on the other side than in exact arithmetic; a
 * whole dO is then in or out of the gradients.  A group that holds
 * an infinity or a NaN gives NaN, and only that group.  Every result is reproducible.
 *
 * Storage: channels are neighbours; position p of image n starts at p ld + n ldb values,
 * ld >= c, ldb >= (s - 1) ld + c.  Any address that the type allows is taken; where a
 * position does not start at 16 bytes, loads are as wide as the hardware serves them.
 *
 * Rules as in linear.h.  O may be I itself and dI may be dO or I itself (with the same
 * ld and ldb); no other overlaps.  Return value: 0, -i when argument i (1-based) is
 * invalid, with nothing enqueued, or LINEAR_ERR_HIP_BASE - e.
 */
#ifndef GROUP_NORM_H
#define GROUP_NORM_H

#include <stdint.h>
#include <hip/hip_runtime_api.h>

#include "linear.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of workspace of the two calls (host only), or -i when argument i is invalid. */
int64_t convgemm_group_norm_workspace(int dtype, int64_t c, int64_t s, int64_t b, int64_t groups);
int64_t convgemm_group_norm_backward_workspace(int dtype, int64_t c, int64_t s, int64_t b, int64_t groups);

/* O, mean and rstd.
 *   c, s, b           : sizes (>= 0; c and s below 2^24, b below 2^31, c s b below 2^40);
 *   groups            : >= 1, divides c;
 *   weight, bias      : c values each, or NULL (1 and 0);
 *   eps               : >= 0;
 *   mean, rstd        : groups x b values, groups fastest, or NULL; NaN where c s = 0. */
int convgemm_group_norm(int dtype, int64_t c, int64_t s, int64_t b, int64_t groups, const void* I, int64_t ldi, int64_t ldbi,
                        const void* weight, const void* bias, double eps, int act, void* O, int64_t ldo, int64_t ldbo,
                        float* mean, float* rstd, void* workspace, int64_t workspace_bytes, hipStream_t stream);

/* dI, dweight and dbias from dO and what the call above gave; each of the three may be
 * NULL and is then not computed. */
int convgemm_group_norm_backward(int dtype, int64_t c, int64_t s, int64_t b, int64_t groups, const void* I, int64_t ldi,
                                 int64_t ldbi, const void* dO, int64_t lddo, int64_t ldbdo, const void* weight,
                                 const void* bias, int act, const float* mean, const float* rstd, void* dI, int64_t lddi,
                                 int64_t ldbdi, void* dweight, void* dbias, void* workspace, int64_t workspace_bytes,
                                 hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* GROUP_NORM_H */
