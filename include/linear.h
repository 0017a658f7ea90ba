/*
 * linear.h -- C ABI of the MI355X (gfx950) layer operators that stand around a
 * convolution or alone: the fully connected layer with its epilogue, the
 * layer's gradients, and the norm and clipping of many gradients together.
 *
 * The layer.  F is kn x ci (kn outputs of ci inputs each), X is ci x t (one
 * column per token or image), and
 *        Z = F X + bias 1^T,        O = act(Z) + residual       (kn x t),
 * which is convgemm_f32 (convgemm.h) for 1 x 1 filters, with the layer's bias,
 * activation and residual in the product's epilogue.  Activations:
 *        0 none        z
 *        1 relu        z where z > 0, else 0 (a NaN stays a NaN)
 *        2 gelu        z Phi(z), Phi the normal distribution function
 *        3 gelu_tanh   z (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3))) / 2
 *        4 silu        z / (1 + exp(-z))
 *
 * Its gradients, for dO = dL/dO (the residual's gradient is dO itself):
 *        dZ = dO act'(Z),   dX = F^T dZ,   dF = dZ X^T,   dbias = dZ 1.
 * relu's dZ is 0 where z <= 0 and dO elsewhere.
 *
 * Clipping.  Over all tensors g together,
 *        norm = sqrt(sum g^2),   c = min(1, max_norm / norm),   out = c g,
 * with c = 1 where norm = 0.  norm and c are computed in fp64, c is applied to
 * fp32's precision at any size, and norm is returned in fp32: one above that range
 * is returned as infinity, though c goes by its value.  An infinite or NaN gradient
 * gives c = 0 or a NaN c, as the formula says; the caller reads norm where that
 * matters.
 *
 * Types: LINEAR_F32, LINEAR_BF16, LINEAR_F16; all tensors of one layer have the
 * same type.  Products are summed in fp32 on the matrix cores and the epilogue
 * is computed in fp32; each result is rounded to the type once.  Between the
 * two products of the gradients dZ is held in the layer's type, one more rounding
 * (exact for relu and without an activation): a 16-bit dX or dF is then off by
 * about 1.4 roundings in its norm instead of one.  fp16 holds dZ times a power of
 * two that is taken from the largest finite |dO|, so that no dZ overflows and
 * small ones keep their digits.  dbias is summed from the values before that
 * rounding.  norm is summed in fp64.  Every result is reproducible: no sum
 * depends on the order in which workgroups run.
 *
 * Storage: X, O, residual, Z, dO and dX have their first index fastest and a
 * leading dimension (elements from one token to the next) of at least their
 * first extent.  F and dF have either index fastest, by f_order: 0 = kn fastest
 * (the convolution's filters: F[k][c] at F[k + ldf c]), 1 = ci fastest (F[k][c]
 * at F[c + ldf k]).  Any leading dimension and any address that the type
 * allows are taken; operands whose addresses, leading dimensions or contiguous
 * extents are not multiples of 16 bytes cost narrower loads (fp32), a padded copy
 * (16-bit types) or, up to 64 tokens, loads through registers; lines of 2^22 fp32
 * or 2^23 16-bit values and more always go through registers.
 *
 * Rules (as in ltlt.h): pointers are DEVICE pointers of the current HIP device
 * unless marked HOST; calls are stream-ordered and asynchronous; the caller
 * owns every buffer, the workspace among them, and nothing is retained.  A
 * workspace may be reused as soon as later work on the same stream needs it.
 * Return value: 0 on success (empty problems included: a product over no terms
 * is zero); -i when argument i (1-based) is invalid, with nothing enqueued;
 * LINEAR_ERR_HIP_BASE - e for a HIP runtime error e.  Outputs may not overlap
 * inputs, except that out may be g itself in convgemm_grad_clip and O may be
 * the residual itself (same leading dimension).
 */
#ifndef LINEAR_H
#define LINEAR_H

#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

#define LINEAR_OK 0
#define LINEAR_ERR_HIP_BASE (-1000) /* returned as LINEAR_ERR_HIP_BASE - (int)hipError_t */

#define LINEAR_F32 1
#define LINEAR_BF16 4
#define LINEAR_F16 5

#define LINEAR_ACT_NONE 0
#define LINEAR_ACT_RELU 1
#define LINEAR_ACT_GELU 2
#define LINEAR_ACT_GELU_TANH 3
#define LINEAR_ACT_SILU 4

/* Bytes of workspace that convgemm_linear needs for a layer of these sizes on
 * the current device (0 where none; host only), or -i when argument i is
 * invalid.  aligned = 1 says that F and X have 16-byte aligned addresses and
 * leading dimensions of whole 16 bytes, below 2^22 bytes; what 0 gives is enough
 * for any. */
int64_t convgemm_linear_workspace(int dtype, int64_t kn, int64_t ci, int64_t t, int f_order, int aligned);

/* The kernel that convgemm_linear takes for a layer on the current device (host
 * only; without a device, on one of 256 CUs; `aligned` as above).  HOST int
 * out[6]:
 *   out[0] = 1 the 256 x 256 tile's kernel, 2 a kernel with another tile, 3 one
 *            that loads single fp32 values, 4 loads through registers; 0 where
 *            there is nothing to do;
 *   out[1], out[2] = its tile, outputs x tokens;
 *   out[3] = workgroups that share a tile's contraction (added in a fixed order);
 *   out[4] = operands that are copied first;
 *   out[5] = the kernel's number among those of family 1 to 3 (two kernels may
 *            have the same tile). */
int convgemm_linear_choice(int dtype, int64_t kn, int64_t ci, int64_t t, int f_order, int aligned, int* out);

/* O = act(F X + bias) + residual.
 *   dtype             : LINEAR_*;
 *   kn, ci, t         : sizes (>= 0, below 2^24; kn t, kn ci and ci t below 2^40);
 *   F, f_order, ldf   : the weights;
 *   X, ldx            : the input;
 *   bias              : kn values, or NULL;
 *   act               : LINEAR_ACT_*;
 *   residual, ldr     : kn x t, or NULL (ldr is then not looked at);
 *   Z, ldz            : kn x t for the pre-activation, or NULL;
 *   O, ldo            : the result;
 *   workspace, workspace_bytes : at least convgemm_linear_workspace() bytes,
 *                       16-byte aligned, or NULL where that is 0.
 * Leading dimensions are below 2^24.  */
int convgemm_linear(int dtype, int64_t kn, int64_t ci, int64_t t, const void* F, int f_order, int64_t ldf,
                    const void* X, int64_t ldx, const void* bias, int act, const void* residual, int64_t ldr,
                    void* Z, int64_t ldz, void* O, int64_t ldo, void* workspace, int64_t workspace_bytes,
                    hipStream_t stream);

/* Bytes of workspace that convgemm_linear_backward needs (host only), or -i
 * when argument i is invalid.  aligned: as above, of F, X and dO. */
int64_t convgemm_linear_backward_workspace(int dtype, int64_t kn, int64_t ci, int64_t t, int f_order, int act,
                                           int aligned);

/* dX, dF and dbias from dO; each of the three may be NULL and is then not
 * computed (the bytes that the query names are enough all the same).  F may be
 * NULL where dX is, X where dF is.  Z is the pre-activation that convgemm_linear
 * wrote; it is not looked at where act is LINEAR_ACT_NONE.  dF has F's order; its
 * leading dimension is lddf. */
int convgemm_linear_backward(int dtype, int64_t kn, int64_t ci, int64_t t, const void* F, int f_order, int64_t ldf,
                             const void* X, int64_t ldx, const void* dO, int64_t lddo, const void* Z, int64_t ldz,
                             int act, void* dX, int64_t lddx, void* dF, int64_t lddf, void* dbias, void* workspace,
                             int64_t workspace_bytes, hipStream_t stream);

/* Bytes of workspace that the two calls below need (host only). */
int64_t convgemm_grad_workspace(int count);

/* norm (one float) of `count` tensors together.  HOST arrays: g[i] the tensor's
 * device address, n[i] < 2^37 its number of values (stored without gaps, in any
 * order), dtype[i] its LINEAR_* type. */
int convgemm_grad_norm(int count, const void* const* g, const int64_t* n, const int* dtype, float* norm,
                       void* workspace, int64_t workspace_bytes, hipStream_t stream);

/* The same, and out[i] = c g[i] with c = min(1, max_norm / norm); out[i] has
 * g[i]'s type and order and may be g[i] itself (then nothing is written where
 * c = 1); the out[i] may not overlap one another.  max_norm >= 0. */
int convgemm_grad_clip(int count, const void* const* g, void* const* out, const int64_t* n, const int* dtype,
                       double max_norm, float* norm, void* workspace, int64_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* LINEAR_H */
