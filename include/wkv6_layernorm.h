/*
 * wkv6_layernorm.h -- LayerNorm over whole rows, with its gradients.  (wkv6.h has the LayerNorm whose statistics a prefill leaves.)
 *
 *     y = u gamma + beta,  u = (x - mean) rstd,  rstd = 1 / sqrt(var + eps)       over the D values of a row, var dividing by D
 *
 *   M            rows, fewer than 2^24 (0: nothing to do)
 *   D            width, a multiple of 8 up to 16384 (others: WKV6_ERR_UNSUPPORTED)
 *   x            [M][D] of the wkv6_dtype dtype; y [M][D] of out_dtype: any pair
 *   gamma, beta  [D] fp32
 *   mean_rstd    [M][2] fp32
 * Device pointers, 16-byte aligned.  fp32 arithmetic, one rounding of the results.  Everything else (ownership, streams, errors
 * before any launch) is as in wkv6.h.
 */
#ifndef WKV6_LAYERNORM_H
#define WKV6_LAYERNORM_H

#include "wkv6.h"

#ifdef __cplusplus
extern "C" {
#endif

/* mean_rstd may be NULL (not written): the backward call needs it.  y may equal x if they have one type. */
int wkv6_layernorm_forward(long long M, int D, const void *x, const float *gamma, const float *beta, float eps,
                           void *y, float *mean_rstd, int dtype, int out_dtype, void *stream);

/*
 * Gradients: dy [M][D] of out_dtype, dx [M][D] of dtype,
 *     dx = rstd (a - mean(a) - u mean(a u)),  a = gamma dy        dgamma = sum over the rows of dy u        dbeta = sum over the rows of dy
 * dgamma and dbeta may both be NULL (frozen weights: no workspace then).  M = 0 leaves them nought.  The sums over the rows have a fixed order:
 * the same bits from call to call.  dx may equal dy or x if they have one type.  workspace: device memory of the caller of at least
 * wkv6_layernorm_backward_workspace_bytes, used during the call's kernels only (less: WKV6_ERR_WORKSPACE).
 */
int wkv6_layernorm_backward(long long M, int D, const void *x, const float *mean_rstd, const float *gamma, const void *dy,
                            void *dx, float *dgamma, float *dbeta, int dtype, int out_dtype,
                            void *workspace, long long workspace_bytes, void *stream);

/* Bytes of that workspace, -1 for invalid sizes. */
long long wkv6_layernorm_backward_workspace_bytes(long long M, int D);

#ifdef __cplusplus
}
#endif
#endif /* WKV6_LAYERNORM_H */
