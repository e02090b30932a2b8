/*
 * wkv6_selective_scan.h -- the recurrence whose decays are formed from a step size: one decay per channel, state and token, beside the ones of
 * wkv6.h (per key channel) and wkv6_head_decay.h (per head): prompts, single tokens, gradients.  The short convolution in front
 * of it is in wkv6_short_conv.h.
 *
 * For every (sequence, channel d) independently, with N states n,
 *
 *     dt_t = softplus(delta_t + delta_bias)           softplus(v) = log(1 + exp(v)); with softplus = 0 dt_t = delta_t + delta_bias
 *     h_t[n] = exp(dt_t a[n]) h_{t-1}[n] + dt_t b_t[n] x_t                              t = 1..len
 *     out_t = (sum over n of c_t[n] h_t[n] + skip x_t) silu(z_t)                          silu(v) = v / (1 + exp(-v))
 *
 * b and c are shared by all channels of a token.
 *
 * Layout (row-major, innermost index last):
 *   B, T, D, N    sequences, tokens of the longest one (at most 2^30), channels (a multiple of 8 up to 65536), states: 8, 16, 32 or 64
 *   rows          rows of the tensors below
 *   offsets       [B + 1] int32, device: sequence b has the rows offsets[b] .. offsets[b+1] - 1, as in wkv6_head_decay.h: rows that belong to
 *                 nobody are not read and keep what they hold; an offset outside 0 .. rows is taken as the nearer of the
 *                 two, a longer sequence ends after T tokens, one that ends in front of its start has none, and sequences may lie in any order;
 *                 where they overlap, what their rows and the sums over tokens get is not defined.  NULL: B sequences of T rows each, and rows must be B T.  A sequence of no tokens has
 *                 state_out = state_in.
 *   x, delta, z   [rows][D], rows x_stride, delta_stride, z_stride ELEMENTS apart (at least D, at most 2^22, a multiple of 16 bytes), so that they may be
 *                 parts of a projection's rows.  z may be NULL: no gate.  dx, ddelta, dz likewise, with the same strides
 *   b, c          [rows][N], rows bc_stride elements apart (at least N, at most 2^22, a multiple of 16 bytes).  db, dc likewise
 *   a             [D][N] fp32: negative numbers as a rule; positive ones (states grow) are taken as they are, as far as a token's exp(dt a), states (and, of the
 *                 backward call, their gradients) and what each token leaves in them stay inside fp32's range; an infinity counts as fp32's largest number,
 *                 a NaN reaches all that its state has a part in
 *   delta_bias, skip   [D] fp32, may be NULL (nought)
 *   state_in      [B][D][N] fp32, NULL means zero.  state_out the same, NULL means "do not write"; it may equal state_in
 *   out, dout     [rows][D]
 * Device pointers, 16-byte aligned but for offsets (4); `out` and the gradients must not alias any input or each other.
 * dtype is the wkv6_dtype of x, delta, z, b, c (and, of the backward call, dout, dx, ddelta, dz, db, dc), out_dtype that of out: bf16 rows with
 * either, fp32 rows with fp32.
 *
 * Arithmetic: fp32 throughout, one rounding of the results.  A decay is rounded to fp32 token by token, as the recurrence is written, and its exponent, its product
 * and the sum with it: a state that remembers M tokens is off by (250 + 8 M) 2^-24 of its terms' magnitudes at most (one that grows by four times that), and by M 2^-24 or so where all its tokens have
 * the same step size, by the root of M where they differ.  Values have to be finite: a NaN or infinity in a row reaches other tokens of its
 * sequence, also earlier ones, not other sequences.
 *
 * Workspace: device memory of the caller, 16-byte aligned, as many bytes as the function beside the call says (none where that is 0),
 * used during the call's kernels only; calls that share one must be ordered.  Its contents need not be set.
 *
 * Everything else (ownership, streams, errors before any launch) is as in wkv6.h.  Too small a workspace: WKV6_ERR_WORKSPACE.
 */
#ifndef WKV6_SELECTIVE_SCAN_H
#define WKV6_SELECTIVE_SCAN_H

#include "wkv6.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Whole sequences.  At few (sequence, channel) units the token axis is cut and the pieces' states are formed first, in the workspace. */
int wkv6_selective_scan_prefill(int B, int T, int D, int N, long long rows,
                                const void *x, long long x_stride, const void *delta, long long delta_stride,
                                const float *delta_bias, int softplus, const float *a,
                                const void *b, const void *c, long long bc_stride, const float *skip,
                                const void *z, long long z_stride, const int *offsets, const float *state_in,
                                void *out, float *state_out, int dtype, int out_dtype,
                                void *workspace, long long workspace_bytes, void *stream);

/* Bytes of that workspace (0: none is needed), -1 for invalid sizes. */
long long wkv6_selective_scan_workspace_bytes(int B, int T, int D, int N);

/* One token of every sequence: x, delta, z [B][D], b, c [B][N] (rows their strides apart), out [B][D]. */
int wkv6_selective_scan_decode(int B, int D, int N,
                               const void *x, long long x_stride, const void *delta, long long delta_stride,
                               const float *delta_bias, int softplus, const float *a,
                               const void *b, const void *c, long long bc_stride, const float *skip,
                               const void *z, long long z_stride, const float *state_in,
                               void *out, float *state_out, int dtype, int out_dtype, void *stream);

/*
 * Gradients of a prefill: from dout and dstate_out (NULL means zero) those of its inputs.  States and read-outs are formed again from the
 * inputs; nothing has to be kept from the forward call.
 *   rows      at most 2^26 - 16
 *   dx, ddelta, db, dc, dz          rows (dz only if there is a z; NULL there: not written)
 *   da [D][N], dskip, ddelta_bias [D] fp32: sums over all tokens; each may be NULL (not written).  Without tokens they are nought.
 *   dstate_in [B][D][N] fp32, may be NULL
 * Results are the same bits from call to call.
 */
int wkv6_selective_scan_backward(int B, int T, int D, int N, long long rows,
                                 const void *x, long long x_stride, const void *delta, long long delta_stride,
                                 const float *delta_bias, int softplus, const float *a,
                                 const void *b, const void *c, long long bc_stride, const float *skip,
                                 const void *z, long long z_stride, const int *offsets, const float *state_in,
                                 const void *dout, const float *dstate_out,
                                 void *dx, void *ddelta, void *db, void *dc, void *dz,
                                 float *da, float *dskip, float *ddelta_bias, float *dstate_in, int dtype,
                                 void *workspace, long long workspace_bytes, void *stream);

/* Bytes of that workspace, -1 for invalid sizes. */
long long wkv6_selective_scan_backward_workspace_bytes(int B, int T, int D, int N, long long rows);

#ifdef __cplusplus
}
#endif
#endif /* WKV6_SELECTIVE_SCAN_H */
