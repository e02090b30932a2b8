/*
 * wkv6_head_decay.h -- time mix with one decay per head and token, beside the per-channel one of wkv6.h: prompts, single
 * tokens, gradients.
 *
 * For every (sequence, head) independently
 *
 *     S_t = exp(g_t) S_{t-1} + k_t^T v_t        o_t = r_t S_t        t = 1..len
 *
 * S is a (key channel) x (value channel) matrix as in wkv6.h.  The token itself is part of its read-out, there is no bonus, and the
 * decay is given as its logarithm.  A scale of the read-out goes into r.
 *
 * Layout (row-major, innermost index last):
 *   B, T, H, N    sequences, tokens of the longest one (at most 2^30), heads (at most 65536), head size, which must be 64
 *   rows          rows of the tensors below
 *   offsets       [B + 1] int32, device: sequence b has the rows offsets[b] .. offsets[b+1] - 1, one sequence behind the other, none longer
 *                 than T.  Rows in front of offsets[0] and from offsets[B] on belong to nobody: they are not read, and what a
 *                 call writes leaves them as they were.  An offset is only known on the device: one outside 0 .. rows is taken as the
 *                 nearer of the two, a longer sequence ends after T tokens, and one that ends in front of its start has
 *                 none, so nothing outside the tensors is touched; where sequences overlap, what their rows get is not defined.
 *                 NULL: B sequences of T rows each, and rows must be B T.  A sequence of no tokens has state_out = state_in.
 *   r, k, v       [rows][H][N], rows token_stride ELEMENTS apart (at least H N, at most 2^22; rows a multiple of 16 bytes): they may be
 *                 parts of one tensor [rows][3][H][N], as one projection leaves them.  dr, dk, dv likewise, with the same stride
 *   g             [rows][H] fp32, rows g_stride elements apart (at least H), or one decay a head for all tokens: [H] with g_stride = 0.
 *                 Meant for g <= 0, but a finite g above nought (states grow) is taken as it is, as far as states stay inside fp32's range;
 *                 -inf (forget everything) is taken as -128, whose exponential is nothing in fp32.
 *   state_in      [B][H][N][N] fp32, NULL means zero.  state_out the same, NULL means "do not write"; it may equal state_in
 *   out, dout     [rows][H][N]
 * Device pointers, 16-byte aligned but for g, dg and offsets (4); `out` and the gradients must not alias any input.
 * dtype is the wkv6_dtype of r, k, v (and, of the backward call, dout, dr, dk, dv), out_dtype that of out: bf16 rows with either, fp32
 * rows with fp32.
 *
 * Arithmetic: fp32 states, sums and decays.  Of bf16 rows the products are formed on the bf16 matrix cores; operands that are no rows
 * (states, scores, decayed values) enter as sums of bf16 that hold fp32 values whole, over fp32's range (2^-17 of them where only bf16
 * read-outs depend on it).  fp32 rows: fp32 throughout.
 * Values have to be finite: a NaN or infinity in a row reaches other tokens of its sequence, also earlier ones, not other sequences.
 *
 * Workspace: device memory of the caller, 16-byte aligned, as many bytes as the function beside the call says (none where that is 0),
 * used during the call's kernels only; calls that share one must be ordered.  Its contents need not be set.
 *
 * Everything else (ownership, streams, errors before any launch) is as in wkv6.h.  Too small a workspace: WKV6_ERR_WORKSPACE.
 */
#ifndef WKV6_HEAD_DECAY_H
#define WKV6_HEAD_DECAY_H

#include "wkv6.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Whole sequences.  At few (sequence, head) units the token axis is cut and the pieces' states are formed first, in the workspace. */
int wkv6_head_decay_prefill(int B, int T, int H, int N, long long rows,
                            const void *r, const void *k, const void *v, long long token_stride,
                            const float *g, long long g_stride, const int *offsets, const float *state_in,
                            void *out, float *state_out, int dtype, int out_dtype,
                            void *workspace, long long workspace_bytes, void *stream);

/* Bytes of that workspace (0: none is needed), -1 for invalid sizes. */
long long wkv6_head_decay_workspace_bytes(int B, int T, int H, int N);

/* One token of every sequence: r, k, v [B][H][N] (rows token_stride apart), g [B][H] or [H], out [B][H][N]. */
int wkv6_head_decay_decode(int B, int H, int N,
                           const void *r, const void *k, const void *v, long long token_stride,
                           const float *g, long long g_stride, const float *state_in,
                           void *out, float *state_out, int dtype, int out_dtype, void *stream);

/*
 * Gradients of a prefill: from dout and dstate_out (NULL means zero) those of r, k, v, g and state_in (dstate_in NULL: not written).
 * State and read-outs are formed again from the inputs; nothing has to be kept from the forward call.
 *   dg   [rows][H] fp32, or [H] with g_stride = 0: then summed over all tokens
 *        A g that stands for -inf (below -128) gets the gradient of the value that it is taken as: nought but for rounding.
 * Results are the same bits from call to call.  With B = 0, T = 0 or rows = 0, dg of g_stride = 0 is nought.
 */
int wkv6_head_decay_backward(int B, int T, int H, int N, long long rows,
                             const void *r, const void *k, const void *v, long long token_stride,
                             const float *g, long long g_stride, const int *offsets, const float *state_in,
                             const void *dout, const float *dstate_out,
                             void *dr, void *dk, void *dv, float *dg, float *dstate_in, int dtype,
                             void *workspace, long long workspace_bytes, void *stream);

/* Bytes of that workspace, -1 for invalid sizes. */
long long wkv6_head_decay_backward_workspace_bytes(int B, int T, int H, int N, long long rows);

#ifdef __cplusplus
}
#endif
#endif /* WKV6_HEAD_DECAY_H */
