/*
 * wkv6_short_conv.h -- the short causal convolution over a token's own channel, in front of wkv6_selective_scan.h: prompts, single tokens,
 * gradients.  (With two taps it is a token shift with a weight a channel.)
 *
 *     p_t[d] = bias[d] + sum over j < W of w[d][j] x_{t-W+1+j}[d]        out = silu(p) = p / (1 + exp(-p)), or p with silu = 0
 *
 * The inputs in front of a sequence's first token are its state: the last W - 1 inputs of what came before.
 *
 *   B, T, D, W    sequences, tokens of the longest one (at most 2^30), channels (a multiple of 8 up to 65536), taps: 2, 3 or 4
 *   rows, offsets as in wkv6_selective_scan.h
 *   x             [rows][D], rows x_stride ELEMENTS apart (at least D, at most 2^22, a multiple of 16 bytes); dx likewise, with the same stride
 *   w, dw         [D][W] fp32; bias, dbias [D] fp32, bias may be NULL (nought)
 *   state_in      [B][W - 1][D] of dtype, the latest input last; NULL means zero.  state_out the same, after the last token; NULL means
 *                 "do not write"; it may equal state_in.  A sequence of no tokens has state_out = state_in
 *   out, dout     [rows][D]
 * Device pointers, 16-byte aligned but for offsets (4); out and the gradients must not alias any input or each other.  dtype: the wkv6_dtype of all but
 * w, bias, dw, dbias.  fp32 arithmetic, one rounding of the results; states are kept as they are.  A NaN or infinity in a row
 * reaches, of its own channel, only the tokens that have it under their taps; of the gradients dx (and dstate_in) of the W - 1 tokens in front of it
 * and behind it, dw and dbias.
 * Workspace, ownership, streams, errors before any launch: as in wkv6_selective_scan.h.
 */
#ifndef WKV6_SHORT_CONV_H
#define WKV6_SHORT_CONV_H

#include "wkv6.h"

#ifdef __cplusplus
extern "C" {
#endif

int wkv6_short_conv_prefill(int B, int T, int D, int W, long long rows, const void *x, long long x_stride,
                            const float *w, const float *bias, int silu, const int *offsets, const void *state_in,
                            void *out, void *state_out, int dtype, void *stream);

/* One token of every sequence: x [B][D] (rows x_stride apart), out [B][D]. */
int wkv6_short_conv_decode(int B, int D, int W, const void *x, long long x_stride, const float *w, const float *bias, int silu,
                           const void *state_in, void *out, void *state_out, int dtype, void *stream);

/*
 * Gradients of a prefill: from dout and dstate_out (NULL means zero) those of x, w, bias and state_in (dstate_in NULL: not written; dw, dbias
 * NULL, both or neither: frozen weights).  dw and dbias are sums over all tokens, in a fixed order; without tokens they are nought.
 */
int wkv6_short_conv_backward(int B, int T, int D, int W, long long rows, const void *x, long long x_stride,
                             const float *w, const float *bias, int silu, const int *offsets, const void *state_in,
                             const void *dout, const void *dstate_out, void *dx, float *dw, float *dbias, void *dstate_in,
                             int dtype, void *workspace, long long workspace_bytes, void *stream);

/* Bytes of that workspace, -1 for invalid sizes. */
long long wkv6_short_conv_backward_workspace_bytes(int B, int T, int D, int W, long long rows);

#ifdef __cplusplus
}
#endif
#endif /* WKV6_SHORT_CONV_H */
