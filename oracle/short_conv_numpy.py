"""The short causal convolution and its gradients in float64, one token at a time -- TEST INFRASTRUCTURE, NOT PRODUCT CODE.

    p_t[d] = bias[d] + sum_j w[d][j] x_{t-W+1+j}[d]        out = silu(p), or p

Rows are [row][D]; sequence i has the rows of ``spans[i]``, and in front of them its state, the last W - 1 inputs.
Pins (tests/test_scan_operators_cpu.py): a case worked by hand, gradients against differences, a sequence cut in two.
"""
import numpy as np

from .selective_scan_numpy import dsilu, silu


def short_conv_numpy(x, w, spans, bias=None, use_silu=True, state_in=None):
    """(out, state); out is NaN in rows that belong to no sequence."""
    x, w = np.asarray(x, dtype=np.float64), np.asarray(w, dtype=np.float64)
    D, W = w.shape
    state = np.zeros((len(spans), W - 1, D)) if state_in is None else np.array(state_in, dtype=np.float64)
    out = np.full(x.shape, np.nan)
    for i, (first, end) in enumerate(spans):
        for t in range(first, end):
            taps = np.concatenate([state[i], x[t:t + 1]])
            p = (taps * w.T).sum(0) + (0 if bias is None else bias)
            out[t] = silu(p) if use_silu else p
            state[i] = taps[1:]
    return out, state


def short_conv_gradients_numpy(x, w, spans, dout, bias=None, use_silu=True, state_in=None, dstate_out=None, magnitudes=False):
    """(dx, dw, dbias, dstate_in); NaN in rows that belong to no sequence.  magnitudes: of the terms, one by one."""
    x, w, dout = (np.asarray(a, dtype=np.float64) for a in (x, w, dout))
    of = np.abs if magnitudes else lambda v: v
    D, W = w.shape
    state_in = np.zeros((len(spans), W - 1, D)) if state_in is None else np.asarray(state_in, dtype=np.float64)
    dstate = np.zeros((len(spans), W - 1, D)) if dstate_out is None else np.array(dstate_out, dtype=np.float64)
    dx, dw, dbias, first_states = np.full(x.shape, np.nan), np.zeros((D, W)), np.zeros(D), np.zeros(state_in.shape)
    for i, (first, end) in enumerate(spans):
        all_in = np.concatenate([state_in[i], x[first:end]])
        grad = np.zeros(all_in.shape)
        grad[end - first:] += of(dstate[i])
        for t in range(end - first):
            p = (all_in[t:t + W] * w.T).sum(0) + (0 if bias is None else bias)
            size = (np.abs(all_in[t:t + W] * w.T)).sum(0) + (0 if bias is None else np.abs(bias))
            dp = dout[first + t] * (dsilu(p) if use_silu else 1.0)
            if magnitudes:             # the slope of silu changes by at most one half a unit of p
                dp = np.abs(dout[first + t]) * (np.abs(dsilu(p)) + 1 + 0.5 * size if use_silu else 1.0)
            grad[t:t + W] += of(dp * w.T)
            dw += of(dp * all_in[t:t + W]).T
            dbias += of(dp)
        first_states[i], dx[first:end] = grad[:W - 1], grad[W - 1:]
    return dx, dw, dbias, first_states
