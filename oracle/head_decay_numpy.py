"""The head-decay time mix and its gradients in float64, one token at a time -- TEST INFRASTRUCTURE, NOT PRODUCT CODE.

    S_t = exp(g_t) S_{t-1} + k_t^T v_t        o_t = r_t S_t

for every (sequence, head).  Rows are [row][H][N]; sequence b has the rows of ``spans[b]``.  The gradients are those of the
recurrence, step by step backwards: with dS the gradient of S_t from everything behind token t,

    dS += r_t^T do_t    dr_t = do_t S_t^T    dk_t = v_t dS^T    dv_t = k_t dS    dg_t = <dS, exp(g_t) S_{t-1}>    dS <- exp(g_t) dS

Pins (tests/test_operators_cpu.py): a case worked by hand, gradients against differences, a sequence cut in two.
"""
import numpy as np


def _per_row(g, rows):
    g = np.asarray(g, dtype=np.float64)
    return np.broadcast_to(g, (rows, g.shape[-1])) if g.ndim == 1 else g


def head_decay_numpy(r, k, v, g, spans, state_in=None):
    """(out, state): out is NaN in rows that belong to no sequence."""
    r, k, v = (np.asarray(a, dtype=np.float64) for a in (r, k, v))
    rows, H, N = r.shape
    w = np.exp(_per_row(g, rows))
    S = np.zeros((len(spans), H, N, N)) if state_in is None else np.array(state_in, dtype=np.float64)
    out = np.full(v.shape, np.nan)
    for b, (first, end) in enumerate(spans):
        for t in range(first, end):
            S[b] = w[t][:, None, None] * S[b] + k[t][:, :, None] * v[t][:, None, :]
            out[t] = (r[t][:, :, None] * S[b]).sum(1)
    return out, S


def head_decay_gradients_numpy(r, k, v, g, spans, dout, state_in=None, dstate_out=None):
    """(dr, dk, dv, dg [rows][H], dstate_in); NaN in rows that belong to no sequence."""
    r, k, v, dout = (np.asarray(a, dtype=np.float64) for a in (r, k, v, dout))
    rows, H, N = r.shape
    w = np.exp(_per_row(g, rows))
    dr, dk, dv = (np.full(r.shape, np.nan) for _ in range(3))
    dg = np.full((rows, H), np.nan)
    d0 = np.zeros((len(spans), H, N, N)) if dstate_out is None else np.array(dstate_out, dtype=np.float64)
    for b, (first, end) in enumerate(spans):
        S = np.zeros((H, N, N)) if state_in is None else np.array(state_in[b], dtype=np.float64)
        before = []
        for t in range(first, end):
            before.append(S)
            S = w[t][:, None, None] * S + k[t][:, :, None] * v[t][:, None, :]
        dS = d0[b]
        for t in reversed(range(first, end)):
            dS = dS + r[t][:, :, None] * dout[t][:, None, :]
            dr[t] = (S * dout[t][:, None, :]).sum(2)
            dk[t] = (dS * v[t][:, None, :]).sum(2)
            dv[t] = (dS * k[t][:, :, None]).sum(1)
            S = before.pop()
            decayed = w[t][:, None, None] * dS
            dg[t] = (decayed * S).sum((1, 2))
            dS = decayed
        d0[b] = dS
    return dr, dk, dv, dg, d0
