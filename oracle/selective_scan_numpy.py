"""The selective scan and its gradients in float64, one token at a time -- TEST INFRASTRUCTURE, NOT PRODUCT CODE.

    dt_t = softplus(delta_t + bias)    h_t[d][n] = exp(dt_t[d] a[d][n]) h_{t-1}[d][n] + dt_t[d] b_t[n] x_t[d]
    out_t[d] = (sum_n c_t[n] h_t[d][n] + skip[d] x_t[d]) silu(z_t[d])

Rows are [row][D], b and c [row][N]; sequence i has the rows of ``spans[i]``.  The gradients are those of the recurrence, step by step
backwards: with G the gradient of h_t from everything behind token t and dy = dout silu(z),

    G += dy_t c_t    k = G exp(dt a) h_{t-1}    dx_t = dt sum_n G b + skip dy    d(dt) = x sum_n G b + sum_n k a    db = sum_d G dt x
    dc = sum_d dy h_t    da += k dt    G <- exp(dt a) G

The recurrences take step sizes, exponents and gates, so that a caller can put others there.
Pins (tests/test_scan_operators_cpu.py): a case worked by hand, gradients against differences, a sequence cut in two.
"""
import numpy as np


def softplus(v):
    return np.logaddexp(v, 0.0)


def sigmoid(v):
    return 0.5 * (1 + np.tanh(0.5 * np.asarray(v)))


def silu(v):
    return v * sigmoid(v)


def dsilu(v):
    s = sigmoid(v)
    return s * (1 + v * (1 - s))


def scan_recurrence(dt, exponents, x, b, c, skip, gate, spans, state_in):
    """(out, state, read-outs in front of the gate); NaN in rows that belong to no sequence."""
    out, y = np.full(x.shape, np.nan), np.full(x.shape, np.nan)
    h = np.array(state_in, dtype=np.float64)
    for i, (first, end) in enumerate(spans):
        for t in range(first, end):
            h[i] = np.exp(exponents[t]) * h[i] + (dt[t] * x[t])[:, None] * b[t]
            y[t] = (h[i] * c[t]).sum(1) + skip * x[t]
            out[t] = y[t] * gate[t]
    return out, h, y


def scan_gradients(dt, exponents, a, x, b, c, skip, gate, dgate, slope, spans, state_in, dout, dstate_out):
    """{name: gradient}; `slope` is that of the step size.  NaN in rows that belong to no sequence."""
    rows, D = x.shape
    res = {n: np.full(s, np.nan) for n, s in (("dx", x.shape), ("ddelta", x.shape), ("dz", x.shape), ("db", b.shape), ("dc", c.shape))}
    da, dskip, dbias = np.zeros(a.shape), np.zeros(D), np.zeros(D)
    g_in = np.array(dstate_out, dtype=np.float64)
    for i, (first, end) in enumerate(spans):
        h, before = np.array(state_in[i], dtype=np.float64), []
        for t in range(first, end):
            before.append(h)
            h = np.exp(exponents[t]) * h + (dt[t] * x[t])[:, None] * b[t]
        G = g_in[i]
        for t in reversed(range(first, end)):
            dy = dout[t] * gate[t]
            G = G + dy[:, None] * c[t]
            res["dz"][t] = dout[t] * ((h * c[t]).sum(1) + skip * x[t]) * dgate[t]
            res["dc"][t] = (h * dy[:, None]).sum(0)
            h = before.pop()
            k = G * np.exp(exponents[t]) * h
            into = (G * b[t]).sum(1)
            res["dx"][t] = into * dt[t] + skip * dy
            res["ddelta"][t] = (into * x[t] + (k * a).sum(1)) * slope[t]
            res["db"][t] = (G * (dt[t] * x[t])[:, None]).sum(0)
            da += k * dt[t][:, None]
            dskip += dy * x[t]
            dbias += res["ddelta"][t]
            G = np.exp(exponents[t]) * G
        g_in[i] = G
    return {**res, "da": da, "dskip": dskip, "dbias": dbias, "dstate_in": g_in}


def selective_scan_parts(x, delta, a, b, c, spans, bias=None, use_softplus=True, skip=None, z=None, state_in=None):
    """The arguments of the recurrences from those of a call."""
    x, delta, a, b, c = (np.asarray(v, dtype=np.float64) for v in (x, delta, a, b, c))
    v = delta if bias is None else delta + bias
    dt = softplus(v) if use_softplus else v
    return dict(dt=dt, exponents=dt[:, :, None] * a, a=a, x=x, b=b, c=c, skip=np.zeros(x.shape[1]) if skip is None else np.asarray(skip, dtype=np.float64),
                gate=np.ones(x.shape) if z is None else silu(np.asarray(z, dtype=np.float64)),
                dgate=np.zeros(x.shape) if z is None else dsilu(np.asarray(z, dtype=np.float64)),
                slope=sigmoid(v) if use_softplus else np.ones(x.shape), spans=spans,
                state_in=np.zeros((len(spans),) + a.shape) if state_in is None else np.asarray(state_in, dtype=np.float64))


def selective_scan_numpy(**call):
    p = selective_scan_parts(**call)
    for n in ("a", "dgate", "slope"):
        p.pop(n)
    return scan_recurrence(**p)[:2]


def selective_scan_gradients_numpy(dout, dstate_out=None, **call):
    p = selective_scan_parts(**call)
    return scan_gradients(**p, dout=np.asarray(dout, dtype=np.float64),
                          dstate_out=np.zeros(p["state_in"].shape) if dstate_out is None else np.asarray(dstate_out, dtype=np.float64))
