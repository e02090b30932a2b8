"""The selective scan (a decay per channel and state, formed from a step size per token) and the short causal convolution in
front of it, prompts, single tokens and gradients, as a serving or training program calls them, beside the same operators in
plain torch operations.

    p_t[d] = bias_d + sum_j w[d][j] x_{t-W+1+j}[d]        y = silu(p)                                      (convolution, W taps)

    dt_t[d] = softplus(delta_t[d] + bias_d)
    h_t[d][n] = exp(dt_t[d] a[d][n]) h_{t-1}[d][n] + dt_t[d] b_t[n] x_t[d]
    out_t[d] = (sum_n c_t[n] h_t[d][n] + skip_d x_t[d]) silu(z_t[d])                                       (scan, N states a channel)

Rows are [row][channel].  Sequences are B of T rows each, or packed one behind the other with their first rows in `offsets`.
"""
import math
import random

import torch

own = False               # set by whoever runs the file: the library's kernels instead of the plain form

WIDTHS = (8, 64, 200, 768, 1000, 1024, 1536, 2048, 2056, 4096, 8192)
STATES = (8, 16, 16, 16, 32, 64)
MOST = 131072 * 2048 * 16   # (row, channel, state) triples of the largest scan
SLAB = 1 << 27              # the plain form's triples at once


def _library():
    import paper_2407_12077_amd
    return paper_2407_12077_amd


def listed():
    return [
        # one layer over a batch of eight full-context prompts, gated; z is one half of a projection's rows, b and c parts of another's
        {"name": "scan eight prompts", "kind": "scan", "B": 8, "T": 4096, "D": 4096, "N": 16, "packed": 0, "state": False,
         "gate": True, "fused": True, "dtype": "bf16", "out": "bf16"},
        # one long context: few channels for the compute units there are
        {"name": "scan long context", "kind": "scan", "B": 1, "T": 131072, "D": 2048, "N": 16, "packed": 0, "state": False,
         "gate": True, "fused": True, "dtype": "bf16", "out": "bf16"},
        # requests of all lengths packed into one call, continued from carried states, read-outs not rounded, no gate
        {"name": "scan packed requests", "kind": "scan", "B": 37, "T": 2011, "D": 1536, "N": 16, "packed": 5, "state": True,
         "gate": False, "fused": False, "dtype": "bf16", "out": "f32"},
        # all-fp32 tensors with many states a channel, as in a parity run of a small model
        {"name": "scan fp32 small model", "kind": "scan", "B": 2, "T": 531, "D": 1000, "N": 64, "packed": 0, "state": True,
         "gate": True, "fused": False, "dtype": "f32", "out": "f32"},
        # a decode step of a full server, and of a single user
        {"name": "scan step full server", "kind": "scan_step", "B": 1024, "D": 4096, "N": 16, "gate": True, "fused": True,
         "dtype": "bf16", "out": "bf16"},
        {"name": "scan step one user", "kind": "scan_step", "B": 1, "D": 4096, "N": 16, "gate": True, "fused": True,
         "dtype": "bf16", "out": "bf16"},
        # the gradients of a training step's layer: full batch, and packed documents of a small fp32 model from carried states
        {"name": "scan backward training", "kind": "scan_backward", "B": 8, "T": 2048, "D": 4096, "N": 16, "packed": 0,
         "state": False, "gate": True, "fused": True, "dtype": "bf16"},
        {"name": "scan backward packed", "kind": "scan_backward", "B": 9, "T": 1531, "D": 768, "N": 16, "packed": 3,
         "state": True, "gate": False, "fused": False, "dtype": "f32"},
        # the convolution in front of the layer: a prompt batch whose x is one half of a projection's rows, one new token a user
        {"name": "conv prompt batch", "kind": "conv", "B": 8, "T": 4096, "D": 4096, "W": 4, "packed": 0, "state": False,
         "fused": True, "dtype": "bf16"},
        {"name": "conv step one token each", "kind": "conv_step", "B": 24, "D": 4096, "W": 4, "fused": True, "dtype": "bf16"},
        # its gradients: a training batch, and packed documents of a small fp32 model
        {"name": "conv backward training", "kind": "conv_backward", "B": 8, "T": 2048, "D": 4096, "W": 4, "packed": 0,
         "state": False, "fused": True, "dtype": "bf16"},
        {"name": "conv backward packed", "kind": "conv_backward", "B": 9, "T": 1531, "D": 768, "W": 3, "packed": 3,
         "state": True, "fused": False, "dtype": "f32"},
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, uniform over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["scan", "scan", "scan_step", "scan_backward", "scan_backward", "conv", "conv_step", "conv_backward"])
    D = rng.choice(WIDTHS)
    case = {"kind": kind, "D": D, "fused": rng.random() < 0.5, "dtype": rng.choice(["bf16", "bf16", "bf16", "f32"])}
    half = 2 if case["dtype"] == "f32" else 1
    if kind.startswith("conv"):
        case["W"] = rng.choice([2, 3, 4, 4])
        most = (8192 * 4096 if kind == "conv" else 8192 * 2048) // half // D * 4
    else:
        case["N"] = rng.choice(STATES)
        case["gate"] = rng.random() < 0.6
        most = MOST // 8 // (4 if kind == "scan_backward" else 1) // half // D // case["N"] * 8
    if kind.endswith("step"):
        case["B"] = _log(rng, 1, max(1, min(4096, (1 << 26) // D // case.get("N", 4))))
    else:
        case["B"] = _log(rng, 1, min(256, most))
        case["T"] = _log(rng, 1, max(1, min(65536, most // case["B"])))
        case["packed"] = rng.randrange(1, 1000) if rng.random() < 0.5 else 0
        case["state"] = rng.random() < 0.5
    if kind in ("scan", "scan_step"):
        case["out"] = "f32" if case["dtype"] == "f32" else rng.choice(["bf16", "bf16", "f32"])
    return case


# ----------------------------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------------------------
def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, scale, dtype):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _empty(shape, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda")


def _lengths(case):
    """Tokens of every sequence; packed ones from one token (now and then none) to T, the first of them T long."""
    B, T = case["B"], case.get("T", 1)
    if not case.get("packed"):
        return [T] * B
    rng = random.Random(case["packed"])
    return [T] + [0 if rng.random() < 0.05 else _log(rng, 1, T) for _ in range(B - 1)]


def _rank(D):
    """Columns of the projection that b and c follow in its rows."""
    return max(8, D // 16 // 8 * 8)


def _inputs(case, seed):
    g = _gen(seed)
    kind, B, D, f32 = case["kind"], case["B"], case["D"], torch.float32
    dtype = _dtype(case["dtype"])
    lengths = _lengths(case)
    rows = sum(lengths)
    s = {"case": case, "lengths": lengths, "rows": rows, "offsets": None}
    if case.get("packed"):
        first = torch.zeros(B + 1, dtype=torch.int32)
        first[1:] = torch.cumsum(torch.tensor(lengths), 0)
        s["offsets"] = first.cuda()
    carried = case.get("state", True)
    if kind.startswith("conv"):
        W = case["W"]
        if case["fused"]:                                      # x and z as one projection writes them
            s["xz"] = _normal(g, (rows, 2, D), 1.0, dtype)
            s["x"] = s["xz"][:, 0]
        else:
            s["x"] = _normal(g, (rows, D), 1.0, dtype)
        s["w"], s["bias"] = _normal(g, (D, W), W ** -0.5, f32), _normal(g, (D,), 0.2, f32)
        s["state_in"] = _normal(g, (B, W - 1, D), 1.0, dtype) if carried else None
        if kind == "conv_backward":
            s["dout"] = _normal(g, (rows, D), 1.0, dtype)
            s["dstate_out"] = _normal(g, (B, W - 1, D), 0.3, dtype) if carried else None
        return s
    N = case["N"]
    x = torch.randn((rows, D), generator=g, device="cuda")
    s["x"] = (x * torch.sigmoid(x)).to(dtype)                  # what the convolution leaves
    s["delta"] = _normal(g, (rows, D), 0.5, dtype)
    # step sizes between 1/1000 and 1/10, decays from one state to the next 1, 2, 3, ...: memories from one token to a thousand
    step = torch.exp(torch.rand((D,), generator=g, device="cuda", dtype=torch.float64) * math.log(100) + math.log(1e-3))
    s["bias"] = torch.log(torch.expm1(step)).float()
    s["a"] = -torch.arange(1, N + 1, device="cuda") * torch.exp(_normal(g, (D, N), 0.1, f32))
    if case["fused"]:
        R = _rank(D)
        s["rbc"] = _normal(g, (rows, R + 2 * N), 1.0, dtype)
        s["b"], s["c"] = s["rbc"][:, R:R + N], s["rbc"][:, R + N:]
        s["xz"] = _normal(g, (rows, 2, D), 1.0, dtype) if case["gate"] else None
        s["z"] = s["xz"][:, 1] if case["gate"] else None
    else:
        s["b"], s["c"] = (_normal(g, (rows, N), 1.0, dtype) for _ in range(2))
        s["z"] = _normal(g, (rows, D), 1.0, dtype) if case["gate"] else None
    s["skip"] = 1 + _normal(g, (D,), 0.1, f32)
    s["state_in"] = _normal(g, (B, D, N), 0.3, f32) if carried else None
    if kind == "scan_backward":
        s["dout"] = _normal(g, (rows, D), 1.0, dtype)
        s["dstate_out"] = _normal(g, (B, D, N), 0.3, f32) if carried else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    kind, B, T, D, rows, f32 = case["kind"], case["B"], case.get("T", 1), case["D"], s["rows"], torch.float32
    dtype, fused, carried = _dtype(case["dtype"]), case["fused"], case.get("state", True)
    size = 0
    if kind == "conv_backward":
        W = case["W"]
        s["dx"] = _empty((rows, 2, D), dtype)[:, 0] if fused else _empty((rows, D), dtype)
        s["dw"], s["dbias"] = _empty((D, W), f32), _empty((D,), f32)
        s["dstate_in"] = _empty((B, W - 1, D), dtype) if carried else None
        if own:
            size = _library().wkv6_short_conv_backward_workspace_bytes(B, T, D, W, rows)
    elif kind.startswith("conv"):
        s["out"], s["state_out"] = _empty((rows, D), dtype), _empty((B, case["W"] - 1, D), dtype)
    elif kind == "scan_backward":
        N = case["N"]
        s["dx"], s["ddelta"] = _empty((rows, D), dtype), _empty((rows, D), dtype)
        if fused:                                              # where the projections' own gradients want them
            drbc = _empty((rows, _rank(D) + 2 * N), dtype)
            s["db"], s["dc"] = drbc[:, -2 * N:-N], drbc[:, -N:]
            s["dz"] = _empty((rows, 2, D), dtype)[:, 1] if case["gate"] else None
        else:
            s["db"], s["dc"] = _empty((rows, N), dtype), _empty((rows, N), dtype)
            s["dz"] = _empty((rows, D), dtype) if case["gate"] else None
        s["da"], s["dskip"], s["dbias"] = _empty((D, N), f32), _empty((D,), f32), _empty((D,), f32)
        s["dstate_in"] = _empty((B, D, N), f32) if carried else None
        if own:
            size = _library().wkv6_selective_scan_backward_workspace_bytes(B, T, D, N, rows)
    else:
        s["out"], s["state_out"] = _empty((rows, D), _dtype(case["out"])), _empty((B, D, case["N"]), f32)
        if own and kind == "scan":
            size = _library().wkv6_selective_scan_workspace_bytes(B, T, D, case["N"])
    s["workspace"] = _empty((max(16, size),), torch.uint8)
    return s


# ----------------------------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        return {"scan": _plain_scan, "scan_step": _plain_scan, "scan_backward": _plain_scan_backward, "conv": _plain_conv,
                "conv_step": _plain_conv, "conv_backward": _plain_conv_backward}[kind](s)
    wkv = _library()
    code = {"bf16": wkv.WKV6_DTYPE_BF16, "f32": wkv.WKV6_DTYPE_F32}
    B, T, D, rows, dtype, ws = case["B"], case.get("T", 1), case["D"], s["rows"], code[case["dtype"]], s["workspace"]
    if kind.startswith("conv"):
        W, stride = case["W"], 2 * D if case["fused"] else D
        if kind == "conv":
            wkv.wkv6_short_conv_prefill(B, T, D, W, rows, s["x"], stride, s["w"], s["bias"], 1, s["offsets"], s["state_in"],
                                        s["out"], s["state_out"], dtype)
            return s["out"], s["state_out"]
        if kind == "conv_step":
            wkv.wkv6_short_conv_decode(B, D, W, s["x"], stride, s["w"], s["bias"], 1, s["state_in"], s["out"], s["state_out"],
                                       dtype)
            return s["out"], s["state_out"]
        wkv.wkv6_short_conv_backward(B, T, D, W, rows, s["x"], stride, s["w"], s["bias"], 1, s["offsets"], s["state_in"],
                                     s["dout"], s["dstate_out"], s["dx"], s["dw"], s["dbias"], s["dstate_in"], dtype, ws,
                                     ws.numel())
        return [s["dx"], s["dw"], s["dbias"]] + ([s["dstate_in"]] if case["state"] else [])
    N = case["N"]
    bc_stride, z_stride = (_rank(D) + 2 * N, 2 * D) if case["fused"] else (N, D)
    inputs = (s["x"], D, s["delta"], D, s["bias"], 1, s["a"], s["b"], s["c"], bc_stride, s["skip"], s["z"], z_stride)
    if kind == "scan_step":
        wkv.wkv6_selective_scan_decode(B, D, N, *inputs, s["state_in"], s["out"], s["state_out"], dtype, code[case["out"]])
        return s["out"], s["state_out"]
    if kind == "scan":
        wkv.wkv6_selective_scan_prefill(B, T, D, N, rows, *inputs, s["offsets"], s["state_in"], s["out"], s["state_out"], dtype,
                                        code[case["out"]], ws, ws.numel())
        return s["out"], s["state_out"]
    wkv.wkv6_selective_scan_backward(B, T, D, N, rows, *inputs, s["offsets"], s["state_in"], s["dout"], s["dstate_out"], s["dx"],
                                     s["ddelta"], s["db"], s["dc"], s["dz"], s["da"], s["dskip"], s["dbias"], s["dstate_in"],
                                     dtype, ws, ws.numel())
    return [s["dx"], s["ddelta"], s["db"], s["dc"], s["da"], s["dskip"], s["dbias"]] + \
        ([s["dz"]] if case["gate"] else []) + ([s["dstate_in"]] if case["state"] else [])


# ----------------------------------------------------------------------------------------------
# the plain form: all sequences at once, a slab of tokens by doubling
# ----------------------------------------------------------------------------------------------
def _places(s):
    """[B][T] row numbers, and which of them exist."""
    lengths = torch.tensor(s["lengths"], device="cuda")
    at = torch.arange(s["case"].get("T", 1), device="cuda")[None]
    return (torch.cumsum(lengths, 0) - lengths)[:, None] + at, at < lengths[:, None]


def _padded(s, rows, kind=torch.float32):
    """[rows][C] to [B][T][C], zeros where a sequence has ended."""
    rows = rows.to(kind)
    if not s["case"].get("packed"):
        return rows.reshape(s["case"]["B"], -1, rows.shape[1])
    places, there = _places(s)
    return rows[places.clamp(max=rows.shape[0] - 1)] * there[..., None]


def _rows(s, t, dtype):
    """[B][T][C] back to [rows][C]."""
    return (t.flatten(0, 1) if not s["case"].get("packed") else t[_places(s)[1]]).to(dtype)


def _silu(v):
    return v * torch.sigmoid(v)


def _dsilu(v):
    s = torch.sigmoid(v)
    return s * (1 + v * (1 - s))


def _steps(s):
    """Step sizes [B][T][D], none behind a sequence's end, and what their gradients are times to be those of delta."""
    v = s["delta"].float() + s["bias"]
    dt = v.clamp(min=0) + torch.log1p(torch.exp(-v.abs()))
    return _padded(s, dt), _padded(s, torch.sigmoid(v))


def _doubled(a, v, h):
    """h_t = a_t h_{t-1} + v_t over the second axis, from h on."""
    n = 1
    while n < a.shape[1]:
        v = torch.cat([v[:, :n], torch.addcmul(v[:, n:], a[:, n:], v[:, :-n])], 1)
        a = torch.cat([a[:, :n], a[:, n:] * a[:, :-n]], 1)
        n *= 2
    return torch.addcmul(v, a, h[:, None])


def _slab(case):
    most = max(1, SLAB // (case["B"] * case["D"] * case["N"]))
    return min(256, 1 << int(math.log2(most)))


def _slabs(case):
    n, T = _slab(case), case.get("T", 1)
    return [slice(t, min(t + n, T)) for t in range(0, T, n)]


def _start(s, state, kind=torch.float32):
    case = s["case"]
    if state is None:
        return torch.zeros((case["B"], case["D"], case["N"]), dtype=kind, device="cuda")
    return state.to(kind)


def _plain_scan(s):
    dt, _ = _steps(s)
    x, b, c = (_padded(s, s[n]) for n in ("x", "b", "c"))
    h, y = _start(s, s["state_in"]), torch.empty_like(x)
    for at in _slabs(s["case"]):
        states = _doubled(torch.exp(dt[:, at, :, None] * s["a"]), (dt * x)[:, at, :, None] * b[:, at, None], h)
        y[:, at] = (states * c[:, at, None]).sum(3)
        h = states[:, -1]
    y = _rows(s, y + s["skip"] * x, torch.float32)
    if s["z"] is not None:
        y = y * _silu(s["z"].float())
    return y.to(s["out"].dtype), h.clone()


def _plain_scan_backward(s):
    case, f64 = s["case"], torch.float64
    dt, sig = _steps(s)
    x, b, c, do = (_padded(s, s[n]) for n in ("x", "b", "c", "dout"))
    z = None if s["z"] is None else _padded(s, s["z"])
    dy = do if z is None else do * _silu(z)
    a, skip = s["a"], s["skip"]
    slabs = _slabs(case)
    decays = lambda at: torch.exp(dt[:, at, :, None] * a)  # noqa: E731
    inputs = lambda at: (dt * x)[:, at, :, None] * b[:, at, None]  # noqa: E731
    kept = [_start(s, s["state_in"])]
    for at in slabs[:-1]:
        kept.append(_doubled(decays(at), inputs(at), kept[-1])[:, -1].clone())
    g = _start(s, s["dstate_out"])                             # of the state behind the slab
    y, dx, ddt = (torch.empty_like(x) for _ in range(3))
    db, dc = torch.empty_like(b), torch.empty_like(c)
    da = torch.zeros(a.shape, dtype=f64, device="cuda")
    for at, h in zip(reversed(slabs), reversed(kept)):
        w = decays(at)
        states = _doubled(w, inputs(at), h)
        before = torch.cat([h[:, None], states[:, :-1]], 1)
        behind = torch.cat([w[:, 1:], torch.ones_like(w[:, :1])], 1)
        ds = torch.flip(_doubled(torch.flip(behind, (1,)), torch.flip(c[:, at, None] * dy[:, at, :, None], (1,)), g), (1,))
        g = w[:, 0] * ds[:, 0]
        y[:, at] = (states * c[:, at, None]).sum(3)
        dc[:, at] = (states * dy[:, at, :, None]).sum(2)
        db[:, at] = (ds * (dt * x)[:, at, :, None]).sum(2)
        into = (ds * b[:, at, None]).sum(3)
        dx[:, at] = into * dt[:, at]
        left = ds * before * w
        ddt[:, at] = into * x[:, at] + (left * a).sum(3)
        da += (left * dt[:, at, :, None]).sum((0, 1), dtype=f64)
    dx, ddelta, dtype = dx + skip * dy, ddt * sig, s["dx"].dtype
    res = [_rows(s, t, dtype) for t in (dx, ddelta, db, dc)]
    res += [da.float(), (dy * x).sum((0, 1), dtype=f64).float(), ddelta.sum((0, 1), dtype=f64).float()]
    if z is not None:
        res.append(_rows(s, do * (y + skip * x) * _dsilu(z), dtype))
    return res + ([g] if case["state"] else [])


def _windows(s, kind=torch.float32):
    """Inputs with the W - 1 in front of them, [B][W - 1 + T][D]."""
    x = _padded(s, s["x"], kind)
    front = s["state_in"]
    front = x.new_zeros((x.shape[0], s["case"]["W"] - 1, x.shape[2])) if front is None else front.to(kind)
    return torch.cat([front, x], 1)


def _last(s):
    """[B][W - 1] places in _windows() of every sequence's last inputs."""
    return torch.tensor(s["lengths"], device="cuda")[:, None] + torch.arange(s["case"]["W"] - 1, device="cuda")


def _before(s, xs):
    T = s["case"].get("T", 1)
    return s["bias"] + sum(xs[:, j:j + T] * s["w"][:, j] for j in range(s["case"]["W"]))


def _plain_conv(s):
    xs = _windows(s)
    each = torch.arange(xs.shape[0], device="cuda")[:, None]
    return _rows(s, _silu(_before(s, xs)), s["out"].dtype), xs[each, _last(s)].to(s["out"].dtype)


def _plain_conv_backward(s):
    W, T, f64 = s["case"]["W"], s["case"]["T"], torch.float64
    xs = _windows(s)
    dp = _padded(s, s["dout"]) * _dsilu(_before(s, xs))
    dxs = torch.zeros_like(xs)
    for j in range(W):
        dxs[:, j:j + T] += dp * s["w"][:, j]
    if s["dstate_out"] is not None:
        each = torch.arange(xs.shape[0], device="cuda")[:, None]
        dxs[each, _last(s)] += s["dstate_out"].float()
    dw = torch.stack([(dp * xs[:, j:j + T]).sum((0, 1), dtype=f64) for j in range(W)], 1).float()
    res = [_rows(s, dxs[:, W - 1:], s["dx"].dtype), dw, dp.sum((0, 1), dtype=f64).float()]
    return res + ([dxs[:, :W - 1].to(s["dx"].dtype)] if s["case"]["state"] else [])


# ----------------------------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------------------------
def work(case):
    kind, B, D = case["kind"], case["B"], case["D"]
    size = {"bf16": 2, "f32": 4}
    rows, item = sum(_lengths(case)), size[case["dtype"]]
    offsets = 4 * (B + 1) if case.get("packed") else 0
    carried = 1 if case.get("state", True) else 0
    if kind.startswith("conv"):
        W = case["W"]
        taps, state = 4 * D * (W + 1), B * (W - 1) * D * item
        if kind == "conv_backward":
            return {"bytes": 3 * rows * D * item + 2 * taps + offsets + 3 * carried * state, "flops": rows * D * (6 * W + 12)}
        return {"bytes": 2 * rows * D * item + taps + offsets + (1 + carried) * state, "flops": rows * D * (2 * W + 5)}
    N, gate = case["N"], 1 if case["gate"] else 0
    weights, state = 4 * D * (N + 2), 4 * B * D * N
    if kind == "scan_backward":
        # per state: decay, state, its gradient, and the products with b, c, x, dy, the step size and a
        return {"bytes": rows * D * item * (5 + 2 * gate) + 4 * rows * N * item + 2 * weights + offsets + 3 * carried * state,
                "flops": rows * D * (20 * N + 30)}
    return {"bytes": rows * D * ((2 + gate) * item + size[case["out"]]) + 2 * rows * N * item + weights + offsets +
            (1 + carried) * state, "flops": rows * D * (7 * N + 15)}


# ----------------------------------------------------------------------------------------------
# the same in 64 bits: the recurrence itself, token by token
# ----------------------------------------------------------------------------------------------
def _block(case):
    return max(1, min(64, (1 << 27) // (case["B"] * case["D"] * case["N"])))


def _walk(w, v, h):
    """States behind each token of a block, [B][t][D][N]; h is left behind the last one."""
    res = torch.empty_like(v)
    for t in range(v.shape[1]):
        h.mul_(w[:, t]).add_(v[:, t])
        res[:, t] = h
    return res


def _exact_steps(s):
    v = s["delta"].double() + s["bias"].double()
    return _padded(s, torch.logaddexp(v, torch.zeros_like(v)), v.dtype), _padded(s, 1 / (1 + torch.exp(-v)), v.dtype)


def _exact_scan(s):
    case, f64 = s["case"], torch.float64
    dt, _ = _exact_steps(s)
    x, b, c = (_padded(s, s[n], f64) for n in ("x", "b", "c"))
    a, n, h = s["a"].double(), _block(case), _start(s, s["state_in"], f64).clone()
    y = torch.empty_like(x)
    for t in range(0, case.get("T", 1), n):
        at = slice(t, t + n)
        h_all = _walk(torch.exp(dt[:, at, :, None] * a), (dt[:, at] * x[:, at])[..., None] * b[:, at, None], h)
        y[:, at] = torch.matmul(h_all, c[:, at, :, None])[..., 0]
    y = _rows(s, y + s["skip"].double() * x, f64)
    if s["z"] is not None:
        z = s["z"].double()
        y = y * z / (1 + torch.exp(-z))
    return y, h


def _exact_scan_backward(s):
    case, f64 = s["case"], torch.float64
    T, n = case["T"], max(1, _block(case) // 4)
    dt, sig = _exact_steps(s)
    x, b, c, do = (_padded(s, s[k], f64) for k in ("x", "b", "c", "dout"))
    gate = dgate = None
    dy = do
    if s["z"] is not None:
        z = _padded(s, s["z"], f64)
        q = 1 / (1 + torch.exp(-z))
        gate, dgate = z * q, q + z * q * (1 - q)
        dy = do * gate
    a, skip = s["a"].double(), s["skip"].double()
    places = [slice(t, min(t + n, T)) for t in range(0, T, n)]
    w_of = lambda at: torch.exp(dt[:, at, :, None] * a)  # noqa: E731
    v_of = lambda at: (dt[:, at] * x[:, at])[..., None] * b[:, at, None]  # noqa: E731
    h, kept = _start(s, s["state_in"], f64).clone(), []
    for at in places:
        kept.append(h.clone())
        _walk(w_of(at), v_of(at), h)
    g = _start(s, s["dstate_out"], f64).clone()
    y, dx, ddt, db, dc = (torch.empty_like(t) for t in (x, x, x, b, c))
    da = torch.zeros_like(a)
    for at, first in zip(reversed(places), reversed(kept)):
        w = w_of(at)
        h_all = _walk(w, v_of(at), first.clone())
        ds = torch.empty_like(h_all)
        for t in reversed(range(h_all.shape[1])):
            g.add_(c[:, at][:, t, None] * dy[:, at][:, t, :, None])
            ds[:, t] = g
            g.mul_(w[:, t])
        y[:, at] = torch.matmul(h_all, c[:, at, :, None])[..., 0]
        dc[:, at] = torch.matmul(dy[:, at, None], h_all)[:, :, 0]
        db[:, at] = torch.matmul((dt * x)[:, at, None], ds)[:, :, 0]
        into = torch.matmul(ds, b[:, at, :, None])[..., 0]
        dx[:, at] = into * dt[:, at]
        left = ds * w * torch.cat([first[:, None], h_all[:, :-1]], 1)
        ddt[:, at] = into * x[:, at] + (left * a).sum(3)
        da += (left * dt[:, at, :, None]).sum((0, 1))
    ddelta = ddt * sig
    res = [_rows(s, t, f64) for t in (dx + skip * dy, ddelta, db, dc)] + [da, (dy * x).sum((0, 1)), ddelta.sum((0, 1))]
    if gate is not None:
        res.append(_rows(s, do * (y + skip * x) * dgate, f64))
    return res + ([g] if case["state"] else [])


def _exact_conv(s):
    """Output row by output row of the padded sequences, tap by tap, in 64 bits; the gradients from the transposed taps."""
    case, f64 = s["case"], torch.float64
    W, T = case["W"], case.get("T", 1)
    xs, w = _windows(s, f64), s["w"].double()
    taps = xs.unfold(1, W, 1)                                  # [B][T][D][W]
    p = torch.matmul(taps.unsqueeze(3), w[:, :, None])[..., 0, 0] + s["bias"].double()
    q = 1 / (1 + torch.exp(-p))
    each = torch.arange(xs.shape[0], device="cuda")[:, None]
    if case["kind"] != "conv_backward":
        return _rows(s, p * q, f64), xs[each, _last(s)]
    dp = _padded(s, s["dout"], f64) * (q + p * q * (1 - q))
    wide = torch.zeros((dp.shape[0], T + 2 * W - 2, dp.shape[2]), dtype=f64, device="cuda")
    wide[:, W - 1:W - 1 + T] = dp
    dxs = torch.matmul(wide.unfold(1, W, 1).unsqueeze(3), torch.flip(w, (1,))[:, :, None])[..., 0, 0]
    if s["dstate_out"] is not None:
        dxs[each, _last(s)] += s["dstate_out"].double()
    res = [_rows(s, dxs[:, W - 1:], f64), (taps * dp[..., None]).sum((0, 1)), dp.sum((0, 1))]
    return res + ([dxs[:, :W - 1]] if case["state"] else [])


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"].startswith("conv"):
        return _exact_conv(s)
    return _exact_scan_backward(s) if case["kind"] == "scan_backward" else _exact_scan(s)
