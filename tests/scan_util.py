"""What the GPU tests of the selective scan and the short convolution share: inputs, calls, and how far a result may be off.

Bounds of the scan.  Roundings are half steps of fp32, 2^-24 of a value.  A step size from v = delta + bias, |v| <= 8: the sum moves v by 2^-24 |v|, the argument
log2(e) |v| by two more such, and softplus(v) by no more than that share of itself; its exponential, sum, logarithm and products are within 12 roundings: 8 * 3 + 12 = 36.  An
exponent dt a log2(e) adds three: 39 roundings of X, and X exp(-X) <= 0.74 exp(-X / 2): 29 of the term with half its exponent.  A term: dt x b with 36 + 2, products with c, skip,
gate (sigmoid of |z| <= 8: 8 * 3 + 8) or its slope (twice that), dy, a, x: 38 + 2 * 32 + 8.  Sums: 64 states, 64 lanes in six, 16 blocks, 20 more in the folds: 106.  In the state, and in its
gradient, a token multiplies by an exponential (its own error: two) and adds: four roundings a token.  Together K(T) = 250 + 8 T roundings of m, the sum of the terms' magnitudes
with halved exponents: the oracle on absolute values.  (Exponents above nought grow by X exp(X): tests of them keep X below 3, and take 4 K.)  Sums over all tokens add T / 16 + 16 + B
roundings, within the 8 T.  Results rounded to bf16 are off by 2^-8 of the value more.

Bounds of the convolution.  out: W + 2 roundings in p, times silu's slope, at most 1.1; of silu itself 32 for |p| <= 8: 48 of sum |w x| + |bias|.  Gradients: the same 48 of p, and of the products
and sums 16 (and T of the sums over tokens, fewer in fact), of the terms' magnitudes with the slope's own change (oracle).
"""
import numpy as np
import torch

import paper_2407_12077_amd as wkv
from oracle.selective_scan_numpy import scan_gradients, scan_recurrence, selective_scan_gradients_numpy, selective_scan_numpy, selective_scan_parts
from oracle.short_conv_numpy import short_conv_gradients_numpy, short_conv_numpy

CODE = {torch.bfloat16: wkv.WKV6_DTYPE_BF16, torch.float32: wkv.WKV6_DTYPE_F32}
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
BF16, F32 = torch.bfloat16, torch.float32
UNTOUCHED = 77.0


def np64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def check(name, got, want, bound, covered=None, untouched=UNTOUCHED):
    """Within `bound` and the rounding to got's type; rows that nobody owns as they were."""
    value = np64(got)
    assert np.isfinite(value).all(), f"{name}: not finite"
    if covered is not None:
        assert (value[~covered] == untouched).all(), f"{name}: rows of nobody were written"
        value, want, bound = value[covered], want[covered], bound[covered]
    limit = bound + HALF[got.dtype] * np.abs(want) + 1e-37
    over = np.abs(value - want) / limit
    assert value.shape == want.shape and (over.size == 0 or over.max() <= 1), (name, over.max(), np.unravel_index(over.argmax(), over.shape))


class Rows:
    """B x T, or sequences packed with `front` rows in front of and `tail` rows behind them."""

    def __init__(self, B=None, T=None, lengths=None, front=0, tail=0, longest=None):
        self.offsets = None
        if lengths is None:
            self.B, self.T, self.rows = B, T, B * T
            self.spans = [(b * T, (b + 1) * T) for b in range(B)]
        else:
            ends = front + np.cumsum([0] + list(lengths))
            self.B, self.T, self.rows = len(lengths), max(lengths) if longest is None else longest, int(ends[-1]) + tail
            self.spans = [(int(ends[i]), int(ends[i]) + min(n, self.T)) for i, n in enumerate(lengths)]
            self.offsets = torch.tensor(ends, dtype=torch.int32).cuda()
        self.covered = np.zeros(self.rows, dtype=bool)
        for first, end in self.spans:
            self.covered[first:end] = True
        self.longest = max([e - f for f, e in self.spans] + [0])


class Workspace:
    """Stands for exactly `n` bytes of workspace in a call; nothing in it has to be set, and what lies behind it has to stay as it is."""

    GUARD = 4096

    def __init__(self, n):
        assert n >= 0 and n % 4 == 0
        self.all = torch.full((n // 4 + self.GUARD,), float("nan"), device="cuda")
        self.all[n // 4:] = 7.0
        self.n = n

    def data_ptr(self):
        return self.all.data_ptr()

    def check(self):
        assert bool((self.all[self.n // 4:] == 7).all()), "behind the workspace"


class Scan(Rows):
    def __init__(self, seed, D, N, dtype=BF16, gate=True, skip=True, bias=True, softplus=True, state=True, fused=False, growing=False, **rows):
        super().__init__(**rows)
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        normal = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
        R = self.rows
        self.D, self.N, self.dtype, self.softplus = D, N, dtype, softplus
        self.whole = {}                                        # what the strided parts lie in
        if fused:                                              # x and z of one projection, b and c behind eight columns of another
            self.whole["xz"] = normal(R, 2, D).to(dtype)
            self.whole["rbc"] = normal(R, 8 + 2 * N).to(dtype)
            self.x, z = self.whole["xz"].unbind(1)
            self.b, self.c = self.whole["rbc"][:, 8:8 + N], self.whole["rbc"][:, 8 + N:]
            self.x_stride, self.bc_stride = 2 * D, 8 + 2 * N
        else:
            self.x, z, self.b, self.c = (normal(R, w).to(dtype) for w in (D, D, N, N))
            self.x_stride, self.bc_stride = D, N
        self.z = z if gate else None
        self.delta = (normal(R, D) * (0.5 if softplus else 0.02) + (0 if softplus else 0.1)).to(dtype)
        self.bias = normal(D) - 2.5 if bias and softplus else normal(D) * 0.02 if bias else None
        self.a = -torch.exp(normal(D, N)) * (1 + torch.arange(N, device="cuda") / 4)
        if growing:
            self.a = self.a.abs() * 1e-3
        self.skip = normal(D) if skip else None
        self.state_in = normal(self.B, D, N) if state else None
        self.dout = normal(R, D).to(dtype)
        self.dstate_out = normal(self.B, D, N) if state else None
        self.scale = 4 if growing else 1

    def inputs(self):
        return (self.x, self.x_stride, self.delta, self.D, self.bias, int(self.softplus), self.a, self.b, self.c, self.bc_stride, self.skip, self.z,
                self.x_stride)

    def blank(self, width, dtype, stride=None):
        t = torch.full((self.rows, stride or width), UNTOUCHED, dtype=dtype, device="cuda")
        return t[:, :width]

    def prefill(self, out_dtype=None, state_out="new", workspace=None, stream=None):
        out_dtype = out_dtype or self.dtype
        out = self.blank(self.D, out_dtype)
        if isinstance(state_out, str):
            state_out = torch.full((self.B, self.D, self.N), float("nan"), device="cuda")
        n = wkv.wkv6_selective_scan_workspace_bytes(self.B, self.T, self.D, self.N)
        ws = workspace or Workspace(n)
        wkv.wkv6_selective_scan_prefill(self.B, self.T, self.D, self.N, self.rows, *self.inputs(), self.offsets, self.state_in, out, state_out,
                                        CODE[self.dtype], CODE[out_dtype], ws, n, stream=stream)
        if workspace is None:
            ws.check()
        return out, state_out

    def backward(self, workspace=None, weights=True):
        D, N, dt = self.D, self.N, self.dtype
        g = dict(dx=self.blank(D, dt, self.x_stride), ddelta=self.blank(D, dt), db=self.blank(N, dt, self.bc_stride), dc=self.blank(N, dt, self.bc_stride),
                 dz=self.blank(D, dt, self.x_stride) if self.z is not None else None)
        for name, shape in (("da", (D, N)), ("dskip", (D,)), ("dbias", (D,))):
            g[name] = torch.full(shape, float("nan"), device="cuda") if weights else None
        g["dstate_in"] = torch.full((self.B, D, N), float("nan"), device="cuda")
        n = wkv.wkv6_selective_scan_backward_workspace_bytes(self.B, self.T, D, N, self.rows)
        ws = workspace or Workspace(n)
        wkv.wkv6_selective_scan_backward(self.B, self.T, D, N, self.rows, *self.inputs(), self.offsets, self.state_in, self.dout, self.dstate_out,
                                         *g.values(), CODE[dt], ws, n)
        if workspace is None:
            ws.check()
        return g

    # ------------------------------------------------------------------ oracle
    def call(self):
        return dict(x=np64(self.x), delta=np64(self.delta), a=np64(self.a), b=np64(self.b), c=np64(self.c), spans=self.spans, bias=np64(self.bias),
                    use_softplus=self.softplus, skip=np64(self.skip), z=np64(self.z), state_in=np64(self.state_in))

    def magnitude_parts(self):
        p = selective_scan_parts(**self.call())
        p["exponents"] = np.maximum(p["exponents"], p["exponents"] / 2)
        for n in ("dt", "a", "x", "b", "c", "skip", "gate", "state_in"):
            p[n] = np.abs(p[n])
        if self.z is not None:                                 # the slope's terms one by one
            z = np.abs(np64(self.z))
            p["dgate"] = 1 + z
        return p

    def steps(self):
        return (250 + 8 * self.longest) * self.scale * 2.0 ** -24

    def want(self):
        out, state = selective_scan_numpy(**self.call())
        p = self.magnitude_parts()
        for n in ("a", "dgate", "slope"):
            p.pop(n)
        m_out, m_state, _ = scan_recurrence(**p)
        return (out, state), (self.steps() * m_out, self.steps() * m_state)

    def want_gradients(self):
        want = selective_scan_gradients_numpy(np64(self.dout), np64(self.dstate_out), **self.call())
        p = self.magnitude_parts()
        zero = np.zeros(p["state_in"].shape)
        m = scan_gradients(**p, dout=np.abs(np64(self.dout)), dstate_out=zero if self.dstate_out is None else np.abs(np64(self.dstate_out)))
        return want, {n: self.steps() * v for n, v in m.items()}

    def check_prefill(self, out, state):
        want, bound = self.want()
        check("out", out, want[0], bound[0], self.covered)
        if state is not None:
            check("state", state, want[1], bound[1])

    def check_backward(self, got):
        want, bound = self.want_gradients()
        for name, g in got.items():
            if g is not None:
                check(name, g, want[name], bound[name], self.covered if g.shape[0] == self.rows and name in ("dx", "ddelta", "db", "dc", "dz") else None)


class Conv(Rows):
    def __init__(self, seed, D, W, dtype=BF16, bias=True, silu=True, state=True, fused=False, **rows):
        super().__init__(**rows)
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        normal = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
        R = self.rows
        self.D, self.W, self.dtype, self.silu = D, W, dtype, silu
        self.stride = 2 * D if fused else D
        self.whole = normal(R, self.stride).to(dtype)
        self.x = self.whole[:, :D]
        self.w, self.bias = normal(D, W) * 0.5, normal(D) if bias else None
        self.state_in = normal(self.B, W - 1, D).to(dtype) if state else None
        self.dout = normal(R, D).to(dtype)
        self.dstate_out = normal(self.B, W - 1, D).to(dtype) if state else None

    def blank_out(self):
        return torch.full((self.rows, self.D), UNTOUCHED, dtype=self.dtype, device="cuda")

    def prefill(self, state_out="new"):
        out = self.blank_out()
        if isinstance(state_out, str):
            state_out = torch.full((self.B, self.W - 1, self.D), float("nan"), dtype=self.dtype, device="cuda")
        wkv.wkv6_short_conv_prefill(self.B, self.T, self.D, self.W, self.rows, self.x, self.stride, self.w, self.bias, int(self.silu), self.offsets,
                                    self.state_in, out, state_out, CODE[self.dtype])
        return out, state_out

    def backward(self, weights=True):
        dx = torch.full((self.rows, self.stride), UNTOUCHED, dtype=self.dtype, device="cuda")[:, :self.D]
        dw, db = (torch.full(s, float("nan"), device="cuda") if weights else None for s in ((self.D, self.W), (self.D,)))
        ds = torch.full((self.B, self.W - 1, self.D), float("nan"), dtype=self.dtype, device="cuda")
        n = wkv.wkv6_short_conv_backward_workspace_bytes(self.B, self.T, self.D, self.W, self.rows)
        ws = Workspace(n if weights else 0)
        wkv.wkv6_short_conv_backward(self.B, self.T, self.D, self.W, self.rows, self.x, self.stride, self.w, self.bias, int(self.silu), self.offsets,
                                     self.state_in, self.dout, self.dstate_out, dx, dw, db, ds, CODE[self.dtype], ws, ws.n)
        ws.check()
        return dx, dw, db, ds

    def call(self):
        return dict(x=np64(self.x), w=np64(self.w), spans=self.spans, bias=np64(self.bias), use_silu=self.silu, state_in=np64(self.state_in))

    def check_prefill(self, out, state):
        want, want_state = short_conv_numpy(**self.call())
        c = self.call()
        c = {**c, "x": abs(c["x"]), "w": abs(c["w"]), "bias": None if c["bias"] is None else abs(c["bias"]),
             "state_in": None if c["state_in"] is None else abs(c["state_in"]), "use_silu": False}
        check("out", out, want, 48 * 2.0 ** -24 * short_conv_numpy(**c)[0], self.covered)
        if state is not None:
            assert (np64(state) == want_state).all()

    def check_backward(self, got):
        args = dict(**self.call(), dout=np64(self.dout), dstate_out=np64(self.dstate_out))
        want = short_conv_gradients_numpy(**args)
        size = short_conv_gradients_numpy(**args, magnitudes=True)
        for i, name in enumerate(("dx", "dw", "dbias", "dstate_in")):
            if got[i] is not None:
                steps = (64 + (self.longest if name in ("dw", "dbias") else 0)) * 2.0 ** -24
                check(name, got[i], want[i], steps * size[i], self.covered if name == "dx" else None)
