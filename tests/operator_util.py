"""What the GPU tests of the head-decay time mix share: inputs, calls, and how far a result may be off.

Bounds.  A result in fp32 is a sum of terms, each a product of input values and a decay.  With half a step of fp32, 2^-24, for each rounding a term
passes: up to 64 in the product of two rows or of a row with a state, up to 80 in the sums over a chunk, 8 in factors, and 8 a chunk
of 32 tokens while it is part of the state.  A decay 2^-X over tokens of a block has an exponent that is off by up to 18 roundings of X (sixteen
additions, the factor log2 e, a difference), so it is off by 18 X 2^-24 of itself; X 2^-X <= 1.07 2^(-X/2), so that is 20 roundings
of the term with half the logarithm of its decay.  Together K(T) = 64 + 80 + 8 + 20 + 8 ceil(T / 32) roundings of m, the sum of
the terms' magnitudes with halved logarithms: the oracle on absolute values and g / 2.  Read-outs that are rounded to bf16 have computed
operands of two bf16, 2^-17 of a term, and the rounding itself, 2^-8 of the value.
"""
import math

import numpy as np
import torch

import paper_2407_12077_amd as wkv
from oracle.head_decay_numpy import head_decay_gradients_numpy, head_decay_numpy

N = 64
CODE = {torch.bfloat16: wkv.WKV6_DTYPE_BF16, torch.float32: wkv.WKV6_DTYPE_F32}


def roundings(T):
    return 64 + 80 + 8 + 20 + 8 * math.ceil(T / 32)


def np64(t):
    return None if t is None else t.detach().double().cpu().numpy()


class Mix:
    """Inputs of a call on the GPU.  lengths: sequences packed with `front` rows before and `tail` rows behind them, else B x T."""

    def __init__(self, seed, H, B=None, T=None, lengths=None, front=0, tail=0, dtype=torch.bfloat16, decay="token", fused=False, state=True,
                 longest=None, scale=0.25, gradients=False):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        normal = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
        self.H, self.dtype, self.decay = H, dtype, decay
        if lengths is None:
            self.B, self.T, self.rows, self.offsets = B, T, B * T, None
            self.spans = [(b * T, b * T + T) for b in range(B)]
        else:
            first = [front]
            for n in lengths:
                first.append(first[-1] + n)
            self.B, self.T, self.rows = len(lengths), longest or max(lengths + [0]), first[-1] + tail
            self.spans = list(zip(first[:-1], first[1:]))
            self.offsets = torch.tensor(first, dtype=torch.int32, device="cuda")
        rows = self.rows
        if fused:
            self.rkv = (normal(rows, 3, H, N) * scale).to(dtype)
            self.r, self.k, self.v = self.rkv.unbind(1)
        else:
            self.r, self.k, self.v = ((normal(rows, H, N) * scale).to(dtype) for _ in range(3))
        self.stride = (3 if fused else 1) * H * N
        if decay == "head":
            self.g = -torch.exp(torch.rand(H, generator=gen, device="cuda") * 7 - 7)
        else:
            self.g = -torch.exp(torch.rand((rows, H), generator=gen, device="cuda") * 7 - 6)
        self.g_stride = 0 if decay == "head" else H
        self.state_in = normal(self.B, H, N, N) * 0.1 if state else None
        self.dout = normal(rows, H, N).to(dtype) if gradients else None
        self.dstate_out = normal(self.B, H, N, N) * 0.1 if gradients and state else None
        self.covered = torch.zeros(rows, dtype=torch.bool)
        for a, b in self.spans:
            self.covered[a:b] = True

    def arrays(self):
        return tuple(np64(a) for a in (self.r, self.k, self.v, self.g))

    def workspace(self, gradients=False):
        n = wkv.wkv6_head_decay_backward_workspace_bytes(self.B, self.T, self.H, N, self.rows) if gradients else \
            wkv.wkv6_head_decay_workspace_bytes(self.B, self.T, self.H, N)
        assert n >= 0
        return torch.full((max(16, n) // 4,), float("nan"), device="cuda")     # nothing in it has to be set

    def prefill(self, out_dtype=torch.float32, state_out="new", workspace=None, out=None):
        out = torch.full((self.rows, self.H, N), 7.0, dtype=out_dtype, device="cuda") if out is None else out
        if isinstance(state_out, str):
            state_out = torch.full((self.B, self.H, N, N), float("nan"), device="cuda")
        ws = self.workspace() if workspace is None else workspace
        wkv.wkv6_head_decay_prefill(self.B, self.T, self.H, N, self.rows, self.r, self.k, self.v, self.stride, self.g, self.g_stride, self.offsets,
                                    self.state_in, out, state_out, CODE[self.dtype], CODE[out_dtype], ws, ws.numel() * 4)
        return out, state_out

    def backward(self, workspace=None, into=None):
        if into is None:
            fused = self.stride != self.H * N
            if fused:
                grads = torch.full((self.rows, 3, self.H, N), 7.0, dtype=self.dtype, device="cuda").unbind(1)
            else:
                grads = [torch.full((self.rows, self.H, N), 7.0, dtype=self.dtype, device="cuda") for _ in range(3)]
            into = [*grads, torch.full(self.g.shape, 7.0, device="cuda"),
                    torch.full((self.B, self.H, N, N), float("nan"), device="cuda") if self.state_in is not None else None]
        ws = self.workspace(True) if workspace is None else workspace
        wkv.wkv6_head_decay_backward(self.B, self.T, self.H, N, self.rows, self.r, self.k, self.v, self.stride, self.g, self.g_stride, self.offsets,
                                     self.state_in, self.dout, self.dstate_out, *into, CODE[self.dtype], ws, ws.numel() * 4)
        return into

    # ------------------------------------------------------------------ oracle and bounds
    def exact(self):
        r, k, v, g = self.arrays()
        return head_decay_numpy(r, k, v, g, self.spans, np64(self.state_in))

    def magnitudes(self):
        r, k, v, g = self.arrays()
        s = np64(self.state_in)
        return head_decay_numpy(abs(r), abs(k), abs(v), np.maximum(g, -300.) / 2, self.spans, None if s is None else abs(s))

    def exact_gradients(self):
        r, k, v, g = self.arrays()
        return list(head_decay_gradients_numpy(r, k, v, g, self.spans, np64(self.dout), np64(self.state_in), np64(self.dstate_out)))

    def gradient_bounds(self):
        """(of dr, dk, dv, dg [rows][H], dstate_in) in fp32."""
        r, k, v, g = self.arrays()
        s, d = np64(self.state_in), np64(self.dstate_out)
        g = np.broadcast_to(np.maximum(g, -300.) / 2, (self.rows, self.H))
        absolute = [abs(r), abs(k), abs(v), g, self.spans]
        dr, dk, dv, dg, d0 = head_decay_gradients_numpy(*absolute, abs(np64(self.dout)), None if s is None else abs(s), None if d is None else abs(d))
        _, last = head_decay_numpy(*absolute, None if s is None else abs(s))
        # dg: the sums of r . dr and k . dk (another 64 roundings) from a token to the end of its block, here of its sequence, and <dS, S> behind
        each = (abs(r) * dr).sum(2) + (abs(k) * dk).sum(2)
        total = np.full(each.shape, np.nan)
        for b, (first, end) in enumerate(self.spans):
            total[first:end] = np.cumsum(each[first:end][::-1], 0)[::-1]
            if d is not None:
                total[first:end] += (abs(d[b]) * last[b]).sum((1, 2))
        step = 2.0 ** -24
        K = roundings(self.T)
        return [step * K * a for a in (dr, dk, dv)] + [step * (K + 64) * total, step * K * d0]


def check(name, got, want, bound, covered=None, dtype=torch.float32):
    """Every element within its bound (plus the rounding to bf16); rows of nobody as they were (7)."""
    got = np64(got)
    if covered is not None:
        mask = covered.numpy()
        assert (got[~mask] == 7.0).all(), f"{name}: rows of no sequence were written"
        got, want, bound = got[mask], want[mask], bound[mask]
    limit = bound + (2.0 ** -8 * abs(want) if dtype == torch.bfloat16 else 0) + 1e-30
    off = abs(got - want)
    assert np.isfinite(got).all(), f"{name}: not finite"
    if off.size:
        worst = np.unravel_index(np.argmax(off / limit), off.shape)
        assert (off <= limit).all(), f"{name}: {off[worst]:.3e} off {want[worst]:.3e} at {worst}, bound {limit[worst]:.3e}"
