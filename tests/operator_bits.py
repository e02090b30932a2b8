"""How far the gradient of the head-decay mix's decays may be off, as roundings fall: root mean squares, beside the worst cases of tests/operator_util.py.

    dg_t = sum_{t <= s <= a} (r_s . dr_s - k_s . dk_s) + w_{a+1} <dS_{a+1}, S_a>,      a the end of t's block of 1024 tokens or of its sequence

is a sum of products of two numbers.  As root mean squares a number that is a sum over a chunk is off by sqrt(8) steps of 2^-24 of its size (seven
levels of additions and the factors, 1 / sqrt(3) of a step each, and the state's and the decays' own few), the 64 products of a row by seven levels more
(a level's additions together are one rounding of all products in quadrature), so by sqrt(8 + 8 / 3) < 3.3 steps of sqrt(sum of the products' squares).
Rows of dr and dk of one sequence share errors of the states that they are formed from, so twice that is allowed: 6.6 steps."""
import numpy as np

from operator_util import N, np64
from oracle.head_decay_numpy import head_decay_gradients_numpy, head_decay_numpy

BLOCK = 1024
STEPS = 6.6 * 2.0 ** -24


class Parts:
    """dg [rows][H] in 64 bits, and what it consists of."""

    def __init__(self, r, k, v, g, spans, dout, state_in=None, dstate_out=None):
        rows, H = r.shape[:2]
        g = np.broadcast_to(g, (rows, H))
        dr, dk, _, self.dg, _ = head_decay_gradients_numpy(r, k, v, g, spans, dout, state_in, dstate_out)
        self.each = (r * dr - k * dk).sum(2)
        products = ((r * dr) ** 2 + (k * dk) ** 2).sum(2)
        self.anchor, self.ahead = np.full((rows, H), np.nan), np.full((rows, H), np.nan)      # <dS, S> at the block's end, and w in front of it
        self.spread = np.full((rows, H), np.nan)               # sqrt of the sum of all products' squares
        self.blocks = []
        for b, (first, end) in enumerate(spans):
            start = None if state_in is None else state_in[b:b + 1]
            for t0 in range(first, end, BLOCK):
                t1 = min(t0 + BLOCK, end)
                _, start = head_decay_numpy(r, k, v, g, [(t0, t1)], start)
                dS = None if dstate_out is None else dstate_out[b:b + 1]
                if t1 < end:                                   # w_{t1} dS_{t1}: what the rest of the sequence hands back
                    dS = head_decay_gradients_numpy(r, k, v, g, [(t1, end)], dout, None, dS)[4]
                at = np.zeros((H, N, N)) if dS is None else (dS * start)[0]
                self.blocks.append((t0, t1))
                self.anchor[t0:t1] = at.sum((1, 2))
                self.ahead[t0:t1] = np.exp(g[t1]) if t1 < end else 1.
                self.spread[t0:t1] = np.sqrt(np.cumsum(products[t0:t1][::-1], 0)[::-1] + (at ** 2).sum((1, 2)))

    def sums(self, stride=BLOCK):
        """The sums from a token on; with a smaller stride without what is carried from one stride (from the block's end) to the next."""
        res = np.full(self.each.shape, np.nan)
        for t0, t1 in self.blocks:
            for e in range(t1, t0, -stride):
                s = max(t0, e - stride)
                res[s:e] = np.cumsum(self.each[s:e][::-1], 0)[::-1]
        return res


def parts_of(x):
    r, k, v, g = x.arrays()
    return Parts(r, k, v, g, x.spans, np64(x.dout), np64(x.state_in), np64(x.dstate_out))


def off(got, parts):
    """Error beside the spread, a root mean square over every block of every head: [blocks][H], in units of what is allowed."""
    return np.array([np.sqrt((((got - parts.dg)[a:b] / parts.spread[a:b]) ** 2).mean(0)) for a, b in parts.blocks]) / STEPS


def head_off(got, parts, spans):
    """The same of dg [H], a sum over all tokens: an error of a token's product is in the sums of all tokens in front of it, of its block."""
    rows = np.concatenate([np.arange(a, b) for a, b in spans])
    weight = sum(((parts.spread[a:b] ** 2).sum(0) * (b - a)) for a, b in parts.blocks)
    return abs(got - parts.dg[rows].sum(0)) / np.sqrt(weight) / STEPS
