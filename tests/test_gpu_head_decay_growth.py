"""The head-decay time mix where g is above nought, so that states grow, against the recurrence in 64 bits.

Bounds: those of tests/operator_util.py, but for the exponents.  There a decay's logarithm X is as far off as 18 roundings of it, and X 2^-X stays
small; here X grows with 2^X, so a term has 18 |X| roundings more, |X| at most what all tokens of the longest sequence make of it, and its
magnitude is that with the decays as they are."""
import numpy as np
import pytest
import torch

import paper_2407_12077_amd as wkv
from operator_util import CODE, N, Mix, check, np64, roundings
from oracle.head_decay_numpy import head_decay_gradients_numpy, head_decay_numpy

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
STEP = 2.0 ** -24


def steps_of(x):
    g = np.broadcast_to(abs(np64(x.g)), (x.rows, x.H))
    return STEP * (roundings(x.T) + 18 * np.log2(np.e) * max(g[a:b].sum(0).max() for a, b in x.spans))


def magnitudes(x):
    r, k, v, g = x.arrays()
    s = np64(x.state_in)
    return head_decay_numpy(abs(r), abs(k), abs(v), g, x.spans, None if s is None else abs(s))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("g", [0.004, 0.02, 0.1, 0.3])
def test_prefill(gpu_device, g, dtype):
    x = Mix(1, H=2, B=2, T=150, dtype=dtype, decay="head")
    x.g[:] = g
    out, state = x.prefill()
    (want, last), (m, m_last) = x.exact(), magnitudes(x)
    check("out", out, want, steps_of(x) * m)
    check("state", state, last, steps_of(x) * m_last)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_prefill_in_pieces_with_decays_and_growth(gpu_device, dtype):
    x = Mix(2, H=2, B=1, T=1500, dtype=dtype)
    x.g[:, 0] = 0.02
    x.g[:, 1] = x.g[:, 1].abs() * 0.1 * torch.where(torch.arange(1500, device="cuda") % 3 == 0, 1., -0.5)
    assert wkv.wkv6_head_decay_workspace_bytes(x.B, x.T, x.H, N) > 0
    out, state = x.prefill()
    (want, last), (m, m_last) = x.exact(), magnitudes(x)
    check("out", out, want, steps_of(x) * m)
    check("state", state, last, steps_of(x) * m_last)


def test_prefill_and_single_tokens_agree(gpu_device):
    x = Mix(3, H=2, B=1, T=70, dtype=F32, decay="head")
    x.g[:] = 0.05
    out, state = x.prefill()
    s, o = x.state_in.clone(), torch.empty((1, 2, N), device="cuda")
    steps = []
    for t in range(x.T):
        wkv.wkv6_head_decay_decode(1, 2, N, x.r[t:], x.k[t:], x.v[t:], 2 * N, x.g, 0, s, o, s, CODE[F32], CODE[F32])
        steps.append(o.clone())
    m, m_last = magnitudes(x)
    check("out", out, np64(torch.cat(steps)), 2 * steps_of(x) * m)
    check("state", state, np64(s), 2 * steps_of(x) * m_last)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_gradients(gpu_device, dtype):
    x = Mix(4, H=2, lengths=[100, 33, 0, 70], dtype=dtype, gradients=True)
    x.g[:] = 0.03
    got, want = x.backward(), x.exact_gradients()
    r, k, v, g = x.arrays()
    absolute = [abs(r), abs(k), abs(v), g, x.spans]
    s, d = abs(np64(x.state_in)), abs(np64(x.dstate_out))
    m = list(head_decay_gradients_numpy(*absolute, abs(np64(x.dout)), s, d))
    _, last = head_decay_numpy(*absolute, s)
    each = (abs(r) * m[0]).sum(2) + (abs(k) * m[1]).sum(2)     # dg: sums of r . dr and k . dk from a token on, and <dS, S> behind
    for b, (first, end) in enumerate(x.spans):
        m[3][first:end] = np.cumsum(each[first:end][::-1], 0)[::-1] + (d[b] * last[b]).sum((1, 2))
    K = steps_of(x)
    for name, a, w, b in zip(("dr", "dk", "dv"), got, want, m):
        check(name, a, w, K * b, x.covered, dtype)
    check("dg", got[3], want[3], (K + 64 * STEP) * m[3], x.covered)
    check("dstate_in", got[4], want[4], K * m[4])
