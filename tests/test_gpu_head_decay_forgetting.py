"""A state that a chunk, or a run of chunks, forgets nearly all of: what is left of it keeps its bits, relative to itself.

Bounds.  Behind T tokens a decay 2^-X has an exponent that is off by 18 roundings of X (tests/operator_util.py) and, over chunks, 4 roundings a chunk of
32 tokens (its factor's, the product's, and a cut's); rows are so small that nothing else is in the results, or nought."""
import math

import numpy as np
import pytest
import torch

import paper_2407_12077_amd as wkv
from operator_util import N, Mix, check, np64

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
STEP = 2.0 ** -24


def relative(x):
    X = np.log2(np.e) * np.broadcast_to(-np64(x.g), (x.rows, x.H))
    return STEP * (18 * max(X[a:b].sum(0).max() for a, b in x.spans) + 4 * math.ceil(x.T / 32) + 8)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,g", [(32, -0.25), (64, -0.1), (64, -0.5), (128, -0.2), (200, -0.2), (300, -0.07), (2000, -0.02), (2000, -0.03)])
def test_state_alone(gpu_device, T, g, dtype):
    """No keys: the state behind is the state in front, decayed; with 2000 tokens in pieces, whose total decays are kept."""
    x = Mix(T, H=2, B=1, T=T, dtype=dtype, decay="head")
    x.g[:] = g
    x.k.zero_()
    assert T < 2000 or wkv.wkv6_head_decay_workspace_bytes(1, T, 2, N) > 0
    out, state = x.prefill()
    want, last = x.exact()
    check("state", state, last, relative(x) * abs(last))
    # a read-out adds 64 products with a state
    S = abs(np64(x.state_in))[0]
    r, decay = abs(np64(x.r)), np.exp(g * np.arange(1, T + 1))[:, None, None]
    check("out", out, want, (relative(x) + 72 * STEP) * decay * (r[..., None] * S).sum(2))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_states_gradient_alone(gpu_device, dtype):
    """No queries: the gradient of the state in front is that of the state behind, decayed."""
    x = Mix(5, H=2, lengths=[192, 0, 40], dtype=dtype, decay="head", gradients=True)
    x.g[:] = -0.15
    x.r.zero_()
    x.dout.zero_()
    want = x.exact_gradients()[4]
    check("dstate_in", x.backward()[4], want, relative(x) * abs(want))
