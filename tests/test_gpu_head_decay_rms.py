"""How many bits the head-decay time mix keeps: root mean squares of errors against 64 bits, beside those of the results.

The bounds of tests/operator_util.py hold for every element and assume that all roundings fall the same way; these take them as they fall.  A rounding
is at most half a step, 2^-24, evenly spread: 2^-24 / sqrt(3) at most as a root mean square.  A state with a decay w a token is rounded once a
chunk of C = 64 tokens (32 of fp32 rows) and remembers M = 1 / (1 - w^(2 C)) of these in quadrature: sqrt(M / 3) steps.  Three steps more: the factor
log2 e of a decay that is the same for all tokens and the decay's own factor, which fall the same way in every chunk, and a chunk's own sum, whose
roundings are of its size."""
import math

import numpy as np
import pytest
import torch

import paper_2407_12077_amd as wkv
from operator_bits import STEPS, head_off, off, parts_of
from operator_util import N, Mix, np64

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
STEP = 2.0 ** -24


def rms(t):
    return float(t.double().square().mean().sqrt())


def walk(x, last=0):
    """The state behind a whole call's tokens, and the read-outs of the last ones, in 64 bits on the GPU."""
    r, k, v = (t.view(x.B, x.T, x.H, N) for t in (x.r, x.k, x.v))
    w = torch.exp(x.g.double())
    w = w.expand(x.B, x.T, x.H) if x.decay == "head" else w.view(x.B, x.T, x.H)
    S = torch.zeros((x.B, x.H, N, N), dtype=torch.float64, device="cuda") if x.state_in is None else x.state_in.double()
    out = []
    for t in range(x.T):
        S = w[:, t, :, None, None] * S + k[:, t].double()[..., None] * v[:, t].double()[:, :, None]
        if t >= x.T - last:
            out.append((r[:, t].double()[..., None] * S).sum(2))
    return S, torch.stack(out, 1) if out else None


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("B,T", [(64, 4096), (1, 6000)], ids=["whole", "pieces"])
def test_states_with_long_memories(gpu_device, B, T, dtype):
    x = Mix(3, H=4, B=B, T=T, dtype=dtype, decay="head", state=False)
    x.g.copy_(torch.log1p(-torch.exp2(-torch.tensor([9., 10., 11., 12.], device="cuda", dtype=torch.float64))).float())
    _, state = x.prefill()
    want, _ = walk(x)
    for h in range(4):
        M = 1 / (1 - math.exp(2 * (64 if dtype == BF16 else 32) * float(x.g[h])))
        assert rms(state[:, h].double() - want[:, h]) <= STEP * (math.sqrt(M / 3) + 3) * rms(want[:, h]), h


@pytest.mark.parametrize("g", [-0.02, -0.3])
def test_the_factor_of_the_first_token(gpu_device, g):
    """With queries and read-outs' gradients of nought dstate_in is exp(g) dstate_out: four logarithms near g.  The factor: half a step of its exponent, X = g log2 e,
    which is X ln 2 steps of its value and falls as it does; its own, evenly spread; and the series' 2^-25 at the most.  The product: a rounding."""
    x = Mix(6, H=4, B=512, T=1, dtype=F32, gradients=True)
    x.g.copy_(g * (1 + torch.rand((512, 4), device="cuda", generator=torch.Generator("cuda").manual_seed(1)) / 4))
    x.r.zero_()
    x.dout.zero_()
    got = x.backward()[4].double()
    want = torch.exp(x.g.double())[:, :, None, None] * x.dstate_out.double()
    error = (got - want) / want
    assert rms(error) <= STEP * math.sqrt(((1.25 * g) ** 2 + 2) / 3 + 0.25)
    assert float(error.abs().max()) <= STEP * (1.25 * abs(g) + 2.5)


# Sums and factors that no long memory is in: chains of up to forty additions (an fp32 score has sixteen of four products, a read-out eight over keys and sixteen
# over the state), whose partial sums have half the result's square on average, sqrt(40 / 2 / 3) < 2.6 steps, ten more roundings, sqrt(10 / 3) < 1.9; and the three
# steps of above.  Two bf16 terms of a state or a score, in the place of three, are 41 steps of it off (tests/test_operator_bits_cpu.py)
SUMS = 2.6 + 1.9 + 3


def memory(x, h):
    g = x.g[h] if x.decay == "head" else x.g[:, h].mean()
    return 1 / (1 - math.exp(2 * (64 if x.dtype == BF16 else 32) * float(g)))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("decay", ["token", "head"])
@pytest.mark.parametrize("case", [dict(B=65, T=200, H=4), dict(B=300, T=70, H=1), dict(B=1, T=1500, H=2), dict(lengths=[900, 0, 33, 130, 64], H=3)], ids=str)
def test_results_in_fp32(gpu_device, case, decay, dtype):
    """Among them more units than the card has compute units, whole: a second round of workgroups."""
    x = Mix(7, dtype=dtype, decay=decay, gradients=True, **case)
    out, state = x.prefill(F32)
    want, last = x.exact()
    results = [("out", out, want), ("state", state, last)]
    exact, got = x.exact_gradients(), x.backward()
    if dtype == F32:
        results += [(n, got[i], exact[i]) for i, n in enumerate(("dr", "dk", "dv"))]
    results.append(("dstate_in", got[4], exact[4]))
    for name, a, b in results:
        b = torch.from_numpy(b).cuda()
        for h in range(x.H):
            u, v = a[:, h].double(), b[:, h]
            if name in ("out", "dr", "dk", "dv"):
                u, v = u[x.covered], v[x.covered]
            assert rms(u - v) <= STEP * (math.sqrt(memory(x, h) / 3) + SUMS) * rms(v), (name, h)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("decay", ["token", "head"])
@pytest.mark.parametrize("case", [dict(B=2, T=2100, H=2), dict(B=65, T=200, H=4), dict(lengths=[2100, 0, 1024, 1025, 5, 300], H=2, tail=3)], ids=str)
def test_gradients_of_decays(gpu_device, case, decay, dtype):
    """Over several blocks, and from short and empty sequences, per token and summed a head; the bounds are a small part of what they bound."""
    x = Mix(8, dtype=dtype, decay=decay, gradients=True, **case)
    got, parts = np64(x.backward()[3]), parts_of(x)
    if decay == "head":
        assert head_off(got, parts, x.spans).max() < 1
    else:
        assert off(got, parts).max() < 1
    assert np.median(parts.spread[x.covered.numpy()] * STEPS / abs(parts.dg[x.covered.numpy()])) < 0.01
