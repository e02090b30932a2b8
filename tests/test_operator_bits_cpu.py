"""The bounds of tests/operator_bits.py refuse what a wrong kernel would give: gradients of the decays that are nought, that lack a block's anchor or its decay, or
what is carried from 256 tokens to the next; and they take the right one with every product rounded to fp32."""
import numpy as np
import pytest
import torch

from operator_bits import Parts, head_off, off
from operator_util import N

SPANS = [(0, 2100), (2100, 3124), (3124, 4149), (4149, 4149), (4149, 4154)]


@pytest.fixture(scope="module", params=["states", "no_states"])
def parts(request):
    rng = np.random.default_rng(7)
    rows, H, B = SPANS[-1][1], 2, len(SPANS)
    r, k, v = (rng.standard_normal((rows, H, N)) * 0.25 for _ in range(3))
    g = -np.exp(rng.random((rows, H)) * 7 - 6)
    g[:, 1] = -np.exp(-5.)                                     # one decay for all tokens
    states = [rng.standard_normal((B, H, N, N)) * 0.1 if request.param == "states" else None for _ in range(2)]
    return Parts(r, k, v, g, SPANS, rng.standard_normal((rows, H, N)), *states)


def test_the_parts_make_the_whole(parts):
    whole = parts.sums() + parts.anchor
    assert np.allclose(whole, parts.dg, rtol=0, atol=1e-11 * parts.spread.max())


def test_rounded_sums_pass(parts):
    rng = np.random.default_rng(8)
    near = parts.dg + 2.0 ** -24 * parts.spread * rng.standard_normal(parts.dg.shape)
    assert off(near, parts).max() < 1 and head_off(near.sum(0), parts, SPANS).max() < 1


def test_wrong_gradients_are_refused(parts):
    inner = [i for i, (a, b) in enumerate(parts.blocks) if b not in {e for _, e in SPANS}]       # blocks with tokens of their sequence behind them
    assert len(inner) == 3
    assert (off(np.zeros_like(parts.dg), parts) > 1).all()
    assert (off(parts.sums(), parts)[inner] > 1).all()
    assert (off(parts.sums() + parts.anchor / parts.ahead, parts)[inner] > 1).all()
    long = [i for i, (a, b) in enumerate(parts.blocks) if b - a > 256]
    assert (off(parts.sums(256) + parts.anchor, parts)[long] > 1).all()


def test_wrong_sums_over_all_tokens_are_refused(parts):
    for wrong in (np.zeros_like(parts.dg), parts.sums(), parts.sums(256) + parts.anchor, parts.sums() + parts.anchor / parts.ahead):
        assert (head_off(wrong.sum(0), parts, SPANS) > 1).all()
    for a, b in parts.blocks:                                  # one block's share left out
        left = parts.dg.copy()
        left[a:b] = 0
        assert (head_off(left.sum(0), parts, SPANS) > 1).all() or b - a < 8


def test_two_bf16_terms_are_refused():
    """What a state or a score in two bf16 terms, in the place of three, is off: beyond every bound of tests/test_gpu_head_decay_rms.py."""
    x = torch.from_numpy(np.random.default_rng(9).standard_normal(1 << 16))

    def error(terms):
        left = x
        for _ in range(terms):
            left = left - left.bfloat16().double()
        return float((left.square().mean() / x.square().mean()).sqrt()) * 2 ** 24
    assert 40 < error(2) < 42 and error(3) < 0.2
