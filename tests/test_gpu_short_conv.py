"""The short causal convolution against its oracle in 64 bits: prompts, packed prompts, single tokens, gradients."""
import pytest
import torch

import paper_2407_12077_amd as wkv
from scan_util import BF16, CODE, F32, Conv

pytestmark = pytest.mark.gpu
ROWS = [dict(B=2, T=35), dict(lengths=[17, 0, 1, 2, 3, 70, 4], front=3, tail=2), dict(B=3, T=1), dict(B=1, T=300), dict(lengths=[40, 3], longest=30)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("rows", ROWS, ids=str)
@pytest.mark.parametrize("D", [8, 72, 520])
def test_prompts_and_gradients(gpu_device, D, rows, W, dtype):
    c = Conv(1, D=D, W=W, dtype=dtype, fused=D != 8, **rows)
    c.check_prefill(*c.prefill())
    c.check_backward(c.backward())


@pytest.mark.parametrize("off", ["bias", "silu", "state"])
def test_without(gpu_device, off):
    c = Conv(2, D=64, W=4, lengths=[2, 30, 1], **{off: False})
    c.check_prefill(*c.prefill())
    c.check_backward(c.backward())


@pytest.mark.parametrize("D,T", [(2048, 2500), (8, 9000), (768, 1000)])
def test_long_runs(gpu_device, D, T):
    """Many workgroups, and runs of tokens as long as they get."""
    c = Conv(3, D=D, W=4, lengths=[T, 5, T // 3])
    c.check_prefill(*c.prefill())
    c.check_backward(c.backward())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("B,D", [(1, 8), (3, 200), (70, 520)])
def test_single_tokens(gpu_device, B, D, W, dtype):
    c = Conv(4, D=D, W=W, dtype=dtype, fused=B == 3, state=B != 70, B=B, T=1)
    out = torch.empty((B, D), dtype=dtype, device="cuda")
    state = c.state_in.clone() if B == 1 else torch.empty((B, W - 1, D), dtype=dtype, device="cuda")
    wkv.wkv6_short_conv_decode(B, D, W, c.x, c.stride, c.w, c.bias, 1, state if B == 1 else c.state_in, out, state, CODE[dtype])
    c.check_prefill(out, state)


def test_no_tokens(gpu_device):
    for rows in (dict(B=2, T=0), dict(lengths=[0, 0], front=2, longest=4)):
        c = Conv(5, D=64, W=4, **rows)
        out, state = c.prefill()
        assert torch.equal(state, c.state_in) and bool((out == 77).all())
        _, dw, db, ds = c.backward()
        assert torch.equal(ds, c.dstate_out) and not dw.any() and not db.any()


@pytest.mark.parametrize("T", [1, 2, 3, 200])
def test_state_in_place(gpu_device, T):
    c = Conv(6, D=128, W=4, B=2, T=T)
    out, state = c.prefill()
    alone, _ = c.prefill(state_out=None)
    c.state_in = c.state_in.clone()
    again, same = c.prefill(state_out=c.state_in)
    assert torch.equal(out, again) and torch.equal(state, same) and torch.equal(out, alone)


def test_the_same_bits_and_weights_not_wanted(gpu_device):
    c = Conv(7, D=200, W=3, lengths=[90, 300, 7])
    first, second, frozen = c.backward(), c.backward(), c.backward(weights=False)
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    assert torch.equal(first[0], frozen[0]) and torch.equal(first[3], frozen[3])


def test_nan_stays_under_its_taps(gpu_device):
    c = Conv(8, D=64, W=4, lengths=[50, 50])
    clean, _ = c.prefill()
    c.x[49, 3] = float("nan")
    out, _ = c.prefill()
    assert out[49, 3].isnan() and torch.equal(out[50:], clean[50:]) and torch.equal(out[:49], clean[:49])


@pytest.mark.parametrize("where", ["x", "dout"])
def test_nan_stays_under_its_taps_in_gradients(gpu_device, where):
    c = Conv(9, D=64, W=4, lengths=[300, 50])
    clean = c.backward()
    for row in (150, 299):
        c.x, c.dout = c.x.clone(), c.dout.clone()
        given = getattr(c, where)
        was = given[row, 3].clone()
        given[row, 3] = float("nan")
        dx, dw, dbias, ds = c.backward()
        given[row, 3] = was
        near = torch.zeros_like(dx, dtype=torch.bool)
        near[row - 3:min(row + 4, 300), 3] = True
        assert dx[row, 3].isnan() and dw[3].isnan().any() and dbias[3].isnan()
        assert torch.equal(dx[~near], clean[0][~near]) and torch.equal(ds, clean[3])
        assert torch.equal(dw[:3], clean[1][:3]) and torch.equal(dw[4:], clean[1][4:]) and not dbias[4:].isnan().any()


def test_many_short_sequences_where_long_ones_may_come(gpu_device):
    """A launch has places for the longest sequence that may come: threads take more tokens one behind the other, so that most have some."""
    c = Conv(10, D=16, W=4, lengths=[3, 1, 0, 7] * 511 + [3000, 2, 90, 1], front=1, tail=3, longest=65536)
    c.check_prefill(*c.prefill())
    c.check_backward(c.backward())
