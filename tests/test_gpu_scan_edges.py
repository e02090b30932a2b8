"""Calls of the selective scan and the short convolution at the edges of what their headers allow, on the GPU."""
import numpy as np
import pytest
import torch

import paper_2407_12077_amd as wkv
from scan_util import BF16, CODE, F32, Conv, Scan, Workspace

pytestmark = pytest.mark.gpu
# offsets that fall, that lie outside the rows, and sequences longer than T; no two sequences overlap
ORDERS = [([2000, 3500, 3500, 0, 1500], 9000), ([2000, 3500, 3500, 0, 1500], 400), ([200, 0, 2500], 5000), ([100, 200, 0, 90], 200),
          ([-5, 30, 30, 900, 900, 5000], 2000), ([40, -7, 30, 30, 17], 64), ([600, 300, 500, 0, 200, 210, 211, 290], 300), ([20, 28, 5, 9, 9, 2, 4], 8)]


def in_any_order(cls, seed, offsets, longest, **sizes):
    """A call with these offsets, 1200 rows behind the largest one that there may be."""
    rows = max(o for o in offsets if o < 5000) + 1200
    x = cls(seed, lengths=[0] * (len(offsets) - 1), tail=rows, longest=longest, **sizes)
    x.offsets.copy_(torch.tensor(offsets, dtype=torch.int32))
    at = np.clip(offsets, 0, rows)
    x.spans = [(int(f), int(f + min(max(e - f, 0), longest))) for f, e in zip(at[:-1], at[1:])]
    for f, e in x.spans:
        assert not x.covered[f:e].any()
        x.covered[f:e] = True
    x.longest = max(e - f for f, e in x.spans)
    return x


@pytest.mark.parametrize("N", [8, 16, 32, 64])
@pytest.mark.parametrize("T", [1, 5, 19, 700])
def test_a_weight_that_is_no_number_shows(gpu_device, T, N):
    """A NaN in a[d][n] reaches channel d's read-outs and state n, its da and the gradients of its rows; other channels keep their bits."""
    s, d, n = Scan(1, D=72, N=N, lengths=[T, 3, 0]), 5, N - 1
    rows, others = slice(0, T + 3), [i for i in range(72) if i != d]
    clean_out, clean_state = s.prefill()
    clean = s.backward()
    s.a[d, n] = float("nan")
    out, state = s.prefill()
    assert bool(out[rows, d].isnan().all()) and torch.equal(out[:, others], clean_out[:, others])
    assert bool(state[:2, d, n].isnan().all())
    state[:2, d, n] = clean_state[:2, d, n]
    assert torch.equal(state, clean_state)                     # the sequence of no tokens among them
    g = s.backward()
    assert bool(g["da"][d, n].isnan()) and torch.equal(g["da"][others], clean["da"][others])
    assert bool(g["ddelta"][rows, d].isnan().all()) and bool(g["dbias"][d].isnan()) and bool(g["dstate_in"][:2, d, n].isnan().all())
    for name in ("dx", "ddelta", "dz"):
        assert torch.equal(g[name][:, others], clean[name][:, others])
    assert torch.equal(g["dstate_in"][2], clean["dstate_in"][2])


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("N", [8, 16, 32, 64])
def test_a_weight_that_is_no_number_shows_in_single_tokens(gpu_device, N, dtype):
    s = Scan(2, D=72, N=N, dtype=dtype, B=3, T=1)
    results = []
    for value in (None, float("nan")):
        if value is not None:
            s.a[7, 2] = value
        out, state = s.blank(72, dtype), torch.empty_like(s.state_in)
        wkv.wkv6_selective_scan_decode(3, 72, N, *s.inputs(), s.state_in, out, state, CODE[dtype], CODE[dtype])
        results.append((out, state))
    (clean_out, clean_state), (out, state) = results
    assert bool(out[:, 7].isnan().all()) and bool(state[:, 7, 2].isnan().all())
    out[:, 7], state[:, 7, 2] = clean_out[:, 7], clean_state[:, 7, 2]
    assert torch.equal(out, clean_out) and torch.equal(state, clean_state)


@pytest.mark.parametrize("N", [8, 16, 32, 64])
@pytest.mark.parametrize("rows", [dict(B=1, T=700), dict(lengths=[3, 700, 40], front=1)], ids=str)
@pytest.mark.parametrize("state", ["nought", "small"])
def test_a_piece_may_grow_more_than_fp32_holds(gpu_device, state, rows, N):
    """Every other state grows, over 32 tokens by more than fp32's largest number (exp(7) a token, or exp(2.9)), but from nought, or from 1e-25 to 1e16, and no gradient comes
    from there: whatever pieces the tokens are cut into, states and gradients are as token by token, within the bounds for growing states (scan_util)."""
    s = Scan(3, D=72, N=N, dtype=F32, softplus=False, bias=False, state=False, gate=True, **rows)
    s.scale = 4                                                # as for `growing`
    first, end = max(s.spans, key=lambda span: span[1] - span[0])
    s.a[:, ::2] = 0.70 + 0.04 * torch.rand(72, N // 2, device="cuda")
    grows = slice(first + 320, first + 352)
    s.delta[:] = 0.02
    s.delta[grows] = 10.0 if state == "nought" else 4.0
    if state == "nought":
        s.x[first:first + 352] = 0
    else:
        s.x *= 1e-25
    s.dout[first + 320:end] = 0
    s.check_prefill(*s.prefill())
    s.check_backward(s.backward())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("N", [8, 16, 64])
@pytest.mark.parametrize("offsets,longest", ORDERS, ids=str)
def test_sequences_in_any_order(gpu_device, offsets, longest, N, dtype):
    s = in_any_order(Scan, 4, offsets, longest, D=72, N=N, dtype=dtype, fused=N == 16)
    s.check_prefill(*s.prefill())
    g = s.backward()
    s.check_backward(g)
    for name, again in s.backward().items():
        assert torch.equal(g[name], again), name


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D,W", [(72, 4), (520, 2)])
@pytest.mark.parametrize("offsets,longest", ORDERS, ids=str)
def test_convolutions_in_any_order(gpu_device, offsets, longest, D, W, dtype):
    c = in_any_order(Conv, 5, offsets, longest, D=D, W=W, dtype=dtype, fused=D == 72)
    c.check_prefill(*c.prefill())
    g = c.backward()
    c.check_backward(g)
    for a, b in zip(g, c.backward()):
        assert torch.equal(a, b)


@pytest.mark.parametrize("T", [0, 9, 70000])
def test_weights_of_no_sequence(gpu_device, T):
    """No sequence, however long one may be: sums over nothing are nought, without a workspace."""
    D, rows, offsets = 72, 5, torch.zeros(1, dtype=torch.int32, device="cuda")
    t, dx = torch.full((rows, D), 7.0, dtype=BF16, device="cuda"), torch.full((rows, D), 7.0, dtype=BF16, device="cuda")
    w, dw, db = torch.ones(D, 4, device="cuda"), torch.full((D, 4), 7.0, device="cuda"), torch.full((D,), 7.0, device="cuda")
    assert wkv.wkv6_short_conv_backward_workspace_bytes(0, T, D, 4, rows) == 0 == wkv.wkv6_selective_scan_backward_workspace_bytes(0, T, D, 16, rows)
    wkv.wkv6_short_conv_backward(0, T, D, 4, rows, t, D, w, None, 1, offsets, None, t, None, dx, dw, db, None, CODE[BF16], None, 0)
    assert not dw.any() and not db.any() and bool((dx == 7).all())
    a, bc = -torch.ones(D, 16, device="cuda"), torch.ones(rows, 16, dtype=BF16, device="cuda")
    da, dskip, dbias = torch.full((D, 16), 7.0, device="cuda"), torch.full((D,), 7.0, device="cuda"), torch.full((D,), 7.0, device="cuda")
    dbc = bc.clone()
    wkv.wkv6_selective_scan_backward(0, T, D, 16, rows, t, D, t, D, None, 1, a, bc, bc, 16, None, None, 0, offsets, None, t, None, dx, dx, dbc, dbc, None, da, dskip, dbias, None,
                                     CODE[BF16], None, 0)
    assert not da.any() and not dskip.any() and not dbias.any() and bool((dx == 7).all()) and torch.equal(dbc, bc)


def test_a_state_that_is_no_number_passes_a_sequence_of_no_tokens(gpu_device):
    """It comes out as it is, its gradient is that of the state behind, and nothing else changes."""
    c = Conv(6, D=72, W=4, lengths=[3, 0, 40, 1], front=2)
    clean_out, clean_state = c.prefill()
    clean = c.backward()
    c.state_in[1, 1, 3], c.state_in[1, 2, 9] = float("nan"), float("inf")
    out, state = c.prefill()
    assert torch.equal(out, clean_out) and bool(state[1, 1, 3].isnan()) and bool(state[1, 2, 9].isinf())
    state[1, 1, 3], state[1, 2, 9] = clean_state[1, 1, 3], clean_state[1, 2, 9]
    assert torch.equal(state, clean_state)
    for got, want in zip(c.backward(), clean):
        assert torch.equal(got, want)


@pytest.mark.parametrize("longest", [60, 2000])
def test_a_captured_call_follows_its_offsets(gpu_device, longest):
    """One graph and one workspace, replayed with other offsets each time: every replay as a call of its own, whatever the one before has left in the workspace."""
    orders = [[0, 300, 620, 900, 901], [901, 40, 100, 0, 33], [100, 200, 200, 260, 700], [1500, -3, 5, 70, 2000], [0, 0, 0, 0, 0], [0, 300, 620, 900, 901]]
    s = in_any_order(Scan, 7, orders[0], longest, D=72, N=16)
    c = in_any_order(Conv, 8, orders[0], longest, D=72, W=4)
    s.offsets = c.offsets
    own = Workspace(wkv.wkv6_selective_scan_backward_workspace_bytes(s.B, s.T, s.D, s.N, s.rows))
    conv_own = Workspace(wkv.wkv6_short_conv_backward_workspace_bytes(c.B, c.T, c.D, c.W, c.rows))

    def calls(space, conv_space):
        dx = torch.full((c.rows, c.stride), 77.0, dtype=c.dtype, device="cuda")
        dw, db, ds = torch.zeros_like(c.w), torch.zeros_like(c.bias), torch.zeros_like(c.state_in)
        wkv.wkv6_short_conv_backward(c.B, c.T, c.D, c.W, c.rows, c.x, c.stride, c.w, c.bias, 1, c.offsets, c.state_in, c.dout, c.dstate_out, dx, dw, db, ds, CODE[c.dtype],
                                     conv_space, conv_own.n)
        return [*s.backward(workspace=space).values(), dx, dw, db, ds]
    calls(own, conv_own)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        kept = calls(own, conv_own)
    for offsets in orders:
        c.offsets.copy_(torch.tensor(offsets, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        want = calls(Workspace(own.n), Workspace(conv_own.n))
        for a, b in zip(kept, want):
            assert torch.equal(a, b), offsets
    own.check()
    conv_own.check()


@pytest.mark.parametrize("D", [136, 264, 384, 896, 1056, 2056])
def test_convolutions_of_widths_that_leave_lanes_idle(gpu_device, D):
    """As many threads side by side as there are groups of four channels, or half or a quarter as many, and some without one."""
    c = Conv(9, D=D, W=4, lengths=[70, 3, 0, 130], front=1, tail=2)
    c.check_prefill(*c.prefill())
    c.check_backward(c.backward())
