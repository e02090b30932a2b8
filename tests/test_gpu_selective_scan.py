"""The selective scan against its oracle in 64 bits: prompts, packed prompts, pieces, single tokens, gradients."""
import pytest
import torch

import paper_2407_12077_amd as wkv
from scan_util import BF16, CODE, F32, Scan

pytestmark = pytest.mark.gpu
PACKED = [17, 0, 1, 33, 16, 5]


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (BF16, F32), (F32, F32)], ids=["bf16", "bf16-f32", "f32"])
@pytest.mark.parametrize("N", [8, 16, 32, 64])
@pytest.mark.parametrize("rows", [dict(B=2, T=35), dict(lengths=PACKED, front=3, tail=2), dict(B=3, T=1)], ids=["whole", "packed", "single"])
def test_prompts(gpu_device, rows, N, dtype, out):
    s = Scan(1, D=72, N=N, dtype=dtype, fused=True, **rows)
    s.check_prefill(*s.prefill(out))


@pytest.mark.parametrize("D", [8, 64, 128, 136, 200])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_widths(gpu_device, D, dtype):
    s = Scan(2, D=D, N=16, dtype=dtype, lengths=[40, 3], longest=30)
    s.check_prefill(*s.prefill())
    s.check_backward(s.backward())


@pytest.mark.parametrize("off", ["gate", "skip", "bias", "softplus", "state"])
def test_without(gpu_device, off):
    s = Scan(3, D=64, N=16, dtype=F32, B=2, T=19, **{off: False})
    s.check_prefill(*s.prefill())
    s.check_backward(s.backward())


@pytest.mark.parametrize("N", [8, 16, 64])
@pytest.mark.parametrize("rows", [dict(B=1, T=700), dict(lengths=[520, 1, 256, 0, 255], front=1), dict(lengths=[130, 128], longest=1000)], ids=str)
def test_pieces(gpu_device, rows, N):
    s = Scan(4, D=72, N=N, dtype=F32, **rows)
    assert wkv.wkv6_selective_scan_workspace_bytes(s.B, s.T, s.D, N) > 0
    s.check_prefill(*s.prefill())
    s.check_backward(s.backward())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("N", [8, 16, 32, 64])
@pytest.mark.parametrize("rows", [dict(B=2, T=35), dict(lengths=PACKED, front=3, tail=2), dict(B=3, T=1)], ids=["whole", "packed", "single"])
def test_gradients(gpu_device, rows, N, dtype):
    s = Scan(5, D=72, N=N, dtype=dtype, fused=True, **rows)
    s.check_backward(s.backward())


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (BF16, F32), (F32, F32)], ids=["bf16", "bf16-f32", "f32"])
@pytest.mark.parametrize("N", [8, 16, 32, 64])
@pytest.mark.parametrize("B,D", [(1, 8), (3, 200), (5, 1000)])
def test_single_tokens(gpu_device, B, D, N, dtype, out):
    s = Scan(6, D=D, N=N, dtype=dtype, fused=B == 3, gate=B != 1, B=B, T=1)
    y = torch.empty((B, D), dtype=out, device="cuda")
    h = s.state_in.clone()
    wkv.wkv6_selective_scan_decode(B, D, N, *s.inputs(), h, y, h, CODE[dtype], CODE[out])       # in place
    s.check_prefill(y, h)


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (BF16, F32), (F32, F32)], ids=["bf16", "bf16-f32", "f32"])
@pytest.mark.parametrize("N", [8, 16, 32, 64])
@pytest.mark.parametrize("rows", [dict(B=3, T=2), dict(B=2, T=8), dict(lengths=[8, 0, 1, 5, 3, 4], front=3, tail=2), dict(lengths=[1, 0, 1], front=1),
                                  dict(lengths=[9, 20], longest=7)], ids=str)
def test_few_tokens(gpu_device, rows, N, dtype, out):
    s = Scan(12, D=200, N=N, dtype=dtype, fused=True, gate=N != 32, state=N != 16, **rows)
    s.check_prefill(*s.prefill(out))
    if s.state_in is not None:
        alone, want = s.prefill(out)
        s.state_in = s.state_in.clone()
        again, state = s.prefill(out, state_out=s.state_in)
        assert torch.equal(again, alone) and torch.equal(state, want)


def test_a_prompt_of_one_token_is_a_single_token(gpu_device):
    s = Scan(13, D=136, N=16, B=4, T=1)
    out, state = s.prefill()
    y, h = torch.empty_like(out), torch.empty_like(state)
    wkv.wkv6_selective_scan_decode(4, 136, 16, *s.inputs(), s.state_in, y, h, CODE[BF16], CODE[BF16])
    assert torch.equal(out, y) and torch.equal(state, h)


@pytest.mark.parametrize("T", [5, 19, 700])
def test_states_of_one_token(gpu_device, T):
    """a as low as fp32 goes: a state forgets everything, and the rows behind a sequence's end change nothing."""
    s = Scan(14, D=72, N=16, dtype=F32, lengths=[T, 3, 0])
    s.a[:, 1] = s.a[5] = -torch.finfo(F32).max
    s.check_prefill(*s.prefill())
    s.check_backward(s.backward())


def test_states_grow(gpu_device):
    s = Scan(7, D=64, N=16, dtype=F32, B=2, T=300, growing=True)
    s.check_prefill(*s.prefill())
    s.check_backward(s.backward())


@pytest.mark.parametrize("rows", [dict(B=2, T=0), dict(lengths=[0, 0], front=3, longest=5), dict(lengths=[0, 0], longest=0)], ids=str)
def test_no_tokens(gpu_device, rows):
    s = Scan(8, D=64, N=16, **rows)
    out, state = s.prefill()
    assert torch.equal(state, s.state_in) and bool((out == 77).all())
    g = s.backward()
    assert torch.equal(g["dstate_in"], s.dstate_out) and all(not g[n].any() for n in ("da", "dskip", "dbias"))


@pytest.mark.parametrize("T", [40, 700])
def test_state_in_place_and_not_wanted(gpu_device, T):
    s = Scan(9, D=64, N=16, B=1, T=T)
    out, state = s.prefill()
    alone, _ = s.prefill(state_out=None)
    s.state_in = s.state_in.clone()
    again, same = s.prefill(state_out=s.state_in)
    assert torch.equal(out, again) and torch.equal(state, same) and torch.equal(out, alone)


def test_cut_in_two(gpu_device):
    """A prompt in two calls, and its last token by decode: the whole prompt's, within the bounds."""
    s = Scan(10, D=72, N=16, dtype=F32, B=1, T=50)
    parts, state = [], s.state_in
    for first, end in ((0, 33), (33, 49), (49, 50)):
        p = Scan(10, D=72, N=16, dtype=F32, B=1, T=end - first)
        p.x, p.delta, p.z, p.b, p.c = (t[first:end].contiguous() for t in (s.x, s.delta, s.z, s.b, s.c))
        p.a, p.bias, p.skip, p.state_in = s.a, s.bias, s.skip, state
        if end - first > 1:
            out, state = p.prefill()
        else:
            out, new = torch.empty((1, 72), device="cuda"), torch.empty_like(state)
            wkv.wkv6_selective_scan_decode(1, 72, 16, *p.inputs(), state, out, new, CODE[F32], CODE[F32])
            state = new
        parts.append(out)
    s.check_prefill(torch.cat(parts), state)


def test_the_same_bits_and_weights_not_wanted(gpu_device):
    s = Scan(11, D=136, N=16, lengths=[90, 300, 7])
    first, second, frozen = s.backward(), s.backward(), s.backward(weights=False)
    for name, g in first.items():
        assert torch.equal(g, second[name]) and (frozen[name] is None or torch.equal(g, frozen[name])), name
