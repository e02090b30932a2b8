"""The selective scan over calls whose token axis is cut (tests/scan_pieces.py), against its oracle in 64 bits."""
import pytest
import torch

from scan_pieces import CUT, D, MANY, MANY_D, STATES
from scan_util import BF16, F32, Scan

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (BF16, F32), (F32, F32)], ids=["bf16", "bf16-f32", "f32"])
@pytest.mark.parametrize("N", STATES)
@pytest.mark.parametrize("rows", CUT, ids=str)
def test_pieces_of_strided_rows(gpu_device, rows, N, dtype, out):
    s = Scan(21, D=D, N=N, dtype=dtype, fused=True, gate=N != 16, state=N != 8, **rows)
    s.check_prefill(*s.prefill(out))
    s.check_backward(s.backward())


@pytest.mark.parametrize("softplus", [True, False])
def test_pieces_without_softplus_or_bias(gpu_device, softplus):
    s = Scan(22, D=D, N=32, softplus=softplus, bias=False, skip=False, B=1, T=700)
    s.check_prefill(*s.prefill())
    s.check_backward(s.backward())


@pytest.mark.parametrize("N,dtype", [(16, BF16), (8, F32)], ids=str)
def test_one_long_sequence_among_many(gpu_device, N, dtype):
    s = Scan(23, D=MANY_D, N=N, dtype=dtype, **MANY)
    s.check_prefill(*s.prefill())
    g = s.backward()
    s.check_backward(g)
    for name, again in s.backward().items():
        assert torch.equal(g[name], again), name
