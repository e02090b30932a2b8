"""Calls of the head-decay time mix at the edges of what its header allows, on the GPU."""
import pytest
import torch

import paper_2407_12077_amd as wkv
from operator_util import CODE, N

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("B,T,rows,packed", [(0, 0, 0, False), (0, 9, 0, False), (0, 9, 4, True), (2, 0, 0, False), (2, 9, 0, True)])
def test_gradient_of_a_head_s_decay_without_tokens(gpu_device, B, T, rows, packed):
    H = 5
    t = torch.full((max(rows, 1), H, N), 7.0, dtype=BF16, device="cuda")
    dr, dk, dv = (torch.full_like(t, 7.0) for _ in range(3))
    g, dg = torch.zeros(H, device="cuda"), torch.full((H + 1,), 7.0, device="cuda")
    n = wkv.wkv6_head_decay_backward_workspace_bytes(B, T, H, N, rows)
    ws = torch.empty(max(16, n), dtype=torch.uint8, device="cuda")
    offsets = torch.zeros(B + 1, dtype=torch.int32, device="cuda") if packed else None
    wkv.wkv6_head_decay_backward(B, T, H, N, rows, t, t, t, H * N, g, 0, offsets, None, t, None, dr, dk, dv, dg, None, CODE[BF16], ws, n)
    assert bool((dg[:H] == 0).all()) and float(dg[H]) == 7 and all(bool((a == 7).all()) for a in (dr, dk, dv))
