"""The operators write nothing behind the workspace that their functions ask for: a guard behind exactly that many bytes stays as it was, and the results are those with
a workspace to spare."""
import pytest
import torch

import paper_2407_12077_amd as wkv
from operator_util import CODE, N, Mix

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
GUARD = 1 << 16


class Guarded:
    """Stands for a workspace of `n` bytes in a call; nothing in it has to be set."""

    def __init__(self, n):
        assert n >= 0 and n % 4 == 0
        self.all = torch.full((n // 4 + GUARD,), float("nan"), device="cuda")
        self.all[n // 4:] = 7.0
        self.n = n

    def data_ptr(self):
        return self.all.data_ptr()

    def numel(self):
        return self.n // 4

    def check(self):
        assert bool((self.all[self.n // 4:] == 7).all())


CASES = [dict(B=1, T=1500, H=2), dict(B=2, T=200, H=3), dict(lengths=[2100, 0, 64, 700, 1], H=1), dict(lengths=[2100, 0, 64, 700, 1], H=1, longest=9000),
         dict(B=130, T=70, H=2), dict(lengths=[300] * 40 + [1, 0, 2000], H=7)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("decay", ["token", "head"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_mix(gpu_device, case, decay, dtype):
    x = Mix(1, dtype=dtype, decay=decay, gradients=True, **case)
    want = (*x.prefill(), *x.backward())
    first = Guarded(wkv.wkv6_head_decay_workspace_bytes(x.B, x.T, x.H, N))
    second = Guarded(wkv.wkv6_head_decay_backward_workspace_bytes(x.B, x.T, x.H, N, x.rows))
    got = (*x.prefill(workspace=first), *x.backward(workspace=second))
    first.check()
    second.check()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("M,D", [(1, 8), (3, 520), (1531, 768), (5000, 2048), (700, 8200), (2, 16384)])
def test_norm(gpu_device, M, D, dtype):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(M)
    x, dy = (torch.randn((M, D), generator=gen, device="cuda").to(dtype) for _ in range(2))
    stats = torch.rand((M, 2), generator=gen, device="cuda")
    gamma = torch.rand(D, generator=gen, device="cuda")
    n = wkv.wkv6_layernorm_backward_workspace_bytes(M, D)
    res = []
    for space in (torch.empty(n // 4 + GUARD, device="cuda"), Guarded(n)):
        dx, dg, db = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(gamma)
        wkv.wkv6_layernorm_backward(M, D, x, stats, gamma, dy, dx, dg, db, CODE[dtype], CODE[dtype], space, n)
        res.append((dx, dg, db))
    space.check()
    for a, b in zip(*res):
        assert torch.equal(a, b)
