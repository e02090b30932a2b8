"""A layer as a training program runs it: the head-decay time mix over packed sequences, the LayerNorm over all heads of its read-outs, and both
gradients back to r, k, v, the decays and the norm's weights; then the same layer serving, a prompt and single tokens behind it."""
import numpy as np
import pytest
import torch

import paper_2407_12077_amd as wkv
from operator_util import CODE, N, Mix, check, np64, roundings
from oracle.head_decay_numpy import head_decay_gradients_numpy, head_decay_numpy
from oracle.layernorm_rows_numpy import layernorm_rows_gradients_numpy, layernorm_rows_numpy

pytestmark = pytest.mark.gpu
EPS = 1e-5


def norm(o, gamma, beta, dtype):
    M, D = o.shape[0], o.shape[1] * N
    y, stats = torch.empty((M, D), dtype=dtype, device="cuda"), torch.empty((M, 2), device="cuda")
    wkv.wkv6_layernorm_forward(M, D, o, gamma, beta, EPS, y, stats, CODE[o.dtype], CODE[dtype])
    return y, stats


def norm_backward(o, stats, gamma, dy):
    M, D = o.shape[0], o.shape[1] * N
    do, dg, db = torch.empty_like(o), torch.empty_like(gamma), torch.empty_like(gamma)
    n = wkv.wkv6_layernorm_backward_workspace_bytes(M, D)
    wkv.wkv6_layernorm_backward(M, D, o, stats, gamma, dy, do, dg, db, CODE[o.dtype], CODE[dy.dtype], torch.empty(n // 4, device="cuda"), n)
    return do, dg, db


def test_gradients_of_a_layer_against_differences(gpu_device):
    """fp32 rows; the loss, and its change along a direction, in 64 bits from the inputs alone.  The gradients' roundings: those of the mix
    (operator_util), and of the norm's, 100 steps of every term, both ways: 1e-4 of the sum of all terms' magnitudes is twice their sum."""
    x = Mix(1, H=3, lengths=[60, 17, 1, 35], dtype=torch.float32, fused=True, gradients=True)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(9)
    gamma, beta = torch.rand(3 * N, generator=gen, device="cuda") + 0.5, torch.randn(3 * N, generator=gen, device="cuda")
    dy = torch.randn((x.rows, 3 * N), generator=gen, device="cuda")
    out, _ = x.prefill()
    _, stats = norm(out, gamma, beta, torch.float32)
    x.dout, dgamma, dbeta = norm_backward(out, stats, gamma, dy)
    x.dstate_out = None
    grads = dict(zip(("r", "k", "v", "g", "state_in", "gamma", "beta"), [np64(a) for a in (*x.backward(), dgamma, dbeta)]))
    base = dict(r=np64(x.r), k=np64(x.k), v=np64(x.v), g=np64(x.g), state_in=np64(x.state_in), gamma=np64(gamma), beta=np64(beta))

    def loss(p):
        o, _ = head_decay_numpy(p["r"], p["k"], p["v"], p["g"], x.spans, p["state_in"])
        return (layernorm_rows_numpy(o.reshape(x.rows, -1), p["gamma"], p["beta"], EPS)[0] * np64(dy)).sum()
    rng = np.random.default_rng(2)
    for name, grad in grads.items():
        step = rng.standard_normal(grad.shape)
        diff = (loss({**base, name: base[name] + 1e-6 * step}) - loss({**base, name: base[name] - 1e-6 * step})) / 2e-6
        assert abs((grad * step).sum() - diff) <= 1e-4 * abs(grad * step).sum(), (name, (grad * step).sum(), diff)


def test_bf16_layer_step_by_step(gpu_device):
    """Every call in 64 bits from what the call before it handed over."""
    x = Mix(2, H=4, lengths=[130, 64, 0, 9, 300], fused=True, gradients=True)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    gamma, beta = torch.rand(4 * N, generator=gen, device="cuda") + 0.5, torch.randn(4 * N, generator=gen, device="cuda")
    out, _ = x.prefill(torch.bfloat16)
    y, stats = norm(out, gamma, beta, torch.bfloat16)
    dy = torch.randn(y.shape, generator=gen, device="cuda").to(torch.bfloat16)
    do, dgamma, dbeta = norm_backward(out, stats, gamma, dy)
    x.dout = do
    got = x.backward()
    flat = np64(out).reshape(x.rows, -1)
    want_y, want_stats = layernorm_rows_numpy(flat, np64(gamma), np64(beta), EPS)
    want_d = layernorm_rows_gradients_numpy(flat, np64(stats), np64(gamma), np64(dy))
    spread = 2.0 ** -18 * (1 + abs(flat).max() * want_stats[:, 1:])       # 64 steps of fp32 about values of this size
    check("y", y, want_y, spread * (1 + abs(want_y)), None, torch.bfloat16)
    check("do", do.view(x.rows, -1), want_d[0], spread * (1 + abs(want_d[0])) * want_stats[:, 1:], None, torch.bfloat16)
    check("dgamma", dgamma, want_d[1], 2.0 ** -18 * abs(want_d[1]).max() * np.ones_like(want_d[1]))
    check("dbeta", dbeta, want_d[2], 2.0 ** -18 * abs(np64(dy)).sum(0))
    want = head_decay_gradients_numpy(*x.arrays(), x.spans, np64(do), np64(x.state_in), np64(x.dstate_out))
    for name, a, w, b in zip(("dr", "dk", "dv", "dg"), got, want, x.gradient_bounds()):
        check(name, a, w, b, x.covered, torch.bfloat16 if name != "dg" else torch.float32)


def test_a_prompt_and_single_tokens_served_from_graphs(gpu_device):
    """The prompt eagerly, then steps of decode and norm in one captured graph, replayed token by token: as a longer prompt."""
    B, H, T, more = 3, 2, 70, 4
    x = Mix(4, H=H, B=B, T=T + more, dtype=torch.float32)
    gamma, beta = torch.ones(H * N, device="cuda"), torch.zeros(H * N, device="cuda")
    whole, _ = x.prefill()
    want, _ = norm(whole, gamma, beta, torch.float32)
    rows = lambda t, a, b: t.view(B, T + more, *t.shape[1:])[:, a:b].reshape(B * (b - a), *t.shape[1:]).contiguous()  # noqa: E731
    y = Mix(4, H=H, B=B, T=T, dtype=torch.float32)
    y.r, y.k, y.v, y.g = (rows(t, 0, T) for t in (x.r, x.k, x.v, x.g))
    y.state_in = x.state_in
    _, state = y.prefill()
    r, k, v, g = (rows(t, T, T + 1) for t in (x.r, x.k, x.v, x.g))
    o, z, stats = torch.empty((B, H, N), device="cuda"), torch.empty((B, H * N), device="cuda"), torch.empty((B, 2), device="cuda")

    def step():
        wkv.wkv6_head_decay_decode(B, H, N, r, k, v, H * N, g, H, state, o, state, CODE[torch.float32], CODE[torch.float32])
        wkv.wkv6_layernorm_forward(B, H * N, o, gamma, beta, EPS, z, stats, CODE[torch.float32], CODE[torch.float32])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        step()
    m, _ = x.magnitudes()
    for t in range(T, T + more):
        for dst, src in zip((r, k, v, g), (x.r, x.k, x.v, x.g)):
            dst.copy_(rows(src, t, t + 1))
        graph.replay()
        torch.cuda.synchronize()
        at = torch.arange(B) * (T + more) + t
        check("out", o, np64(whole)[at], 2 * 2.0 ** -24 * roundings(T + more) * m[at])
        # the norm's rows follow: what the read-outs may differ by, times rstd, to first order (every value may differ)
        off = 2 * 2.0 ** -24 * roundings(T + more) * m[at].reshape(B, -1)
        slack = np64(stats)[:, 1:] * (off + off.mean(1, keepdims=True)) * 4 + 1e-5
        check("normed", z, np64(want)[at], slack * (1 + abs(np64(want)[at])))
