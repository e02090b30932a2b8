"""LayerNorm over rows and its gradients against 64 bits (oracle/layernorm_rows_numpy.py), element by element.

Bounds.  A sum over a row's D values passes at most 40 roundings a term (eight values in three steps, up to eight pieces of a lane, six steps over a
wave, five over waves, and what the values themselves have been rounded), each half a step of fp32, 2^-24.  With A the mean of |x|:
mean is off by 40 A steps; x - mean by |x| + |mean| + 40 A; rstd by 48 of itself (a square doubles what its root halves) plus, where var is
small, rstd^2 times the square of the mean's error.  The gradients take the statistics as given.  A column's sum over M rows: M / 512 + 1 rows in a
lane's own sum, four waves, eight rows and six steps of the fold, and five roundings of each term."""
import numpy as np
import pytest
import torch

import paper_2407_12077_amd as wkv
from operator_util import CODE, check, np64
from oracle.layernorm_rows_numpy import layernorm_rows_gradients_numpy, layernorm_rows_numpy

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
PAIRS = [(BF16, BF16), (BF16, F32), (F32, BF16), (F32, F32)]
IDS = ["bf16_bf16", "bf16_f32", "f32_bf16", "f32_f32"]
STEP, EPS = 2.0 ** -24, 1e-5
WIDTHS = [8, 64, 72, 504, 512, 520, 768, 1000, 1024, 2048, 2056, 4096, 4104, 8192, 8200, 16384]


def inputs(seed, M, D, x_dtype, y_dtype, offset=0.5):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    x = (normal(M, D) * 1.5 + normal(M, 1) + offset).to(x_dtype)
    return x, torch.rand(D, generator=gen, device="cuda") + 0.5, normal(D) * 0.3, normal(M, D).to(y_dtype)


def forward(x, gamma, beta, y_dtype, y=None, stats=True):
    M, D = x.shape
    y = torch.full((M, D), 7.0, dtype=y_dtype, device="cuda") if y is None else y
    s = torch.full((M, 2), float("nan"), device="cuda") if stats else None
    wkv.wkv6_layernorm_forward(M, D, x, gamma, beta, EPS, y, s, CODE[x.dtype], CODE[y_dtype])
    return y, s


def gradients(x, stats, gamma, dy, dx=None, frozen=False):
    M, D = x.shape
    dx = torch.full((M, D), 7.0, dtype=x.dtype, device="cuda") if dx is None else dx
    if frozen:
        wkv.wkv6_layernorm_backward(M, D, x, stats, gamma, dy, dx, None, None, CODE[x.dtype], CODE[dy.dtype], None, 0)
        return dx
    dg, db = (torch.full((D,), float("nan"), device="cuda") for _ in range(2))
    n = wkv.wkv6_layernorm_backward_workspace_bytes(M, D)
    ws = torch.full((max(4, n // 4),), float("nan"), device="cuda")
    wkv.wkv6_layernorm_backward(M, D, x, stats, gamma, dy, dx, dg, db, CODE[x.dtype], CODE[dy.dtype], ws, n)
    return dx, dg, db


def check_forward(x, gamma, beta, y, stats):
    want, want_stats = layernorm_rows_numpy(np64(x), np64(gamma), np64(beta), EPS)
    v = np64(x)
    mean, rstd = want_stats[:, :1], want_stats[:, 1:]
    A = abs(v).mean(1, keepdims=True)
    d_mean = 40 * STEP * A
    d_rstd = rstd * (48 * STEP + (rstd * d_mean) ** 2)
    u = abs(v - mean) * rstd
    d_u = (STEP * (abs(v) + abs(mean)) + d_mean) * rstd + abs(v - mean) * d_rstd
    bound = (d_u + 4 * STEP * u) * abs(np64(gamma)) + STEP * (abs(want) + abs(np64(beta)))
    check("y", y, want, bound, None, y.dtype)
    check("mean", stats[:, :1], mean, d_mean + STEP * abs(mean))
    check("rstd", stats[:, 1:], rstd, d_rstd + STEP * rstd)


def check_gradients(x, stats, gamma, dy, dx, dg, db):
    want = layernorm_rows_gradients_numpy(np64(x), np64(stats), np64(gamma), np64(dy))
    v, d = np64(x), abs(np64(dy))
    mean, rstd = np64(stats)[:, :1], np64(stats)[:, 1:]
    u, a = abs(v - mean) * rstd, d * abs(np64(gamma))
    d_u = 3 * STEP * (abs(v) + abs(mean)) * rstd
    m1 = (a * u).mean(1, keepdims=True)
    d_m0 = 44 * STEP * a.mean(1, keepdims=True)
    d_m1 = 44 * STEP * m1 + (a * d_u).mean(1, keepdims=True)
    bound = rstd * (6 * STEP * (a + a.mean(1, keepdims=True) + u * m1) + d_m0 + u * d_m1 + d_u * m1)
    check("dx", dx, want[0], bound, None, x.dtype)
    n = STEP * (x.shape[0] / 512 + 24)
    check("dgamma", dg, want[1], n * (d * u).sum(0) + (d * d_u).sum(0))
    check("dbeta", db, want[2], n * d.sum(0))


@pytest.mark.parametrize("x_dtype,y_dtype", PAIRS, ids=IDS)
@pytest.mark.parametrize("D", WIDTHS)
def test_widths(gpu_device, D, x_dtype, y_dtype):
    """Seven rows, and so many that bf16 rows of up to 2048 columns are a wave's each."""
    for M in (7, 4099 if D in (1000, 2048) else 1030 if D <= 4096 else 600):
        x, gamma, beta, dy = inputs(D, M, D, x_dtype, y_dtype)
        y, stats = forward(x, gamma, beta, y_dtype)
        check_forward(x, gamma, beta, y, stats)
        check_gradients(x, stats, gamma, dy, *gradients(x, stats, gamma, dy))


@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 511, 513, 2047, 2049, 9001])
def test_rows(gpu_device, M):
    x, gamma, beta, dy = inputs(M, M, 136, BF16, BF16)
    y, stats = forward(x, gamma, beta, BF16)
    check_forward(x, gamma, beta, y, stats)
    check_gradients(x, stats, gamma, dy, *gradients(x, stats, gamma, dy))


def test_constant_rows_and_far_means(gpu_device):
    x, gamma, beta, dy = inputs(3, 6, 768, F32, F32)
    x[0] = 0.
    x[1] = 3.
    x[2] += 1000.
    x[3] *= 1e-6
    y, stats = forward(x, gamma, beta, F32)
    check_forward(x, gamma, beta, y, stats)
    assert torch.allclose(y[0], beta) and float(stats[0, 0]) == 0
    check_gradients(x, stats, gamma, dy, *gradients(x, stats, gamma, dy))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("M,D", [(3, 520), (1500, 2048), (5, 8200)])
def test_in_place_frozen_and_without_statistics(gpu_device, M, D, dtype):
    x, gamma, beta, dy = inputs(5, M, D, dtype, dtype)
    y, stats = forward(x, gamma, beta, dtype)
    assert torch.equal(forward(x, gamma, beta, dtype, stats=False)[0], y)
    copy = x.clone()
    assert torch.equal(forward(copy, gamma, beta, dtype, y=copy)[0], y)
    dx, dg, db = gradients(x, stats, gamma, dy)
    assert torch.equal(gradients(x, stats, gamma, dy, frozen=True), dx)
    for alias in (0, 1):                                       # dx in the place of x, of dy
        a, b = x.clone(), dy.clone()
        got = gradients(a, stats, gamma, b, dx=b if alias else a)
        assert torch.equal(got[0], dx) and torch.equal(got[1], dg) and torch.equal(got[2], db)


def test_no_rows(gpu_device):
    x, gamma, beta, dy = inputs(6, 0, 64, BF16, BF16)
    forward(x, gamma, beta, BF16)
    _, dg, db = gradients(x, torch.empty((0, 2), device="cuda"), gamma, dy)
    assert bool((dg == 0).all()) and bool((db == 0).all())


def test_rows_past_four_gigabytes(gpu_device):
    M, D = 300_000, 8192
    x = torch.zeros((M, D), dtype=BF16, device="cuda")
    few, gamma, beta, dy = inputs(9, 600, D, BF16, BF16)
    x[-600:] = few
    y, stats = forward(x, gamma, beta, BF16)
    want, want_stats = forward(few, gamma, beta, BF16)
    assert torch.equal(y[-600:], want) and torch.equal(stats[-600:], want_stats)
    y.zero_()
    y[-600:] = dy                                              # a gradient of nought for the rows before
    got = gradients(x, stats, gamma, y)
    want = gradients(few, want_stats, gamma, dy)
    assert torch.equal(got[0][-600:], want[0]) and not bool(got[0][:-600].any())
    # other shares of the columns' sums: 24 roundings of each term more
    u = (few.float() - want_stats[:, :1]) * want_stats[:, 1:]
    assert bool(((got[1] - want[1]).abs() <= 64 * STEP * (dy.float() * u).abs().sum(0)).all())
    assert bool(((got[2] - want[2]).abs() <= 64 * STEP * dy.float().abs().sum(0)).all())


def test_gradients_against_differences(gpu_device):
    x, gamma, beta, dy = inputs(7, 9, 200, F32, F32)
    _, stats = forward(x, gamma, beta, F32)
    got = [np64(a) for a in gradients(x, stats, gamma, dy)]
    args = [np64(a) for a in (x, gamma, beta)]
    rng = np.random.default_rng(0)
    for i, grad in enumerate(got):
        step = rng.standard_normal(grad.shape)
        ends = [(layernorm_rows_numpy(*[a + s * step if j == i else a for j, a in enumerate(args)], EPS)[0] * np64(dy)).sum() for s in (1e-5, -1e-5)]
        # 100 roundings of every term, which covers the statistics' own, and the differences' error of second order
        assert abs((grad * step).sum() - (ends[0] - ends[1]) / 2e-5) <= (100 * STEP + 1e-6) * abs(grad * step).sum() + 1e-6


def test_captured_with_eager_work_between(gpu_device):
    x, gamma, beta, dy = inputs(8, 700, 1024, BF16, BF16)
    y, stats = forward(x, gamma, beta, BF16)
    want = gradients(x, stats, gamma, dy)
    n = wkv.wkv6_layernorm_backward_workspace_bytes(700, 1024)
    ws = torch.empty((n // 4,), device="cuda")
    y2, s2, dx, dg, db = torch.empty_like(y), torch.empty_like(stats), torch.empty_like(want[0]), torch.empty_like(gamma), torch.empty_like(gamma)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        wkv.wkv6_layernorm_forward(700, 1024, x, gamma, beta, EPS, y2, s2, CODE[BF16], CODE[BF16])
        wkv.wkv6_layernorm_backward(700, 1024, x, s2, gamma, dy, dx, dg, db, CODE[BF16], CODE[BF16], ws, n)
    for replay in range(3):
        for t in (y2, s2, dx, dg, db, ws):
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((y2, s2, dx, dg, db), (y, stats, *want)):
            assert torch.equal(a, b), replay
