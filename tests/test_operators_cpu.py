"""The head-decay time mix and the LayerNorm with gradients on the CPU: refusals (before anything is launched), sizes of workspaces,
which kernels a call launches (tests/launch_util.py), the headers, the binding, and the oracles' pins."""
import ctypes
import inspect
import os
import re
import subprocess

import numpy as np
import pytest

import launch_util as lu
import paper_2407_12077_amd as wkv
from oracle.head_decay_numpy import head_decay_gradients_numpy, head_decay_numpy
from oracle.layernorm_rows_numpy import layernorm_rows_gradients_numpy, layernorm_rows_numpy
from paper_2407_12077_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADERS = ("wkv6_head_decay.h", "wkv6_layernorm.h")
OK, NULL, SHAPE, UNSUPPORTED, LAUNCH, ALIGN, WORKSPACE = range(7)
BF16, F32 = 0, 1
P = ctypes.c_void_p
A = P(0x1000)                  # aligned, never dereferenced
BIG = 1 << 40


def _raw(name):
    return getattr(binding.load(), name)


# ---------------------------------------------------------------------------------------------- headers and binding
def test_every_declared_function_is_exported_and_bound():
    text = "".join(open(os.path.join(ROOT, "include", h)).read() for h in HEADERS)
    names = set(re.findall(r"\b(wkv6_[a-z0-9_]+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S)))
    assert names == set(binding.OPERATOR_EXPORTS)
    for name in names:
        fn = getattr(wkv, name)
        params = [p for p in inspect.signature(fn).parameters]
        assert len(params) == len(_raw(name).argtypes), name
        assert name.endswith("_bytes") or params[-1] == "stream", name


@pytest.mark.parametrize("header", HEADERS)
def test_headers_are_plain_c(header):
    src = f'#include "{header}"\nint main(void) {{ return 0; }}\n'
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Wextra", "-pedantic", "-Werror", "-fsyntax-only", "-I", os.path.join(ROOT, "include"), "-x", "c", "-"],
                   input=src, text=True, check=True)


class Address:
    def data_ptr(self):
        return 0x1000


def test_binding_refuses_fractions_and_reports_statuses():
    a = Address()
    with pytest.raises(TypeError):
        wkv.wkv6_head_decay_decode(0, 2, 64, a, a, a, 128.5, a, 2, a, a, a, BF16, BF16, stream=0)
    with pytest.raises(TypeError):
        wkv.wkv6_layernorm_forward(0.5, 64, a, a, a, 1e-5, a, a, BF16, BF16, stream=0)
    wkv.wkv6_head_decay_decode(0, 2, 64, a, a, a, 128, a, 2, a, a, a, BF16, BF16, stream=0)           # no sequence: nothing to launch
    with pytest.raises(wkv.Wkv6Error) as e:
        wkv.wkv6_layernorm_forward(1, 60, a, a, a, 1e-5, a, a, BF16, BF16, stream=0)
    assert e.value.status == UNSUPPORTED


# ---------------------------------------------------------------------------------------------- refusals
def prefill(**over):
    p = dict(B=2, T=8, H=2, N=64, rows=16, r=A, k=A, v=A, token_stride=128, g=A, g_stride=2, offsets=None, state_in=None, out=A, state_out=A,
             dtype=BF16, out_dtype=BF16, workspace=A, workspace_bytes=BIG, stream=None)
    assert not set(over) - set(p)
    return _raw("wkv6_head_decay_prefill")(*{**p, **over}.values())


def decode(**over):
    p = dict(B=2, H=2, N=64, r=A, k=A, v=A, token_stride=128, g=A, g_stride=2, state_in=A, out=A, state_out=A, dtype=BF16, out_dtype=BF16, stream=None)
    assert not set(over) - set(p)
    return _raw("wkv6_head_decay_decode")(*{**p, **over}.values())


def backward(**over):
    p = dict(B=2, T=8, H=2, N=64, rows=16, r=A, k=A, v=A, token_stride=128, g=A, g_stride=2, offsets=None, state_in=None, dout=A, dstate_out=None,
             dr=A, dk=A, dv=A, dg=A, dstate_in=None, dtype=BF16, workspace=A, workspace_bytes=BIG, stream=None)
    assert not set(over) - set(p)
    return _raw("wkv6_head_decay_backward")(*{**p, **over}.values())


@pytest.mark.parametrize("call", [prefill, decode, backward], ids=["prefill", "decode", "backward"])
def test_mix_refuses_wrong_sizes_types_and_strides(call):
    assert call(N=32) == UNSUPPORTED
    assert call(dtype=2) == UNSUPPORTED
    assert call(H=0) == SHAPE and call(H=65537) == SHAPE and call(B=-1) == SHAPE
    assert call(token_stride=127) == SHAPE                     # less than a row
    assert call(token_stride=132) == ALIGN                     # rows not a multiple of 16 bytes
    assert call(token_stride=(1 << 22) + 8) == SHAPE
    assert call(g_stride=1) == SHAPE and call(g_stride=-2) == SHAPE
    for name in ("r", "k", "v"):
        assert call(**{name: None}) == NULL
        assert call(**{name: P(0x1008)}) == ALIGN
    assert call(g=None) == NULL and call(g=P(0x1002)) == ALIGN
    assert call(state_in=P(0x1008)) == ALIGN
    assert call(B=0, **({} if call is decode else {"rows": 0})) == OK


def test_prefill_refuses():
    assert prefill(dtype=F32, out_dtype=BF16) == UNSUPPORTED and prefill(out_dtype=7) == UNSUPPORTED
    assert prefill(T=-1) == SHAPE and prefill(rows=15) == SHAPE and prefill(rows=-1, offsets=A) == SHAPE
    assert prefill(rows=1 << 31, offsets=A) == SHAPE
    assert prefill(T=(1 << 30) + 1, offsets=A) == SHAPE and backward(T=(1 << 30) + 1, offsets=A) == SHAPE
    assert prefill(out=None) == NULL and prefill(out=P(0x1004)) == ALIGN and prefill(state_out=P(0x1004)) == ALIGN
    assert prefill(offsets=P(0x1001)) == ALIGN
    assert prefill(B=1 << 20, T=0, H=64, rows=0) == SHAPE      # more workgroups than a launch has
    need = wkv.wkv6_head_decay_workspace_bytes(1, 4096, 32, 64)
    assert need > 0
    long = dict(B=1, T=4096, H=32, rows=4096, token_stride=2048, g_stride=32)
    assert prefill(**long, workspace=None) == NULL and prefill(**long, workspace=P(0x1008)) == ALIGN
    assert prefill(**long, workspace_bytes=16) == WORKSPACE


def test_decode_refuses():
    assert decode(dtype=F32, out_dtype=BF16) == UNSUPPORTED
    assert decode(out=None) == NULL and decode(out=P(0x1004)) == ALIGN and decode(state_out=P(0x1004)) == ALIGN
    assert decode(B=1 << 20, H=64, token_stride=4096, g_stride=64) == SHAPE


def test_backward_refuses():
    for name in ("dout", "dr", "dk", "dv", "dg"):
        assert backward(**{name: None}) == NULL
        assert backward(**{name: P(0x1002)}) == ALIGN
    assert backward(dstate_out=P(0x1004)) == ALIGN and backward(dstate_in=P(0x1004)) == ALIGN
    assert backward(workspace=None) == NULL
    need = wkv.wkv6_head_decay_backward_workspace_bytes(2, 8, 2, 64, 16)
    assert need > 0 and backward(workspace_bytes=need // 8) == WORKSPACE
    assert backward(rows=17) == SHAPE


def test_layernorm_refuses():
    f = _raw("wkv6_layernorm_forward")
    assert f(4, 64, A, A, A, 1e-5, A, A, 2, BF16, None) == UNSUPPORTED
    for D in (0, 4, 12, 16392):
        assert f(4, D, A, A, A, 1e-5, A, A, BF16, BF16, None) == UNSUPPORTED
    assert f(-1, 64, A, A, A, 1e-5, A, A, BF16, BF16, None) == SHAPE and f(1 << 24, 64, A, A, A, 1e-5, A, A, BF16, BF16, None) == SHAPE
    assert f(4, 64, A, A, A, -1e-5, A, A, BF16, BF16, None) == SHAPE and f(4, 64, A, A, A, float("nan"), A, A, BF16, BF16, None) == SHAPE
    for i in (2, 3, 4, 6):
        args = [4, 64, A, A, A, 1e-5, A, A, BF16, BF16, None]
        args[i] = None
        assert f(*args) == NULL
        args[i] = P(0x1008)
        assert f(*args) == ALIGN
    assert f(0, 64, None, None, None, 1e-5, None, None, BF16, BF16, None) == OK
    g = _raw("wkv6_layernorm_backward")
    base = [4, 64, A, A, A, A, A, A, A, BF16, BF16, A, BIG, None]
    for i in (2, 3, 4, 5, 6, 7, 8):                            # one of dgamma, dbeta alone too
        args = list(base)
        args[i] = None
        assert g(*args) == NULL
        args[i] = P(0x1008)
        assert g(*args) == ALIGN
    assert g(*base[:11], None, 0, None) == NULL and g(*base[:11], A, 16, None) == WORKSPACE
    assert g(0, 64, None, None, None, None, None, None, None, BF16, BF16, None, 0, None) == OK


# ---------------------------------------------------------------------------------------------- workspaces
def test_workspace_sizes():
    mix, back, norm = wkv.wkv6_head_decay_workspace_bytes, wkv.wkv6_head_decay_backward_workspace_bytes, wkv.wkv6_layernorm_backward_workspace_bytes
    assert mix(8, 4096, 32, 64) == 0                           # 256 units fill the compute units: one walk each
    assert mix(0, 10, 4, 64) == 0 and mix(1, 0, 4, 64) == 0 and mix(1, 1, 1, 64) == 0
    for bad in ((1, 8, 2, 32), (-1, 8, 2, 64), (1, -8, 2, 64), (1, 8, 0, 64), (1 << 20, 8, 64, 64), (1, (1 << 30) + 1, 2, 64)):
        assert mix(*bad) == -1 and back(*bad, 8) == -1
    assert back(1, 8, 2, 64, -1) == -1
    # anchors of both directions, two sums a row and head, partial sums of a head
    assert back(8, 4096, 32, 64, 32768) == 4 * (2 * 256 * 4 * 4096 + 2 * 32 * 32768 + 8 * 4 * 32)
    assert norm(0, 64) == 0 and norm(1, 64) == 512 and norm(32768, 2048) == 512 * 2 * 2048 * 4
    assert norm(4, 12) == -1 and norm(-1, 64) == -1


# ---------------------------------------------------------------------------------------------- launches
@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return lu.build_fake(tmp_path_factory.mktemp("fake_hip"))


def mix_call(B, T, H, dtype=BF16, out=BF16, packed=False):
    return ("wkv6_head_decay_prefill", [B, T, H, 64, B * T, lu.at(0), lu.at(1), lu.at(2), H * 64, lu.at(3), H, lu.at(4) if packed else None, lu.at(5),
                                        lu.at(6), lu.at(7), dtype, out, lu.at(8), BIG, None])


def back_call(B, T, H, dtype=BF16, g_stride=None):
    return ("wkv6_head_decay_backward", [B, T, H, 64, B * T, lu.at(0), lu.at(1), lu.at(2), H * 64, lu.at(3), H if g_stride is None else g_stride, None,
                                         lu.at(4), lu.at(5), lu.at(6), lu.at(7), lu.at(8), lu.at(9), lu.at(10), lu.at(11), dtype, lu.at(12), BIG, None])


def test_launches_of_the_mix(fake):
    """Pieces only where compute units would idle; the gradients are three walks in one launch, and dg."""
    calls = [mix_call(8, 4096, 32), mix_call(1, 4096, 32), mix_call(1, 200, 32), mix_call(1, 200, 32, F32, F32), mix_call(5, 1, 1),
             back_call(8, 4096, 32), back_call(1, 4096, 32), back_call(2, 3, 1, g_stride=0), back_call(2, 0, 3, g_stride=0)]
    got = [[e for e in ev if e.kind == "launch"] for ev in lu.events(fake, calls)]
    assert [[e.base for e in ev] for ev in got] == [
        ["mix_kernel"], ["mix_kernel"] * 2, ["mix_kernel"], ["mix_kernel"] * 2, ["mix_kernel"], ["mix_kernel", "decay_gradient_kernel"],
        ["mix_kernel"] * 2 + ["decay_gradient_kernel"], ["mix_kernel", "decay_gradient_kernel", "head_sums_kernel"],
        ["mix_kernel", "head_sums_kernel"]]
    assert [ev[-1].grid[0] for ev in got[:3]] == [256, 256, 32]
    assert got[5][0].grid[0] == 3 * 256 and all(e.bytes <= 160 * 1024 for ev in got for e in ev)


def test_workspace_holds_whatever_the_lengths_are(fake):
    """A packed call is cut by its rows too, which the prefill's workspace function does not know."""
    rng = np.random.default_rng(5)
    calls = []
    for _ in range(60):
        B, H, T = int(rng.integers(1, 40)), int(rng.integers(1, 20)), int(2 ** rng.uniform(0, 14))
        rows, dtype = int(rng.integers(0, B * T + 100)), int(rng.integers(0, 2))
        for n in (rows, T):
            name, args = mix_call(B, T, H, dtype, dtype, packed=True)
            args[4], args[-2] = n, wkv.wkv6_head_decay_workspace_bytes(B, T, H, 64)
            calls.append((name, args))
            name, args = back_call(B, T, H, dtype)
            args[4], args[11], args[-2] = n, lu.at(13), wkv.wkv6_head_decay_backward_workspace_bytes(B, T, H, 64, n)
            calls.append((name, args))
    for ev in lu.events(fake, calls):
        assert [e for e in ev if e.kind == "launch"]


def test_first_call_raises_every_limit(fake):
    for first in (mix_call(1, 5, 1), back_call(1, 5, 1, F32)):
        calls = [first, mix_call(8, 300, 32), mix_call(1, 4096, 32, BF16, F32), mix_call(1, 4096, 32, F32, F32), back_call(1, 4096, 32), back_call(1, 4096, 32, F32)]
        per_call = lu.events(fake, calls)
        limit = {e.kernel: e.bytes for e in per_call[0] if e.kind == "attribute"}
        for ev in per_call[1:]:
            assert not [e for e in ev if e.kind == "attribute"]
            for e in ev:
                assert e.bytes <= max(65536, limit.get(e.kernel, 0)), e.kernel


@pytest.mark.parametrize("M,D,lanes", [(1, 64, 64), (3, 1024, 64), (4095, 1032, 256), (4096, 2048, 64), (4096, 2056, 256), (3, 16384, 256)])
def test_lanes_of_a_norm_row(fake, M, D, lanes):
    ev = lu.events(fake, [("wkv6_layernorm_forward", [M, D, lu.at(0), lu.at(1), lu.at(2), 1e-5, lu.at(3), None, BF16, BF16, None])])[0]
    assert [e.base for e in ev] == ["norm_kernel"] and f", {lanes}, " in ev[0].kernel.replace("(int)", "")
    assert ev[0].grid[0] == (M if lanes == 256 else (M + 3) // 4)


@pytest.mark.parametrize("M,D,dtype,lanes", [(1, 64, BF16, 64), (4096, 2048, BF16, 64), (4095, 2048, BF16, 256), (4096, 2048, F32, 256), (3, 1024, F32, 64),
                                             (5000, 8192, BF16, 256), (5000, 8200, BF16, 512)])
def test_lanes_of_a_norm_row_s_gradients(fake, M, D, dtype, lanes):
    call = ("wkv6_layernorm_backward", [M, D] + [lu.at(i) for i in range(7)] + [dtype, dtype, lu.at(8), BIG, None])
    frozen = ("wkv6_layernorm_backward", [M, D] + [lu.at(i) for i in range(5)] + [None, None, dtype, dtype, None, 0, None])
    ev, without = ([e for e in x if e.kind == "launch"] for x in lu.events(fake, [call, frozen]))
    assert [e.base.split("(")[0] for e in ev] == ["norm_backward_kernel", "norm_fold_kernel"]
    assert [e.base for e in without] == ["norm_backward_kernel"]
    assert f", {lanes}, " in ev[0].kernel.replace("(int)", "")
    assert ev[0].grid[0] == min(512, M if lanes > 64 else (M + 3) // 4) and ev[1].grid[0] == D // 8
    assert ev[0].grid[0] * D * 8 <= wkv.wkv6_layernorm_backward_workspace_bytes(M, D)


# ---------------------------------------------------------------------------------------------- oracles
def _mix(rng, rows, H, B, N=4):
    return dict(r=rng.standard_normal((rows, H, N)), k=rng.standard_normal((rows, H, N)), v=rng.standard_normal((rows, H, N)),
                g=-rng.random((rows, H)), state_in=rng.standard_normal((B, H, N, N)))


def test_mix_oracle_by_hand():
    # one head, two channels: S_1 = k_1^T v_1, S_2 = S_1 / 2 + k_2^T v_2
    r = np.array([[[1., 0.]], [[2., 3.]]])
    k = np.array([[[1., 2.]], [[0., 1.]]])
    v = np.array([[[4., 8.]], [[1., 1.]]])
    out, S = head_decay_numpy(r, k, v, np.log([[1.], [.5]]), [(0, 2)])
    assert np.allclose(S[0, 0], [[2, 4], [5, 9]]) and np.allclose(out[:, 0], [[4, 8], [2 * 2 + 3 * 5, 2 * 4 + 3 * 9]])


def test_mix_oracle_cut_in_two_and_forgetting():
    rng = np.random.default_rng(3)
    x = _mix(rng, 9, 2, 1)
    whole, S = head_decay_numpy(spans=[(0, 9)], **x)
    a, S1 = head_decay_numpy(spans=[(0, 4)], **x)
    b, S2 = head_decay_numpy(spans=[(4, 9)], **{**x, "state_in": S1})
    assert np.allclose(whole, np.where(np.isnan(a), b, a)) and np.allclose(S, S2)
    x["g"][4] = -np.inf                                        # nothing passes token 4
    cut, _ = head_decay_numpy(spans=[(0, 9)], **x)
    fresh, _ = head_decay_numpy(spans=[(4, 9)], **{**x, "state_in": None})
    assert np.allclose(cut[4:], fresh[4:])


def test_mix_gradients_against_differences():
    rng = np.random.default_rng(4)
    spans, rows, B = [(1, 6), (6, 6), (6, 8)], 9, 3
    x = _mix(rng, rows, 2, B)
    dout, dS = rng.standard_normal((rows, 2, 4)), rng.standard_normal((B, 2, 4, 4))

    def loss(y):
        out, S = head_decay_numpy(spans=spans, **y)
        return np.nansum(out * dout) + (S * dS).sum()
    grads = dict(zip(("r", "k", "v", "g", "state_in"),
                     head_decay_gradients_numpy(x["r"], x["k"], x["v"], x["g"], spans, dout, x["state_in"], dS)))
    for name, grad in grads.items():
        step = rng.standard_normal(x[name].shape)
        diff = (loss({**x, name: x[name] + 1e-6 * step}) - loss({**x, name: x[name] - 1e-6 * step})) / 2e-6
        assert abs(np.nansum(grad * step) - diff) < 1e-6 * (1 + abs(diff)), name
    assert np.isnan(grads["r"][[0, 8]]).all() and np.allclose(grads["state_in"][1], dS[1])


def test_layernorm_oracle_and_its_gradients():
    import torch
    rng = np.random.default_rng(5)
    x, gamma, beta, dy = rng.standard_normal((5, 24)) * 2 + 1, rng.random(24), rng.standard_normal(24), rng.standard_normal((5, 24))
    y, stats = layernorm_rows_numpy(x, gamma, beta, 1e-5)
    lib = torch.nn.functional.layer_norm(*(torch.from_numpy(a) if isinstance(a, np.ndarray) else a for a in (x, (24,), gamma, beta, 1e-5)))
    assert np.allclose(y, lib.numpy(), atol=1e-12)
    dx, dgamma, dbeta = layernorm_rows_gradients_numpy(x, stats, gamma, dy)
    for i, grad in enumerate((dx, dgamma, dbeta)):
        args = [x, gamma, beta]
        step = rng.standard_normal(args[i].shape)
        ends = [(layernorm_rows_numpy(*[a + s * step if j == i else a for j, a in enumerate(args)], 1e-5)[0] * dy).sum() for s in (1e-6, -1e-6)]
        assert abs((grad * step).sum() - (ends[0] - ends[1]) / 2e-6) < 1e-6
