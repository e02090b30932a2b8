"""The selective scan and the short convolution on the CPU: refusals (before anything is launched), sizes of workspaces, which kernels a
call launches (tests/launch_util.py), the headers, the binding, and the oracles' pins."""
import ctypes
import inspect
import os
import re
import subprocess

import numpy as np
import pytest

import launch_util as lu
import paper_2407_12077_amd as wkv
from oracle.selective_scan_numpy import selective_scan_gradients_numpy, selective_scan_numpy
from oracle.short_conv_numpy import short_conv_gradients_numpy, short_conv_numpy
from paper_2407_12077_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADERS = ("wkv6_selective_scan.h", "wkv6_short_conv.h")
OK, NULL, SHAPE, UNSUPPORTED, LAUNCH, ALIGN, WORKSPACE = range(7)
BF16, F32 = 0, 1
P = ctypes.c_void_p
A = P(0x1000)                  # aligned, never dereferenced
BIG = 1 << 50


def _raw(name):
    return getattr(binding.load(), name)


# ---------------------------------------------------------------------------------------------- headers and binding
def test_every_declared_function_is_exported_and_bound():
    text = "".join(open(os.path.join(ROOT, "include", h)).read() for h in HEADERS)
    names = set(re.findall(r"\b(wkv6_[a-z0-9_]+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S)))
    assert names == set(binding.SCAN_EXPORTS)
    for name in names:
        params = list(inspect.signature(getattr(wkv, name)).parameters)
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
        wkv.wkv6_short_conv_decode(0, 64, 4, a, 64.5, a, a, 1, a, a, a, BF16, stream=0)
    wkv.wkv6_short_conv_decode(0, 64, 4, a, 64, a, a, True, a, a, a, BF16, stream=0)                # no sequence: nothing to launch
    wkv.wkv6_selective_scan_decode(0, 64, 16, a, 64, a, 64, a, True, a, a, a, 16, a, None, 0, a, a, a, BF16, BF16, stream=0)
    with pytest.raises(wkv.Wkv6Error) as e:
        wkv.wkv6_short_conv_decode(1, 60, 4, a, 64, a, a, 1, a, a, a, BF16, stream=0)
    assert e.value.status == UNSUPPORTED


# ---------------------------------------------------------------------------------------------- refusals
INPUTS = dict(x=A, x_stride=64, delta=A, delta_stride=64, delta_bias=A, softplus=1, a=A, b=A, c=A, bc_stride=16, skip=A, z=A, z_stride=64)


def scan(**over):
    p = dict(B=2, T=8, D=64, N=16, rows=16, **INPUTS, offsets=None, state_in=None, out=A, state_out=A, dtype=BF16, out_dtype=BF16, workspace=A,
             workspace_bytes=BIG, stream=None)
    assert not set(over) - set(p)
    return _raw("wkv6_selective_scan_prefill")(*{**p, **over}.values())


def scan_step(**over):
    p = dict(B=2, D=64, N=16, **INPUTS, state_in=A, out=A, state_out=A, dtype=BF16, out_dtype=BF16, stream=None)
    assert not set(over) - set(p)
    return _raw("wkv6_selective_scan_decode")(*{**p, **over}.values())


def scan_back(**over):
    p = dict(B=2, T=8, D=64, N=16, rows=16, **INPUTS, offsets=None, state_in=None, dout=A, dstate_out=None, dx=A, ddelta=A, db=A, dc=A, dz=A, da=A,
             dskip=A, ddelta_bias=A, dstate_in=None, dtype=BF16, workspace=A, workspace_bytes=BIG, stream=None)
    assert not set(over) - set(p)
    return _raw("wkv6_selective_scan_backward")(*{**p, **over}.values())


CONV = dict(x=A, x_stride=64, w=A, bias=A, silu=1)


def conv(**over):
    p = dict(B=2, T=8, D=64, W=4, rows=16, **CONV, offsets=None, state_in=None, out=A, state_out=A, dtype=BF16, stream=None)
    assert not set(over) - set(p)
    return _raw("wkv6_short_conv_prefill")(*{**p, **over}.values())


def conv_step(**over):
    p = dict(B=2, D=64, W=4, **CONV, state_in=A, out=A, state_out=A, dtype=BF16, stream=None)
    assert not set(over) - set(p)
    return _raw("wkv6_short_conv_decode")(*{**p, **over}.values())


def conv_back(**over):
    p = dict(B=2, T=8, D=64, W=4, rows=16, **CONV, offsets=None, state_in=None, dout=A, dstate_out=None, dx=A, dw=A, dbias=A, dstate_in=None,
             dtype=BF16, workspace=A, workspace_bytes=BIG, stream=None)
    assert not set(over) - set(p)
    return _raw("wkv6_short_conv_backward")(*{**p, **over}.values())


SCANS, CONVS = (scan, scan_step, scan_back), (conv, conv_step, conv_back)


@pytest.mark.parametrize("call", SCANS + CONVS, ids=lambda f: f.__name__)
def test_wrong_sizes_types_and_strides(call):
    assert call(dtype=2) == UNSUPPORTED and call(dtype=-1) == UNSUPPORTED
    assert call(D=60) == UNSUPPORTED and call(D=0) == SHAPE and call(D=-8) == SHAPE and call(D=65544) == SHAPE and call(B=-1) == SHAPE
    assert call(x_stride=56) == SHAPE and call(x_stride=-64) == SHAPE and call(x_stride=68) == ALIGN and call(x_stride=(1 << 22) + 8) == SHAPE
    assert call(x=None) == NULL and call(x=P(0x1008)) == ALIGN
    assert call(state_in=P(0x1008)) == ALIGN
    if call not in (scan_step, conv_step):
        assert call(T=-1) == SHAPE and call(rows=15) == SHAPE and call(rows=-1, offsets=A) == SHAPE and call(rows=1 << 31, offsets=A) == SHAPE
        assert call(T=(1 << 30) + 1, offsets=A) == SHAPE and call(offsets=P(0x1002)) == ALIGN
        assert call(B=1 << 30, T=0, rows=0) == SHAPE           # more workgroups than a launch has


@pytest.mark.parametrize("call", SCANS, ids=lambda f: f.__name__)
def test_scan_refuses(call):
    for N in (0, 4, 12, 24, 128):
        assert call(N=N) == UNSUPPORTED
    for name in ("delta", "a", "b", "c"):
        assert call(**{name: None}) == NULL
        assert call(**{name: P(0x1008)}) == ALIGN
    for name in ("delta_bias", "skip", "z"):
        assert call(**{name: P(0x1008)}) == ALIGN
    for name in ("delta_stride", "z_stride"):
        assert call(**{name: 56}) == SHAPE and call(**{name: 65}) == ALIGN
    assert call(bc_stride=8) == SHAPE and call(bc_stride=17) == ALIGN
    if call is not scan_back:
        assert call(dtype=F32, out_dtype=BF16) == UNSUPPORTED and call(out_dtype=3) == UNSUPPORTED
        assert call(out=None) == NULL and call(out=P(0x1004)) == ALIGN and call(state_out=P(0x1004)) == ALIGN
        assert call(B=0, **({} if call is scan_step else {"rows": 0})) == OK


def test_scan_gradients_refuse():
    for name in ("dout", "dx", "ddelta", "db", "dc"):
        assert scan_back(**{name: None}) == NULL
    for name in ("dout", "dx", "ddelta", "db", "dc", "dz", "da", "dskip", "ddelta_bias", "dstate_out", "dstate_in"):
        assert scan_back(**{name: P(0x1004)}) == ALIGN
    need = wkv.wkv6_selective_scan_backward_workspace_bytes(2, 8, 64, 16, 16)
    assert need > 0 and scan_back(workspace_bytes=need // 8) == WORKSPACE and scan_back(workspace=None) == NULL and scan_back(workspace=P(0x1004)) == ALIGN
    assert scan_back(B=0, rows=0, da=None, dskip=None, ddelta_bias=None) == OK


def test_scan_workspace_refused():
    long = dict(B=1, T=4096, rows=4096)
    need = wkv.wkv6_selective_scan_workspace_bytes(1, 4096, 64, 16)
    assert need > 0 and scan(**long, workspace_bytes=16) == WORKSPACE and scan(**long, workspace=None) == NULL
    assert scan(**long, workspace=P(0x1008)) == ALIGN


@pytest.mark.parametrize("call", CONVS, ids=lambda f: f.__name__)
def test_conv_refuses(call):
    for W in (0, 1, 5):
        assert call(W=W) == UNSUPPORTED
    assert call(w=None) == NULL and call(w=P(0x1004)) == ALIGN and call(bias=P(0x1004)) == ALIGN
    if call is conv_back:
        for name in ("dout", "dx", "dw", "dbias", "workspace"):
            assert call(**{name: None}) == NULL and call(**{name: P(0x1004)}) == ALIGN
        assert call(dstate_out=P(0x1004)) == ALIGN and call(dstate_in=P(0x1004)) == ALIGN
        need = wkv.wkv6_short_conv_backward_workspace_bytes(2, 8, 64, 4, 16)
        assert need > 0 and call(workspace_bytes=need - 1) == WORKSPACE
        assert call(B=0, rows=0, dw=None, dbias=None) == OK
    else:
        assert call(out=None) == NULL and call(out=P(0x1004)) == ALIGN and call(state_out=P(0x1004)) == ALIGN
        assert call(B=0, **({} if call is conv_step else {"rows": 0})) == OK


# ---------------------------------------------------------------------------------------------- workspaces
def test_workspace_sizes():
    fore, back, taps = wkv.wkv6_selective_scan_workspace_bytes, wkv.wkv6_selective_scan_backward_workspace_bytes, wkv.wkv6_short_conv_backward_workspace_bytes
    assert fore(0, 10, 64, 16) == 0 and fore(1, 0, 64, 16) == 0 and fore(1, 1, 64, 16) == 0
    for bad in ((1, 8, 60, 16), (1, 8, 64, 12), (-1, 8, 64, 16), (1, -8, 64, 16), (1, 8, 0, 16), (1, (1 << 30) + 1, 64, 16)):
        assert fore(*bad) == -1 and back(*bad, 8) == -1
    assert back(1, 8, 64, 16, -1) == -1 and back(0, 8, 64, 16, 0) == 0
    assert taps(1, 8, 64, 5, 8) == -1 and taps(1, 8, 60, 4, 8) == -1 and taps(1, 8, 64, 4, -1) == -1
    for B, T, D, N in ((1, 100000, 2048, 16), (3, 700, 200, 64)):
        assert fore(B, T, D, N) % 16 == 0 and back(B, T, D, N, B * T) % 16 == 0


# ---------------------------------------------------------------------------------------------- launches
@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return lu.build_fake(tmp_path_factory.mktemp("fake_hip"))


def scan_call(B, T, D, N, rows=None, dtype=BF16, out=BF16, space=BIG, gate=True):
    inputs = [lu.at(0), D, lu.at(1), D, lu.at(2), 1, lu.at(3), lu.at(4), lu.at(5), N, lu.at(6), lu.at(7) if gate else None, D]
    return ("wkv6_selective_scan_prefill", [B, T, D, N, B * T if rows is None else rows, *inputs, None if rows is None else lu.at(8), lu.at(9), lu.at(10), lu.at(11),
                                            dtype, out, lu.at(12), space, None])


def back_call(B, T, D, N, rows=None, dtype=BF16, space=BIG, weights=True):
    inputs = [lu.at(0), D, lu.at(1), D, lu.at(2), 1, lu.at(3), lu.at(4), lu.at(5), N, lu.at(6), lu.at(7), D]
    w = [lu.at(20 + i) if weights else None for i in range(3)]
    return ("wkv6_selective_scan_backward", [B, T, D, N, B * T if rows is None else rows, *inputs, None if rows is None else lu.at(8), lu.at(9), lu.at(10), lu.at(11),
                                             *(lu.at(13 + i) for i in range(5)), *w, lu.at(18), dtype, lu.at(12), space, None])


def conv_back_call(B, T, D, W, rows=None, dtype=BF16, space=BIG, weights=True):
    return ("wkv6_short_conv_backward", [B, T, D, W, B * T if rows is None else rows, lu.at(0), D, lu.at(1), lu.at(2), 1, None if rows is None else lu.at(3), lu.at(4),
                                         lu.at(5), lu.at(6), lu.at(7), lu.at(8) if weights else None, lu.at(9) if weights else None, lu.at(10), dtype, lu.at(11), space, None])


def test_launches(fake):
    """Pieces only where compute units would idle, or one long sequence would go on alone."""
    calls = [scan_call(8, 4096, 4096, 16), scan_call(1, 4096, 2048, 16), scan_call(1, 20, 64, 16), scan_call(37, 2011, 1536, 16, rows=13900),
             scan_call(8, 4096, 4096, 16, rows=32768), scan_call(2, 0, 64, 8), back_call(8, 2048, 4096, 16), back_call(1, 4096, 2048, 16),
             back_call(1, 20, 64, 64, weights=False), back_call(2, 0, 64, 8), conv_back_call(2, 9, 64, 4), conv_back_call(2, 9, 64, 2, weights=False),
             conv_back_call(2, 0, 64, 3)]
    got = [[e for e in ev if e.kind == "launch"] for ev in lu.events(fake, calls)]
    assert [[e.base for e in ev] for ev in got] == [
        ["scan_kernel"], ["scan_pieces_kernel", "scan_kernel"], ["scan_kernel"], ["scan_pieces_kernel", "scan_kernel"], ["scan_kernel"], ["scan_kernel"],
        ["scan_backward_kernel", "scan_folds_kernel"],
        ["scan_pieces_kernel", "scan_backward_kernel", "scan_folds_kernel"], ["scan_backward_kernel", "scan_folds_kernel"],
        ["scan_backward_kernel", "scan_weights_kernel"], ["conv_backward_kernel", "conv_fold_kernel"], ["conv_backward_kernel"],
        ["conv_backward_kernel", "conv_fold_kernel"]]
    assert got[0][0].grid[0] == 512 and got[0][0].block == 256 and got[6][0].grid[0] == 512
    # nothing to add up: the folds alone
    none = [back_call(0, 5, 64, 16), conv_back_call(0, 5, 64, 4)]
    assert [[e.base for e in ev if e.kind == "launch"] for ev in lu.events(fake, none)] == [["scan_weights_kernel"], ["conv_fold_kernel"]]


def test_launches_of_few_tokens(fake):
    """Up to eight tokens a sequence: no chunks."""
    calls = [scan_call(3, 1, 4096, 64), scan_call(64, 8, 2048, 32), scan_call(64, 8, 2048, 32, rows=100), scan_call(64, 9, 2048, 32), scan_call(2, 0, 64, 8)]
    got = [[(e.base, e.grid[0], e.block) for e in ev if e.kind == "launch"] for ev in lu.events(fake, calls)]
    assert got == [[("scan_step_kernel", 3 * 256, 256)], [("scan_step_kernel", 64 * 64, 256)], [("scan_step_kernel", 64 * 64, 256)], [("scan_kernel", 64 * 32, 512)],
                   [("scan_kernel", 2, 128)]]


def test_folds_of_as_many_rows_as_there_may_be(fake):
    """One launch for both folds as long as one holds them."""
    rows = 2 ** 26 - 16
    fits, whole = lu.events(fake, [back_call(1, 4096, 64, 8), back_call(4096, 2 ** 14, 8, 8, rows=rows)])
    assert [(e.base, e.grid[0], e.block) for e in fits if e.kind == "launch"][-1] == ("scan_folds_kernel", 64 * 10 // 64 + 4096 // 16, 1024)
    assert [(e.base, e.grid[0]) for e in whole if e.kind == "launch"][-2:] == [("scan_folds_kernel", rows // 16), ("scan_weights_kernel", 2)]
    assert [wkv.wkv6_selective_scan_backward_workspace_bytes(4096, 2 ** 14, 8, 8, n) > 0 for n in (rows, rows + 1)] == [True, False]


def test_empty_workgroups_are_few(fake):
    """Thousands of packed sequences, one of them long: a launch stays a small multiple of the work, and is not refused for its size."""
    calls = [conv_back_call(4096, 65536, 4096, 4, rows=10 ** 6), conv_back_call(1024, 32768, 2048, 4, rows=500000), conv_back_call(8, 65536, 4096, 4, rows=8 * 65536)]
    got = [ev[0].grid[0] for ev in lu.events(fake, calls)]
    for n, (B, D, rows) in zip(got, ((4096, 4096, 10 ** 6), (1024, 2048, 500000), (8, 4096, 8 * 65536))):
        assert n <= 16 * (rows // 128 + B) * D // 256


def test_workspace_holds_whatever_the_lengths_are(fake):
    rng = np.random.default_rng(5)
    calls = []
    for _ in range(150):
        B, D, T, N = int(rng.integers(1, 60)), 8 * int(rng.integers(1, 300)), int(2 ** rng.uniform(0, 14)), int(rng.choice([8, 16, 32, 64]))
        rows, dtype = int(rng.integers(0, B * T + 100)), int(rng.integers(0, 2))
        for n in (None, rows, T):
            calls.append(scan_call(B, T, D, N, n, dtype, dtype, wkv.wkv6_selective_scan_workspace_bytes(B, T, D, N)))
            m = B * T if n is None else n
            calls.append(back_call(B, T, D, N, n, dtype, wkv.wkv6_selective_scan_backward_workspace_bytes(B, T, D, N, m)))
            calls.append(conv_back_call(B, T, D, 4, n, dtype, wkv.wkv6_short_conv_backward_workspace_bytes(B, T, D, 4, m)))
    for ev in lu.events(fake, calls):
        assert [e for e in ev if e.kind == "launch"]


# ---------------------------------------------------------------------------------------------- oracles
def _call(rng, rows, spans, D=3, N=4, **over):
    return {**dict(x=rng.standard_normal((rows, D)), delta=rng.standard_normal((rows, D)), a=-rng.random((D, N)), b=rng.standard_normal((rows, N)),
                   c=rng.standard_normal((rows, N)), spans=spans, bias=rng.standard_normal(D), skip=rng.standard_normal(D), z=rng.standard_normal((rows, D)),
                   state_in=rng.standard_normal((len(spans), D, N))), **over}


def test_scan_oracle_by_hand():
    # one channel, two states, step size 1: h_1 = x_1 b_1, h_2 = h_1 / 2 or h_1 / 4, + x_2 b_2
    out, h = selective_scan_numpy(x=[[2.], [1.]], delta=[[1.], [1.]], a=np.log([[.5, .25]]), b=[[1., 2.], [3., 0.]], c=[[1., 1.], [2., 4.]], spans=[(0, 2)],
                                  use_softplus=False, skip=[10.])
    assert np.allclose(h, [[[1 + 3, 1]]]) and np.allclose(out, [[2 + 4 + 20], [2 * 4 + 4 * 1 + 10]])
    out, h = selective_scan_numpy(x=[[1.]], delta=[[0.]], a=[[0.]], b=[[1.]], c=[[1.]], spans=[(0, 1)], z=[[1.]])
    assert np.allclose(h, np.log(2)) and np.allclose(out, np.log(2) / (1 + np.exp(-1)))


def test_scan_oracle_cut_in_two():
    rng = np.random.default_rng(3)
    x = _call(rng, 9, [(0, 9)])
    whole, h = selective_scan_numpy(**x)
    a, h1 = selective_scan_numpy(**{**x, "spans": [(0, 4)]})
    b, h2 = selective_scan_numpy(**{**x, "spans": [(4, 9)], "state_in": h1})
    assert np.allclose(whole, np.where(np.isnan(a), b, a)) and np.allclose(h, h2)


@pytest.mark.parametrize("softplus", [True, False])
def test_scan_gradients_against_differences(softplus):
    rng = np.random.default_rng(4)
    spans, rows = [(1, 6), (6, 6), (6, 8)], 9
    x = _call(rng, rows, spans, use_softplus=softplus)
    dout, dh = rng.standard_normal((rows, 3)), rng.standard_normal((3, 3, 4))

    def loss(p):
        out, h = selective_scan_numpy(**p)
        return np.nansum(out * dout) + (h * dh).sum()
    grads = selective_scan_gradients_numpy(dout, dh, **x)
    # The loss's own roundings: at most 64 of 2^-53 of its terms' magnitudes (of steps up to six tokens grow states without softplus), in each of two losses, over 2e-6.
    out, h = selective_scan_numpy(**x)
    noise = 64 * 2.0 ** -53 * (np.nansum(abs(out * dout)) + abs(h * dh).sum()) / 1e-6
    names = dict(x="dx", delta="ddelta", a="da", b="db", c="dc", bias="dbias", skip="dskip", z="dz", state_in="dstate_in")
    for name, of in names.items():
        step = rng.standard_normal(np.shape(x[name]))
        diff = (loss({**x, name: x[name] + 1e-6 * step}) - loss({**x, name: x[name] - 1e-6 * step})) / 2e-6
        assert abs(np.nansum(grads[of] * step) - diff) < 1e-6 * (1 + abs(diff)) + noise, name
    assert np.isnan(grads["dx"][[0, 8]]).all() and np.allclose(grads["dstate_in"][1], dh[1])


def test_conv_oracle_by_hand_and_cut_in_two():
    out, state = short_conv_numpy([[1.], [2.], [3.]], [[10., 1.]], [(0, 3)], bias=[.5], use_silu=False, state_in=[[[7.]]])
    assert np.allclose(out, [[71.5], [12.5], [23.5]]) and np.allclose(state, 3)
    rng = np.random.default_rng(5)
    x, w, s = rng.standard_normal((7, 3)), rng.standard_normal((3, 4)), rng.standard_normal((1, 3, 3))
    whole, last = short_conv_numpy(x, w, [(0, 7)], state_in=s)
    a, s1 = short_conv_numpy(x, w, [(0, 2)], state_in=s)
    b, s2 = short_conv_numpy(x, w, [(2, 7)], state_in=s1)
    assert np.allclose(whole, np.where(np.isnan(a), b, a)) and np.allclose(last, s2) and np.allclose(last[0], x[4:])


@pytest.mark.parametrize("silu", [True, False])
def test_conv_gradients_against_differences(silu):
    rng = np.random.default_rng(6)
    spans, rows = [(1, 6), (6, 6), (6, 8)], 9
    x = dict(x=rng.standard_normal((rows, 3)), w=rng.standard_normal((3, 4)), bias=rng.standard_normal(3), state_in=rng.standard_normal((3, 3, 3)))
    dout, ds = rng.standard_normal((rows, 3)), rng.standard_normal((3, 3, 3))

    def loss(p):
        out, s = short_conv_numpy(spans=spans, use_silu=silu, **p)
        return np.nansum(out * dout) + (s * ds).sum()
    grads = dict(zip(("x", "w", "bias", "state_in"), short_conv_gradients_numpy(spans=spans, use_silu=silu, dout=dout, dstate_out=ds, **x)))
    for name, grad in grads.items():
        step = rng.standard_normal(x[name].shape)
        diff = (loss({**x, name: x[name] + 1e-6 * step}) - loss({**x, name: x[name] - 1e-6 * step})) / 2e-6
        assert abs(np.nansum(grad * step) - diff) < 1e-6 * (1 + abs(diff)), name
