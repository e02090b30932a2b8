"""The selective scan's calls that tests/scan_pieces.py says are cut are cut: a change of what a call is modelled to take would else leave pieces untested."""
import pytest

import launch_util as lu
from scan_pieces import CUT, D, MANY, MANY_D, STATES, sizes
from test_scan_operators_cpu import BF16, F32, back_call, scan_call


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return lu.build_fake(tmp_path_factory.mktemp("fake_hip"))


def calls_of(call, width, N):
    B, T, rows = sizes(call)
    return [scan_call(B, T, width, N, rows, dtype, dtype) for dtype in (BF16, F32)] + [back_call(B, T, width, N, rows, dtype) for dtype in (BF16, F32)]


@pytest.mark.parametrize("N", STATES)
def test_cut_calls_are_cut(fake, N):
    calls = [c for call in CUT for c in calls_of(call, D, N)]
    for args, names in zip(calls, lu.launched(fake, calls)):
        assert names[:2] in (["scan_pieces_kernel", "scan_kernel"], ["scan_pieces_kernel", "scan_backward_kernel"]), (args[1][:5], names)


@pytest.mark.parametrize("N", STATES)
def test_one_long_sequence_among_many_is_cut(fake, N):
    """Into no more pieces than a packed call with work for every compute unit may have."""
    units = sizes(MANY)[0] * MANY_D // 64
    assert units > 256
    for ev in lu.events(fake, calls_of(MANY, MANY_D, N)):
        launches = [e for e in ev if e.kind == "launch"]
        assert launches[0].base == "scan_pieces_kernel" and units < launches[1].grid[0] <= 16 * units
