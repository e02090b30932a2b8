"""How many threads of the short convolution lie side by side over a row's groups of four channels: half as many where that leaves fewer without a group."""
import pytest

import launch_util as lu
from test_scan_operators_cpu import conv_back_call


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return lu.build_fake(tmp_path_factory.mktemp("fake_hip"))


@pytest.mark.parametrize("D,lanes", [(136, 64), (200, 64), (264, 32), (384, 32), (520, 32), (768, 64), (896, 32), (1056, 64), (2056, 64), (64, 16), (8, 2)])
def test_lanes(fake, D, lanes):
    """A row in one workgroup's reach of tokens: as many workgroups as lanes go into the groups."""
    ev = lu.events(fake, [conv_back_call(3, 9, D, 4)])[0]
    assert ev[0].base == "conv_backward_kernel" and ev[0].grid[0] == 3 * -(-D // 4 // lanes)
