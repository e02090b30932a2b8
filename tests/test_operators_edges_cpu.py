"""Calls of the head-decay time mix at the edges of what its header allows, without a GPU: what they launch (tests/launch_util.py) and what they refuse."""
import ctypes

import pytest

import launch_util as lu
from paper_2407_12077_amd import binding

OK, NULL, SHAPE, UNSUPPORTED, LAUNCH, ALIGN, WORKSPACE = range(7)
BF16, F32 = 0, 1
BIG = 1 << 50


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return lu.build_fake(tmp_path_factory.mktemp("fake_hip"))


def launches(fake, calls):
    return [[e for e in ev if e.kind == "launch"] for ev in lu.events(fake, calls)]


def backward(B, T, H, rows, g_stride=None, packed=False, dtype=BF16, dg=lu.at(10), workspace_bytes=BIG):
    return ("wkv6_head_decay_backward", [B, T, H, 64, rows, lu.at(0), lu.at(1), lu.at(2), H * 64, lu.at(3), H if g_stride is None else g_stride,
                                         lu.at(13) if packed else None, lu.at(4), lu.at(5), lu.at(6), lu.at(7), lu.at(8), lu.at(9), dg, lu.at(11), dtype,
                                         lu.at(12), workspace_bytes, None])


def status(call):
    name, args = call
    return getattr(binding.load(), name)(*[ctypes.c_void_p(a) if isinstance(a, int) and a >= 1 << 36 and a != BIG else a for a in args])


def test_gradient_of_a_head_s_decay_with_no_sequence_is_written(fake):
    """dg [H] is a sum over no tokens: nought, not what was there before."""
    got = launches(fake, [backward(0, 0, 3, 0, g_stride=0), backward(0, 8, 3, 0, g_stride=0), backward(0, 8, 3, 5, g_stride=0, packed=True),
                          backward(0, 8, 3, 0), backward(0, 8, 3, 0, g_stride=0, dg=None)])
    assert [[e.base for e in ev] for ev in got] == [["head_sums_kernel"]] * 3 + [[], []]
    assert got[0][0].grid[0] == 3
    assert status(backward(0, 0, 3, 0, g_stride=0, dg=lu.at(10, 2))) == ALIGN


def test_gradient_of_a_head_s_decay_without_a_workspace_is_written(fake):
    """Without tokens no workspace is needed, and none may be given."""
    calls = [backward(2, 0, 3, 0, g_stride=0, workspace_bytes=0), backward(2, 9, 3, 0, g_stride=0, packed=True, workspace_bytes=0)]
    for _, args in calls:
        args[-3] = None
    assert [[e.base for e in ev][-1:] for ev in launches(fake, calls)] == [["head_sums_kernel"]] * 2


def packed_need(B, T, H, rows):
    """Bytes of a packed gradient call with 256 units or more, which stay whole: anchors of both directions, two sums a row and head, a partial sum a block and head.  A head
    has an anchor a block of 1024 tokens of every sequence, at most rows / 1024 blocks that are not a sequence's last and B that are."""
    longest = min(T, rows)
    block = min(1024, (longest + 63) // 64 * 64)
    blocks = -(-longest // block)
    four = lambda n: (n + 3) // 4 * 4  # noqa: E731
    return 4 * (2 * min(B * blocks, rows // block + B) * H * 4096 + 2 * four(H * rows) + four(B * blocks * H))


@pytest.mark.parametrize("B,T,H,rows", [(64, 131072, 32, 131072), (64, 131072, 32, 5000), (300, 1 << 30, 4, 9000), (2048, 131072, 32, 131072), (16, 4096, 16, 65536),
                                        (16, 4096, 16, 65535), (256, 100, 1, 300)])
def test_packed_gradients_take_what_their_rows_need(fake, B, T, H, rows):
    """64 documents in 131072 rows took 8.7 GB of anchors where 0.2 hold them; T may be an upper bound, and 2048 x 32 units of 128 blocks fit a launch."""
    need = binding.load().wkv6_head_decay_backward_workspace_bytes(B, T, H, 64, rows)
    assert need == packed_need(B, T, H, rows)
    ev, = launches(fake, [backward(B, T, H, rows, packed=True, workspace_bytes=need)])
    assert [e.base for e in ev] == ["mix_kernel", "decay_gradient_kernel"]
    longest = min(T, rows)
    assert ev[1].grid[0] == B * -(-longest // min(1024, (longest + 63) // 64 * 64)) * H
    assert status(backward(B, T, H, rows, packed=True, workspace_bytes=need - 1)) == WORKSPACE


def prefill(B, T, H, rows, packed, dtype, workspace_bytes):
    return ("wkv6_head_decay_prefill", [B, T, H, 64, rows, lu.at(0), lu.at(1), lu.at(2), H * 64, lu.at(3), H, lu.at(13) if packed else None, lu.at(4),
                                        lu.at(5), lu.at(6), dtype, dtype, lu.at(12), workspace_bytes, None])


@pytest.mark.parametrize("B,T,H,rows", [(1, 4096, 32, None), (1, 1500, 2, None), (4, 700, 8, None), (2, 512, 16, None), (20, 8000, 8, 60000), (6, 2111, 1, 3000),
                                        (3, 130, 5, 200), (9, 1531, 12, 7000)])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_a_call_takes_exactly_the_workspace_of_its_pieces(fake, B, T, H, rows, dtype):
    """Counted from what is launched: a state and four floats a piece and unit, of gradients for two states, and what packed_need counts."""
    packed, rows = rows is not None, B * T if rows is None else rows
    units = B * H
    ev, back = launches(fake, [prefill(B, T, H, rows, packed, dtype, BIG), backward(B, T, H, rows, packed=packed, dtype=dtype)])
    pieces = ev[0].grid[0] // units if len(ev) == 2 else 0
    assert [e.grid[0] for e in ev] == [pieces * units] * 2 if pieces else [units]
    need = 4 * pieces * units * 4100
    assert need <= binding.load().wkv6_head_decay_workspace_bytes(B, T, H, 64)
    launches(fake, [prefill(B, T, H, rows, packed, dtype, need)])
    if need:
        assert status(prefill(B, T, H, rows, packed, dtype, need - 1)) == WORKSPACE
    pieces = back[0].grid[0] // (2 * units) if len(back) == 3 else 0
    assert back[-2].grid[0] == 3 * units * max(1, pieces)
    longest = min(T, rows)
    block = min(1024, (longest + 63) // 64 * 64)
    blocks = -(-longest // block)
    four = lambda n: (n + 3) // 4 * 4  # noqa: E731
    places = min(B * blocks, rows // block + B) if packed else B * blocks
    need = 4 * (2 * pieces * units * 4100 + 2 * places * H * 4096 + 2 * four(H * rows) + four(units * blocks))
    assert need <= binding.load().wkv6_head_decay_backward_workspace_bytes(B, T, H, 64, rows)
    launches(fake, [backward(B, T, H, rows, packed=packed, dtype=dtype, workspace_bytes=need)])
    assert status(backward(B, T, H, rows, packed=packed, dtype=dtype, workspace_bytes=need - 1)) == WORKSPACE
