"""Buffers of the gradients' norm that lie over each other (no GPU; csrc/tower.cpp with stand-ins for its launches).  A result inside the
workspace is written while other workgroups still read the parts' sums, a workspace over a gradient while its squares are
still being read, and anything over the handle's tables would send workgroups anywhere: all of them are refused."""
import pytest

from paper_2010_11305_amd import emb_cache as ec
from tower_host import Clip

A, B, R, W = 1 << 30, 2 << 30, 3 << 30, 4 << 30    # addresses that no call touches
SIZES = [5000, 70]


@pytest.fixture(scope="module")
def clip():
    c = Clip(SIZES)
    assert c.sizes.workspace_bytes == 256     # 4 parts of 8 bytes, rounded up
    return c


def ends(size, at, width):
    """Places of `width` bytes that share a byte with `size` bytes at `at`, and two beside them."""
    return [at - width + 4, at, at + size - 4], [at - width, at + size]


def both(clip, good, grads, result, workspace):
    for f in (clip.norm, clip.apply):
        st, names = f(grads, result, workspace)
        assert (st == 0) == good and (names != []) == good, (f.__name__, st, names)
        assert good or st == ec.EMB_EINVAL


def test_apart(clip):
    both(clip, True, [A, B], R, W)
    assert clip.scale([A, B], R) == (0, ["scale"])


def test_the_result_in_the_workspace(clip):
    shared, beside = ends(256, W, 8)
    for r in shared:
        both(clip, False, [A, B], r, W)
    for r in beside:
        both(clip, True, [A, B], r, W)


@pytest.mark.parametrize("which", [0, 1])
def test_the_workspace_over_a_gradient(clip, which):
    at, size = (A, B)[which], SIZES[which] * 4
    base = -(-(at + size) // 256) * 256
    for ws in (at, base - 256):
        both(clip, False, [A, B], R, ws)
    for ws in (at - 256, base):
        both(clip, True, [A, B], R, ws)
    both(clip, True, [A if which else None, None if which else B], R, at)     # a gradient that is not there


@pytest.mark.parametrize("which", [0, 1])
def test_the_result_in_a_gradient(clip, which):
    shared, beside = ends(SIZES[which] * 4, (A, B)[which], 8)
    for r in shared:
        both(clip, False, [A, B], r, W)
    for r in beside:
        both(clip, True, [A, B], r, W)


def test_over_the_tables(clip):
    """Neither may anything that a call writes lie over them."""
    n = clip.sizes.state_bytes
    shared, beside = ends(n, clip.state, 8)
    for r in shared:
        both(clip, False, [A, B], r, W)
    for r in beside:
        both(clip, True, [A, B], r, W)
    for ws in range(clip.state, clip.state + n, 256):
        both(clip, False, [A, B], R, ws)
    both(clip, True, [A, B], R, clip.state + n)
    for g in (clip.state, clip.state - 4, clip.state + n - 4):
        assert clip.apply([A, g], R, W) == (ec.EMB_EINVAL, [])
        assert clip.scale([A, g], R) == (ec.EMB_EINVAL, [])


def test_gradients_over_each_other(clip):
    """May be read, not scaled."""
    assert clip.norm([A, A + 16], R, W) == (0, ["squares", "join"])
    for grads in ([A, A + 16], [A + 4996 * 4, A + 4996 * 4 + 8], [A, A - 4]):
        assert clip.apply(grads, R, W) == (ec.EMB_EINVAL, []) and clip.scale(grads, R) == (ec.EMB_EINVAL, [])
    for f in (19996, 0, 4):
        assert clip.scale([A, B], A + f) == (ec.EMB_EINVAL, [])
    assert clip.scale([A, B], A + 20000) == (0, ["scale"])


def test_nothing_to_read():
    """Tensors without elements need no workspace, wherever they are said to be."""
    c = Clip([0, 0])
    assert c.sizes.workspace_bytes == 0
    assert c.norm([A, A], A, None) == (0, ["join"]) and c.apply([None, A], A, A) == (0, ["join"])
    assert c.scale([A, A], A) == (0, [])
    assert c.norm([A, A], c.state, None) == (ec.EMB_EINVAL, [])


def test_many_tensors_are_joined_once():
    """Every workgroup of a launch that joins and scales adds up all parts, so that is left to what one launch carries: with a launch
    for each 480 tensors the work would grow with their square."""
    for n, want in ((1, ["squares", "join_scale"]), (480, ["squares", "join_scale"]), (481, 2 * ["squares"] + ["join"] + 2 * ["scale"]),
                    (20000, 42 * ["squares"] + ["join"] + 42 * ["scale"])):
        c = Clip([3] * n)
        assert c.apply([A + 16 * k for k in range(n)], R, W) == (0, want)
        assert c.apply([A] * n, R, W) == ((0, want) if n == 1 else (ec.EMB_EINVAL, []))
