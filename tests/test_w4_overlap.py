"""Plain codes, scales and biases over a W4 matrix, or over each other where they are written (no GPU; csrc/tower.cpp with
stand-ins for its launches): workgroups would read what others had written."""
import pytest

from paper_2010_11305_amd import emb_cache as ec
from tower_host import launches, load

A, Q = 1 << 30, 5 << 30
ROWS, COLS, GROUP = 20, 201, 32
SIZE = {"q": 2 * 2 * 1024 + 2 * 8 * 64, "codes": 20 * 101, "scales": 20 * 7 * 2, "biases": 20 * 7 * 2}


@pytest.fixture(scope="module")
def L():
    return load()


def call(L, name, **at):
    p = dict(codes=A, scales=2 * A, biases=3 * A, q=Q)
    p.update(at)
    if name == "pack":
        st = L.emb_w4_pack(p["codes"], p["scales"], p["biases"], ROWS, COLS, GROUP, p["q"], None)
    else:
        st = L.emb_w4_unpack(p["q"], ROWS, COLS, GROUP, p["codes"], p["scales"], p["biases"], None)
    return st, launches(L)


def around(base, size, width, step):
    """Places of `width` bytes over `size` bytes at `base`, and the nearest beside them, on multiples of `step`."""
    return [base, base + (size - 1) // step * step, base - (width - 1) // step * step], [base + -(-size // step) * step, base - -(-width // step) * step]


@pytest.mark.parametrize("name", ["pack", "unpack"])
@pytest.mark.parametrize("part", ["codes", "scales", "biases"])
def test_over_the_matrix(L, name, part):
    assert call(L, name) == (0, [name])
    shared, beside = around(Q, SIZE["q"], SIZE[part], 1 if part == "codes" else 2)
    for at in shared:
        assert call(L, name, **{part: at}) == (ec.EMB_EINVAL, [])
    for at in beside:
        assert call(L, name, **{part: at}) == (0, [name])


@pytest.mark.parametrize("part,other", [("codes", "scales"), ("codes", "biases"), ("scales", "biases")])
def test_over_each_other(L, part, other):
    """Read, they may lie as they like."""
    base = {"scales": 2 * A, "biases": 3 * A}[other]
    shared, beside = around(base, SIZE[other], SIZE[part], 1 if part == "codes" else 2)
    for at in shared:
        assert call(L, "unpack", **{part: at}) == (ec.EMB_EINVAL, []) and call(L, "pack", **{part: at}) == (0, ["pack"])
    for at in beside:
        assert call(L, "unpack", **{part: at}) == (0, ["unpack"])
