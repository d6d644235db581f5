"""Buffers of a call that overlap.  The two results of a quantisation are refused.  An output over its own input: the
linear layer's route that quantises its rows inside the product refuses it (its workgroups read all of x while
others write y).  No GPU: a call that passes the checks ends at the launch."""
import ctypes
import os

import pytest

from paper_2010_11305_amd import dense_lib
from paper_2010_11305_amd import emb_cache as ec

FAKE = 1 << 20


@pytest.fixture(scope="module")
def L():
    import torch
    if torch.cuda.is_available():
        pytest.skip("the calls use addresses that no GPU may touch")
    if not os.path.exists(ec.LIB_PATH):
        from paper_2010_11305_amd import build
        build.build()
    return dense_lib.load()


@pytest.mark.parametrize("y,ldx,ldy,shared", [
    (0, 64, 64, True), (-1, 64, 64, True), (3 * 64 + 63, 64, 64, True), (3 * 64 + 64, 64, 64, False), (-4 * 64, 64, 64, False),
    (-3 * 64 - 1, 64, 64, True), (64, 128, 128, False), (63, 128, 128, True), (-64, 128, 128, False), (-63, 128, 128, True),
    (128 + 64, 128, 128, False), (-128 - 64, 128, 128, False), (2 * 128 + 65, 128, 128, True), (64, 128, 129, True),
    # rows that lie differently far apart: between each other, or not
    (70, 140, 139, False), (-70, 139, 140, False), (70, 140, 150, True), (-3 * 140 + 70, 139, 140, False), (-3 * 140 + 75, 139, 140, False),
    (-3 * 140 + 76, 139, 140, True),
])
def test_rows_quantised_inside(L, y, ldx, ldy, shared):
    """x [4][64] and y [4][64], `y` elements behind x."""
    n = ctypes.c_size_t(1)
    assert L.emb_mx4_linear_workspace(4, 64, 64, ctypes.byref(n)) == 0 and n.value == 0
    for type, b in ((0, 4), (1, 2)):
        st = L.emb_mx4_linear(FAKE, type, 4, 64, ldx, 2 * FAKE, 64, FAKE + y * b, ldy, None, 0, None)
        assert (st == ec.EMB_EINVAL) == shared


def test_rows_quantised_before(L):
    """With a workspace the rows are read before anything is written."""
    n = ctypes.c_size_t()
    assert L.emb_mx4_linear_workspace(200, 64, 64, ctypes.byref(n)) == 0 and n.value
    assert L.emb_mx4_linear(FAKE, 1, 200, 64, 64, 2 * FAKE, 64, FAKE, 64, 3 * FAKE, n.value, None) != ec.EMB_EINVAL


@pytest.mark.parametrize("columns,shared", [(0, True), (256, True), (-256, True), (4 * 1280, False), (-4 * 1280, False),
                                            (4 * 1280 - 256, True)])
def test_both_results_of_a_quantisation(L, columns, shared):
    """[64][64]: 4 tiles and 4 pieces of scale bytes either way."""
    n = ctypes.c_size_t()
    assert L.emb_mx4_query_bytes(64, 64, ctypes.byref(n)) == 0 and n.value == 4 * 1280
    st = L.emb_mx4_quantize(FAKE, 0, 64, 64, 64, 4 * FAKE, 4 * FAKE + columns, 0, 0, 0, None)
    assert (st == ec.EMB_EINVAL) == shared
    m = L.emb_mx4_linear_train(FAKE, 0, 64, 64, 64, 2 * FAKE, 16, 3 * FAKE, 16, 4 * FAKE + columns, 0, 0, 0, 4 * FAKE, 4 * 1280,
                               None)
    assert (m == ec.EMB_EINVAL) == shared


def test_against_every_element(L):
    """Drawn strides and places against sets of elements."""
    import random

    r, seen = random.Random(4), set()
    for _ in range(400):
        m, k, n = r.randint(1, 9), r.randint(1, 40), r.randint(1, 40)
        ldx, ldy = k + r.randint(0, 60), n + r.randint(0, 60)
        if r.random() < 0.5:
            ldx = ldy = max(ldx, ldy)
        y = r.randint(-m * ldy - 5, m * ldx + 5)
        shared = bool({i * ldx + j for i in range(m) for j in range(k)} & {y + i * ldy + j for i in range(m) for j in range(n)})
        st = L.emb_mx4_linear(FAKE, 0, m, k, ldx, 2 * FAKE, n, FAKE + 4 * y, ldy, None, 0, None)
        assert (st == ec.EMB_EINVAL) == shared, (m, k, n, ldx, ldy, y)
        seen.add((shared, ldx == ldy))
    assert len(seen) == 4
