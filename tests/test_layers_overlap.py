"""Which buffers of a call may share memory, against sets of addresses: outputs of the norm over its inputs, of a product over its
rows, gradients over each other.  No GPU: a call that passes the checks ends at the launch."""
import ctypes
import os
import random

import pytest

from paper_2010_11305_amd import dense_lib
from paper_2010_11305_amd import emb_cache as ec

FAKE, FAR = 1 << 20, 1 << 30


@pytest.fixture(scope="module")
def L():
    import torch
    if torch.cuda.is_available():
        pytest.skip("the calls use addresses that no GPU may touch")
    if not os.path.exists(ec.LIB_PATH):
        from paper_2010_11305_amd import build
        build.build()
    return dense_lib.load()


def places(at, rows, cols, ld, size):
    return {at + size * (r * ld + c) + k for r in range(rows) for c in range(cols) for k in range(size)}


def test_the_norm_over_its_input(L):
    """y over x: exactly, or with no byte in common.  All strides, also equal ones, and offsets of whole elements."""
    rng = random.Random(1)
    seen = set()
    for _ in range(4000):
        rows, cols = rng.randint(1, 5), rng.randint(1, 6)
        type, size = rng.choice([(0, 4), (1, 2)])
        ldx = cols + rng.choice([0, 0, 1, 3, 7])
        ldy = rng.choice([ldx, ldx, cols + rng.randint(0, 8)])
        off = rng.randint(-(rows * ldx + 2), rows * ldx + 2) * size
        st = L.emb_rmsnorm_forward(FAKE, type, rows, cols, ldx, None, 0, None, 0, 1e-6, None, 0, FAKE + off, ldy, None, None)
        shared = bool(places(FAKE, rows, cols, ldx, size) & places(FAKE + off, rows, cols, ldy, size))
        same = off == 0 and (ldx == ldy or rows == 1)
        assert (st == ec.EMB_EINVAL) == (shared and not same), (rows, cols, ldx, ldy, off, size)
        seen.add((shared, same))
    assert seen == {(True, True), (True, False), (False, False)}


def test_a_sum_over_another_stride(L):
    """The sum over the residual, both with strides of their own, and 8-bit codes among FP32 rows."""
    rng = random.Random(2)
    for _ in range(3000):
        rows, cols = rng.randint(1, 4), rng.randint(1, 5)
        ldr, ldh, off = cols + rng.randint(0, 9), cols + rng.randint(0, 9), rng.randint(-30, 30) * 4
        st = L.emb_rmsnorm_forward(FAR, 0, rows, cols, cols, FAKE, ldr, None, 0, 1e-6, FAKE + off, ldh, 2 * FAR, cols, None, None)
        shared = bool(places(FAKE, rows, cols, ldr, 4) & places(FAKE + off, rows, cols, ldh, 4))
        same = off == 0 and (ldr == ldh or rows == 1)
        assert (st == ec.EMB_EINVAL) == (shared and not same)
        ldc, at = cols + rng.randint(0, 40), FAKE + rng.randint(-120, 120)
        st = L.emb_rmsnorm_forward8(FAKE, 0, rows, cols, ldr, None, 0, None, 0, 1e-6, None, 0, at, ldc, FAR, None)
        assert (st == ec.EMB_EINVAL) == bool(places(FAKE, rows, cols, ldr, 4) & places(at, rows, cols, ldc, 1))


def test_products_over_their_rows(L):
    rng = random.Random(3)
    n = ctypes.c_size_t(1)
    for _ in range(2000):
        m, k, o = rng.randint(1, 4), rng.randint(1, 6), rng.randint(1, 6)
        assert L.emb_w4_linear_workspace(1, m, o, k, 32, ctypes.byref(n)) == 0 and n.value == 0
        ldx, ldy, off = k + rng.randint(0, 8), o + rng.randint(0, 8), rng.randint(-40, 40) * 2
        st = L.emb_w4_linear(FAKE, 1, None, m, k, ldx, FAR, o, 32, None, 0, FAKE + off, 1, ldy, None, 0, None)
        assert (st == ec.EMB_EINVAL) == bool(places(FAKE, m, k, ldx, 2) & places(FAKE + off, m, o, ldy, 2))
