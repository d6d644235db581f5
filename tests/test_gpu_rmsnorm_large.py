"""Gradients of the norm whose row sums leave FP32: the mean over a row is taken in FP64 at every width, and its error is that
of its terms, not of their number."""
import numpy as np
import pytest

import layers_ref as ref
from layers_ref import DTYPES, U, f64

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module")
def torch():
    import torch as t
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2010_11305_amd import dense_lib
    dense_lib.load()
    return t


def check(dx, dy, h, gain, dh, dtype):
    """Roundings of FP32 in dx = (dn - n mean) inverse + dh.  dn has 1; n has 2 (that of inverse, its own).  The mean has those of
    its terms, 3, of mean |dn n|, and its own, the products and sums between being exact to FP64: 4.  n mean has 4 + 2 + 1,
    and both go through the difference, the product with inverse, which has 1 itself, and the last sum."""
    D, H, G = f64(dy), f64(h), f64(gain)
    want, _, along = ref.norm_gradients(D, H, G, EPS)
    n, inverse = ref.norm(H, 1.0, EPS)
    extra = 0.0 if dh is None else f64(dh)
    want = want + extra
    slack = 1.01 * U * (4 * np.abs(D * G) * inverse + 10 * np.abs(n) * along * inverse + np.abs(extra) + np.abs(want))
    off = np.abs(f64(dx) - want)
    assert np.isfinite(f64(dx)).all()
    assert (off <= ref.rounded(want, dtype) + slack * (1 + ref.HALF_STEP[dtype])).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows", [3, 100])
@pytest.mark.parametrize("cols", [7, 300, 1500, 2050, 8192, 12800, 16384, 16391, 20000])
def test_row_sums_beyond_fp32(torch, cols, rows, dtype):
    """Terms of 2^123 and more of one sign in a row: 2^128 is passed from 32 columns on.  Rows take turns in their sign, so that
    the gain's sums over rows, which are of FP32, stay in range."""
    from paper_2010_11305_amd import rmsnorm

    r = np.random.default_rng(cols + rows)
    sign = np.where(r.random((rows, cols)) < 0.5, -1.0, 1.0)
    x = sign * (1 + 0.2 * r.random((rows, cols)))
    dy = sign * np.where(np.arange(rows) % 2, -1.0, 1.0)[:, None] * 2.0**123 * (1 + 0.5 * r.random((rows, cols)))
    t = lambda v: torch.from_numpy(v).to(DTYPES[dtype]).cuda()  # noqa: E731
    x, dy, dh = t(x), t(dy), t(r.standard_normal((rows, cols)) * 2.0**120)
    gain = torch.from_numpy(1 + 0.2 * r.random(cols)).float().cuda()
    _, h, inverse = rmsnorm.norm_train(x, gain, eps=EPS)
    n, _ = ref.norm(f64(h), 1.0, EPS)
    for past in (None, dh):
        dx, dgain = rmsnorm.backward(dy, h, inverse, gain, dh=past)
        check(dx, dy, h, gain, past, dtype)
        assert (np.abs(f64(dgain) - (f64(dy) * n).sum(0)) <= 264 * U * np.abs(f64(dy) * n).sum(0)).all()
        dx, _ = rmsnorm.backward(dy, h, inverse, None, dh=past)
        check(dx, dy, h, torch.ones_like(gain), past, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (5, 31), (9, 416), (33, 1029), (3, 4100), (1100, 2049), (130, 16384), (3, 16391), (2, 70001)])
def test_the_mean_has_its_terms_error(torch, rows, cols, dtype):
    from paper_2010_11305_amd import rmsnorm

    r = np.random.default_rng(rows * 31 + cols)
    t = lambda s: torch.from_numpy(r.standard_normal((rows, cols)) * s).to(DTYPES[dtype]).cuda()  # noqa: E731
    x, dy, dh = t(1.0), t(0.1), t(0.1)
    gain = torch.from_numpy(1 + 0.3 * r.standard_normal(cols)).float().cuda()
    _, h, inverse = rmsnorm.norm_train(x, gain, eps=EPS)
    dx, _ = rmsnorm.backward(dy, h, inverse, gain, dh=dh)
    check(dx, dy, h, gain, dh, dtype)
