"""The root-mean-square norm against its formula in 64 bits: types, widths from one column to rows that no register
holds, residuals, strides, work in place, 8 bits, gradients (against the formula's and against differences), values
that are not finite, graphs and streams."""
import numpy as np
import pytest

import layers_ref as ref
from layers_ref import DTYPES, U, f64

pytestmark = pytest.mark.gpu
EPS = 1e-6
SIZES = [(1, 1), (3, 2), (1, 8), (5, 31), (2, 64), (7, 416), (4, 513), (33, 1029), (2, 2048), (3, 2049), (2, 4100), (2, 8192), (2, 8200),
         (1, 12800), (2, 16384), (2, 16391), (1, 70001), (700, 40), (1000, 257)]


@pytest.fixture(scope="module")
def torch():
    import torch as t
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2010_11305_amd import dense_lib
    dense_lib.load()
    return t


def inputs(torch, rows, cols, dtype, seed=0, gain_dtype=None):
    r = np.random.default_rng(seed + rows * 7919 + cols)

    def matrix(scale=1.0):
        v = r.standard_normal((rows, cols)) * scale * np.exp2(r.integers(-6, 7, (rows, 1)))
        return torch.from_numpy(v).to(DTYPES[dtype]).cuda()

    gain = torch.from_numpy(1 + 0.3 * r.standard_normal(cols)).to(DTYPES[gain_dtype or "fp32"]).cuda()
    return matrix(), matrix(), gain, matrix(0.01), matrix(0.01)


def summed(x, r):
    """x + r of their type, as FP32 adds and the type rounds."""
    return (x.float() + r.float()).to(x.dtype)


def check_y(y, h, gain, dtype):
    """inverse is rounded once, and two products follow: 3 roundings of FP32 and that of the type."""
    want, _ = ref.norm(f64(h), f64(gain) if gain is not None else 1.0, EPS)
    off = np.abs(f64(y) - want)
    assert (off <= ref.rounded(want, dtype) + 3.01 * U * np.abs(want) * (1 + ref.HALF_STEP[dtype])).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward(torch, rows, cols, dtype):
    from paper_2010_11305_amd import rmsnorm

    x, r, gain, _, _ = inputs(torch, rows, cols, dtype)
    y, h = rmsnorm.norm(x, gain, residual=r, eps=EPS)
    assert torch.equal(h, summed(x, r))
    check_y(y, h, gain, dtype)
    y, h, inverse = rmsnorm.norm_train(x, gain, eps=EPS)
    assert h is x
    check_y(y, x, gain, dtype)
    want = ref.norm(f64(x), 1.0, EPS)[1][:, 0]
    assert (np.abs(f64(inverse) - want) <= 1.01 * U * want).all()
    check_y(rmsnorm.norm(x, eps=EPS)[0], x, None, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,cols", [(9, 416), (3, 8200), (2, 17000)])
def test_gain_of_the_type(torch, rows, cols, dtype):
    from paper_2010_11305_amd import rmsnorm

    x, r, gain, dy, dh = inputs(torch, rows, cols, dtype, gain_dtype=dtype)
    y, h, inverse = rmsnorm.norm_train(x, gain, residual=r, eps=EPS)
    check_y(y, h, gain, dtype)
    dx, dgain = rmsnorm.backward(dy, h, inverse, gain, dh=dh)
    check_gradients(dx, dgain, dy, h, gain, dh, dtype, dtype)


def check_gradients(dx, dgain, dy, h, gain, dh, dtype, gain_dtype="fp32"):
    """Roundings of FP32: dn one, n two; the row's mean takes products of those (4) and sums of at most 80 terms in
    FP32; then four operations and the type.  The gain's: products of 4 roundings, sums of at most 256 rows."""
    D, H, G = f64(dy), f64(h), f64(gain) if gain is not None else np.ones(h.shape[1])
    want, wg, along = ref.norm_gradients(D, H, G, EPS)
    n, inverse = ref.norm(H, 1.0, EPS)
    size = (np.abs(D * G) + np.abs(n) * along) * inverse
    extra = 0.0 if dh is None else f64(dh)
    want = want + extra
    slack = U * (8 * size + 90 * np.abs(n) * along * inverse + np.abs(extra) + np.abs(want))
    off = np.abs(f64(dx) - want)
    assert (off <= ref.rounded(want, dtype) + slack * (1 + ref.HALF_STEP[dtype])).all(), off.max()
    if gain is None:
        assert dgain is None
        return
    assert dgain.dtype == gain.dtype
    magnitude = np.abs(D * n).sum(0)
    assert (np.abs(f64(dgain) - wg) <= 264 * U * magnitude + ref.rounded(wg, gain_dtype)).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_backward(torch, rows, cols, dtype):
    from paper_2010_11305_amd import rmsnorm

    x, r, gain, dy, dh = inputs(torch, rows, cols, dtype)
    _, h, inverse = rmsnorm.norm_train(x, gain, residual=r, eps=EPS)
    dx, dgain = rmsnorm.backward(dy, h, inverse, gain, dh=dh)
    check_gradients(dx, dgain, dy, h, gain, dh, dtype)
    dx, dgain = rmsnorm.backward(dy, h, inverse, gain)
    check_gradients(dx, dgain, dy, h, gain, None, dtype)
    dx, none = rmsnorm.backward(dy, h, inverse)
    check_gradients(dx, none, dy, h, None, None, dtype)


def test_backward_over_many_rows(torch):
    """Rows of several slabs, few columns: the partial sums' join."""
    from paper_2010_11305_amd import rmsnorm

    for rows, cols in ((20000, 24), (5000, 600), (257, 3)):
        x, _, gain, dy, _ = inputs(torch, rows, cols, "fp32", 5)
        _, h, inverse = rmsnorm.norm_train(x, gain, eps=EPS)
        dx, dgain = rmsnorm.backward(dy, h, inverse, gain)
        check_gradients(dx, dgain, dy, h, gain, None, "fp32")
        again = rmsnorm.backward(dy, h, inverse, gain)
        assert torch.equal(dx, again[0]) and torch.equal(dgain, again[1])


@pytest.mark.parametrize("dtype,rows,cols", [("bf16", 17, 2048), ("fp16", 40, 8), ("fp32", 33, 16383), ("bf16", 257, 8160), ("fp32", 1024, 1024),
                                             ("fp32", 1024, 1028), ("bf16", 1024, 29), ("bf16", 1025, 29), ("fp16", 1023, 2049)])
def test_backward_of_few_rows(torch, dtype, rows, cols):
    """Both sides of the rule by which both gradients go in one launch; results do not depend on where dx lies."""
    from paper_2010_11305_amd import rmsnorm

    x, _, gain, dy, dh = inputs(torch, rows, cols, dtype, 6, gain_dtype=dtype)
    _, h, inverse = rmsnorm.norm_train(x, gain, eps=EPS)
    dx, dgain = rmsnorm.backward(dy, h, inverse, gain.float(), dh=dh)
    check_gradients(dx, dgain, dy, h, gain.float(), dh, dtype)
    for over in range(3):
        t = [v.clone() for v in (dy, h, dh)]
        got = rmsnorm.backward(t[0], t[1], inverse, gain, dh=t[2], out=t[over])
        assert torch.equal(got[0], dx) and torch.equal(got[1], dgain.to(gain.dtype))
    wide = torch.full((rows, cols + 5), 7.0, dtype=x.dtype, device="cuda")
    got = rmsnorm.backward(dy, h, inverse, gain, dh=dh, out=wide[:, 2:-3])
    assert torch.equal(wide[:, 2:-3], dx) and (wide[:, :2] == 7).all() and (wide[:, -3:] == 7).all()


def test_gradients_against_differences(torch):
    """Central differences of sum(w y) in 64 bits around FP32 inputs: steps of 2^-10 of values near 1 leave an error of
    their square, 2^-20, times third derivatives of a few units."""
    from paper_2010_11305_amd import rmsnorm

    r = np.random.default_rng(4)
    x, g, w = r.standard_normal((3, 37)), 1 + 0.3 * r.standard_normal(37), r.standard_normal((3, 37))
    x, g, w = (v.astype(np.float32).astype(np.float64) for v in (x, g, w))
    t = lambda v: torch.from_numpy(v).float().cuda()  # noqa: E731
    _, h, inverse = rmsnorm.norm_train(t(x), t(g), eps=EPS)
    dx, dgain = rmsnorm.backward(t(w), h, inverse, t(g))
    f = lambda x, g: (w * ref.norm(x, g, EPS)[0]).sum()  # noqa: E731
    for got, of in ((f64(dx), 0), (f64(dgain), 1)):
        base = [x, g]
        for i in np.ndindex(*base[of].shape):
            up, down = [v.copy() for v in base], [v.copy() for v in base]
            up[of][i] += 2.0**-10
            down[of][i] -= 2.0**-10
            assert abs((f(*up) - f(*down)) * 2.0**9 - got[i]) < 1e-4


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_in_8_bits(torch, rows, cols, dtype):
    """v carries 3 roundings of FP32, the scale those and one division, the reciprocal and the product two more: 9 of
    at most 127 units, below 1e-4."""
    from paper_2010_11305_amd import rmsnorm

    x, r, gain, _, _ = inputs(torch, rows, cols, dtype, 1)
    for residual in (None, r):
        q, h = rmsnorm.norm8(x, gain, residual=residual, eps=EPS)
        assert q.shape == (rows, cols) and torch.equal(h, x if residual is None else summed(x, r))
        v, _ = ref.norm(f64(h), f64(gain), EPS)
        scale = np.abs(v).max(1) / 127
        assert (np.abs(f64(q.scales) - scale) <= 5 * U * scale).all()
        code = f64(q.codes)
        assert (np.abs(code - v / scale[:, None]) <= 0.5 + 1e-4).all() and (np.abs(code).max(1) == 127).all()
        for name, t in DTYPES.items():
            want = code * f64(q.scales)[:, None]
            assert (np.abs(f64(q.dequantize(t)) - want) <= ref.rounded(want, name) + U * np.abs(want) * (1 + ref.HALF_STEP[name])).all()


def test_extreme_rows(torch):
    """Zeros, values whose squares leave FP32 either way, subnormal ones."""
    from paper_2010_11305_amd import rmsnorm

    for cols in (40, 3000, 20000):
        x = torch.zeros((6, cols), device="cuda")
        x[1], x[2, 3], x[3], x[4] = 3e30, 1e38, 1e-30, 1e-41
        x[5, ::2], x[5, 1::2] = 3e38, -3e38
        y, _, inverse = rmsnorm.norm_train(x, eps=1e-12)
        want, wi = ref.norm(f64(x), 1.0, 1e-12)
        eps32 = float(np.float32(1e-12))
        want, wi = ref.norm(f64(x), 1.0, eps32)
        assert (np.abs(f64(inverse) - wi[:, 0]) <= 1.01 * U * wi[:, 0] + 2.0**-149).all()
        # inverse may be subnormal (rms above 2^126): the error of its last bit grows with h
        assert (np.abs(f64(y) - want) <= 4 * U * np.abs(want) + np.abs(f64(x)) * 2.0**-149 + 2.0**-149).all()
        q, _ = rmsnorm.norm8(x, eps=1e-12)
        assert (q.codes[0] == 0).all() and q.scales[0] == 2.0**-126
        assert (q.codes[1] == 127).all() and q.codes[2, 3] == 127
        assert torch.isfinite(q.dequantize()).all()


def test_values_that_are_not_finite(torch):
    """Only their own rows are spoilt; in 8 bits a row stands for NaN as a whole."""
    from paper_2010_11305_amd import rmsnorm

    for cols in (33, 1500, 17000):
        x = torch.randn((5, cols), device="cuda")
        x[1, 5], x[3, cols - 1] = float("nan"), float("inf")
        gain = torch.ones(cols, device="cuda")
        y, h, inverse = rmsnorm.norm_train(x, gain)
        assert torch.isnan(y[1]).all() and torch.isnan(y[3, cols - 1]) and (y[3, : cols - 1] == 0).all()
        fine = [0, 2, 4]
        assert torch.equal(y[fine], rmsnorm.norm(x[fine].contiguous(), gain)[0])
        q, _ = rmsnorm.norm8(x, gain)
        assert torch.isnan(q.dequantize()[[1, 3]]).all() and (q.codes[[1, 3]] == 0).all()
        assert torch.equal(q.codes[fine], rmsnorm.norm8(x[fine].contiguous(), gain)[0].codes)
        dx, dgain = rmsnorm.backward(torch.ones_like(x), h, inverse, gain)
        assert torch.isfinite(dx[fine]).all() and torch.isnan(dgain[5])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("cols", [100, 1029, 4097, 16500])
def test_strides_and_odd_addresses(torch, cols, dtype):
    """Rows inside wider matrices, from an odd element on; what lies between them is left as it was."""
    from paper_2010_11305_amd import rmsnorm

    x, r, gain, dy, dh = inputs(torch, 6, cols, dtype, 2)

    def inside(t, start, pad):
        wide = torch.full((6, cols + pad), 7.0, dtype=t.dtype, device="cuda")
        v = wide[:, start:start + cols]
        v.copy_(t)
        return v, wide

    def untouched(wide, start):
        return bool((wide[:, :start] == 7).all() and (wide[:, start + cols:] == 7).all())

    y, h, inverse = rmsnorm.norm_train(x, gain, residual=r, eps=EPS)
    dx, dgain = rmsnorm.backward(dy, h, inverse, gain, dh=dh)
    (xv, _), (rv, _), (yv, yw), (hv, hw) = inside(x, 1, 3), inside(r, 3, 9), inside(x, 1, 2), inside(x, 5, 6)
    out = rmsnorm.norm_train(xv, gain, residual=rv, eps=EPS, out=yv, sum_out=hv)
    assert torch.equal(yv, y) and torch.equal(hv, h) and torch.equal(out[2], inverse) and untouched(yw, 1) and untouched(hw, 5)
    (dyv, _), (dhv, _), (dxv, dxw) = inside(dy, 3, 4), inside(dh, 1, 1), inside(dy, 7, 8)
    got = rmsnorm.backward(dyv, hv, inverse, gain, dh=dhv, out=dxv)
    assert torch.equal(dxv, dx) and torch.equal(got[1], dgain) and untouched(dxw, 7)
    assert torch.equal(rmsnorm.norm8(xv, gain, residual=rv, eps=EPS)[0].codes, rmsnorm.norm8(x, gain, residual=r, eps=EPS)[0].codes)
    # the gain at an odd element
    g = torch.zeros(cols + 1, device="cuda")[1:]
    g.copy_(gain)
    assert torch.equal(rmsnorm.norm(x, g, residual=r, eps=EPS)[0], y)


@pytest.mark.parametrize("cols", [96, 1500, 9000, 17000])
def test_in_place(torch, cols):
    from paper_2010_11305_amd import rmsnorm

    x, r, gain, dy, dh = inputs(torch, 5, cols, "bf16", 3)
    y, h, inverse = rmsnorm.norm_train(x, gain, residual=r)
    for over_y, over_h in (("x", "r"), ("r", "x"), ("x", None), (None, "r")):
        t = {"x": x.clone(), "r": r.clone(), None: None}
        got = rmsnorm.norm(t["x"], gain, residual=t["r"], out=t[over_y], sum_out=t[over_h])
        assert torch.equal(got[0], y) and torch.equal(got[1], h)
    q, _ = rmsnorm.norm8(x, gain, residual=r)
    for over in (0, 1):
        t = [x.clone(), r.clone()]
        got, sum_out = rmsnorm.norm8(t[0], gain, residual=t[1], sum_out=t[over])
        assert sum_out is t[over] and torch.equal(sum_out, h) and torch.equal(got.codes, q.codes) and torch.equal(got.scales, q.scales)
    dx, dgain = rmsnorm.backward(dy, h, inverse, gain, dh=dh)
    for over in range(3):
        t = [v.clone() for v in (dy, h, dh)]
        got = rmsnorm.backward(t[0], t[1], inverse, gain, dh=t[2], out=t[over])
        assert torch.equal(got[0], dx) and torch.equal(got[1], dgain) and got[0] is t[over]
    both = torch.randn((5, 2 * cols), device="cuda")
    with pytest.raises(Exception, match="emb_rmsnorm_forward"):
        rmsnorm.norm(both[:, :cols], out=both[:, 1:cols + 1])
    rmsnorm.norm(both[:, :cols], out=both[:, cols:])    # beside each other


def test_no_rows(torch):
    from paper_2010_11305_amd import rmsnorm

    x, gain = torch.zeros((0, 40), device="cuda"), torch.ones(40, device="cuda")
    y, h, inverse = rmsnorm.norm_train(x, gain)
    assert y.shape == (0, 40) and inverse.shape == (0,)
    dx, dgain = rmsnorm.backward(x, h, inverse, gain)
    assert dx.shape == (0, 40) and (dgain == 0).all()
    assert rmsnorm.norm8(x, gain)[0].dequantize().shape == (0, 40)


def test_refusals(torch):
    from paper_2010_11305_amd import rmsnorm

    x, g = torch.zeros((4, 40), device="cuda"), torch.ones(40, device="cuda")
    for bad in (lambda: rmsnorm.norm(x.t()), lambda: rmsnorm.norm(x.cpu()), lambda: rmsnorm.norm(x, g[:39]), lambda: rmsnorm.norm(x, g.bfloat16()),
                lambda: rmsnorm.norm(x, g, residual=x[:3]), lambda: rmsnorm.norm(x, g, residual=x.half()), lambda: rmsnorm.norm(x, sum_out=x),
                lambda: rmsnorm.norm(x, out=x.half()), lambda: rmsnorm.norm(x, residual=x, sum_out=x.half()), lambda: rmsnorm.norm(x.double()),
                lambda: rmsnorm.backward(x, x, torch.ones(3, device="cuda"), g), lambda: rmsnorm.backward(x, x[:3], torch.ones(4, device="cuda"), g),
                lambda: rmsnorm.backward(x, x, torch.ones(4, device="cuda"), g, dh=x.half()),
                lambda: rmsnorm.Rows8(x, g), lambda: rmsnorm.Rows8(x.to(torch.int8), torch.ones(3, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: rmsnorm.norm(x, eps=0.0), lambda: rmsnorm.norm(x, eps=float("nan")), lambda: rmsnorm.norm(x[:, :0])):
        with pytest.raises(Exception, match="emb_rmsnorm_forward"):
            bad()


def test_written_tensors_count_as_changed(torch):
    from paper_2010_11305_amd import rmsnorm

    for call in (lambda o, x: rmsnorm.norm(x, out=o), lambda o, x: rmsnorm.norm(x, residual=x, sum_out=o), lambda o, x: rmsnorm.norm8(x, residual=x, sum_out=o),
                 lambda o, x: rmsnorm.backward(x, x, torch.ones(4, device="cuda"), out=o)):
        o, x = torch.zeros(4, 40, device="cuda"), torch.ones(4, 40, device="cuda")
        z = (torch.ones_like(o, requires_grad=True) * o).sum()
        call(o, x)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            z.backward()


def test_graph_and_streams(torch):
    """Captured once and replayed with new inputs, with eager work between; and on a stream of its own."""
    from paper_2010_11305_amd import rmsnorm

    for rows, cols in ((3, 40), (300, 1029), (2, 17000)):
        x, r, gain, dy, dh = inputs(torch, rows, cols, "bf16", 6)

        def step():
            y, h, inverse = rmsnorm.norm_train(x, gain, residual=r)
            return (y, h, *rmsnorm.backward(dy, h, inverse, gain, dh=dh), rmsnorm.norm8(x, gain, residual=r)[0].dequantize())

        step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            held = step()
        for k in range(3):
            x.copy_(torch.randn_like(x))
            g.replay()
            for a, b in zip(held, step()):
                assert torch.equal(a, b)
            torch.cuda.synchronize()
        want = step()
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got = step()
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
