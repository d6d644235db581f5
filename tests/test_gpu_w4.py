"""4-bit weights with group scales against numpy in 64 bits: quantisation bit for bit, the plain form and back, expansion, and
products of one row to many with every type of rows, group and ragged size."""
import numpy as np
import pytest

import layers_ref as ref
from layers_ref import DTYPES, U, f64

pytestmark = pytest.mark.gpu
GROUPS = (32, 64, 128)
SHAPES = [(1, 1), (3, 31), (16, 128), (17, 129), (5, 33), (40, 416), (33, 1000), (2, 4100), (100, 257)]


@pytest.fixture(scope="module")
def torch():
    import torch as t
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2010_11305_amd import dense_lib
    dense_lib.load()
    return t


def weight(n, k, seed=0):
    r = np.random.default_rng(seed + 31 * n + k)
    w = r.standard_normal((n, k)) * np.exp2(r.integers(-4, 5, (n, 1)))
    w[r.random((n, k)) < 0.02] *= 20
    w[n // 2, : k // 2] = 0.75           # groups without a range
    return w


def plain(w):
    codes, scales, biases = (t.cpu().numpy() for t in w.to_codes())
    return codes, scales, biases


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("group", GROUPS)
@pytest.mark.parametrize("n,k", SHAPES)
def test_quantisation(torch, n, k, group, dtype):
    """Every code, scale and bias, and the values they stand for (one FP32 sum of an exact product)."""
    from paper_2010_11305_amd import w4

    x = torch.from_numpy(weight(n, k)).to(DTYPES[dtype]).cuda()
    q = w4.quantize(x, group)
    want = ref.w4_quantize(x.float().cpu().numpy(), group)
    codes, scales, biases = plain(q)
    assert np.array_equal(codes, ref.pack(want[0]))
    assert np.array_equal(scales.view(np.uint16), want[1].view(np.uint16)) and np.array_equal(biases.view(np.uint16), want[2].view(np.uint16))
    values = ref.w4_values(*want, group)
    for name, t in DTYPES.items():
        got = f64(q.dequantize(t))
        assert (np.abs(got - values) <= U * np.abs(values) * (1 + ref.HALF_STEP[name]) + ref.rounded(values, name)).all()
    assert torch.equal(q.dequantize(torch.float32), torch.from_numpy(values).float().cuda())


@pytest.mark.parametrize("group", GROUPS)
@pytest.mark.parametrize("n,k", SHAPES + [(31, 7)])
def test_plain_form_and_back(torch, n, k, group):
    """Any codes, scales and biases; what pads the buffer is 0 whatever was there."""
    from paper_2010_11305_amd import w4

    r = np.random.default_rng(n * k + group)
    codes, groups = r.integers(0, 16, (n, k), dtype=np.uint8), -(-k // group)
    scales, biases = (r.standard_normal((n, groups)).astype(np.float16) for _ in range(2))
    packed = ref.pack(codes)
    if k % 2:
        packed[:, -1] |= 0xF0            # a half byte that is no column's
    t = [torch.from_numpy(v).cuda() for v in (packed, scales, biases)]
    q = w4.W4Matrix(n, k, group)
    q.data.fill_(255)
    w4.from_codes(*t, k, group, out=q)
    back = plain(q)
    assert np.array_equal(back[0], ref.pack(codes)) and np.array_equal(back[1], scales) and np.array_equal(back[2], biases)
    data = q.data.cpu().numpy()
    rt, kt = -(-n // 16), -(-k // 128)
    want = np.zeros((rt, kt, 4, 16, 4), np.uint32)      # dwords: row tile, column tile, b, r, i
    for row in range(n):
        for c in range(k):
            j = c % 8
            want[row // 16, c // 128, c // 8 % 4, row % 16, c // 32 % 4] |= np.uint32(codes[row, c]) << (8 * j if j < 4 else 8 * (j - 4) + 4)
    assert np.array_equal(data[: want.nbytes].view(np.uint32), want.ravel())
    pairs = np.zeros((rt, kt * 128 // group, 16, 2), np.float16)
    for row in range(n):
        pairs[row // 16, :groups, row % 16, 0], pairs[row // 16, :groups, row % 16, 1] = scales[row], biases[row]
    assert np.array_equal(data[want.nbytes:].view(np.float16), pairs.ravel()) and len(data) == want.nbytes + pairs.nbytes


def test_extreme_groups(torch):
    """Constants, subnormal scales, zeros of both signs, and groups that FP16 or FP32 do not hold."""
    from paper_2010_11305_amd import w4

    x = np.random.default_rng(0).standard_normal((8, 256)).astype(np.float32)
    x[0], x[1], x[2] = 0.0, -0.0, 3e-8
    x[3, 5], x[4, 200], x[5, 100], x[6, 0] = np.nan, np.inf, -65520.0, 65519.0
    x[7] *= 1e-6
    for group in GROUPS:
        want = ref.w4_quantize(x, group)
        q = w4.quantize(torch.from_numpy(x).cuda(), group)
        codes, scales, biases = plain(q)
        for got, w in ((scales, want[1]), (biases, want[2])):
            assert np.array_equal(got, w, equal_nan=True)
        assert np.array_equal(codes, ref.pack(want[0]))
        v = q.dequantize().cpu().numpy()
        at = [np.arange(256) // group == c // group for c in (5, 200, 100)]
        for row, spoilt in zip((3, 4, 5), at):
            assert np.isnan(v[row, spoilt]).all() and np.isfinite(v[row, ~spoilt]).all()
        assert np.isfinite(v[[0, 1, 2, 6, 7]]).all()


def rows_of(torch, m, k, dtype, seed=0):
    """(what linear takes, its values in 64 bits)"""
    from paper_2010_11305_amd.rmsnorm import Rows8

    r = np.random.default_rng(seed + m * 131 + k)
    if dtype == "int8":
        codes, scales = r.integers(-127, 128, (m, k)).astype(np.int8), np.exp2(r.uniform(-6, 2, m)).astype(np.float32)
        return Rows8(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()), codes * scales.astype(np.float64)[:, None]
    x = torch.from_numpy(r.standard_normal((m, k)) * np.exp2(r.integers(-4, 5, (m, 1))) + 0.5).to(DTYPES[dtype]).cuda()
    return x, f64(x)


def check(torch, y, X, parts, group, dtype, y_name, bias=None, relu=False):
    """Products are exact.  Their sums: an FP32 addition a product (three for FP32 rows, which are split in three),
    none inside a group of 8-bit rows, and two a group; none is off by more than 2^-23 of the magnitudes summed."""
    codes, scales, biases = parts
    k = codes.shape[1]
    want = X @ ref.w4_values(codes, scales, biases, group).T
    adds = 2 * -(-k // group) + 40 + (0 if dtype == "int8" else 3 * k if dtype == "fp32" else k)
    slack = adds * 2.0**-23 * 1.01 * ref.w4_magnitudes(X, codes, scales, biases, group)
    if bias is not None:
        want = want + bias
        slack = slack + U * (np.abs(want) + np.abs(bias))
    if relu:
        want = np.maximum(want, 0)
    got = f64(y)
    if y_name == "fp16":      # from 65520 on, halfway to 2^16, a value rounds to infinity
        beyond = np.abs(want) - slack >= 65520
        assert np.array_equal(got[beyond], np.copysign(np.inf, want[beyond]))
        edge = np.isinf(got) & (np.abs(want) + slack >= 65520)
        got = np.where(edge, want, got)
    assert (np.abs(got - want) <= slack * (1 + ref.HALF_STEP[y_name]) + ref.rounded(want, y_name)).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16", "int8"])
@pytest.mark.parametrize("group", GROUPS)
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 16, 128), (2, 40, 416), (7, 33, 1000), (16, 17, 129), (17, 100, 257), (33, 16, 300), (64, 130, 640),
                                   (65, 20, 31), (130, 48, 520), (1, 700, 4100), (5, 2100, 96), (20, 1040, 2100)])
def test_products(torch, m, n, k, group, dtype):
    from paper_2010_11305_amd import w4

    parts = ref.w4_quantize(weight(n, k, 1), group)
    w = w4.from_codes(*(torch.from_numpy(v).cuda() for v in (ref.pack(parts[0]), *parts[1:])), k, group)
    x, X = rows_of(torch, m, k, dtype)
    b = torch.from_numpy(np.random.default_rng(m).standard_normal(n)).float().cuda()
    y_names = ["fp32", "bf16"] if dtype == "int8" else [dtype]
    for name in y_names:
        y = w4.linear(x, w, dtype=DTYPES[name])
        assert y.shape == (m, n) and y.dtype == DTYPES[name]
        check(torch, y, X, parts, group, dtype, name)
        check(torch, w4.linear(x, w, bias=b, dtype=DTYPES[name]), X, parts, group, dtype, name, f64(b))
        check(torch, w4.linear(x, w, bias=b, relu=True, dtype=DTYPES[name]), X, parts, group, dtype, name, f64(b), True)
        assert torch.equal(y, w4.linear(x, w, dtype=DTYPES[name]))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16", "int8"])
def test_exact_products(torch, dtype):
    """Small whole numbers, of which every sum is exact: each element, every column's place and every row."""
    from paper_2010_11305_amd import w4
    from paper_2010_11305_amd.rmsnorm import Rows8

    r = np.random.default_rng(2)
    for m, n, k, group in ((3, 50, 700, 32), (20, 35, 390, 64), (70, 64, 1000, 128), (1, 1, 5, 128)):
        codes, groups = r.integers(0, 16, (n, k), dtype=np.uint8), -(-k // group)
        scales, biases = r.integers(1, 4, (n, groups)).astype(np.float16), r.integers(-20, 1, (n, groups)).astype(np.float16)
        w = w4.from_codes(*(torch.from_numpy(v).cuda() for v in (ref.pack(codes), scales, biases)), k, group)
        X = r.integers(-8, 9, (m, k))
        x = torch.from_numpy(X).cuda()
        x = Rows8(x.to(torch.int8), torch.full((m,), 0.5, device="cuda")) if dtype == "int8" else x.to(DTYPES[dtype])
        want = X @ ref.w4_values(codes, scales, biases, group).T * (0.5 if dtype == "int8" else 1.0)
        assert np.array_equal(f64(w4.linear(x, w, dtype=torch.float32)), want)


def test_fp32_rows_keep_all_their_bits(torch):
    """One column, a code of 1, scale 1 and bias 0: y is x, bit for bit."""
    from paper_2010_11305_amd import w4

    codes, one, zero = torch.ones((1, 1), dtype=torch.uint8, device="cuda"), torch.ones((1, 1), device="cuda").half(), torch.zeros((1, 1), device="cuda").half()
    w = w4.from_codes(codes, one, zero, 1, 32)
    x = torch.randn((64, 1), device="cuda") * torch.exp2(torch.randint(-90, 90, (64, 1), device="cuda").float())
    assert torch.equal(w4.linear(x, w), x)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "int8"])
def test_strides_and_odd_addresses(torch, dtype):
    from paper_2010_11305_amd import w4
    from paper_2010_11305_amd.rmsnorm import Rows8

    for m, n, k in ((5, 37, 301), (40, 100, 530)):
        w = w4.quantize(torch.from_numpy(weight(n, k)).float().cuda(), 64)
        x, _ = rows_of(torch, m, k, dtype)
        y = w4.linear(x, w, dtype=torch.bfloat16)
        t = x.codes if dtype == "int8" else x
        wide = torch.full((m, k + 6), 100, dtype=t.dtype, device="cuda") if dtype == "int8" else torch.full((m, k + 6), float("nan"), dtype=t.dtype, device="cuda")
        v = wide[:, 3:3 + k]
        v.copy_(t)
        v = Rows8(v, x.scales) if dtype == "int8" else v
        out = torch.full((m, n + 5), 7.0, dtype=torch.bfloat16, device="cuda")
        w4.linear(v, w, out=out[:, 1:n + 1])
        assert torch.equal(out[:, 1:n + 1], y) and (out[:, 0] == 7).all() and (out[:, n + 1:] == 7).all()
    x = torch.from_numpy(weight(9, 200)).float().cuda()
    wide = torch.zeros((9, 207), device="cuda")
    wide[:, 5:205].copy_(x)
    assert torch.equal(w4.quantize(wide[:, 5:205], 32).data, w4.quantize(x, 32).data)
    w4.quantize(x, 32).dequantize(out=wide[:, 3:203])
    assert torch.equal(wide[:, 3:203], w4.quantize(x, 32).dequantize()) and (wide[:, :3] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_subnormal_rows(torch, dtype):
    """One column, a code of 1, scale 1 and bias 0, by both routes: values below the normal numbers arrive as they are."""
    from paper_2010_11305_amd import w4

    least = {"bf16": -133, "fp16": -24}[dtype]
    for m, n, k in ((16, 1, 1), (16, 20, 8200)):
        codes, scales = torch.zeros((n, -(-k // 2)), dtype=torch.uint8, device="cuda"), torch.ones((n, -(-k // 32)), device="cuda").half()
        codes[:, 0] = 1
        w = w4.from_codes(codes, scales, torch.zeros_like(scales), k, 32)
        x = torch.zeros((m, k), dtype=DTYPES[dtype], device="cuda")
        x[:, 0] = torch.tensor([(1 + e % 7) * 2.0 ** (least + e // 2) for e in range(m)], dtype=torch.float64).to(x.dtype)
        assert (x[:, 0] != 0).all()
        assert torch.equal(w4.linear(x, w, dtype=torch.float32), x[:, :1].float().expand(m, n))


def test_rows_that_are_not_finite(torch):
    """They spoil their own outputs alone, also where the activation follows; a row in 8 bits whose scale is NaN too."""
    from paper_2010_11305_amd import rmsnorm, w4

    w = w4.quantize(torch.from_numpy(weight(40, 500)).float().cuda(), 64)
    for m in (3, 30):
        for dt in DTYPES.values():
            x = torch.randn((m, 500), device="cuda").to(dt)
            fine = w4.linear(x, w, relu=True)
            x[1, 499], x[2, 7] = float("nan"), float("inf")
            y = w4.linear(x, w, relu=True)
            assert torch.isnan(y[1]).all() and not torch.isfinite(y[2]).all()
            keep = [i for i in range(m) if i not in (1, 2)]
            assert torch.equal(y[keep], fine[keep])
        q, _ = rmsnorm.norm8(x)
        assert torch.isnan(w4.linear(q, w, relu=True)[1:3]).all() and torch.isfinite(w4.linear(q, w)[keep]).all()


def test_nothing_to_do(torch):
    from paper_2010_11305_amd import w4

    w = w4.quantize(torch.zeros((5, 40), device="cuda"))
    assert w4.linear(torch.zeros((0, 40), device="cuda"), w).shape == (0, 5)
    none = w4.quantize(torch.zeros((0, 40), device="cuda"))
    assert w4.linear(torch.zeros((3, 40), device="cuda"), none).shape == (3, 0)
    empty = w4.quantize(torch.zeros((5, 0), device="cuda"))
    b = torch.tensor([1.0, -1.0, 0.0, 2.0, -2.0], device="cuda")
    for m in (3, 40):
        assert torch.equal(w4.linear(torch.zeros((m, 0), device="cuda"), empty, bias=b, relu=True), b.clamp(min=0).expand(m, 5))


def test_refusals(torch):
    from paper_2010_11305_amd import w4

    x, w = torch.zeros((4, 40), device="cuda"), w4.quantize(torch.zeros((8, 40), device="cuda"), 32)
    codes, scales, biases = w.to_codes()
    for bad in (lambda: w4.linear(x[:, :39], w), lambda: w4.linear(x.t(), w), lambda: w4.linear(x, w, bias=torch.zeros(7, device="cuda")),
                lambda: w4.linear(x, w, bias=torch.zeros(8, device="cuda").half()), lambda: w4.linear(x, w, out=torch.zeros((4, 7), device="cuda")),
                lambda: w4.from_codes(codes, scales[:, :1], biases, 40, 32), lambda: w4.from_codes(codes[:, :19], scales, biases, 40, 32),
                lambda: w4.from_codes(codes, scales.float(), biases, 40, 32), lambda: w4.quantize(x, 32, out=w),
                lambda: w4.quantize(torch.zeros((8, 40), device="cuda"), 64, out=w), lambda: w4.W4Matrix(8, 40, 32, data=w.data[:100])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(Exception, match="emb_w4_query_bytes"):
        w4.quantize(x, 48)
    with pytest.raises(Exception, match="emb_w4_linear"):
        w4.linear(x, w, out=x[:, :8])


def test_written_tensors_count_as_changed(torch):
    from paper_2010_11305_amd import w4

    x = torch.ones(4, 40, device="cuda")
    w = w4.quantize(torch.ones(8, 40, device="cuda"))
    for o, call in ((torch.zeros(4, 8, device="cuda"), lambda o: w4.linear(x, w, out=o)), (torch.zeros(8, 40, device="cuda"), lambda o: w.dequantize(out=o))):
        z = (torch.ones_like(o, requires_grad=True) * o).sum()
        call(o)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            z.backward()


def test_graph_and_streams(torch):
    """Two graphs and eager calls of the same layer, in turn: each call has its own workspace."""
    from paper_2010_11305_amd import rmsnorm, w4

    w = w4.quantize(torch.from_numpy(weight(600, 2000)).float().cuda(), 128)
    b = torch.randn(600, device="cuda")
    graphs = []
    large = w4.quantize(torch.from_numpy(weight(4000, 2000)).float().cuda(), 64)     # of 40 rows, these go through a workspace
    for m in (1, 40):
        x = torch.randn((m, 2000), device="cuda").bfloat16()
        step = lambda x=x: (w4.linear(x, w, bias=b, relu=True), w4.linear(rmsnorm.norm8(x)[0], w), w4.linear(x, large),  # noqa: E731
                            w4.linear(rmsnorm.norm8(x)[0], large))
        step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        graphs.append((g, x, step, out))
    for k in range(3):
        for g, x, step, out in graphs:
            x.copy_(torch.randn_like(x))
            g.replay()
            assert all(torch.equal(a, c) for a, c in zip(out, step()))
        torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = [graphs[1][2]() for _ in range(4)]
    want = [graphs[0][2]() for _ in range(4)]      # at the same time
    torch.cuda.synchronize()
    for (_, _, step, _), calls in zip(graphs, (want, got)):
        expect = step()
        assert all(torch.equal(a, c) for call in calls for a, c in zip(call, expect))


# the largest rows that k_w4_few holds as operands (16 x 2048 in 16 bits) and as FP32 (16 x 2048), and those past them
LARGE = [(16, 40, 2048), (16, 40, 2049), (5, 40, 6500), (16, 20, 4096), (16, 20, 4097), (16, 33, 8200), (16, 8200, 8200), (17, 4000, 2200), (20, 8200, 1200), (40, 3000, 2100), (48, 8177, 700), (64, 2100, 2100), (70, 8200, 520), (7, 50, 4100),
         (200, 1700, 1000), (33, 8209, 1100), (64, 8257, 600), (128, 4193, 1300), (25, 17000, 900), (24, 4113, 1300), (60, 5000, 400)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16", "int8"])
@pytest.mark.parametrize("group", GROUPS)
@pytest.mark.parametrize("m,n,k", LARGE)
def test_exact_products_of_large_ones(torch, m, n, k, group, dtype):
    """The routes of large products (one block of 16 rows to four of them, one row tile of the weight, two and four), of whole numbers
    whose sums stay below 2^24: every element is exact."""
    from paper_2010_11305_amd import w4
    from paper_2010_11305_amd.rmsnorm import Rows8

    g = torch.Generator(device="cuda")
    g.manual_seed(m + n + k + group)
    rand = lambda lo, hi, *shape: torch.randint(lo, hi, shape, generator=g, device="cuda")  # noqa: E731
    groups = -(-k // group)
    codes, scales, biases = rand(0, 16, n, k + k % 2), rand(1, 4, n, groups), rand(-20, 1, n, groups)
    w = w4.from_codes((codes[:, 0::2] + 16 * codes[:, 1::2]).to(torch.uint8), scales.half(), biases.half(), k, group)
    at = torch.arange(k, device="cuda") // group
    W = (codes[:, :k] * scales[:, at] + biases[:, at]).double()
    X = rand(-8, 9, m, k)
    x = Rows8(X.to(torch.int8), torch.full((m,), 0.5, device="cuda")) if dtype == "int8" else X.to(DTYPES[dtype])
    want = X.double() @ W.t() * (0.5 if dtype == "int8" else 1.0)
    out = torch.full((m, n + 3), 7.0, device="cuda")
    w4.linear(x, w, out=out[:, 1:n + 1])
    assert torch.equal(out[:, 1:n + 1].double(), want) and (out[:, 0] == 7).all() and (out[:, n + 1:] == 7).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "int8"])
def test_large_products(torch, dtype):
    """Values of all magnitudes through the same routes, with bias and activation; what is not finite stays in its row."""
    from paper_2010_11305_amd import w4
    from paper_2010_11305_amd.rmsnorm import Rows8

    for m, n, k, group in ((16, 300, 8200, 64), (33, 2500, 2200, 32), (64, 8200, 700, 128)):
        parts = ref.w4_quantize(weight(n, k, 3), group)
        w = w4.from_codes(*(torch.from_numpy(v).cuda() for v in (ref.pack(parts[0]), *parts[1:])), k, group)
        x, X = rows_of(torch, m, k, dtype, 9)
        b = torch.from_numpy(np.random.default_rng(m).standard_normal(n)).float().cuda()
        y = w4.linear(x, w, bias=b, relu=True, dtype=torch.float32)
        check(torch, y, X, parts, group, dtype, "fp32", f64(b), True)
        wide = torch.zeros((m, k + 5), dtype=(x.codes if dtype == "int8" else x).dtype, device="cuda")
        wide[:, 3:k + 3].copy_(x.codes if dtype == "int8" else x)
        inside = wide[:, 3:k + 3]
        again = w4.linear(Rows8(inside, x.scales) if dtype == "int8" else inside, w, bias=b, relu=True, dtype=torch.float32)
        assert torch.equal(again, y)
        if dtype == "int8":
            x.scales[2] = float("nan")
        else:
            x[2, k - 1] = float("nan")
        z = w4.linear(x, w, bias=b, relu=True, dtype=torch.float32)
        keep = [i for i in range(m) if i != 2]
        assert torch.isnan(z[2]).all() and torch.equal(z[keep], y[keep])
