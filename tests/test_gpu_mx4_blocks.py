"""Blocks that are not finite or lie at the ends of the scale's range, through the product of tiles in each of its sizes and
through a layer's gradients, and the bytes that pad an MX4 matrix."""
import numpy as np
import pytest

import dense_ref as ref
from dense_launch import tile_rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2010_11305_amd import dense_lib
    dense_lib.load()
    return t


def plain(t):
    return t.double().cpu().numpy()


def buffer_of(code, scale, cols):
    """The buffer of an MX4 matrix, byte by byte as its layout says: zeros where no block is."""
    rows = code.shape[0]
    rt, kt = -(-rows // 16), -(-cols // 128)
    kg = -(-kt // 4)
    codes = np.zeros((rt * 16, kt * 128), dtype=np.uint8)
    codes[:rows, :cols] = code
    tiles = (codes[:, 0::2] | codes[:, 1::2] << 4).reshape(rt, 16, kt, 4, 16).transpose(0, 2, 3, 1, 4)
    scales = np.zeros((rt * 16, kg * 16), dtype=np.uint8)
    scales[:rows, :scale.shape[1]] = scale
    pieces = scales.reshape(rt, 16, kg, 4, 4).transpose(0, 2, 4, 1, 3)      # of a lane 16 b + r: four column tiles
    return np.concatenate([tiles.ravel(), pieces.ravel()])


@pytest.mark.parametrize("rounding", ["nearest", "stochastic"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (17, 129), (33, 513), (15, 1100), (130, 70), (600, 31), (48, 1024)])
def test_every_byte_of_a_matrix(torch, rows, cols, dtype, rounding):
    """Into buffers full of ones, with more behind the matrix: the matrix is written whole, and nothing else."""
    from paper_2010_11305_amd import mx4

    r = np.random.default_rng(rows + cols)
    x = torch.from_numpy(r.standard_normal((rows, cols)) * np.exp2(r.integers(-8, 9, (rows, cols)))).to(getattr(torch, dtype)).cuda()
    x[rows // 2, cols - 1] = float("nan")
    x[rows - 1, cols // 3] = float("inf")
    kw = dict(rounding=rounding, seed=4, step=2)

    def full(m, n):
        need = mx4.Mx4Matrix(m, n).data.numel()
        return mx4.Mx4Matrix(m, n, data=torch.full((need + 512,), 255, dtype=torch.uint8, device="cuda"))

    both = mx4.quantize_both(x, out=(full(rows, cols), full(cols, rows)), **kw)
    for tag, q, of in ((0, mx4.quantize(x, out=full(rows, cols), **kw), x),
                       (1, mx4.quantize_columns(x, out=full(cols, rows), **kw), x.t()), (0, both[0], x), (1, both[1], x.t())):
        code, scale = ref.mx4_quantize(plain(of), tag=tag, **kw)
        want = np.concatenate([buffer_of(code, scale, of.shape[1]), np.full(512, 255, dtype=np.uint8)])
        assert np.array_equal(q.data.cpu().numpy(), want)
        again = mx4.from_codes(*q.to_codes(), of.shape[1], out=full(*of.shape))
        assert np.array_equal(again.data.cpu().numpy(), want)


# tiles of 64, 128 and 256 (the last also several to a workgroup), ragged, the last group of columns short
TILES = [(1000, 1029, 700, 64), (1920, 1913, 400, 128), (4090, 4081, 700, 256), (8100, 4090, 130, 256)]


@pytest.mark.parametrize("m,n,k,tile", TILES)
def test_not_finite_blocks_in_tiles(torch, m, n, k, tile):
    """In the last block of the last row and in the first: NaN in exactly their rows and columns, and elsewhere the product."""
    from paper_2010_11305_amd import mx4

    assert tile_rows(m, n) == tile
    print("not finite", m, n, k, flush=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(m)
    a, b = (torch.randn((rows, k), generator=g, device="cuda") for rows in (m, n))
    a4, b4 = mx4.quantize(a), mx4.quantize(b)
    want = a4.dequantize().double() @ b4.dequantize().double().t()
    bound = k * 2.0**-23 * (a4.dequantize().double().abs() @ b4.dequantize().double().abs().t()) + 2.0**-24 * want.abs()
    a[m - 1, k - 1], a[0, 0], b[n - 1, k - 1], b[n // 2, 33] = float("nan"), float("inf"), -float("inf"), float("nan")
    c = mx4.matmul(mx4.quantize(a), mx4.quantize(b), torch.float32).double()
    bad = torch.zeros((m, n), dtype=torch.bool, device="cuda")
    bad[m - 1], bad[0], bad[:, n - 1], bad[:, n // 2] = True, True, True, True
    assert torch.equal(torch.isnan(c), bad)
    assert bool(((c - want).abs() <= bound)[~bad].all())


@pytest.mark.parametrize("m,n,k,tile", TILES)
def test_scales_at_their_ends_in_tiles(torch, m, n, k, tile):
    """Rows of equal values under scale bytes 0, 127 and 254: every sum is exact, or infinite."""
    from paper_2010_11305_amd import mx4

    assert tile_rows(m, n) == tile
    print("scales", m, n, k, flush=True)
    byte = torch.tensor([0, 127, 254], dtype=torch.uint8, device="cuda")
    value = torch.tensor([2.0**-127, 1.0, 2.0**127], dtype=torch.float64, device="cuda")

    def rows_of(rows, first, codes):
        kind = (torch.arange(rows, device="cuda") + first) % 3
        wide = torch.full((rows, -(-k // 2)), codes, dtype=torch.uint8, device="cuda")
        return mx4.from_codes(wide, byte[kind][:, None].expand(rows, -(-k // 32)).contiguous(), k), value[kind]

    (a4, a), (b4, b) = rows_of(m, 0, 0x22), rows_of(n, 1, 0x11)      # codes of 1 and of 1/2
    c = mx4.matmul(a4, b4, torch.float32)
    want = torch.outer(a, b) * (k / 2)     # far below FP32's smallest, far above its largest, or exact
    got, limit = c.double(), 2.0**128
    assert bool((got[want.abs() >= limit] == float("inf")).all())
    assert bool((got[want < 2.0**-200] == 0).all())
    mid = (want < limit) & (want >= 2.0**-200)
    assert int(mid.sum()) > m * n / 2 and bool((got[mid] == want[mid]).all())


@pytest.mark.parametrize("m,n,k", [(300, 200, 700), (4100, 40, 33)])
def test_not_finite_blocks_in_gradients(torch, m, n, k):
    """Both gradients from one launch, and (over more than 4096 rows) from one each."""
    from paper_2010_11305_amd import mx4

    g = torch.Generator(device="cuda")
    g.manual_seed(m)
    x, w, dy = (torch.randn(s, generator=g, device="cuda") for s in ((m, k), (n, k), (m, n)))
    x[m - 1, k - 1], w[n - 1, 0], dy[m - 1, n - 1], dy[0, 1] = float("nan"), float("inf"), float("nan"), -float("inf")
    layer = mx4.Linear(n, k, seed=1)
    layer.load(w)
    y, saved = layer.forward_train(x)
    dx, dw = layer.backward(dy, saved, step=1)

    def lines(shape, rows, cols):
        bad = torch.zeros(shape, dtype=torch.bool, device="cuda")
        bad[rows], bad[:, cols] = True, True
        return bad

    assert torch.equal(torch.isnan(y), lines(y.shape, [m - 1], [n - 1]))
    assert torch.equal(torch.isnan(dx), lines(dx.shape, [0, m - 1], [0]))
    assert torch.equal(torch.isnan(dw), lines(dw.shape, [1, n - 1], [k - 1]))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_expansion_at_the_ends_of_the_scale(torch, dtype):
    """Every code under every scale byte: the value rounded to the type, an infinity beyond its largest."""
    from paper_2010_11305_amd import mx4

    code = np.tile(np.arange(16, dtype=np.uint8), (256, 2))
    scale = np.arange(256, dtype=np.uint8)[:, None]
    q = mx4.from_codes(torch.from_numpy(ref.pack_codes(code)).cuda(), torch.from_numpy(scale).cuda(), 32)
    with np.errstate(over="ignore"):
        want = torch.from_numpy(ref.mx4_values(code, scale, 32)).to(getattr(torch, dtype))
    got = q.dequantize(getattr(torch, dtype)).cpu()
    bits = torch.int32 if dtype == "float32" else torch.int16
    bad = torch.isnan(want)
    assert torch.equal(torch.isnan(got), bad) and torch.equal(got.view(bits)[~bad], want.view(bits)[~bad])
