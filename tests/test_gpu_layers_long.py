"""Offsets that pass 31 and 32 bits: rows far apart, many rows, and tensors of more than 2^31 elements."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2010_11305_amd import dense_lib
    dense_lib.load()
    return t


@pytest.mark.parametrize("rows,cols", [(270_000, 8192), (140_000, 16400), (140_000_000, 16)])
def test_norm_of_many_rows(torch, rows, cols):
    """2^31 elements and more (and 2^27 rows): the last ones as they are by themselves."""
    from paper_2010_11305_amd import rmsnorm

    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda").uniform_(-1, 1)
    gain = torch.rand(cols, device="cuda") + 0.5
    y, h, inverse = rmsnorm.norm_train(x, gain)
    dx, dgain = rmsnorm.backward(x, h, inverse, gain)
    last = x[-37:].clone()
    y1, h1, inverse1 = rmsnorm.norm_train(last, gain)
    assert torch.equal(y[-37:], y1) and torch.equal(inverse[-37:], inverse1)
    assert torch.equal(dx[-37:], rmsnorm.backward(last, h1, inverse1, gain)[0])
    del dx, y
    # the gain's gradient over all rows: a sum of dy * h * inverse, here of squares times inverse
    want = torch.zeros(cols, dtype=torch.float64, device="cuda")
    step = max(1, 50_000_000 // cols)
    for i in range(0, rows, step):
        want += (x[i:i + step].double().square() * inverse[i:i + step].double()[:, None]).sum(0)
    assert ((dgain.double() - want).abs() <= 264 * 2.0**-24 * want).all()     # all terms have one sign
    q, _ = rmsnorm.norm8(x, gain)
    q1, _ = rmsnorm.norm8(last, gain)
    assert torch.equal(q.codes[-37:], q1.codes) and torch.equal(q.scales[-37:], q1.scales)
    v = q.dequantize(torch.bfloat16)
    assert torch.equal(v[-37:], q1.dequantize(torch.bfloat16))


def test_rows_far_apart(torch):
    """Rows 2^30 elements apart."""
    from paper_2010_11305_amd import rmsnorm, w4

    cols, ld = 300, 1 << 30
    wide = torch.empty(19 * ld + 1000, dtype=torch.bfloat16, device="cuda")
    x = wide.as_strided((20, cols), (ld, 1))
    x.copy_(torch.randn(20, cols, device="cuda"))
    near = x.contiguous()
    w = w4.quantize(torch.randn(40, cols, device="cuda"), 64)
    big = w4.quantize(torch.randn(9000, cols, device="cuda"), 64)
    assert torch.equal(w4.linear(x, w), w4.linear(near, w))
    assert torch.equal(w4.linear(x, big), w4.linear(near, big))
    assert torch.equal(w4.quantize(x, 32).data, w4.quantize(near, 32).data)
    y, _, inverse = rmsnorm.norm_train(near)
    out = wide.as_strided((20, cols), (ld, 1), 500)
    rmsnorm.norm(x, out=out)
    assert torch.equal(out, y)
    assert torch.equal(rmsnorm.backward(x, out, inverse)[0], rmsnorm.backward(near, y, inverse)[0])
    w4.linear(near, w, out=wide.as_strided((20, 40), (ld, 1), 900))
    assert torch.equal(wide.as_strided((20, 40), (ld, 1), 900), w4.linear(near, w))


def test_large_weight(torch):
    """A weight whose buffer passes 4 GiB, its last rows against those rows by themselves."""
    from paper_2010_11305_amd import w4

    n, k = 560_000, 16384
    codes = torch.randint(0, 256, (n, k // 2), dtype=torch.uint8, device="cuda")
    scales, biases = torch.rand(n, k // 128, device="cuda").half(), -torch.rand(n, k // 128, device="cuda").half()
    w = w4.from_codes(codes, scales, biases, k, 128)
    assert w.data.numel() > 1 << 32
    part = w4.from_codes(codes[-48:].contiguous(), scales[-48:].contiguous(), biases[-48:].contiguous(), k, 128)
    for m in (1, 20):
        x = torch.randn(m, k, device="cuda").bfloat16()
        # the route, and with it the order of sums, goes by the size: equal up to a rounding of the type and FP32 sums
        a, b = w4.linear(x, w, dtype=torch.float32)[:, -48:], w4.linear(x, part, dtype=torch.float32)
        magnitude = x.double().abs().sum(1, keepdim=True) * 16     # scales and biases are below 1, codes at most 15
        assert ((a - b).abs() <= 2 * (k + 2 * k // 128 + 40) * 2.0**-23 * magnitude).all()
    back = w.to_codes()
    assert torch.equal(back[0], codes) and torch.equal(back[1], scales) and torch.equal(back[2], biases)


def test_clip_of_a_large_tensor(torch):
    from paper_2010_11305_amd.clip import GradClip

    n = (1 << 32) + 12345
    g = [torch.full((n,), 2.0**-8, dtype=torch.bfloat16, device="cuda"), torch.ones(7, device="cuda")]
    g[0][-1] = 3.0
    want = ((n - 1) * 2.0**-16 + 9.0 + 7.0) ** 0.5
    c = GradClip(g, max_norm=want / 2)
    norm, factor = c.clip_(g)
    assert abs(float(norm) - want) <= 1.01 * 2.0**-24 * want and abs(float(factor) - 0.5) < 1e-6
    assert g[0][-1] == 1.5 and g[0][0] == 2.0**-9 and (g[0][-10000:-1] == 2.0**-9).all() and (g[1] == 0.5).all()
