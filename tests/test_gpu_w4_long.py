"""Products with a weight whose buffer passes 4 GiB, of whole numbers whose sums are exact: every output, by both routes."""
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


def test_every_output(torch):
    """|scale sum(q x)| is at most 3 x 15 x 8 x 16384 and |bias sum(x)| 20 x 8 x 16384: 8.6 million together, below 2^24."""
    from paper_2010_11305_amd import w4
    from paper_2010_11305_amd.rmsnorm import Rows8

    n, k, group = 560_000, 16384, 128
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    codes = torch.randint(0, 256, (n, k // 2), dtype=torch.uint8, generator=g, device="cuda")
    scales = torch.randint(1, 4, (n, k // group), generator=g, device="cuda").half()
    biases = torch.randint(-20, 1, (n, k // group), generator=g, device="cuda").half()
    w = w4.from_codes(codes, scales, biases, k, group)
    assert w.data.numel() > 1 << 32
    x = torch.randint(-8, 9, (20, k), generator=g, device="cuda")
    rows = [x[:1].bfloat16(), x.bfloat16(), x[:1].float(), x.float(), Rows8(x.to(torch.int8), torch.ones(20, device="cuda"))]
    got = [w4.linear(v, w, dtype=torch.float32) for v in rows]
    step = 16_000     # 2 GiB of FP64 at a time
    for i in range(0, n, step):
        c = codes[i:i + step]
        v = torch.stack([c & 15, c >> 4], -1).view(len(c), k // group, group).double()
        v = v.mul_(scales[i:i + step, :, None].double()).add_(biases[i:i + step, :, None].double()).view(len(c), k)
        want = x.double() @ v.t()
        for y in got:
            assert torch.equal(y[:, i:i + step].double(), want[:len(y)]), i
        del v
