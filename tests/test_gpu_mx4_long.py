"""A matrix of so many rows that every kernel's workgroups pass one launch (2^31 threads here; HIP takes fewer than
2^32): quantisation, expansion, plain codes and the product with one row.  The values are exact in 4 bits by rows, so
every result is."""
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


def column(torch, rows):
    """[rows, 1]: one of 16 values by the row's number."""
    i = torch.arange(rows, device="cuda", dtype=torch.int64)
    i = (i * 2654435761 >> 13) & 15
    table = torch.tensor([s * m * 2.0**e for s in (1, -1) for m in (1.0, 1.5) for e in (-3, 0, 1, 5)], device="cuda")
    return table.bfloat16()[i][:, None]


def test_more_rows_than_a_launch(torch):
    from paper_2010_11305_amd import mx4

    rows = 2**29 + 5
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("needs 100 GB")
    x = column(torch, rows)
    print("by rows", rows, flush=True)
    q = mx4.quantize(x)
    assert torch.equal(q.dequantize(torch.bfloat16), x)
    one = mx4.quantize(torch.full((1, 1), 3.0, device="cuda"))
    print("products", flush=True)
    assert torch.equal(mx4.matmul(one, q, torch.bfloat16)[0], 3.0 * x[:, 0])
    assert torch.equal(mx4.matmul(q, one, torch.bfloat16), 3.0 * x)
    print("plain codes", flush=True)
    codes, scales = q.to_codes()
    del q
    q = mx4.from_codes(codes, scales, 1)
    del codes, scales
    assert torch.equal(q.dequantize(torch.bfloat16), x)
    del q
    print("by columns", flush=True)
    assert torch.equal(mx4.quantize_columns(x).data, mx4.quantize(x.view(1, rows)).data)
    torch.cuda.empty_cache()
