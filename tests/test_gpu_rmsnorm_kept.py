"""What the backward pass of the norm takes is kept: a training pass whose output would lie over its only h is refused, as its
gradients would be those of other rows, without a word."""
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


def test_training_over_its_rows(torch):
    from paper_2010_11305_amd import rmsnorm

    gain = torch.rand(40, device="cuda") + 0.5
    x, r, dy = (torch.randn(4, 40, device="cuda") for _ in range(3))
    y, h, inverse = rmsnorm.norm_train(x, gain)
    want = rmsnorm.backward(dy, h, inverse, gain)
    before = x.clone()
    for out in (x, x.view(4, 40), x.as_strided((4, 40), (40, 1))):
        with pytest.raises(ValueError, match="out"):
            rmsnorm.norm_train(x, gain, out=out)
    assert torch.equal(x, before)
    t = x.clone()
    assert torch.equal(rmsnorm.norm(t, gain, out=t)[0], y) and torch.equal(t, y)      # no gradients are asked for
    # with a residual h lies elsewhere, or where it is told to
    y2, h2, inverse2 = rmsnorm.norm_train(x, gain, residual=r)
    t = x.clone()
    got = rmsnorm.norm_train(t, gain, residual=r, out=t)
    assert all(torch.equal(a, b) for a, b in zip(got, (y2, h2, inverse2)))
    t, s = x.clone(), r.clone()
    got = rmsnorm.norm_train(t, gain, residual=s, out=t, sum_out=s)
    assert all(torch.equal(a, b) for a, b in zip(got, (y2, h2, inverse2)))
    both = torch.randn(4, 80, device="cuda")
    both[:, :40] = x
    got = rmsnorm.norm_train(both[:, :40], gain, out=both[:, 40:])
    assert torch.equal(got[0], y) and all(torch.equal(a, b) for a, b in zip(rmsnorm.backward(dy, got[1], got[2], gain), want))
    none = torch.zeros((0, 40), device="cuda")
    assert rmsnorm.norm_train(none, gain, out=none)[0].shape == (0, 40)
