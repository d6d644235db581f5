"""A served tower is that of its moment: no later change of any parameter reaches it, nor a captured graph of it."""
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


@pytest.mark.parametrize("widths", [(40, 64, 64, 24), (40,)])
@pytest.mark.parametrize("name", ["weights", "biases", "gains", "last"])
def test_later_changes_do_not_reach_it(torch, name, widths):
    from paper_2010_11305_amd.tower import Tower

    t = Tower(widths, norm=True, seed=3)
    x = torch.randn(5, 40, device="cuda")
    serve = t.serve(32)
    before = serve(x)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = serve(x)
    for v in [t.last] if name == "last" else getattr(t, name):
        v.add_(torch.rand_like(v) + 0.5)
    assert torch.equal(serve(x), before)
    for _ in range(2):
        g.replay()
        assert torch.equal(held, before)
    if name == "last" or len(widths) > 1:
        assert not torch.equal(t.serve(32)(x), before)


def test_training_goes_on_beside_it(torch):
    """One update moves every parameter of the tower, predict follows, the served one stays."""
    from paper_2010_11305_amd.tower import Tower

    t = Tower((40, 64, 64, 24), lr=0.05, norm=True, seed=4)
    x, labels = torch.randn(64, 40, device="cuda"), (torch.arange(64, device="cuda") % 2).float()
    serve = t.serve()
    before, predicted = serve(x), t.predict(x)
    assert torch.equal(t.predict(x), predicted)
    old = [v.clone() for v in (*t.weights, *t.gains, t.last)]
    t.update(t.gradients(x, labels, 0)[1])
    assert not any(torch.equal(a, b) for a, b in zip(old, (*t.weights, *t.gains, t.last)))
    assert torch.equal(serve(x), before)
    assert not torch.equal(t.predict(x), predicted)
