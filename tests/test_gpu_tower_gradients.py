"""Every element of the tower's gradients against its rounded parts in 64 bits.  The output gradients that are rounded
stochastically are taken as the GPU has them (the same torch operations on the same values), so that the codes are the
reference's and each element is within the bound of its FP32 sums: k 2^-23 of the sum of magnitudes."""
import numpy as np
import pytest

import dense_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2010_11305_amd import dense_lib
    dense_lib.load()
    return t


@pytest.mark.parametrize("batch,widths", [(200, (48, 40)), (333, (70, 130, 33)), (64, (5, 1))])
def test_every_element(torch, batch, widths):
    from paper_2010_11305_amd.tower import Tower

    step, seed = 4, 3
    r = np.random.default_rng(batch)
    x = torch.from_numpy(r.standard_normal((batch, widths[0]))).float().cuda()
    labels = torch.from_numpy((r.random(batch) < 0.5).astype(np.float32)).cuda()
    t = Tower(widths, seed=seed)
    _, grads, dx = t.gradients(x, labels, step)
    n = len(t.layers)
    plain = lambda v: v.double().cpu().numpy()  # noqa: E731

    rows, kept = [x], []
    for layer, b in zip(t.layers, t.biases):
        y, saved = layer.forward_train(rows[-1])
        rows.append(torch.relu_(y.add_(b)))
        kept.append(saved)
    d = (torch.sigmoid(rows[-1] @ t.last) - labels) / batch
    down = torch.outer(d, t.last)
    q = ref.mx4_round_trip
    for i in reversed(range(n)):
        dy = down * (rows[i + 1] > 0)
        assert torch.equal(grads[n + i], dy.sum(0))
        D, X, W = plain(dy), plain(rows[i]), plain(t.weights[i])
        kw = dict(rounding="stochastic", seed=seed + i, step=step)
        down, dw = t.layers[i].backward(dy, kept[i], step)
        assert torch.equal(dw, grads[i])
        for got, a, b in ((down, q(D, **kw), q(W.T)), (dw, q(D.T, tag=1, **kw), q(X.T))):
            assert torch.isfinite(got).all()
            want = a @ b.T
            bound = a.shape[1] * 2.0**-23 * (np.abs(a) @ np.abs(b).T) + 2.0**-24 * np.abs(want)
            assert (np.abs(plain(got) - want) <= bound).all()
    assert torch.equal(down, dx) and torch.equal(grads[-1], d @ rows[-1])
