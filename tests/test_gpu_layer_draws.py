"""The random draws of a training layer whose rows, weights and output gradients all round stochastically: operands of
one product draw apart, so that outputs and gradients have the expectation of the unrounded product."""
import numpy as np
import pytest

import dense_ref as ref

pytestmark = pytest.mark.gpu

SEED = 5


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


def spread(rows, cols, seed):
    """Positive values of one scale, 2^0, along both axes (every block holds a 5), none beyond 6."""
    x = np.random.default_rng(seed).uniform(0.3, 5.5, (rows, cols)).astype(np.float32).astype(np.float64)
    x[::16], x[:, ::16] = 5.0, 5.0
    return x


def test_means_of_outputs_and_gradients(torch):
    """Over 400 steps.  A draw's variance is at most (gap / 2)^2 and operands are independent, which bounds the variance
    of a sum of products; 6 sigma of it, the 2^-16 of a gap that 16 bits may shift each operand, and the FP32 sums.  Draws
    shared by the operands move the diagonals by 14 sigma and more."""
    from paper_2010_11305_amd import mx4

    m, n, k, steps = 256, 32, 256, 400
    X, W, D = spread(m, k, 1), spread(n, k, 2), spread(m, n, 3)
    x, w, dy = (torch.from_numpy(v).float().cuda() for v in (X, W, D))
    layer = mx4.Linear(n, k, rounding="stochastic", grad_rounding="stochastic", seed=SEED)
    sums = [0.0, 0.0, 0.0]
    for step in range(steps):
        layer.load(w, step)
        y, saved = layer.forward_train(x, step)
        for i, v in enumerate((y, *layer.backward(dy, saved, step))):
            sums[i] = sums[i] + v.double()

    def gap(v):
        i = np.searchsorted(ref.GRID4, v, side="right") - 1
        return ref.GRID4[i + 1] - ref.GRID4[i]

    for total, a, b in zip(sums, (X, D, D.T), (W, W.T, X.T)):
        ga, gb = gap(a), gap(b)
        var = (ga**2 / 4) @ (b**2 + gb**2 / 4).T + a**2 @ (gb**2 / 4).T
        shift = 2.0**-16 * (ga @ b.T + a @ gb.T + ga @ gb.T)
        want = a @ b.T
        bound = 6 * np.sqrt(var / steps) + shift + a.shape[1] * 2.0**-23 * (a + ga) @ (b + gb).T
        assert (np.abs(plain(total) / steps - want) <= bound).all()


@pytest.mark.parametrize("m,n,k", [(40, 40, 70), (130, 65, 200)])
def test_streams_of_the_operands(torch, m, n, k):
    """Rows draw with 2 and 3 in the counter's last word, output gradients with 0 and 1, weights under a seed of their
    own; within the bound of the FP32 sums."""
    from paper_2010_11305_amd import mx4

    r = np.random.default_rng(m)
    X, W, D = (r.standard_normal(s).astype(np.float32).astype(np.float64) for s in ((m, k), (n, k), (m, n)))
    layer = mx4.Linear(n, k, rounding="stochastic", grad_rounding="stochastic", seed=SEED)
    cuda = lambda v: torch.from_numpy(v).float().cuda()  # noqa: E731
    layer.load(cuda(W), step=7)
    y, saved = layer.forward_train(cuda(X), step=8)
    dx, dw = layer.backward(cuda(D), saved, step=9)

    def q(v, tag, seed, step):
        return ref.mx4_round_trip(v, rounding="stochastic", seed=seed, step=step, tag=tag)

    own = SEED ^ 1 << 63
    for got, a, b in ((y, q(X, 2, SEED, 8), q(W, 0, own, 7)), (dx, q(D, 0, SEED, 9), q(W.T, 1, own, 7)),
                      (dw, q(D.T, 1, SEED, 9), q(X.T, 3, SEED, 8))):
        assert (np.abs(plain(got) - a @ b.T) <= a.shape[1] * 2.0**-23 * (np.abs(a) @ np.abs(b).T) + 2.0**-24 * np.abs(a @ b.T)).all()


def test_serving_draws_nothing(torch):
    """forward() rounds its rows to nearest, also where training rounds them stochastically."""
    from paper_2010_11305_amd import mx4

    x, w = (torch.from_numpy(spread(40, 96, i)).bfloat16().cuda() for i in (1, 2))
    layer = mx4.Linear(40, 96, rounding="stochastic", seed=SEED)
    layer.load(w, step=3)
    want = ref.mx4_round_trip(plain(x)) @ plain(layer.by_rows.dequantize()).T
    for _ in range(2):
        y = plain(layer.forward(x))
        assert (np.abs(y - want) <= (96 * 2.0**-23 + 2.0**-8) * want).all()
    assert torch.equal(layer.forward(x), mx4.linear(x, layer.by_rows))
