"""The ranking model of paper_2010_11305_amd.tower: its gradients against torch's in 64 bits on the rounded values, and
training that learns."""
import numpy as np
import pytest

import dense_ref as ref
from common import custom_cfg

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2010_11305_amd import dense_lib
    dense_lib.load()
    return t


def test_gradients_of_one_layer_are_those_of_its_rounded_parts(torch):
    """One hidden layer written out in 64 bits, with the library's roundings (dense_ref) and nothing else: the parts
    compared are FP32 sums of at most 200 terms over values below 2^3, within 200 2^-23 of the sums of magnitudes."""
    from paper_2010_11305_amd.tower import Tower

    B, K, N, step = 200, 48, 40, 4
    r = np.random.default_rng(1)
    x = torch.from_numpy(r.standard_normal((B, K))).float().cuda()
    labels = torch.from_numpy((r.random(B) < 0.5).astype(np.float32)).cuda()
    t = Tower((K, N), seed=3)
    loss, grads, dx = t.gradients(x, labels, step)
    X, W, last = (v.double().cpu().numpy() for v in (x, t.weights[0], t.last))
    q = ref.mx4_round_trip
    Y = q(X) @ q(W).T + t.biases[0].double().cpu().numpy()
    H = np.maximum(Y, 0)
    z, lab = H @ last, labels.double().cpu().numpy()
    p = 1 / (1 + np.exp(-z))
    assert abs(float(loss) - np.mean(np.maximum(z, 0) - z * lab + np.log1p(np.exp(-np.abs(z))))) < 1e-5
    d = (p - lab) / B
    DY = (np.outer(d, last) * (Y > 0)).astype(np.float32).astype(np.float64)
    slack = 200 * 2.0**-23
    for got, a, b in ((grads[1], np.ones((1, B)), DY), (grads[2], d[None], H)):
        assert (np.abs(got.double().cpu().numpy() - (a @ b)[0]) <= 4 * slack * (np.abs(a) @ np.abs(b))[0] + 1e-9).all()
    # the rounding of dy starts from its FP32 value on the GPU, off by a few ulp from this one: a stochastic code may
    # differ where the two lie on either side of a draw, by one step of its block at most
    kw = dict(rounding="stochastic", seed=3, step=step)
    for got, a, b in ((dx, q(DY, **kw), q(W.T)), (grads[0], q(DY.T, tag=1, **kw), q(X.T))):
        want = a @ b.T
        off = np.abs(got.double().cpu().numpy() - want)
        assert (off > slack * (np.abs(a) @ np.abs(b).T) + 1e-12).mean() < 0.02


@pytest.mark.parametrize("bits", [8, 32])
def test_training_learns(torch, bits):
    """The hidden scores are learnt: the mean loss of the last steps is clearly below a coin's log 2, where it starts."""
    from paper_2010_11305_amd import tower

    cfg = custom_cfg(**dict(tower.MODEL, rows=[500] * 8, batch=2048))
    losses = tower.train(cfg, 120, widths=(64, 32), state_bits=bits)
    assert abs(np.mean(losses[:3]) - np.log(2)) < 0.1
    assert np.mean(losses[-10:]) < np.log(2) - 0.1, losses[::10]


def test_prediction_agrees_with_training_forward(torch):
    from paper_2010_11305_amd.tower import Tower

    x = torch.randn(300, 64, device="cuda")
    t = Tower((64, 96, 33))
    z = t.predict(x)
    loss, _, _ = t.gradients(x, torch.ones(300, device="cuda"), 0)
    want = torch.nn.functional.softplus(-z).mean()
    assert abs(float(loss - want)) < 1e-5
