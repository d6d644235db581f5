"""The ranking model with norms and residuals: its gradients against torch's in 64 bits, training that runs, and serving it with
rows in 8 bits and weights in 4, alone and as a captured graph."""
import numpy as np
import pytest

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


class Exact:
    """A layer in full precision in the place of one in 4 bits."""

    def __init__(self, torch):
        self.torch = torch

    def load(self, w):
        self.w = w

    def forward(self, x):
        return (x.double() @ self.w.double().t()).float()

    def forward_train(self, x):
        return self.forward(x), x

    def backward(self, dy, x, step):
        return (dy.double() @ self.w.double()).float(), (dy.double().t() @ x.double()).float()


def test_gradients(torch):
    """Layers in full precision, so that autograd in 64 bits has the same function: each value passes some ten FP32
    roundings a layer, of sums of at most 64 terms; 1e-5 of the largest magnitude of each gradient is above them."""
    from paper_2010_11305_amd.tower import Tower

    widths, B = (48, 64, 64, 64, 40, 40), 50
    r = np.random.default_rng(1)
    x = torch.from_numpy(r.standard_normal((B, 48))).float().cuda()
    labels = torch.from_numpy((r.random(B) < 0.5).astype(np.float32)).cuda()
    t = Tower(widths, norm=True)
    assert t.adds == [False, True, True, False, True]
    for g in t.gains:
        g.copy_(1 + 0.2 * torch.randn_like(g))
    t.layers = [Exact(torch) for _ in t.layers]
    t.load()
    loss, grads, dx = t.gradients(x, labels, 0)
    p = [v.double().requires_grad_() for v in (*t.weights, *t.biases, t.last, *t.gains, x)]
    n = len(t.layers)
    h, past = p[-1], None
    for i in range(n):
        h = h if past is None else h + past
        rows = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + 1e-6) * p[2 * n + 1 + i]
        y = torch.relu(rows @ p[i].t() + p[n + i])
        past, h = (h if t.adds[i] else None), y
    logits = (h if past is None else h + past) @ p[2 * n]
    want = torch.nn.functional.binary_cross_entropy_with_logits(logits, labels.double())
    want.backward()
    assert abs(float(loss) - float(want.detach())) < 1e-5
    assert (t.predict(x) - logits).abs().max() < 1e-5 * logits.abs().max()
    for got, v in zip([*grads, dx], p):
        assert got.shape == v.shape and (got - v.grad).abs().max() <= 1e-5 * v.grad.abs().max()


def test_training_runs_and_is_served(torch):
    """Tables, deep tower, clipping and optimizer together, in both sizes of state, then another batch through both ways of
    predicting: everything stays finite, every parameter moves, and a step's gradients arrive clipped."""
    from paper_2010_11305_amd import tower

    for bits in (8, 32):
        cfg = custom_cfg(**dict(tower.MODEL, rows=[500] * 8, batch=512))
        seen = []

        def finish(t, x, labels):
            first = tower.Tower((x.shape[1], 64, 64, 32), state_bits=bits, norm=True)
            for a, b in zip((*t.weights, *t.biases, *t.gains, t.last), (*first.weights, *first.biases, *first.gains, first.last)):
                assert torch.isfinite(a).all() and not torch.equal(a, b)
            for group in (32, 64, 128):
                seen.append(t.serve(group)(x))
            seen.append(t.predict(x))
            _, grads, _ = t.gradients(x, labels, 99)
            norm, factor = t.clip.norm(grads)
            want = sum(g.double().square().sum() for g in grads).sqrt()
            assert abs(float(norm) - float(want)) <= 1e-6 * float(want)
            assert abs(float(factor) - min(1.0, t.max_norm / float(want))) <= 1e-6

        losses = tower.train(cfg, 6, widths=(64, 64, 32), state_bits=bits, norm=True, finish=finish)
        assert len(losses) == 6 and np.isfinite(losses).all()
        assert len(seen) == 4 and all(v.shape == (512,) and torch.isfinite(v).all() for v in seen)


def test_served_tower(torch):
    """serve() is its operators called one after the other, on the weights of its moment, and can be captured."""
    from paper_2010_11305_amd import rmsnorm, w4
    from paper_2010_11305_amd.tower import Tower

    t = Tower((96, 256, 256, 64), norm=True, seed=5)
    for b in t.biases:
        b.copy_(torch.randn_like(b))
    serve = t.serve(64)
    for m in (1, 7, 300):
        x = torch.randn(m, 96, device="cuda")
        h, past = x, None
        for w, b, g, adds in zip(t.weights, t.biases, t.gains, t.adds):
            rows, h = rmsnorm.norm8(h, g, residual=past)
            y = w4.linear(rows, w4.quantize(w, 64), bias=b, relu=True, dtype=torch.float32)
            past, h = (h if adds else None), y
        want = (h if past is None else h + past) @ t.last
        got = serve(x)
        assert torch.equal(got, want)
        assert torch.isfinite(t.predict(x)).all()
    x = torch.randn(7, 96, device="cuda")
    serve(x)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = serve(x)
    for _ in range(3):
        x.copy_(torch.randn_like(x))
        g.replay()
        assert torch.equal(out, serve(x))
        torch.cuda.synchronize()
    before = serve(x)
    t.weights[0].add_(1.0)
    assert torch.equal(serve(x), before)
    with pytest.raises(ValueError):
        Tower((8, 8)).serve()
