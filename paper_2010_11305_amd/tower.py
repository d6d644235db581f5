"""A ranking model on the library: cached low-precision tables below, a dense tower in 4 bits above.

One training step puts the operators together as a program would use them:

    pooled rows   emb_cache_forward                            tables in low precision, FP32 cache
    tower         mx4.Linear.forward_train, bias, ReLU         rows and weights in 4 bits, per layer
    gradients     mx4.Linear.backward                          4 bits, rounded stochastically
    tables        emb_cache_backward_update                    with the gradient of the pooled rows
    tower         adamw.AdamW.step, then mx4.Linear.load       FP32 weights, moments in 8 or 32 bits

With `norm` the tower is one that may be deep: each layer's rows are normed on their way in, and a layer as wide as its rows
adds them to what it puts out:

    rows          rmsnorm.norm_train, with the addition       backward: rmsnorm.backward
    gradients     clip.GradClip.norm                           their common norm, for AdamW's factor
    serving       rmsnorm.norm8, then w4.linear                rows in 8 bits, weights in 4 bits by groups of columns

The last layer (one output) stays in FP32.  Labels come from a hidden score of every row, so that there is
something to learn; no data set is used.

    python -m paper_2010_11305_amd.tower [--steps 200] [--batch 4096] [--state-bits 8] [--norm]
"""
from __future__ import annotations

import argparse
import time

import numpy as np

from . import configs, workload

MODEL = dict(rows=[100_000] * 8, dim=16, bits=4, sb_fp16=True, cache_fraction=0.05, assoc=16, policy="lru",
             rounding="stochastic", optimizer="adagrad", lr=0.02, batch=4096, pooling=("fixed", 1), zipf=1.1)


class Tower:
    """Dense layers `widths` (the first is the width of the pooled rows), then one FP32 output.  norm: rows normed before each
    layer, and added to the output of a layer that keeps their width."""

    def __init__(self, widths, lr=1e-3, state_bits=8, max_norm=1.0, seed=1, device="cuda", norm=False):
        import torch

        from . import adamw, clip, mx4, rmsnorm, w4

        self.torch, self.rmsnorm, self.w4, self.max_norm, self.norm = torch, rmsnorm, w4, max_norm, norm
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.weights = [torch.randn((n, k), generator=g, device=device) * (2.0 / k) ** 0.5
                        for k, n in zip(widths, widths[1:])]
        self.biases = [torch.zeros(n, device=device) for n in widths[1:]]
        self.last = torch.randn(widths[-1], generator=g, device=device) * widths[-1] ** -0.5
        self.layers = [mx4.Linear(n, k, seed=seed + i, device=device)
                       for i, (k, n) in enumerate(zip(widths, widths[1:]))]
        self.gains = [torch.ones(k, device=device) for k in widths[:-1]] if norm else []
        self.adds = [norm and k == n for k, n in zip(widths, widths[1:])]
        params = [*self.weights, *self.biases, self.last, *self.gains]
        self.opt = adamw.AdamW(params, lr=lr, weight_decay=[0.01] * len(self.weights) + [0.0] * (len(params) - len(self.weights)),
                               state_bits=state_bits, rounding="stochastic", seed=seed + len(self.layers))
        self.clip = clip.GradClip(params, max_norm=max_norm) if norm else None
        self.load()

    def load(self):
        for layer, w in zip(self.layers, self.weights):
            layer.load(w)

    def predict(self, x):
        """Logits of pooled rows [batch, width]."""
        if self.norm:
            return self._normed(x, lambda i, rows, past: self.rmsnorm.norm(rows, self.gains[i], residual=past),
                                lambda i, rows: self.torch.relu_(self.layers[i].forward(rows).add_(self.biases[i])), self.last)
        for layer, b in zip(self.layers, self.biases):
            x = self.torch.relu_(layer.forward(x).add_(b))
        return x @ self.last

    def _normed(self, x, norm, layer, last):
        """Logits by norm(i, rows, past) -> (normed rows, rows + past), layer(i, normed rows) -> activations, and the last layer."""
        past = None     # the rows that go around the layer before
        for i, adds in enumerate(self.adds):
            rows, x = norm(i, x, past)
            past, x = (x if adds else None), layer(i, rows)
        return (x if past is None else x.add_(past)) @ last

    def serve(self, group=128):
        """A function from pooled rows to logits as predict gives them, for serving a tower with `norm`: its parameters now
        (later changes do not reach it), weights in 4 bits with a scale and a bias for each `group` columns, and rows in 8 bits."""
        if not self.norm:
            raise ValueError("a tower without norms has no rows in 8 bits")
        rmsnorm, w4 = self.rmsnorm, self.w4
        weights = [w4.quantize(w, group) for w in self.weights]
        gains, biases, last = [g.clone() for g in self.gains], [b.clone() for b in self.biases], self.last.clone()
        return lambda x: self._normed(x, lambda i, rows, past: rmsnorm.norm8(rows, gains[i], residual=past),
                                      lambda i, rows: w4.linear(rows, weights[i], bias=biases[i], relu=True, dtype=x.dtype), last)

    def gradients(self, x, labels, step):
        """(loss, gradients of the parameters, gradient of x)."""
        if self.norm:
            return self._normed_gradients(x, labels, step)
        torch, kept = self.torch, []
        for layer, b in zip(self.layers, self.biases):
            y, saved = layer.forward_train(x)
            x = torch.relu_(y.add_(b))
            kept.append((saved, x))
        logits = x @ self.last
        loss = torch.nn.functional.binary_cross_entropy_with_logits(logits, labels)
        d = (torch.sigmoid(logits) - labels) / len(labels)
        d_last, dx = d @ x, torch.outer(d, self.last)
        dws, dbs = [], []
        for layer, (saved, out) in zip(reversed(self.layers), reversed(kept)):
            dy = dx * (out > 0)
            dbs.append(dy.sum(0))
            dx, dw = layer.backward(dy, saved, step)
            dws.append(dw)
        return loss, [*reversed(dws), *reversed(dbs), d_last], dx

    def _normed_gradients(self, x, labels, step):
        torch, kept, past = self.torch, [], None
        for layer, b, g, adds in zip(self.layers, self.biases, self.gains, self.adds):
            rows, x, inverse = self.rmsnorm.norm_train(x, g, residual=past)
            y, saved = layer.forward_train(rows)
            out = torch.relu_(y.add_(b))
            kept.append((saved, out, x, inverse))
            past, x = (x if adds else None), out
        if past is not None:
            x = x + past
        logits = x @ self.last
        loss = torch.nn.functional.binary_cross_entropy_with_logits(logits, labels)
        d = (torch.sigmoid(logits) - labels) / len(labels)
        d_last, dx = d @ x, torch.outer(d, self.last)
        dws, dbs, dgs = [], [], []
        for layer, g, adds, (saved, out, h, inverse) in zip(*map(reversed, (self.layers, self.gains, self.adds, kept))):
            dy = dx * (out > 0)
            dbs.append(dy.sum(0))
            drows, dw = layer.backward(dy, saved, step)
            dx, dg = self.rmsnorm.backward(drows, h, inverse, g, dh=dx if adds else None)
            dws.append(dw)
            dgs.append(dg)
        return loss, [*reversed(dws), *reversed(dbs), d_last, *reversed(dgs)], dx

    def update(self, grads):
        """AdamW on gradients clipped to max_norm by their common norm; it stays on the GPU."""
        if self.norm:
            self.opt.step(grads, grad_scale=self.clip.norm(grads)[1])
            return self.load()
        norm = self.torch.stack([g.norm() for g in grads]).norm()
        self.opt.step(grads, grad_scale=(self.max_norm / norm).clamp(max=1.0))
        self.load()


def labels_of(cfg, indices, step):
    """Clicks drawn from a hidden score of the rows (one lookup per table and sample)."""
    ids = indices.reshape(len(cfg["rows"]), -1).astype(np.uint64)
    mixed = (ids + np.arange(len(ids), dtype=np.uint64)[:, None] * np.uint64(7919)) * np.uint64(0x9E3779B97F4A7C15)
    score = ((mixed >> np.uint64(40)).astype(np.float64) / 2.0**24 - 0.5).sum(0) * 4.0
    return (np.random.default_rng(step).random(len(score)) < 1 / (1 + np.exp(-score))).astype(np.float32)


def train(cfg: dict, steps: int, widths=(512, 256), state_bits=8, progress=None, norm=False, finish=None):
    """Losses of `steps` training steps, as floats.  finish: called in the end with the tower, and the rows and labels of another
    batch."""
    import torch

    from .emb_cache import EmbCache

    T, d, B = len(cfg["rows"]), cfg["dim"], cfg["batch"]
    emb = EmbCache(cfg, max_indices=T * B)
    emb.init_uniform(cfg["init_lo"], cfg["init_hi"], cfg["init_seed"])
    tower = Tower((T * d, *widths), state_bits=state_bits, norm=norm)
    losses = []

    def batch(step):
        idx_np, off_np = workload.make_indices(cfg, step)
        idx, off = torch.from_numpy(idx_np).cuda(), torch.from_numpy(off_np).cuda()
        return idx, off, torch.from_numpy(labels_of(cfg, idx_np, step)).cuda(), emb.forward(idx, off, B)

    for step in range(steps):
        idx, off, labels, pooled = batch(step)
        loss, grads, dx = tower.gradients(pooled.view(B, T * d), labels, step)
        emb.backward_update(idx, off, B, dx.view(B, T, d))
        tower.update(grads)
        losses.append(loss)
        if progress:
            progress(step, loss)
    if finish:
        _, _, labels, pooled = batch(steps)
        finish(tower, pooled.view(B, T * d), labels)
    if emb.check() != 0:
        raise RuntimeError("the embedding step reported an error")
    return [float(v) for v in losses]


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--batch", type=int, default=MODEL["batch"])
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=8)
    ap.add_argument("--norm", action="store_true", help="a deeper tower with norms and residuals, served in the end")
    a = ap.parse_args()
    cfg = configs.get("tiny", **dict(MODEL, batch=a.batch))
    began = time.time()

    def progress(step, loss):
        if step % 20 == 0 or step + 1 == a.steps:
            print(f"step {step:5d}  loss {float(loss):.4f}  {time.time() - began:.1f} s", flush=True)

    def finish(tower, x, labels):
        from torch.nn.functional import binary_cross_entropy_with_logits as loss

        print(f"another batch: loss {float(loss(tower.predict(x), labels)):.4f}, served with rows in 8 bits and weights in 4: "
              f"{float(loss(tower.serve()(x), labels)):.4f}", flush=True)

    if a.norm:
        train(cfg, a.steps, widths=(256, 256, 256), state_bits=a.state_bits, progress=progress, norm=True, finish=finish)
    else:
        train(cfg, a.steps, state_bits=a.state_bits, progress=progress)


if __name__ == "__main__":
    main()
