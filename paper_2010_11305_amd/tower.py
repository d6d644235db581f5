"""A ranking model on the library: cached low-precision tables below, a dense tower in 4 bits above.

One training step puts the operators together as a program would use them:

    pooled rows   emb_cache_forward                            tables in low precision, FP32 cache
    tower         mx4.Linear.forward_train, bias, ReLU         rows and weights in 4 bits, per layer
    gradients     mx4.Linear.backward                          4 bits, rounded stochastically
    tables        emb_cache_backward_update                    with the gradient of the pooled rows
    tower         adamw.AdamW.step, then mx4.Linear.load       FP32 weights, moments in 8 or 32 bits

The last layer (one output) stays in FP32.  Labels come from a hidden score of every row, so that there is
something to learn; no data set is used.

    python -m paper_2010_11305_amd.tower [--steps 200] [--batch 4096] [--state-bits 8]
"""
from __future__ import annotations

import argparse
import time

import numpy as np

from . import configs, workload

MODEL = dict(rows=[100_000] * 8, dim=16, bits=4, sb_fp16=True, cache_fraction=0.05, assoc=16, policy="lru",
             rounding="stochastic", optimizer="adagrad", lr=0.02, batch=4096, pooling=("fixed", 1), zipf=1.1)


class Tower:
    """Dense layers `widths` (the first is the width of the pooled rows), then one FP32 output."""

    def __init__(self, widths, lr=1e-3, state_bits=8, max_norm=1.0, seed=1, device="cuda"):
        import torch

        from . import adamw, mx4

        self.torch, self.max_norm = torch, max_norm
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.weights = [torch.randn((n, k), generator=g, device=device) * (2.0 / k) ** 0.5
                        for k, n in zip(widths, widths[1:])]
        self.biases = [torch.zeros(n, device=device) for n in widths[1:]]
        self.last = torch.randn(widths[-1], generator=g, device=device) * widths[-1] ** -0.5
        self.layers = [mx4.Linear(n, k, seed=seed + i, device=device)
                       for i, (k, n) in enumerate(zip(widths, widths[1:]))]
        params = [*self.weights, *self.biases, self.last]
        self.opt = adamw.AdamW(params, lr=lr, weight_decay=[0.01] * len(self.weights) + [0.0] * (len(self.biases) + 1),
                               state_bits=state_bits, rounding="stochastic", seed=seed + len(self.layers))
        self.load()

    def load(self):
        for layer, w in zip(self.layers, self.weights):
            layer.load(w)

    def predict(self, x):
        """Logits of pooled rows [batch, width]."""
        for layer, b in zip(self.layers, self.biases):
            x = self.torch.relu_(layer.forward(x).add_(b))
        return x @ self.last

    def gradients(self, x, labels, step):
        """(loss, gradients of the parameters, gradient of x)."""
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

    def update(self, grads):
        """AdamW on gradients clipped to max_norm by their common norm; it stays on the GPU."""
        norm = self.torch.stack([g.norm() for g in grads]).norm()
        self.opt.step(grads, grad_scale=(self.max_norm / norm).clamp(max=1.0))
        self.load()


def labels_of(cfg, indices, step):
    """Clicks drawn from a hidden score of the rows (one lookup per table and sample)."""
    ids = indices.reshape(len(cfg["rows"]), -1).astype(np.uint64)
    mixed = (ids + np.arange(len(ids), dtype=np.uint64)[:, None] * np.uint64(7919)) * np.uint64(0x9E3779B97F4A7C15)
    score = ((mixed >> np.uint64(40)).astype(np.float64) / 2.0**24 - 0.5).sum(0) * 4.0
    return (np.random.default_rng(step).random(len(score)) < 1 / (1 + np.exp(-score))).astype(np.float32)


def train(cfg: dict, steps: int, widths=(512, 256), state_bits=8, progress=None):
    """Losses of `steps` training steps, as floats."""
    import torch

    from .emb_cache import EmbCache

    T, d, B = len(cfg["rows"]), cfg["dim"], cfg["batch"]
    emb = EmbCache(cfg, max_indices=T * B)
    emb.init_uniform(cfg["init_lo"], cfg["init_hi"], cfg["init_seed"])
    tower = Tower((T * d, *widths), state_bits=state_bits)
    losses = []
    for step in range(steps):
        idx_np, off_np = workload.make_indices(cfg, step)
        idx, off = torch.from_numpy(idx_np).cuda(), torch.from_numpy(off_np).cuda()
        labels = torch.from_numpy(labels_of(cfg, idx_np, step)).cuda()
        pooled = emb.forward(idx, off, B)
        loss, grads, dx = tower.gradients(pooled.view(B, T * d), labels, step)
        emb.backward_update(idx, off, B, dx.view(B, T, d))
        tower.update(grads)
        losses.append(loss)
        if progress:
            progress(step, loss)
    if emb.check() != 0:
        raise RuntimeError("the embedding step reported an error")
    return [float(v) for v in losses]


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--batch", type=int, default=MODEL["batch"])
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=8)
    a = ap.parse_args()
    cfg = configs.get("tiny", **dict(MODEL, batch=a.batch))
    began = time.time()

    def progress(step, loss):
        if step % 20 == 0 or step + 1 == a.steps:
            print(f"step {step:5d}  loss {float(loss):.4f}  {time.time() - began:.1f} s", flush=True)

    train(cfg, a.steps, state_bits=a.state_bits, progress=progress)


if __name__ == "__main__":
    main()
