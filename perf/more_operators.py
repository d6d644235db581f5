"""Performance cases of the operators between the products of a dense tower: the root-mean-square norm with the
residual's addition, products of few rows with 4-bit weights under group scales, and the gradients' global norm.

A case names its operator in "op":

  norm    a training pass of the norm: h = x + residual, y = h / rms(h) * gain, then the gradients of h (which is that of x
          and of the residual alike, the gradient that reaches h past the norm added) and of the gain
  norm8   the norm with its rows in 8 bits, as serving takes them: int8 codes and one scale a row, given as the values
          they stand for
  w4      the product of few rows with a weight held in 4 bits: a code q of 0 .. 15 stands for q * scale + bias of its group,
          which is `group` consecutive columns of a row
  block   a layer of a served tower: residual's addition and norm to 8 bits, then the product with a 4-bit weight, the
          layer's bias and max(y, 0)
  clip    the norm of all gradients of a model together, and the gradients scaled down to a largest norm
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
EPS = 1e-6
MAX_NORM = 1.0


def _norm(rows, cols, dtype, residual, name=None):
    c = dict(op="norm", rows=rows, cols=cols, dtype=dtype, residual=residual)
    return dict(c, name=name) if name else c


def _norm8(rows, cols, dtype, residual, name=None):
    c = dict(op="norm8", rows=rows, cols=cols, dtype=dtype, residual=residual)
    return dict(c, name=name) if name else c


def _w4(m, n, k, dtype, group, name=None):
    c = dict(op="w4", m=m, n=n, k=k, dtype=dtype, group=group)
    return dict(c, name=name) if name else c


def _block(m, n, k, dtype, group, name=None):
    c = dict(op="block", m=m, n=n, k=k, dtype=dtype, group=group)
    return dict(c, name=name) if name else c


def _clip(tensors, elements, dtype, salt, name=None):
    c = dict(op="clip", tensors=tensors, elements=elements, dtype=dtype, salt=salt)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the pooled rows of the 26 Criteo-Kaggle-shaped tables (26 x 16 columns), batch 2048, ahead of the first layer
        _norm(2048, 416, "fp32", False, "norm_kaggle"),
        # rows as wide as the pooled rows of the 100-table industrial shape (100 x 128 columns), batch 16384, inside a
        # tower with residuals
        _norm(16384, 12800, "bf16", True, "norm_industrial"),
        # an odd layer and a ragged batch
        _norm(1000, 1029, "fp16", True, "norm_ragged"),
        # one request's pooled rows to 8 bits: latency counts
        _norm8(1, 12800, "bf16", False, "norm8_one"),
        # a large batch scored offline
        _norm8(4096, 8192, "bf16", True, "norm8_batch"),
        # one request through the industrial tower's first layer: the weight is read once
        _w4(1, 4096, 12800, "bf16", 128, "w4_one"),
        # a small batch of FP32 rows on an odd layer, the last group of a row short
        _w4(7, 2000, 4100, "fp32", 64, "w4_ragged"),
        # as many rows as the operator is made for, finest scales
        _w4(64, 8192, 12800, "bf16", 32, "w4_batch"),
        # one request through a wide layer of a served tower, and a batch of them
        _block(1, 8192, 8192, "bf16", 128, "block_one"),
        _block(48, 4096, 8192, "bf16", 64, "block_batch"),
        # the tower above the Kaggle-shaped tables: a few small FP32 tensors, latency counts
        _clip(6, 350_000, "fp32", 1, "clip_small"),
        # a model of many tensors of very different and odd sizes, bfloat16 gradients
        _clip(300, 200_000_000, "bf16", 2, "clip_many"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the same ranges: one row to 16384 (64 where the weight is in 4 bits), a few columns to 12800, one
    tensor to 400."""
    op = rng.choice(["norm", "norm", "norm8", "w4", "w4", "block", "clip"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op in ("norm", "norm8"):
        cols = _log_uniform(rng, 1 if op == "norm8" else 16, 12800)
        most = 16384 * 12800 * 2 // (BYTES[dtype] * cols)     # no dearer than the largest
        rows = _log_uniform(rng, 1, min(16384, most))
        return (_norm if op == "norm" else _norm8)(rows, cols, dtype, rng.random() < 0.6)
    if op in ("w4", "block"):
        m, n, k = _log_uniform(rng, 1, 64), _log_uniform(rng, 16, 8192), _log_uniform(rng, 16, 12800)
        return (_w4 if op == "w4" else _block)(m, n, k, dtype, rng.choice([32, 64, 128, 128]))
    tensors = _log_uniform(rng, 1, 400)
    return _clip(tensors, _log_uniform(rng, max(1000, 16 * tensors), 200_000_000), dtype, rng.randrange(1 << 20))


def work(case):
    op, b = case["op"], BYTES[case["dtype"]]
    if op in ("norm", "norm8"):
        n, plus = case["rows"] * case["cols"], case["residual"]
        if op == "norm":
            # x, dy to y, dx; with a residual it, the gradient past the norm, and h as well
            return {"bytes": n * b * (7 if plus else 4) + 8 * case["cols"], "flops": 0}
        # x (and the residual, and h) to codes, the codes to values (bfloat16)
        return {"bytes": n * (b * (3 if plus else 1) + 2 * 1 + 2) + 4 * case["cols"], "flops": 0}
    if op in ("w4", "block"):
        m, n, k = case["m"], case["n"], case["k"]
        weight = n * -(-k // 2) + 4 * n * -(-k // case["group"])
        rows = m * k * (3 if op == "block" else 1)     # x; in a block x, the residual and h
        return {"bytes": weight + b * (rows + m * n) + (4 * (n + k) if op == "block" else 0), "flops": 2 * m * n * k}
    return {"bytes": sum(_sizes(case)) * 3 * b, "flops": 0}     # read for the norm, read and written for the scaling


def _sizes(case):
    """Sizes of the tensors: few of them spread over a factor of four, many over one of a thousand."""
    r = random.Random(case["salt"])
    spread = 1000.0 if case["tensors"] > 20 else 4.0
    w = [math.exp(r.uniform(0.0, math.log(spread))) for _ in range(case["tensors"])]
    return [max(1, int(case["elements"] * v / sum(w))) for v in w]


# ---- inputs -----------------------------------------------------------------------------------
def _matrix(g, rows, cols, scale=1.0):
    """Normal values whose size differs from row to row and, for one column in 64, is larger."""
    x = torch.randn((rows, cols), generator=g, device="cuda") * scale
    x *= torch.exp2(torch.randint(-3, 4, (rows, 1), generator=g, device="cuda").float())
    x *= 1.0 + 7.0 * (torch.rand((1, cols), generator=g, device="cuda") < 1.0 / 64)
    return x


def _gain(g, cols):
    return 1.0 + 0.2 * torch.randn(cols, generator=g, device="cuda")


def _groups(w, group):
    """A weight in 4 bits: codes two a byte (the even column in the low half), scales and biases [n, groups]."""
    n, k = w.shape
    count = -(-k // group)
    pad = torch.nn.functional.pad(w, (0, count * group - k)).view(n, count, group)
    inside = (torch.arange(count * group, device=w.device) < k).view(count, group)
    lo = torch.where(inside, pad, math.inf).amin(-1)
    hi = torch.where(inside, pad, -math.inf).amax(-1)
    scale, bias = ((hi - lo) / 15).half(), lo.half()
    q = ((pad - bias.float()[..., None]) / scale.float()[..., None]).nan_to_num(0.0).round_().clamp_(0, 15)
    q = torch.where(inside, q, 0.0).view(n, -1)[:, : k + k % 2].to(torch.uint8)
    return q[:, 0::2] + 16 * q[:, 1::2], scale, bias


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, dt = case["op"], DTYPES[case["dtype"]]
    s = {"case": dict(case)}
    if op in ("norm", "norm8"):
        rows, cols = case["rows"], case["cols"]
        s["x"] = _matrix(g, rows, cols).to(dt)
        s["r"] = _matrix(g, rows, cols).to(dt) if case["residual"] else None
        s["gain"] = _gain(g, cols)
        if op == "norm":
            s["dy"] = _matrix(g, rows, cols, 2.0**-6).to(dt)
            s["dh"] = _matrix(g, rows, cols, 2.0**-6).to(dt) if case["residual"] else None
    elif op in ("w4", "block"):
        m, n, k = case["m"], case["n"], case["k"]
        s["x"] = _matrix(g, m, k).to(dt)
        s["codes"], s["scales"], s["biases"] = _groups(_matrix(g, n, k, k**-0.5), case["group"])
        if op == "block":
            s["r"] = _matrix(g, m, k).to(dt)
            s["gain"] = _gain(g, k)
            s["bias"] = torch.randn(n, generator=g, device="cuda")
        if own:
            from paper_2010_11305_amd import w4
            s["w"] = w4.from_codes(s["codes"], s["scales"], s["biases"], k, case["group"])
    else:
        sizes = _sizes(case)
        s["g"] = (torch.randn(sum(sizes), generator=g, device="cuda") * 1e-2).to(dt)
        if own:
            from paper_2010_11305_amd import clip
            s["grads"] = list(s["g"].split(sizes))
            s["clip"] = clip.GradClip(s["grads"], max_norm=MAX_NORM)
    return s


# ---- one pass -----------------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    op = s["case"]["op"]
    if op == "norm":
        from paper_2010_11305_amd import rmsnorm
        y, h, inverse = rmsnorm.norm_train(s["x"], s["gain"], residual=s["r"], eps=EPS)
        dx, dgain = rmsnorm.backward(s["dy"], h, inverse, s["gain"], dh=s["dh"])
        out = {"y": y, "dx": dx, "dgain": dgain}
        return out if s["r"] is None else dict(out, h=h)
    if op == "norm8":
        from paper_2010_11305_amd import rmsnorm
        rows, h = rmsnorm.norm8(s["x"], s["gain"], residual=s["r"], eps=EPS)
        out = {"y": rows.dequantize(torch.bfloat16)}
        return out if s["r"] is None else dict(out, h=h)
    if op == "w4":
        from paper_2010_11305_amd import w4
        return w4.linear(s["x"], s["w"])
    if op == "block":
        from paper_2010_11305_amd import rmsnorm, w4
        rows, h = rmsnorm.norm8(s["x"], s["gain"], residual=s["r"], eps=EPS)
        return {"h": h, "y": w4.linear(rows, s["w"], bias=s["bias"], relu=True, dtype=s["x"].dtype)}
    norm, _ = s["clip"].clip_(s["grads"])
    return {"norm": norm, "g": s["g"]}


def _run_plain(s):
    case = s["case"]
    op, dt = case["op"], DTYPES[case["dtype"]]
    if op == "clip":
        norm = s["g"].double().square().sum().sqrt()
        s["g"].copy_(s["g"].float() * (MAX_NORM / norm).clamp(max=1.0).float())
        return {"norm": norm.float(), "g": s["g"]}
    if op == "w4":
        return (s["x"].float() @ _weight(s).t()).to(dt)
    x, r, gain = s["x"], s["r"], s["gain"]
    h = x if r is None else (x.float() + r.float()).to(dt)
    f = h.float()
    inverse = torch.rsqrt(f.square().mean(-1, keepdim=True) + EPS)
    n = f * inverse
    y = n * gain
    if op == "norm":
        dn = s["dy"].float() * gain
        dx = (dn - n * (dn * n).mean(-1, keepdim=True)) * inverse
        if r is not None:
            dx = dx + s["dh"].float()
        out = {"y": y.to(dt), "dx": dx.to(dt), "dgain": (s["dy"].float() * n).sum(0)}
        return out if r is None else dict(out, h=h)
    scale = y.abs().amax(-1, keepdim=True) / 127
    v = torch.round(y / scale.clamp(min=2.0**-126)) * scale
    if op == "norm8":
        out = {"y": v.to(torch.bfloat16)}
        return out if r is None else dict(out, h=h)
    return {"h": h, "y": (v @ _weight(s).t() + s["bias"]).clamp(min=0.0).to(dt)}


def _weight(s):
    k, group = s["case"]["k"], s["case"]["group"]
    q = torch.stack([s["codes"] & 15, s["codes"] >> 4], -1).view(len(s["codes"]), -1)[:, :k].float()
    scale, bias = (s[name].float().repeat_interleave(group, 1)[:, :k] for name in ("scales", "biases"))
    return q * scale + bias


# ---- the definition in 64 bits ---------------------------------------------------------------------
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    op = case["op"]
    if op == "clip":
        g = s["g"].to(torch.float64)
        norm = torch.linalg.vector_norm(g)
        return {"norm": norm, "g": g * min(1.0, MAX_NORM / float(norm))}
    if op == "w4":
        return torch.mm(s["x"].to(torch.float64), _exact_weight(s).t())
    x, r = s["x"].to(torch.float64), s["r"]
    out, h = {}, x
    if r is not None:
        out["h"] = x + r.to(torch.float64)
        h = out["h"].to(s["x"].dtype).to(torch.float64)     # the sum is kept in the type of x, and that is what is normed
    gain = s["gain"].to(torch.float64)
    rms = torch.sqrt((h * h).sum(1) / case["cols" if "cols" in case else "k"] + EPS)[:, None]
    if op == "norm":
        out["y"] = h / rms * gain
        dy = s["dy"].to(torch.float64)
        out["dgain"] = torch.einsum("rc,rc->c", dy, h / rms)
        # d/dh of sum(dy * gain * h / rms): rms depends on every h of its row by h / (cols * rms)
        along = (dy * gain * h).sum(1, keepdim=True) / (case["cols"] * rms**3)
        out["dx"] = dy * gain / rms - along * h + (0.0 if r is None else s["dh"].to(torch.float64))
        return out
    y = h / rms * gain
    step = y.abs().max(1, keepdim=True).values / 127
    v = torch.where(step > 0, torch.round(y / step) * step, 0.0)
    if op == "norm8":
        return dict(out, y=v)
    return dict(out, y=torch.relu(torch.mm(v, _exact_weight(s).t()) + s["bias"].to(torch.float64)))


def _exact_weight(s):
    codes, k = s["codes"].long(), s["case"]["k"]
    q = torch.zeros((codes.shape[0], 2 * codes.shape[1]), dtype=torch.float64, device=codes.device)
    q[:, 0::2], q[:, 1::2] = (codes % 16).double(), torch.div(codes, 16, rounding_mode="floor").double()
    of = torch.arange(k, device=codes.device) // s["case"]["group"]
    return s["biases"].double()[:, of] + s["scales"].double()[:, of] * q[:, :k]
