"""Matrices in microscaled 4-bit floating point and the linear layer on them (include/emb_dense.h).

A block of 32 consecutive values of a row shares a power of two; each value is a 4-bit code
(sign, 2 exponent bits, 1 mantissa bit).  The bindings only marshal arguments; every step
runs in the HIP kernels of libembcache, on the current stream.  None of it is recorded by autograd: what
comes out has no history, whatever went in (Linear.backward gives the gradients).

    w4 = mx4.quantize(w)                   # [n, k]
    y = mx4.linear(x, w4)                  # [m, n] = Q(x) w4^T, x in full precision
    c = mx4.matmul(a4, b4, torch.float32)  # a4 b4^T

    layer = mx4.Linear(n, k)               # training
    layer.load(w)
    y, saved = layer.forward_train(x)
    dx, dw = layer.backward(dy, saved, step)
"""
from __future__ import annotations

import torch

from . import dense_lib as lib

_query = lib.query
_result = lib.result


class Mx4Matrix:
    """rows x cols values in 4 bits, in one device buffer (`data`, uint8)."""

    __slots__ = ("rows", "cols", "data")

    def __init__(self, rows: int, cols: int, device="cuda", data=None):
        need = _query("emb_mx4_query_bytes", rows, cols)
        if data is None:
            data = torch.empty(need, dtype=torch.uint8, device=device)
        elif data.dtype != torch.uint8 or not data.is_cuda or not data.is_contiguous() or data.numel() < need:
            raise ValueError(f"data must be at least {need} contiguous bytes on the GPU")
        self.rows, self.cols, self.data = rows, cols, data

    @property
    def shape(self):
        return (self.rows, self.cols)

    @property
    def device(self):
        return self.data.device

    def dequantize(self, dtype=torch.float32, out=None):
        """The values as a [rows, cols] tensor, exact in float32 and bfloat16 (beyond 2^128, which only imported scale
        bytes 253 and 254 reach, infinite)."""
        rows, cols, dev = self.rows, self.cols, self.data.device
        given = out is not None
        out, p, t, ld = _result(out, rows, cols, dtype, dev)
        lib.call("emb_mx4_dequantize", dev, self.data.data_ptr(), rows, cols, p, t, ld)
        if given:
            lib.written([out])
        return out

    def to_codes(self):
        """(codes [rows, ceil(cols/2)], scales [rows, ceil(cols/32)]) as uint8 tensors, codes two a
        byte with the even column in the low half: the plain form, for checkpoints and exchange."""
        codes = torch.empty((self.rows, -(-self.cols // 2)), dtype=torch.uint8, device=self.device)
        scales = torch.empty((self.rows, -(-self.cols // 32)), dtype=torch.uint8, device=self.device)
        lib.call("emb_mx4_unpack", self.device, self.data.data_ptr(), self.rows, self.cols, codes.data_ptr(),
                 scales.data_ptr())
        return codes, scales


def from_codes(codes, scales, cols: int, out: Mx4Matrix | None = None) -> Mx4Matrix:
    """The inverse of Mx4Matrix.to_codes."""
    rows = codes.shape[0]
    for t, width, what in ((codes, -(-cols // 2), "codes"), (scales, -(-cols // 32), "scales")):
        if t.dtype != torch.uint8 or not t.is_cuda or not t.is_contiguous() or tuple(t.shape) != (rows, width):
            raise ValueError(f"{what} must be a contiguous uint8 tensor [{rows}, {width}] on the GPU")
    if codes.device != scales.device:
        raise ValueError(f"codes and scales must be on one device, not {codes.device} and {scales.device}")
    out = _target(out, rows, cols, codes.device, "out")
    lib.call("emb_mx4_pack", out.device, codes.data_ptr(), scales.data_ptr(), rows, cols, out.data.data_ptr())
    return out


def _target(out, rows, cols, device, what) -> Mx4Matrix:
    if out is None:
        return Mx4Matrix(rows, cols, device)
    if not isinstance(out, Mx4Matrix) or out.shape != (rows, cols) or out.device != device:
        raise ValueError(f"{what} must be an Mx4Matrix [{rows}, {cols}] on {device}")
    return out


def _quantize(x, rows_out, columns_out, rounding, seed, step):
    """rows_out, columns_out: an Mx4Matrix to fill, None for a new one, False for none."""
    p, t, rows, cols, ld = lib.matrix(x, "x")
    by_rows = None if rows_out is False else _target(rows_out, rows, cols, x.device, "the matrix by rows")
    by_columns = None if columns_out is False else _target(columns_out, cols, rows, x.device, "the matrix by columns")
    lib.call("emb_mx4_quantize", x.device, p, t, rows, cols, ld, by_rows and by_rows.data.data_ptr(),
             by_columns and by_columns.data.data_ptr(), lib.rounding_of(rounding), seed, step)
    return by_rows, by_columns


def quantize(x, rounding="nearest", seed=0, step=0, out: Mx4Matrix | None = None) -> Mx4Matrix:
    """x [rows, cols] in 4 bits, blocks along its rows.  Stochastic rounding draws from (seed, step)."""
    return _quantize(x, out, False, rounding, seed, step)[0]


def quantize_columns(x, rounding="nearest", seed=0, step=0, out: Mx4Matrix | None = None) -> Mx4Matrix:
    """The transpose of x in 4 bits, [cols, rows], blocks along the columns of x."""
    return _quantize(x, False, out, rounding, seed, step)[1]


def quantize_both(x, rounding="nearest", seed=0, step=0, out=(None, None)):
    """(quantize(x), quantize_columns(x)) with x read once."""
    return _quantize(x, out[0], out[1], rounding, seed, step)


def matmul(a: Mx4Matrix, b: Mx4Matrix, dtype=torch.bfloat16, out=None):
    """a b^T for a [m, k] and b [n, k]: FP32 sums, one rounding to dtype (or to out's)."""
    if a.cols != b.cols or a.device != b.device:
        raise ValueError(f"a {a.shape} and b {b.shape} must have the same number of columns, on one device")
    dev, given = a.device, out is not None
    out, p, t, ld = _result(out, a.rows, b.rows, dtype, dev)
    lib.call("emb_mx4_matmul", dev, a.data.data_ptr(), b.data.data_ptr(), a.rows, b.rows, a.cols, p, t, ld)
    if given:
        lib.written([out])
    return out


def linear(x, w: Mx4Matrix, out=None):
    """Q(x) w^T for full-precision rows x [m, k] and a weight w [n, k] in 4 bits, in the type of x.  An `out` over x is
    refused where the rows are quantised inside the product (few of them)."""
    p, t, m, k, ld = lib.matrix(x, "x")
    dev, given = x.device, out is not None
    if k != w.cols or w.device != dev:
        raise ValueError(f"x [{m}, {k}] and w {w.shape} must have the same number of columns, on one device")
    out, yp, yt, yld = _result(out, m, w.rows, x.dtype, dev)
    if yt != t:
        raise ValueError("out must have the type of x")
    need = _query("emb_mx4_linear_workspace", m, w.rows, k)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    lib.call("emb_mx4_linear", dev, p, t, m, k, ld, w.data.data_ptr(), w.rows, yp, yld, ws.data_ptr() if need else None, need)
    if given:
        lib.written([out])
    return out


class Linear:
    """The products of a linear layer y = x w^T in 4 bits, forward and backward.

    The full-precision weight stays with the caller (and its optimizer); load() brings it
    here in 4 bits along both axes, after every update.  Rows (of forward_train) and weights round as
    `rounding` says, output gradients as `grad_rounding` does: stochastic rounding keeps
    gradients unbiased.  Weights, rows and output gradients draw from streams of their own; pass the
    number of the training step as `step`, or every step draws the same bits, and give each layer
    its own seed.

        y  = Q(x) Q(w)^T
        dx = Q(dy) Q(w^T)^T        blocks along the outputs
        dw = Q(dy^T) Q(x^T)^T      blocks along the batch
    """

    def __init__(self, out_features: int, in_features: int, rounding="nearest", grad_rounding="stochastic", seed=0,
                 device="cuda"):
        lib.rounding_of(rounding), lib.rounding_of(grad_rounding)
        self.out_features, self.in_features = out_features, in_features
        self.rounding, self.grad_rounding, self.seed = rounding, grad_rounding, seed
        self.weight_seed = seed ^ 1 << 63    # the calls of the library separate rows and output gradients, not the weight
        self.by_rows = Mx4Matrix(out_features, in_features, device)
        self.by_columns = Mx4Matrix(in_features, out_features, device)

    def load(self, weight, step=0):
        """weight [out_features, in_features], full precision."""
        quantize_both(weight, self.rounding, self.weight_seed, step, (self.by_rows, self.by_columns))

    def forward(self, x):
        """y for serving: the rows round to nearest whatever `rounding` says, so that an answer is no draw."""
        return linear(x, self.by_rows)

    def forward_train(self, x, step=0):
        """(y, what backward needs of x: its 4-bit form along the batch)."""
        p, t, m, k, ld = lib.matrix(x, "x")
        n, dev = self.out_features, x.device
        if k != self.in_features or dev != self.by_rows.device:
            raise ValueError(f"x must be [rows, {self.in_features}] on {self.by_rows.device}")
        saved = Mx4Matrix(k, m, dev)
        y = torch.empty((m, n), dtype=x.dtype, device=dev)
        need = _query("emb_mx4_linear_train_workspace", m, n, k)
        ws = torch.empty(need, dtype=torch.uint8, device=dev)
        lib.call("emb_mx4_linear_train", dev, p, t, m, k, ld, self.by_rows.data.data_ptr(), n, y.data_ptr(), max(n, 1),
                 saved.data.data_ptr(), lib.rounding_of(self.rounding), self.seed, step, ws.data_ptr(), need)
        return y, saved

    def backward(self, dy, saved: Mx4Matrix, step=0, weight_grad_dtype=torch.float32):
        """(dx in the type of dy, dw [out_features, in_features])."""
        p, t, m, n, ld = lib.matrix(dy, "dy")
        k, dev = self.in_features, dy.device
        if n != self.out_features or saved.shape != (k, m) or dev != self.by_rows.device or saved.device != dev:
            raise ValueError(f"dy must be [rows, {self.out_features}] and saved [{k}, rows], on {self.by_rows.device}")
        dx = torch.empty((m, k), dtype=dy.dtype, device=dev)
        dw = torch.empty((n, k), dtype=weight_grad_dtype, device=dev)
        need = _query("emb_mx4_linear_grad_workspace", m, n, k)
        ws = torch.empty(need, dtype=torch.uint8, device=dev)
        lib.call("emb_mx4_linear_grad", dev, p, t, m, n, ld, self.by_columns.data.data_ptr(), k, saved.data.data_ptr(),
                 dx.data_ptr(), max(k, 1), dw.data_ptr(), lib.type_of(weight_grad_dtype), max(k, 1),
                 lib.rounding_of(self.grad_rounding), self.seed, step, ws.data_ptr(), need)
        return dx, dw
