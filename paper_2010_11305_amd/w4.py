"""Matrices in 4-bit integer codes with a scale and a bias per group of columns, and their product with few rows
(include/emb_dense.h): weights as a served model holds them.

    w = w4.quantize(weight, group=128)                 # [n, k]; a value is bias + scale * code of its group
    y = w4.linear(x, w, bias=b, relu=True)             # max(x w^T + b, 0), x in full precision
    y = w4.linear(rows, w, dtype=torch.bfloat16)       # rows in 8 bits, from rmsnorm.norm8

Made for few rows.  Of many, w.dequantize() and a full-precision product are faster where the weight is large: measured, with
4096 x 4096 from 550 rows on in 16 bits and 900 in 8 bits, with 8192 x 12800 from 750 and 1400 (float32 rows, or 256 x 256: not up
to 4096 rows).

Every step runs in the HIP kernels of libembcache, on the current stream.  None of it is recorded by autograd.
"""
from __future__ import annotations

import torch

from . import dense_lib as lib
from .rmsnorm import Rows8

INT8 = 3    # the library's type of 8-bit rows


class W4Matrix:
    """rows x cols values in 4 bits with FP16 scales and biases for each `group` (32, 64 or 128) columns of a row, in one device
    buffer (`data`, uint8)."""

    __slots__ = ("rows", "cols", "group", "data")

    def __init__(self, rows: int, cols: int, group: int = 128, device="cuda", data=None):
        need = lib.query("emb_w4_query_bytes", rows, cols, group)
        if data is None:
            data = torch.empty(need, dtype=torch.uint8, device=device)
        elif data.dtype != torch.uint8 or not data.is_cuda or not data.is_contiguous() or data.numel() < need:
            raise ValueError(f"data must be at least {need} contiguous bytes on the GPU")
        self.rows, self.cols, self.group, self.data = rows, cols, group, data

    @property
    def shape(self):
        return (self.rows, self.cols)

    @property
    def device(self):
        return self.data.device

    def dequantize(self, dtype=torch.float32, out=None):
        """The values as a [rows, cols] tensor: bias + scale * code in FP32, rounded to dtype (or to out's)."""
        given = out is not None
        out, p, t, ld = lib.result(out, self.rows, self.cols, dtype, self.device)
        lib.call("emb_w4_dequantize", self.device, self.data.data_ptr(), self.rows, self.cols, self.group, p, t, ld)
        if given:
            lib.written([out])
        return out

    def to_codes(self):
        """(codes [rows, ceil(cols/2)] uint8, two a byte with the even column in the low half, scales and biases
        [rows, ceil(cols/group)] float16): the plain form, for checkpoints and exchange."""
        groups = -(-self.cols // self.group)
        codes = torch.empty((self.rows, -(-self.cols // 2)), dtype=torch.uint8, device=self.device)
        scales, biases = (torch.empty((self.rows, groups), dtype=torch.float16, device=self.device) for _ in range(2))
        lib.call("emb_w4_unpack", self.device, self.data.data_ptr(), self.rows, self.cols, self.group, codes.data_ptr(),
                 scales.data_ptr(), biases.data_ptr())
        return codes, scales, biases


def _target(out, rows, cols, group, device) -> W4Matrix:
    if out is None:
        return W4Matrix(rows, cols, group, device)
    if not isinstance(out, W4Matrix) or out.shape != (rows, cols) or out.group != group or out.device != device:
        raise ValueError(f"out must be a W4Matrix [{rows}, {cols}] with groups of {group} on {device}")
    return out


def quantize(x, group: int = 128, out: W4Matrix | None = None) -> W4Matrix:
    """x [rows, cols] in 4 bits: of each group the least value as bias, a fifteenth of the range as scale (both FP16), and codes
    rounded to nearest."""
    p, t, rows, cols, ld = lib.matrix(x, "x")
    out = _target(out, rows, cols, group, x.device)
    lib.call("emb_w4_quantize", x.device, p, t, rows, cols, ld, group, out.data.data_ptr())
    return out


def from_codes(codes, scales, biases, cols: int, group: int = 128, out: W4Matrix | None = None) -> W4Matrix:
    """The inverse of W4Matrix.to_codes.  Weights whose zero has a code z instead of a bias have the bias -z * scale."""
    rows = codes.shape[0]
    for t, dtype, width, what in ((codes, torch.uint8, -(-cols // 2), "codes"), (scales, torch.float16, -(-cols // group), "scales"),
                                  (biases, torch.float16, -(-cols // group), "biases")):
        if t.dtype != dtype or not t.is_cuda or not t.is_contiguous() or tuple(t.shape) != (rows, width):
            raise ValueError(f"{what} must be a contiguous {dtype} tensor [{rows}, {width}] on the GPU")
    if not codes.device == scales.device == biases.device:
        raise ValueError(f"codes, scales and biases must be on one device, not {codes.device}, {scales.device} and {biases.device}")
    out = _target(out, rows, cols, group, codes.device)
    lib.call("emb_w4_pack", out.device, codes.data_ptr(), scales.data_ptr(), biases.data_ptr(), rows, cols, group, out.data.data_ptr())
    return out


def linear(x, w: W4Matrix, bias=None, relu: bool = False, dtype=None, out=None):
    """x w^T + bias, then max(y, 0) with relu, for rows x [m, k] (a tensor, or Rows8) and a weight w [n, k].  The result has
    `dtype`: that of x, or bfloat16 for Rows8, by default.  bias: n float32 values."""
    dev = x.device
    if isinstance(x, Rows8):
        p, scales, m, k, ld = x.parts()
        t, dtype = INT8, dtype or torch.bfloat16
    else:
        p, t, m, k, ld = lib.matrix(x, "x")
        scales, dtype = None, dtype or x.dtype
    if k != w.cols or w.device != dev:
        raise ValueError(f"x [{m}, {k}] and w {w.shape} must have the same number of columns, on one device")
    n, b = w.rows, None
    if bias is not None:
        if bias.dtype != torch.float32 or bias.shape != (n,) or not bias.is_contiguous() or bias.device != dev:
            raise ValueError(f"bias must be {n} contiguous float32 values on {dev}")
        b = bias.data_ptr()
    given = out is not None
    out, yp, yt, y_ld = lib.result(out, m, n, dtype, dev)
    lib.call_in("emb_w4_linear", dev, lib.query("emb_w4_linear_workspace", t, m, n, k, w.group), p, t, scales, m, k, ld,
                w.data.data_ptr(), n, w.group, b, bool(relu), yp, yt, y_ld)
    if given:
        lib.written([out])
    return out
