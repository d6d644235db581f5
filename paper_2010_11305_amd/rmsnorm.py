"""The root-mean-square norm of rows with the residual's addition, forward and backward, and its output in 8 bits
(include/emb_dense.h).

    y, h = rmsnorm.norm(x, gain, residual=r)              # h = x + r, y = h / rms(h) * gain
    rows, h = rmsnorm.norm8(x, gain, residual=r)          # y in 8 bits, for w4.linear

    y, h, inverse = rmsnorm.norm_train(x, gain, residual=r)
    dx, dgain = rmsnorm.backward(dy, h, inverse, gain, dh=dh)   # dh: what reaches h past the norm

Every step runs in the HIP kernels of libembcache, on the current stream.  None of it is recorded by autograd.
"""
from __future__ import annotations

import torch

from . import dense_lib as lib


class Rows8:
    """Rows in 8 bits: `codes` int8 [rows, cols] (contiguous rows) and one float32 `scales` for each; a value is code * scale."""

    __slots__ = ("codes", "scales")

    def __init__(self, codes, scales):
        if codes.dtype != torch.int8 or codes.dim() != 2 or not codes.is_cuda or (codes.shape[1] > 1 and codes.stride(1) != 1):
            raise ValueError("codes must be an int8 matrix on the GPU whose rows are contiguous")
        if scales.dtype != torch.float32 or scales.shape != codes.shape[:1] or not scales.is_contiguous() or scales.device != codes.device:
            raise ValueError(f"scales must be {len(codes)} contiguous float32 values on {codes.device}")
        self.codes, self.scales = codes, scales

    @property
    def shape(self):
        return tuple(self.codes.shape)

    @property
    def device(self):
        return self.codes.device

    def parts(self):
        """(pointer of the codes, of the scales, rows, cols, row stride)"""
        rows, cols = self.codes.shape
        return (self.codes.data_ptr(), self.scales.data_ptr(), rows, cols,
                self.codes.stride(0) if rows > 1 else max(cols, 1))

    def dequantize(self, dtype=torch.float32, out=None):
        """The values as a [rows, cols] tensor."""
        c, s, rows, cols, ld = self.parts()
        given = out is not None
        out, p, t, ldx = lib.result(out, rows, cols, dtype, self.device)
        lib.call("emb_rows8_dequantize", self.device, c, rows, cols, ld, s, p, t, ldx)
        if given:
            lib.written([out])
        return out


def _gain(gain, cols, x):
    """(pointer, type) of a gain."""
    if gain is None:
        return None, 0
    if gain.shape != (cols,) or not gain.is_contiguous() or gain.device != x.device or gain.dtype not in (torch.float32, x.dtype):
        raise ValueError(f"gain must be {cols} contiguous values on {x.device}, float32 or of the type of x")
    return gain.data_ptr(), lib.TYPES[gain.dtype]


def _inputs(x, gain, residual, sum_out):
    """Arguments of a forward call up to the sum, h, and the tensors given to be written."""
    p, t, rows, cols, ld = lib.matrix(x, "x")
    g, gt = _gain(gain, cols, x)
    if residual is None:
        if sum_out is not None:
            raise ValueError("without a residual there is no sum to write")
        return (p, t, rows, cols, ld, None, 0, g, gt), (None, 0), x, []
    r, rt, r_rows, r_cols, r_ld = lib.matrix(residual, "residual")
    if (r_rows, r_cols, rt) != (rows, cols, t) or residual.device != x.device:
        raise ValueError(f"residual must be [{rows}, {cols}], of the type of x, on {x.device}")
    h, hp, ht, h_ld = lib.result(sum_out, rows, cols, x.dtype, x.device)
    if ht != t:
        raise ValueError("sum_out must have the type of x")
    return (p, t, rows, cols, ld, r, r_ld, g, gt), (hp, h_ld), h, [h] if sum_out is not None else []


def _forward(x, gain, residual, eps, out, sum_out, inverse):
    head, sum_part, h, changed = _inputs(x, gain, residual, sum_out)
    rows, cols = head[2:4]
    y, yp, yt, y_ld = lib.result(out, rows, cols, x.dtype, x.device)
    if yt != head[1]:
        raise ValueError("out must have the type of x")
    inv = torch.empty(rows, dtype=torch.float32, device=x.device) if inverse else None
    lib.call("emb_rmsnorm_forward", x.device, *head, eps, *sum_part, yp, y_ld, inv.data_ptr() if inverse else None)
    if out is not None:
        changed.append(y)
    if changed:
        lib.written(changed)
    return y, h, inv


def norm(x, gain=None, residual=None, eps=1e-6, out=None, sum_out=None):
    """(y, h) for rows x [rows, cols]: h = x + residual (x itself without one), y = h / sqrt(mean(h^2) + eps) * gain.
    out and sum_out may be x or the residual, to work in place (without a residual, out over x leaves no h)."""
    return _forward(x, gain, residual, eps, out, sum_out, False)[:2]


def norm_train(x, gain=None, residual=None, eps=1e-6, out=None, sum_out=None):
    """(y, h, inverse): norm, with the rows' 1 / sqrt(mean(h^2) + eps) that backward takes.  h must keep its values until
    then: without a residual it is x, and out must lie elsewhere."""
    if residual is None and out is not None and out.data_ptr() == x.data_ptr() and x.numel():
        raise ValueError("out lies over x, which is the h that the backward pass takes")
    return _forward(x, gain, residual, eps, out, sum_out, True)


def norm8(x, gain=None, residual=None, eps=1e-6, sum_out=None):
    """(Rows8, h): norm, with y in 8 bits and a scale a row."""
    head, sum_part, h, changed = _inputs(x, gain, residual, sum_out)
    rows, cols = head[2:4]
    q = Rows8.__new__(Rows8)   # made here, so there is nothing to check
    q.codes = codes = torch.empty(rows, cols, dtype=torch.int8, device=x.device)
    q.scales = scales = torch.empty(rows, dtype=torch.float32, device=x.device)
    lib.call("emb_rmsnorm_forward8", x.device, *head, eps, *sum_part, codes.data_ptr(), cols, scales.data_ptr())
    if changed:
        lib.written(changed)
    return q, h


def backward(dy, h, inverse, gain=None, dh=None, out=None):
    """(dx, dgain) for the gradient dy of y: dx is the gradient of x and of the residual alike, with dh added, dgain that of
    the gain in its type (None without a gain).  out may be dy, h or dh, to work in place."""
    p, t, rows, cols, ld = lib.matrix(dy, "dy")
    dev = dy.device
    hp, ht, h_rows, h_cols, h_ld = lib.matrix(h, "h")
    if (h_rows, h_cols, ht) != (rows, cols, t) or h.device != dev:
        raise ValueError(f"h must be [{rows}, {cols}], of the type of dy, on {dev}")
    if inverse.dtype != torch.float32 or inverse.shape != (rows,) or not inverse.is_contiguous() or inverse.device != dev:
        raise ValueError(f"inverse must be {rows} contiguous float32 values on {dev}")
    g, gt = _gain(gain, cols, dy)
    s, s_ld = None, 0
    if dh is not None:
        s, st, s_rows, s_cols, s_ld = lib.matrix(dh, "dh")
        if (s_rows, s_cols, st) != (rows, cols, t) or dh.device != dev:
            raise ValueError(f"dh must be [{rows}, {cols}], of the type of dy, on {dev}")
    dx, xp, xt, x_ld = lib.result(out, rows, cols, dy.dtype, dev)
    if xt != t:
        raise ValueError("out must have the type of dy")
    dgain, need = None, 0
    if gain is not None:
        dgain = torch.empty(cols, dtype=gain.dtype, device=dev)
        need = lib.query("emb_rmsnorm_backward_workspace", t, rows, cols)
    lib.call_in("emb_rmsnorm_backward", dev, need, p, t, rows, cols, ld, hp, h_ld, inverse.data_ptr(), g, gt, s, s_ld, xp, x_ld,
                dgain.data_ptr() if gain is not None else None)
    if out is not None:
        lib.written([out])
    return dx, dgain
