"""Plain numpy forms, in 64 bits, of the operators between a tower's products (norm, 4-bit weights with group scales, the
gradients' norm), and what the tests of them share."""
import numpy as np
import torch

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
U = 2.0**-24                                                   # largest relative error of one FP32 rounding
HALF_STEP = {"fp32": 2.0**-24, "bf16": 2.0**-8, "fp16": 2.0**-11}    # largest relative error of a rounding
LEAST = {"fp32": 2.0**-150, "bf16": 2.0**-134, "fp16": 2.0**-25}   # half the smallest subnormal: the rounding next to zero


def f64(t):
    return t.detach().double().cpu().numpy()


def rounded(t, name):
    """Error of rounding values of magnitude |t| to a type."""
    return np.abs(t) * HALF_STEP[name] + LEAST[name]


def norm(h, gain, eps):
    """(y, inverse) of float64 rows."""
    inverse = 1.0 / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    return h * inverse * gain, inverse


def norm_gradients(dy, h, gain, eps):
    """(gradient of h, of the gain, mean |dn n| of each row), from the formula of y alone."""
    _, inverse = norm(h, gain, eps)
    dn, n = dy * gain, h * inverse
    return (dn - n * (dn * n).mean(-1, keepdims=True)) * inverse, (dy * n).sum(0), np.abs(dn * n).mean(-1, keepdims=True)


def w4_quantize(x, group):
    """(codes [n, k], scales, biases FP16 [n, groups]) of FP32 rows: every operation one of FP32, as the tables' INT4 rows."""
    x = np.asarray(x, dtype=np.float32)
    n, k = x.shape
    groups = -(-k // group)
    codes, scales, biases = np.zeros((n, k), np.uint8), np.zeros((n, groups), np.float16), np.zeros((n, groups), np.float16)
    with np.errstate(all="ignore"):
        for g in range(groups):
            w = x[:, g * group:(g + 1) * group]
            lo, hi = w.min(1) + np.float32(0), w.max(1)
            fine = (np.abs(w) < 65520).all(1)
            s = ((hi - lo) / np.float32(15)).astype(np.float16)
            b = lo.astype(np.float16)
            sf = s.astype(np.float32)[:, None]
            q = np.rint((w - b.astype(np.float32)[:, None]) / np.where(sf == 0, np.float32(1), sf))
            q = np.where((sf == 0) | ~fine[:, None], 0, np.clip(q, 0, 15))
            codes[:, g * group:(g + 1) * group] = q
            scales[:, g], biases[:, g] = np.where(fine, s, np.float16(np.nan)), np.where(fine, b, np.float16(np.nan))
    return codes, scales, biases


def w4_values(codes, scales, biases, group):
    at = np.arange(codes.shape[1]) // group
    return biases.astype(np.float64)[:, at] + scales.astype(np.float64)[:, at] * codes


def pack(codes):
    n, k = codes.shape
    c = np.zeros((n, k + k % 2), np.uint8)
    c[:, :k] = codes
    return c[:, 0::2] | c[:, 1::2] << 4


def w4_magnitudes(x, codes, scales, biases, group):
    """[m, n]: the sum of the magnitudes that a product's sums are made of, codes and biases apart."""
    at = np.arange(codes.shape[1]) // group
    return np.abs(x) @ (np.abs(scales.astype(np.float64))[:, at] * codes + np.abs(biases.astype(np.float64))[:, at]).T
