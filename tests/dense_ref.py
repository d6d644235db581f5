"""Plain numpy forms of the dense operators, in 64 bits, for the tests: the MX4 format, its
random stream, and the AdamW step."""
import numpy as np

GRID4 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
GRID8 = np.concatenate([np.arange(8) * 2.0**-9] + [(8 + np.arange(8)) * 2.0**(e - 3) for e in range(-6, 9)])[:-1]
BF16_STEP = 2.0**-8   # largest relative rounding error of bfloat16; of float16 2^-11, of float32 2^-24


def philox(c0, c1, c2, c3, seed):
    """Philox4x32-10: four uint64 arrays below 2^32."""
    c = [np.asarray(v, dtype=np.uint64) for v in (c0, c1, c2, c3)]
    k0, k1 = int(seed) & 0xFFFFFFFF, int(seed) >> 32
    mask, s = np.uint64(0xFFFFFFFF), np.uint64(32)
    for n in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        ka, kb = np.uint64((k0 + n * 0x9E3779B9) & 0xFFFFFFFF), np.uint64((k1 + n * 0xBB67AE85) & 0xFFFFFFFF)
        c = [(b >> s) ^ c[1] ^ ka, b & mask, (a >> s) ^ c[3] ^ kb, a & mask]
    return c


def mx4_random_bits(rows, cols, seed, step, tag):
    """The 16 random bits of every element [rows, cols]."""
    wide = -(-cols // 8)
    col8, row = np.meshgrid(np.arange(wide), np.arange(rows))
    w = philox(col8, row, np.full_like(row, step), np.full_like(row, tag), seed)
    halves = [h for x in w for h in (x & np.uint64(0xFFFF), x >> np.uint64(16))]
    return np.stack(halves, -1).reshape(rows, wide * 8)[:, :cols].astype(np.int64)


def on_grid(y, grid, bits):
    """Places on a grid of the magnitudes y: nearest (ties to the even place), or up with probability (y - below) /
    (above - below) compared with bits / 2^16."""
    i = np.searchsorted(grid, y, side="right") - 1
    j = np.minimum(i + 1, len(grid) - 1)
    lo, hi = grid[i], grid[j]
    if bits is None:
        up = (y - lo > hi - y) | ((y - lo == hi - y) & (i % 2 == 1))
    else:
        up = bits / 65536.0 * (hi - lo) < y - lo
    return np.where(up, j, i)


def mx4_quantize(x, rounding="nearest", seed=0, step=0, tag=0):
    """(codes [rows, cols], scale bytes [rows, ceil(cols/32)]) of a float64 matrix."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    nb = -(-cols // 32)
    bits = np.zeros((rows, nb * 32), dtype=np.int64)
    if rounding == "stochastic":
        bits[:, :cols] = mx4_random_bits(rows, cols, seed, step, tag)
    b = np.zeros((rows, nb * 32))
    b[:, :cols] = x
    b = b.reshape(rows, nb, 32)
    fine = np.isfinite(b).all(-1)
    safe = np.where(fine[..., None], b, 0.0)
    a = np.abs(safe).max(-1)
    with np.errstate(divide="ignore"):
        s = np.where(a > 0, np.frexp(a)[1] - 1 - 2, -127).clip(-127, 127)
    y = np.abs(safe) / np.exp2(s.astype(np.float64))[..., None]
    code = on_grid(y, GRID4, bits.reshape(b.shape) if rounding == "stochastic" else None)
    code = code + 8 * np.signbit(safe)
    code = np.where(fine[..., None], code, 0).reshape(rows, nb * 32)[:, :cols]
    return code.astype(np.uint8), np.where(fine, s + 127, 255).astype(np.uint8)


def mx4_values(code, scale, cols):
    v = GRID4[code & 7] * np.where(code >= 8, -1.0, 1.0)
    f = np.where(scale == 255, np.nan, np.exp2(scale.astype(np.float64) - 127))
    return v * np.repeat(f, 32, axis=1)[:, :cols]


def pack_codes(code):
    rows, cols = code.shape
    c = np.zeros((rows, cols + cols % 2), dtype=np.uint8)
    c[:, :cols] = code
    return (c[:, 0::2] | c[:, 1::2] << 4).astype(np.uint8)


def mx4_round_trip(x, **kw):
    code, scale = mx4_quantize(x, **kw)
    return mx4_values(code, scale, np.asarray(x).shape[1])


def e4m3_values(elements, scale):
    """Values of E4M3 bytes with a scale byte per 32."""
    v = np.concatenate([GRID8, [np.nan]])[elements & 127] * np.where(elements >= 128, -1.0, 1.0)
    return v * np.repeat(np.where(scale == 255, np.nan, np.exp2(scale.astype(np.float64) - 127)), 32)


def e4m3_scale(block_max):
    """Scale bytes for the largest magnitudes of blocks."""
    with np.errstate(divide="ignore", invalid="ignore"):
        m, e = np.frexp(block_max)          # block_max = m 2^e, m in [0.5, 1); 448 = 0.875 2^9
        s = np.where(block_max > 0, e - 9 + (m > 0.875), -127)
    return (np.maximum(s, -127) + 127).astype(np.int64)


def adamw(p, g, m, v, t, lr, beta1, beta2, eps, decay, scale=1.0):
    """One step in float64: (p, m, v)."""
    g = g * scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    p = p * (1 - lr * decay) - lr / (1 - beta1**t) * m / (np.sqrt(v / (1 - beta2**t)) + eps)
    return p, m, v


def adam_random_bits(places, t, seed):
    """(bits of the first moment, of the second, of the parameter) for elements at these places of the state."""
    places = np.asarray(places, dtype=np.uint64)
    i = places // np.uint64(4)
    w = np.stack(philox(i & np.uint64(0xFFFFFFFF), i >> np.uint64(32), np.full_like(i, t), np.zeros_like(i), seed), -1)
    w = w[np.arange(len(places)), (places % np.uint64(4)).astype(np.int64)].astype(np.int64)
    return w & 0xFFFF, w >> 16, (w & 0xFFFF) ^ (w >> 16)
