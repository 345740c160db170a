"""Microscaled 4-bit numbers and the norm written out from their definitions in 64 bits (numpy, CPU); shares no code with the library."""
import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def words_at(idx, seed):
    """The random words of the elements at positions idx of a matrix, as the public header defines them."""
    mask = np.uint64((1 << 32) - 1)
    idx = np.asarray(idx, dtype=np.uint64)
    x = (idx & mask) ^ np.uint64(seed & 0xFFFFFFFF)
    for shift, left in ((13, True), (17, False), (5, True)):
        x = (x ^ ((x << np.uint64(shift)) if left else (x >> np.uint64(shift)))) & mask
    x = (x + ((idx >> np.uint64(32)) ^ np.uint64(seed >> 32))) & mask
    x ^= x >> np.uint64(16)
    x = (x * np.uint64(0x85EBCA6B)) & mask
    x ^= x >> np.uint64(13)
    x = (x * np.uint64(0xC2B2AE35)) & mask
    return x ^ (x >> np.uint64(16))


def words(rows, cols, seed):
    return words_at(np.arange(rows * cols, dtype=np.uint64).reshape(rows, cols), seed)


def quant(x, h=None):
    """(indices with the sign as bit 3, bytes) of x [rows][k], k along the contraction; h: random words, or None for the nearest."""
    x = np.asarray(x, dtype=np.float64)
    rows, k = x.shape
    nblk = -(-k // 32)
    codes, scales = np.zeros((rows, k), dtype=np.int64), np.zeros((rows, nblk), dtype=np.int64)
    for b in range(nblk):
        part = x[:, 32 * b:32 * b + 32]
        top = np.abs(part).max(axis=1)
        bad = ~np.isfinite(top)
        part, top = np.where(bad[:, None], 0, part), np.where(bad, 0, top)
        frac, e = np.frexp(top)                                   # top = frac * 2^e, 0.5 <= frac < 1
        biased = np.where(top == 0, 0, e - 1 + 127) + ((frac >= 0.875) if h is None else (frac > 0.75))
        s = np.maximum(np.minimum(biased, 254) - 2, 0)
        a = np.ldexp(np.abs(part), (127 - s)[:, None])
        at = np.minimum(np.searchsorted(MAGNITUDES, a, side="right") - 1, 6)
        low, high = MAGNITUDES[at], MAGNITUDES[at + 1]
        if h is None:
            up = (2 * a > low + high) | ((2 * a == low + high) & (at % 2 == 1))
        else:
            # floor(t + h / 2^32) with t = (a - low) / step in [0, 1): t * 2^32 cut to an integer decides as t itself does
            frac32 = np.floor((np.minimum(a, high) - low) / (high - low) * 2.0 ** 32)
            up = frac32 + h[:, 32 * b:32 * b + 32].astype(np.float64) >= 2.0 ** 32
        codes[:, 32 * b:32 * b + 32] = at + up + 8 * np.signbit(part)
        scales[:, b] = np.where(bad, 255, s)
        codes[bad, 32 * b:32 * b + 32] = 0
    return codes, scales


def values(codes, scales):
    v = np.where(codes & 8, -1.0, 1.0) * MAGNITUDES[codes & 7]
    unit = np.where(scales == 255, np.nan, np.ldexp(1.0, scales - 127))
    return v * np.repeat(unit, 32, axis=1)[:, :codes.shape[1]]


def held(x, h=None):
    """The values that an operand holds for x."""
    return values(*quant(x, h))


def norm(total, weight, eps):
    """(n rounded to FP32, 1 / rms) of the sum's rows."""
    s = np.asarray(total, dtype=np.float64)
    rstd = 1.0 / np.sqrt((s * s).sum(axis=1, keepdims=True) / s.shape[1] + np.float64(np.float32(eps)))
    n = s * rstd
    return (n if weight is None else n * np.asarray(weight, dtype=np.float64)).astype(np.float32), rstd[:, 0]


def norm_grad(g, total, rstd, weight, g_sum):
    """(dx, dweight, how large the terms of each are): the terms' magnitudes are what roundings are relative to."""
    g, s, r = (np.asarray(t, dtype=np.float64) for t in (g, total, rstd))
    w = np.ones(g.shape[1]) if weight is None else np.asarray(weight, dtype=np.float64)
    r = r[:, None]
    u = s * r
    through = g * w
    dx = r * (through - u * (through * u).mean(axis=1, keepdims=True))
    size = r * (np.abs(through) + np.abs(u) * np.abs(through * u).mean(axis=1, keepdims=True))
    if g_sum is not None:
        dx, size = dx + g_sum, size + np.abs(g_sum)
    return dx, (g * u).sum(axis=0), size, np.abs(g * u).sum(axis=0)
