"""The serving operators written out from their definitions in 64 bits (numpy, CPU); shares no code with the library."""
import numpy as np


def cached(x):
    """What a cache of 4-bit mantissas holds for x [..., dim]: per block of 32, whole multiples (at most 7, ties to even) of a unit
    that is a quarter of the power of two of the block's largest magnitude, or twice that where the largest would round to 8."""
    x = np.asarray(x, dtype=np.float64)
    out = np.zeros_like(x)
    for d0 in range(0, x.shape[-1], 32):
        part = x[..., d0:d0 + 32]
        top = np.abs(part).max(axis=-1, keepdims=True)
        _, e = np.frexp(top)                                   # top = f * 2^e, 0.5 <= f < 1
        e = np.where(top == 0, -126, np.maximum(e - 1, -126))
        e = np.where(np.rint(np.ldexp(top, 2 - e)) >= 8, e + 1, e)
        out[..., d0:d0 + 32] = np.ldexp(np.rint(np.ldexp(part, 2 - e)), e - 2)
    return out


class Cache:
    def __init__(self, batch, heads, capacity, dim):
        self.k, self.v = (np.zeros((batch, heads, capacity, dim)) for _ in range(2))
        self.capacity = capacity

    def append(self, k, v, lengths):
        tokens = k.shape[1]
        for b, n in enumerate(lengths):
            for t in range(tokens):
                slot = max(int(n), 0) - tokens + t
                if 0 <= slot < self.capacity:
                    self.k[b, :, slot], self.v[b, :, slot] = cached(k[b, t]), cached(v[b, t])


def attend(cache, q, lengths, scale, causal=True, longest=None):
    """(out, lse, spread, noise, p): spread[..., d] = sum p |v|, the scale of an error in the weights; noise[...] the largest
    sum of |scale q k| of a visible key, the scale of an error in the scores; p [batch][token][head][slot] the weights."""
    q = np.asarray(q, dtype=np.float64)
    batch, tokens, heads, dim = q.shape
    group = heads // cache.k.shape[1]
    out, spread = np.zeros(q.shape), np.zeros(q.shape)
    lse, noise = np.full(q.shape[:3], -np.inf), np.zeros(q.shape[:3])
    p = np.zeros(q.shape[:3] + (cache.capacity,))
    for b in range(batch):
        for t in range(tokens):
            n = max(int(lengths[b]), 0)
            n = min(n - tokens + t + 1 if causal else n, cache.capacity if not longest else min(longest, cache.capacity))
            if n <= 0:
                continue
            for h in range(heads):
                k, v = cache.k[b, h // group, :n], cache.v[b, h // group, :n]
                s = scale * (k @ q[b, t, h])
                top = s.max()
                w = np.exp(s - top)
                lse[b, t, h] = top + np.log(w.sum())
                w /= w.sum()
                p[b, t, h, :n] = w
                out[b, t, h] = w @ v
                spread[b, t, h] = w @ np.abs(v)
                noise[b, t, h] = (np.abs(k) @ np.abs(scale * q[b, t, h])).max()
    return out, lse, spread, noise, p


def weigh(p, weights, lengths, decay, kv_heads):
    batch, tokens, heads, slots = p.shape
    got = p.reshape(batch, tokens, kv_heads, heads // kv_heads, slots).sum(axis=(1, 3))
    out = np.zeros_like(got)
    for b, n in enumerate(lengths):
        n = min(max(int(n), 0), slots)
        out[b, :, :n] = decay * weights[b, :, :n] + got[b, :, :n]
    return out


def evict(weights, length, keep, recent):
    """The slots of one head that stay, in order; weights [slots]."""
    n = length
    if n <= keep:
        return list(range(n))
    r = min(recent, keep)
    rank = sorted(range(n - r), key=lambda i: (-np.inf if np.isnan(weights[i]) else weights[i], -i), reverse=True)
    return sorted(rank[:keep - r]) + list(range(n - r, n))


def rows(x):
    """8-bit codes and FP32 scales, the quotients rounded to FP32 as the definition has them."""
    x = np.asarray(x, dtype=np.float32)
    with np.errstate(divide="ignore", invalid="ignore"):
        scale = (np.abs(x).max(axis=1) * np.float32(1 / 127)).astype(np.float32)
        by = np.where(scale == 0, np.float32(1), scale)
        codes = np.clip(np.rint((x / by[:, None]).astype(np.float32)), -127, 127)
    return codes, scale
