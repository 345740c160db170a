"""One attention layer answering for several conversations: 8-bit projections, the 4-bit cache, eviction when it is full.

    python examples/serve_layer.py [--conversations 8] [--steps 96]

Prompts of different length go in at once (padded on the left: the padding's rows see no key), then every conversation gets one token
a step.  When the cache is full, a quarter of each conversation's tokens stays in a second cache, those of the largest attention weight
and the latest, and the two caches change places.  The last line compares the layer with the same layer in FP32, whose weights and
cache are not rounded and whose tokens are evicted alike.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1804_01526_amd import hbfp  # noqa: E402


class Layer:
    """Projections, cache and eviction as a server would keep them: everything is allocated once."""

    def __init__(self, w_qkv, w_out, batch, heads, kv_heads, dim, capacity):
        self.heads, self.kv_heads, self.dim, self.capacity = heads, kv_heads, dim, capacity
        self.w_qkv, self.w_out = hbfp.quant_rows(w_qkv), hbfp.quant_rows(w_out)
        self.cache, self.spare = (hbfp.cache_alloc(batch, kv_heads, capacity, dim) for _ in range(2))
        self.weights, self.spare_weights = (torch.zeros((batch, kv_heads, capacity), device="cuda") for _ in range(2))
        self.lengths = torch.zeros(batch, dtype=torch.int32, device="cuda")

    def step(self, x, new):
        """x [batch, tokens, features]; new: how many of each entry's tokens, counted from the last, are real."""
        batch, tokens, features = x.shape
        self.lengths += new
        y = hbfp.linear_i8(x.reshape(batch * tokens, features), self.w_qkv).view(batch, tokens, self.heads + 2 * self.kv_heads, self.dim)
        q, k, v = y.split([self.heads, self.kv_heads, self.kv_heads], dim=2)       # views: the calls take strides
        hbfp.cache_append(self.cache, k, v, self.lengths)
        out, lse = hbfp.cache_attend(self.cache, q, self.lengths)
        hbfp.cache_weigh(self.cache, q, lse, self.lengths, self.weights, decay=0.97)
        return hbfp.linear_i8(out.view(batch * tokens, self.heads * self.dim), self.w_out).view(batch, tokens, -1)

    def shrink(self, keep, recent):
        """Leaves `keep` tokens of each head; returns the slots that stayed."""
        kept, self.lengths, _ = hbfp.cache_evict(self.cache, self.weights, self.lengths, self.spare, keep, recent, self.spare_weights)
        self.cache, self.spare = self.spare, self.cache
        self.weights, self.spare_weights = self.spare_weights, self.weights
        return kept


class Plain:
    """The same layer in FP32 torch, a conversation at a time."""

    def __init__(self, w_qkv, w_out, batch, heads, kv_heads, dim):
        self.w_qkv, self.w_out, self.heads, self.kv_heads, self.dim = w_qkv.float(), w_out.float(), heads, kv_heads, dim
        self.k, self.v = ([torch.zeros((kv_heads, 0, dim), device="cuda") for _ in range(batch)] for _ in range(2))

    def step(self, x, new):
        out = torch.zeros(x.shape[:2] + (self.w_out.shape[0],), device="cuda")
        group = self.heads // self.kv_heads
        for b, n in enumerate(new):
            y = (x[b, x.shape[1] - n:].float() @ self.w_qkv.t()).view(n, -1, self.dim).transpose(0, 1)
            q, k, v = y.split([self.heads, self.kv_heads, self.kv_heads], dim=0)
            self.k[b], self.v[b] = torch.cat([self.k[b], k], dim=1), torch.cat([self.v[b], v], dim=1)
            keys, values = (t.repeat_interleave(group, dim=0) for t in (self.k[b], self.v[b]))
            s = (q @ keys.transpose(1, 2).contiguous()) / math.sqrt(self.dim)
            at = torch.arange(keys.shape[1], device="cuda")
            s = s.masked_fill(at > (keys.shape[1] - n + torch.arange(n, device="cuda")).unsqueeze(1), -math.inf)
            o = torch.softmax(s, dim=-1) @ values
            out[b, x.shape[1] - n:] = o.transpose(0, 1).reshape(n, self.heads * self.dim) @ self.w_out.t()
        return out

    def shrink(self, kept):
        for b in range(len(self.k)):
            m = int((kept[b, 0] >= 0).sum())
            at = kept[b, :, :m].long().unsqueeze(2).expand(-1, -1, self.dim)
            self.k[b], self.v[b] = self.k[b].gather(1, at), self.v[b].gather(1, at)


def run(conversations=8, steps=96, heads=8, kv_heads=2, dim=64, features=512, prompt=200, capacity=256, keep=64, recent=16, seed=0):
    """(relative error of all outputs against the FP32 layer, evictions)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")
    w_qkv = (randn((heads + 2 * kv_heads) * dim, features) / math.sqrt(features)).bfloat16()
    w_out = (randn(features, heads * dim) / math.sqrt(heads * dim)).bfloat16()
    layer = Layer(w_qkv, w_out, conversations, heads, kv_heads, dim, capacity)
    plain = Plain(w_qkv, w_out, conversations, heads, kv_heads, dim)
    held = [max(1, prompt * (b + 1) // conversations) for b in range(conversations)]   # what the host knows of the lengths
    new, one = torch.tensor(held, dtype=torch.int32, device="cuda"), torch.ones(conversations, dtype=torch.int32, device="cuda")
    error = norm = 0.0
    evictions = 0
    for step in range(steps + 1):
        if max(held) + 1 > capacity:
            plain.shrink(layer.shrink(keep, recent))
            held = [min(n, keep) for n in held]
            evictions += 1
        x = randn(conversations, max(held) if step == 0 else 1, features).bfloat16()
        counts = held if step == 0 else [1] * conversations
        y, want = layer.step(x, new if step == 0 else one).float(), plain.step(x, counts)
        if step:
            held = [n + 1 for n in held]
        for b, n in enumerate(counts):
            error += float((y[b, -n:] - want[b, -n:]).square().sum())
            norm += float(want[b, -n:].square().sum())
    return math.sqrt(error / norm), evictions


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--conversations", type=int, default=8)
    parser.add_argument("--steps", type=int, default=96)
    args = parser.parse_args()
    rel, times = run(args.conversations, args.steps)
    print(f"{args.conversations} conversations, a prompt and {args.steps} steps, {times} evictions: "
          f"relative error against the FP32 layer {rel:.4f}")
