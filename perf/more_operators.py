"""Cases for the operators of 4-bit layers: microscaled 4-bit numbers (quantisation along either axis, products, the three products of a
training step) and the root-mean-square norm that adds the residual and delivers its rows quantised, with its gradient.

``own`` chooses who computes: the plain forms below (elementary torch operations) or the library.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

BLOCK = 32                      # values that share one power of two
EPS = 2.0 ** -20                # of the norms; the same number in 32 and in 64 bits
_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}


# ---------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # a projection for one new token: the weights are read once, at 4.25 bits each
        dict(name="token", kind="linear", rows=1, cols=4096, inner=4096, dtype="bf16", bias=False),
        # a step for a batch of conversations, a layer of a server with wide layers
        dict(name="batch", kind="linear", rows=16, cols=16384, inner=8192, dtype="bf16", bias=False),
        # drafted tokens of a batch, sizes that divide nothing, FP32 in and out
        dict(name="batch_odd", kind="linear", rows=70, cols=5003, inner=2730, dtype="f32", bias=True),
        # a prompt's projection
        dict(name="prompt", kind="linear", rows=4096, cols=8192, inner=4096, dtype="bf16", bias=False),
        # a layer's weights as the optimizer leaves them, for the forward product and for the gradient of its input
        dict(name="weights", kind="quant", rows=8192, cols=4096, dtype="f32", stochastic=False),
        # a ragged batch's gradient, rounded stochastically
        dict(name="gradient_odd", kind="quant", rows=1001, cols=777, dtype="bf16", stochastic=True),
        # a training step of a linear layer: everything quantised anew, forward product, both gradients
        dict(name="train", kind="train", rows=4096, cols=4096, inner=4096, dtype="bf16"),
        # the same for a short sequence and a narrow layer
        dict(name="train_odd", kind="train", rows=501, cols=1100, inner=730, dtype="f32"),
        # one token's norm in front of an 8-bit projection
        dict(name="norm_token", kind="norm", rows=1, cols=4096, dtype="bf16", form="i8"),
        # a prompt's norm in front of an 8-bit projection
        dict(name="norm_prompt", kind="norm", rows=8192, cols=4096, dtype="bf16", form="i8"),
        # training: the norm in front of a 4-bit product, sizes that divide nothing, and back
        dict(name="norm_train_odd", kind="norm_train", rows=777, cols=2730, dtype="f32"),
        # the same at a batch's full size
        dict(name="norm_train", kind="norm_train", rows=8192, cols=4096, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "quant", "train", "norm", "norm_train"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if kind in ("linear", "train"):
        most = 4096 * 8192 * 4096 if kind == "linear" else 4096 ** 3
        while True:
            rows = _log(rng, 1, 4096)
            cols, inner = (_log(rng, 32, 16384), _log(rng, 32, 8192)) if kind == "linear" else (_log(rng, 32, 4096), _log(rng, 32, 4096))
            if rows * cols * inner <= most:
                break
        if kind == "train":
            return dict(kind=kind, rows=rows, cols=cols, inner=inner, dtype=dtype)
        return dict(kind=kind, rows=rows, cols=cols, inner=inner, dtype=dtype, bias=rng.random() < 0.5)
    while True:
        rows, cols = _log(rng, 1, 8192), _log(rng, 32, 16384)
        if rows * cols <= 8192 * 4096:
            break
    if kind == "quant":
        return dict(kind=kind, rows=rows, cols=cols, dtype=dtype, stochastic=rng.random() < 0.5)
    if kind == "norm":
        return dict(kind=kind, rows=rows, cols=cols, dtype=dtype, form=rng.choice(["i8", "mx4"]))
    return dict(kind=kind, rows=rows, cols=cols, dtype=dtype)


# --------------------------------------------------------------------------------------------------------------- inputs
def _activations(gen, rows, cols, dtype):
    """Tokens of different size, some channels several times as large as the others."""
    x = torch.randn((rows, cols), generator=gen, device="cuda")
    x *= torch.exp(0.4 * torch.randn((cols,), generator=gen, device="cuda"))
    x *= torch.exp(0.3 * torch.randn((rows, 1), generator=gen, device="cuda"))
    return x.to(dtype)


def _weights(gen, cols, inner):
    w = torch.randn((cols, inner), generator=gen, device="cuda") / math.sqrt(inner)
    return w.mul_(torch.rand((cols, 1), generator=gen, device="cuda") + 0.5)


def _gradient(gen, rows, cols, dtype):
    """Small, with heavy tails: most of a batch's tokens hardly matter."""
    g = torch.randn((rows, cols), generator=gen, device="cuda") * 2.0 ** -6
    return g.mul_(torch.exp(torch.randn((rows, 1), generator=gen, device="cuda"))).to(dtype)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind, dtype, rows, cols = case["kind"], _DTYPES[case["dtype"]], case["rows"], case["cols"]
    if kind == "quant":
        return dict(x=_gradient(gen, rows, cols, dtype) if case["stochastic"] else _weights(gen, rows, cols).to(dtype))
    if kind == "linear":
        return dict(x=_activations(gen, rows, case["inner"], dtype), w=_weights(gen, cols, case["inner"]).bfloat16(),
                    bias=torch.randn((cols,), generator=gen, device="cuda") if case["bias"] else None)
    if kind == "train":
        return dict(x=_activations(gen, rows, case["inner"], dtype), w=_weights(gen, cols, case["inner"]).to(dtype),
                    dy=_gradient(gen, rows, cols, dtype))
    # what is normalised is a part of a wider projection
    inputs = dict(x=_activations(gen, rows, cols + 64, dtype)[:, :cols], residual=_activations(gen, rows, cols, dtype),
                  weight=1.0 + 0.2 * torch.randn((cols,), generator=gen, device="cuda"))
    if kind == "norm_train":
        inputs.update(g=_gradient(gen, rows, cols, dtype), g_sum=_gradient(gen, rows, cols, dtype))
    return inputs


def prepare(case, seed):
    state = dict(_inputs(case, seed), case=case, seed=seed)
    if case["kind"] == "linear":                                        # the weights are laid out once
        if own:
            from paper_1804_01526_amd import hbfp
            state["w"] = hbfp.quant_mx4(state["w"])
        else:
            state["w"] = _mx4_plain(state["w"])
    return state


# ------------------------------------------------------------------------------------------------------------ plain form
def _hash_plain(rows, cols, seed):
    """The library's random word of every element: a hash of its position and the seed."""
    mask = 0xFFFFFFFF
    idx = torch.arange(rows * cols, device="cuda", dtype=torch.int64)
    x = (idx & mask) ^ (seed & mask)
    x = x ^ ((x << 13) & mask)
    x = x ^ (x >> 17)
    x = x ^ ((x << 5) & mask)
    x = (x + ((idx >> 32) ^ (seed >> 32))) & mask
    x = x ^ (x >> 16)
    x = (x * 0x85EBCA6B) & mask
    x = x ^ (x >> 13)
    x = (x * 0xC2B2AE35) & mask
    return (x ^ (x >> 16)).view(rows, cols)


def _mx4_plain(x, words=None):
    """The values that 4-bit numbers with a power of two per 32 along the last axis hold for x: to nearest (ties to even), or
    stochastically by `words`."""
    cols, pad = x.shape[-1], -x.shape[-1] % BLOCK
    xb = torch.nn.functional.pad(x.float(), (0, pad)).unflatten(-1, (-1, BLOCK))
    bits = xb.abs().amax(dim=-1, keepdim=True).view(torch.int32)
    byte = (((bits + (0x200000 if words is None else 0x3FFFFF)) >> 23).clamp(max=254) - 2).clamp(min=0)
    a = xb.abs() * ((254 - byte) << 23).view(torch.float32)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    if words is None:
        m = torch.round(a / step) * step
    else:
        u = torch.nn.functional.pad(words, (0, pad)).unflatten(-1, (-1, BLOCK)).double() * 2.0 ** -32
        m = (torch.floor((a / step).double() + u) * step).float()
    half = (byte - 127).div(2, rounding_mode="floor")                   # the power of two in two factors: neither ends too early
    unit = [((127 + e) << 23).view(torch.float32) for e in (half, byte - 127 - half)]
    return (torch.copysign(m.clamp(max=6.0), xb) * unit[0] * unit[1]).flatten(-2)[..., :cols]


def _linear_plain(state):
    y = torch.matmul(_mx4_plain(state["x"]), state["w"].t())
    if state["bias"] is not None:
        y = y + state["bias"]
    return y.to(state["x"].dtype)


def _down_plain(x, words=None):
    """Quantised down the columns: the values, transposed."""
    return _mx4_plain(x.t().contiguous(), None if words is None else words.t().contiguous())


def _train_plain(state):
    x, w, dy = state["x"], state["w"], state["dy"]
    words = _hash_plain(*dy.shape, state["seed"])
    y = torch.matmul(_mx4_plain(x), _mx4_plain(w).t())
    dx = torch.matmul(_mx4_plain(dy, words), _down_plain(w).t())
    dw = torch.matmul(_down_plain(dy, words), _down_plain(x).t())
    return y.to(x.dtype), dx.to(x.dtype), dw


def _quant_plain(state):
    x = state["x"]
    words = _hash_plain(*x.shape, state["seed"]) if state["case"]["stochastic"] else None
    return _mx4_plain(x, words).bfloat16(), _down_plain(x, words).bfloat16()


def _norm_plain(state, form):
    """In 64 bits up to the normalised FP32 values, whose codes change at borders."""
    x, weight = state["x"], state["weight"]
    total = (x.float() + state["residual"].float()).to(x.dtype)
    s = total.double()
    rstd = 1.0 / torch.sqrt((s * s).mean(dim=1, keepdim=True) + EPS)
    n = (s * rstd * weight.double()).float()
    if form == "i8":
        scale = n.abs().amax(dim=1, keepdim=True) * (1.0 / 127.0)
        by = torch.where(scale == 0, torch.ones_like(scale), scale)
        values = torch.round(n / by).clamp(-127, 127) * scale
    else:
        values = _mx4_plain(n)
    return total, rstd.float().squeeze(1), values.to(x.dtype)


def _norm_train_plain(state):
    total, rstd, values = _norm_plain(state, "mx4")
    g, s = state["g"].float(), total.float()
    gw = g * state["weight"]
    r = rstd.unsqueeze(1)
    inner = (gw * s).mean(dim=1, keepdim=True) * r * r
    dx = state["g_sum"].float() + r * (gw - s * inner)
    return total, rstd, values, dx.to(state["x"].dtype), (g * s * r).sum(dim=0)


# ------------------------------------------------------------------------------------------------------------------ runs
def run(state):
    case, kind = state["case"], state["case"]["kind"]
    if not own:
        if kind == "linear":
            return _linear_plain(state)
        if kind == "quant":
            return _quant_plain(state)
        if kind == "train":
            return _train_plain(state)
        return _norm_plain(state, case["form"]) if kind == "norm" else _norm_train_plain(state)
    from paper_1804_01526_amd import hbfp
    if kind == "linear":
        return hbfp.linear_mx4(state["x"], state["w"], bias=state["bias"])
    if kind == "quant":
        along, down = hbfp.quant_mx4_both(state["x"], hbfp.STOCHASTIC if case["stochastic"] else hbfp.RNE, state["seed"])
        return hbfp.read_mx4(along, torch.bfloat16), hbfp.read_mx4(down, torch.bfloat16)
    if kind == "train":
        x, w, dy = state["x"], state["w"], state["dy"]
        (x_along, x_down), (w_along, w_down) = hbfp.quant_mx4_both(x), hbfp.quant_mx4_both(w)
        dy_along, dy_down = hbfp.quant_mx4_both(dy, hbfp.STOCHASTIC, state["seed"])
        y = hbfp.gemm_mx4(x_along, w_along, dtype=x.dtype)
        return y, hbfp.gemm_mx4(dy_along, w_down, dtype=x.dtype), hbfp.gemm_mx4(dy_down, x_down)
    x, residual, weight = state["x"], state["residual"], state["weight"]
    if kind == "norm":
        norm = hbfp.norm_i8 if case["form"] == "i8" else hbfp.norm_mx4
        _, total, rstd, values = norm(x, weight, EPS, residual=residual, values=True)
        return total, rstd, values
    _, total, rstd, values = hbfp.norm_mx4(x, weight, EPS, residual=residual, values=True)
    dx, dweight = hbfp.norm_grad(state["g"], total, rstd, weight, g_sum=state["g_sum"])
    return total, rstd, values, dx, dweight


def work(case):
    kind, rows, cols, size = case["kind"], case["rows"], case["cols"], _BYTES[case["dtype"]]

    def held(r, k):                                                     # codes and scales
        return r * (k // 2 + -(-k // BLOCK))
    if kind == "linear":
        inner = case["inner"]
        return {"bytes": rows * inner * size + held(cols, inner) + rows * cols * size + (4 * cols if case["bias"] else 0),
                "flops": 2 * rows * cols * inner}
    if kind == "quant":                                                 # the source, and the values read back
        return {"bytes": rows * cols * (size + 4), "flops": 4 * rows * cols}
    if kind == "train":
        inner = case["inner"]
        inputs = rows * inner + cols * inner + rows * cols
        return {"bytes": inputs * size + rows * (cols + inner) * size + 4 * cols * inner, "flops": 6 * rows * cols * inner}
    if kind == "norm":                                                  # x, residual; sum, values, codes
        code = rows * cols + 4 * rows if case["form"] == "i8" else held(rows, cols)
        return {"bytes": rows * cols * 4 * size + code + 4 * rows + 4 * cols, "flops": 6 * rows * cols}
    # ... and back: both gradients and the sum again; the gradient of x, that of the weight
    return {"bytes": rows * cols * 8 * size + held(rows, cols) + 8 * rows + 12 * cols, "flops": 14 * rows * cols}


# ----------------------------------------------------------------------------------------------------------------- exact
_MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_words(rows, cols, seed):
    with np.errstate(over="ignore"):
        idx = np.arange(rows * cols, dtype=np.uint64)
        x = (idx & np.uint64(0xFFFFFFFF)).astype(np.uint32) ^ np.uint32(seed & 0xFFFFFFFF)
        x ^= x << np.uint32(13)
        x ^= x >> np.uint32(17)
        x ^= x << np.uint32(5)
        x += (idx >> np.uint64(32)).astype(np.uint32) ^ np.uint32(seed >> 32)
        x ^= x >> np.uint32(16)
        x *= np.uint32(0x85EBCA6B)
        x ^= x >> np.uint32(13)
        x *= np.uint32(0xC2B2AE35)
        x ^= x >> np.uint32(16)
    return torch.from_numpy(x.astype(np.float64) / 2.0 ** 32).reshape(rows, cols).cuda()


def _exact_mx4(x, u=None):
    """Block by block: the power of two from the largest magnitude, then the neighbours in the table of magnitudes."""
    x = x.double()
    out = torch.zeros_like(x)
    table = torch.tensor(_MAGNITUDES, dtype=torch.float64, device=x.device)
    for k0 in range(0, x.shape[1], BLOCK):
        part = x[:, k0:k0 + BLOCK]
        top = part.abs().amax(dim=1, keepdim=True)
        frac, e = torch.frexp(top)                                      # top = frac * 2^e, 0.5 <= frac < 1
        e = e - 1 + ((frac >= 0.875) if u is None else (frac > 0.75)).to(e.dtype)
        e = torch.where(top == 0, -125, e).clamp(min=-125) - 2
        unit = ((e.long() + 1023) << 52).view(torch.float64)            # 2^e
        a = part.abs() / unit
        below = (torch.searchsorted(table, a.contiguous(), right=True) - 1).clamp(max=6)
        lo, hi = table[below], table[below + 1]
        if u is None:
            up = (a - lo > hi - a) | ((a - lo == hi - a) & (below % 2 == 1))
        else:
            up = (a - lo) / (hi - lo) + u[:, k0:k0 + BLOCK] >= 1.0
        out[:, k0:k0 + BLOCK] = torch.copysign(torch.where(up, hi, lo), part) * unit
    return out


def _exact_norm(state, form):
    x = state["x"]
    s = (x.float() + state["residual"].float()).to(x.dtype).double()
    mean = torch.linalg.vector_norm(s, dim=1, keepdim=True) ** 2 / s.shape[1]
    rstd = (mean + EPS).rsqrt()
    n = ((s * rstd) * state["weight"].double()).float()
    if form == "mx4":
        return s, rstd.squeeze(1), _exact_mx4(n)
    n = n.cpu().numpy()
    scale = (np.abs(n).max(axis=1) * np.float32(1 / 127)).astype(np.float32)
    by = np.where(scale == 0, np.float32(1), scale)
    codes = np.clip(np.rint((n / by[:, None]).astype(np.float32)), -127, 127).astype(np.float64)
    return s, rstd.squeeze(1), torch.from_numpy(codes * scale[:, None].astype(np.float64)).cuda()


def exact(case, seed):
    kind, state = case["kind"], _inputs(case, seed)
    if kind == "quant":
        x = state["x"]
        u = _exact_words(*x.shape, seed) if case["stochastic"] else None
        return _exact_mx4(x, u), _exact_mx4(x.t(), None if u is None else u.t())
    if kind == "linear":
        y = _exact_mx4(state["x"]) @ _exact_mx4(state["w"]).t().contiguous()
        return y if state["bias"] is None else y + state["bias"].double()
    if kind == "train":
        x, w, dy = state["x"], state["w"], state["dy"]
        u = _exact_words(*dy.shape, seed)
        y = _exact_mx4(x) @ _exact_mx4(w).t().contiguous()
        dx = _exact_mx4(dy, u) @ _exact_mx4(w.t()).t().contiguous()
        return y, dx, _exact_mx4(dy.t(), u.t()) @ _exact_mx4(x.t()).t().contiguous()
    if kind == "norm":
        return _exact_norm(state, case["form"])
    s, rstd, values = _exact_norm(state, "mx4")
    g, weight = state["g"].double(), state["weight"].double()
    unit = s * rstd.unsqueeze(1)                                        # rows of mean square one
    through = g * weight
    dx = rstd.unsqueeze(1) * (through - unit * (through * unit).mean(dim=1, keepdim=True)) + state["g_sum"].double()
    return s, rstd, values, dx, (g * unit).sum(dim=0)
