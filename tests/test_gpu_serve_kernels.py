"""The serving operators' kernels at sizes that reach each of them, against 64 bits on the GPU.

Attention is compared on the values that the cache holds (hbfp_cache_read, itself held to the definition in test_gpu_serve.py).
Tolerances.  With u the unit roundoff of the output's type, w that of the softmax weights as the products take them (2^-16 for bf16
and FP16: two pieces of 8 bits; 2^-24 for FP32) and d the relative error of an exponential,
    d = (dim + 16) 2^-24 max|scale q k| + (64 + keys / 32) 2^-24,
a sum before its rounding is off by e = (w + 2 d) sum p |v|, and an output by e + u (|out| + e); lse by d + 2^-22 (1 + |lse|)."""
import math

import numpy as np
import pytest
import torch

from tests.util import launched_kernels

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
U_WEIGHT = {F32: 2.0 ** -24, BF16: 2.0 ** -16, F16: 2.0 ** -16}


@pytest.fixture(scope="module")
def hb():
    from paper_1804_01526_amd import hbfp
    assert torch.cuda.is_available(), "these tests need the GPU"
    return hbfp


def _lens(lengths):
    return torch.tensor(lengths, dtype=torch.int32, device="cuda")


def _randn(gen, shape, dtype=F32, spread=1):
    x = torch.randn(shape, generator=gen, device="cuda")
    return (x * torch.exp2(torch.randint(-spread, spread + 1, shape, generator=gen, device="cuda").float())).to(dtype)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _filled(hb, gen, batch, heads, capacity, dim, lengths, values=lambda v: v):
    """A cache of `lengths` tokens a batch entry in poisoned buffers, and the FP64 keys and values it holds."""
    cache = hb.cache_alloc(batch, heads, capacity, dim)
    for t in (cache.k, cache.v, cache.k_exps, cache.v_exps):
        t.fill_(255)
    if max(lengths) > 0:
        k, v = (_randn(gen, (batch, max(lengths), heads, dim)) for _ in range(2))
        hb.cache_append(cache, k, values(v), _lens(lengths))
    k, v = hb.cache_read(cache, _lens(lengths))
    return cache, k.double(), v.double()


def _attend64(k, v, q, lengths, scale, causal=True, longest=None):
    """(out, lse, spread, noise) in 64 bits: spread = sum p |v|, noise = the largest sum of |scale q k| of a visible key; and the
    weights that each key of each key head received, [batch][key head][slot]."""
    batch, tokens, heads, dim = q.shape
    kv, capacity = k.shape[1], k.shape[2]
    group = heads // kv
    out, spread = (torch.zeros(q.shape, dtype=torch.float64, device="cuda") for _ in range(2))
    lse = torch.full((batch, tokens, heads), -math.inf, dtype=torch.float64, device="cuda")
    noise = torch.zeros((batch, tokens, heads), dtype=torch.float64, device="cuda")
    got = torch.zeros((batch, kv, capacity), dtype=torch.float64, device="cuda")
    at, t = torch.arange(capacity, device="cuda"), torch.arange(tokens, device="cuda").unsqueeze(1)
    for b, n in enumerate(lengths):
        bound = min(longest or capacity, capacity)
        seen = torch.clamp(n - tokens + t + 1 if causal else torch.full_like(t, n), max=bound)
        hidden = (at >= seen).repeat_interleave(group, dim=0)                    # rows: token, head of the group
        for h in range(kv):
            rows = q[b, :, h * group:(h + 1) * group].double().reshape(tokens * group, dim)
            kt = k[b, h].t().contiguous()
            s = (scale * (rows @ kt)).masked_fill(hidden, -math.inf)
            top = s.amax(dim=1, keepdim=True)
            w = torch.exp(s - torch.where(torch.isinf(top), torch.zeros_like(top), top))
            total = w.sum(dim=1, keepdim=True)
            p = w / torch.where(total == 0, torch.ones_like(total), total)
            put = lambda dst, x: dst[b, :, h * group:(h + 1) * group].copy_(x.reshape(tokens, group, *x.shape[1:]))
            put(out, p @ v[b, h])
            put(spread, p @ v[b, h].abs())
            put(lse, torch.log(total[:, 0]) + torch.where(torch.isinf(top), torch.zeros_like(top), top)[:, 0])
            put(noise, ((scale * rows).abs() @ kt.abs()).masked_fill(hidden, 0).amax(dim=1))
            got[b, h] = p.sum(dim=0)
    return out, lse, spread, noise, got


def _check_attend(got, got_lse, want, dtype, dim, keys):
    out, lse, spread, noise, _ = want
    d = (dim + 16) * 2.0 ** -24 * noise + (64 + keys / 32) * 2.0 ** -24
    e = (U_WEIGHT[dtype] + 2 * d.unsqueeze(-1)) * spread
    tol = e + U[dtype] * (out.abs() + e) + (2.0 ** -25 if dtype == F16 else 2.0 ** -140)
    assert torch.isfinite(got).all()
    ratio = ((got.double() - out).abs() / tol).max().item()
    assert ratio <= 1, f"out: {ratio:.3f} of the tolerance"
    empty = torch.isneginf(lse)
    assert torch.equal(torch.isneginf(got_lse), empty) and (got[empty] == 0).all()
    ratio = ((got_lse.double() - lse).abs() / (d + 2.0 ** -22 * (1 + lse.abs())))[~empty].max().item()
    assert ratio <= 1, f"lse: {ratio:.3f} of the tolerance"


# ------------------------------------------------------------------------------------------------------------- attention
@pytest.mark.parametrize("batch,tokens,kv,group,dim,capacity,lengths", [
    (2, 1, 2, 4, 64, 100, [100, 37]),                # one chunk of keys
    (1, 1, 2, 8, 128, 5000, [4999]),                 # several
    (2, 3, 1, 4, 256, 700, [700, 300]),
    (1, 100, 2, 2, 128, 300, [300]),                 # a prompt
    (2, 70, 1, 3, 72, 900, [900, 100]),
])
def test_bf16_outputs_lose_their_own_rounding_only(hb, batch, tokens, kv, group, dim, capacity, lengths):
    """Softmax weights of bf16 calls enter the products with 16 bits."""
    print(f"[attend] bf16 b{batch} t{tokens} h{kv}x{group} dim {dim} lengths {lengths}", flush=True)
    gen = _gen(dim + tokens)
    cache, k, v = _filled(hb, gen, batch, kv, capacity, dim, lengths)
    q = _randn(gen, (batch, tokens, kv * group, dim), BF16)
    out, lse = hb.cache_attend(cache, q, _lens(lengths))
    _check_attend(out, lse, _attend64(k, v, q, lengths, dim ** -0.5), BF16, dim, capacity)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("batch,tokens,kv,group,dim,capacity,lengths", [
    (2, 1, 2, 4, 64, 100, [100, 37]),
    (1, 2, 1, 4, 128, 3000, [2999]),
    (1, 60, 1, 2, 96, 1200, [1200]),
    (2, 130, 1, 1, 64, 140, [140, 90]),
])
@pytest.mark.parametrize("power", [126, 60, -60])
def test_values_of_every_magnitude(hb, dtype, batch, tokens, kv, group, dim, capacity, lengths, power):
    """Values up to 2^127, all of one sign: sums of many weights times the largest stay finite, equal scores among them."""
    print(f"[attend] values of 2^{power}: {dtype} b{batch} t{tokens} dim {dim} lengths {lengths}", flush=True)
    gen = _gen(dim + tokens)
    cache, k, v = _filled(hb, gen, batch, kv, capacity, dim, lengths, lambda x: (1 + x.abs().clamp(max=8) / 16) * 2.0 ** power)
    q = _randn(gen, (batch, tokens, kv * group, dim), dtype)
    q[:, :, 0] = 0
    out, lse = hb.cache_attend(cache, q, _lens(lengths))
    assert v.max() >= 2.0 ** power
    _check_attend(out, lse, _attend64(k, v, q, lengths, dim ** -0.5), dtype, dim, capacity)


def test_tiny_values_lose_an_absolute_amount_only(hb):
    print("[attend] tiny values", flush=True)
    gen = _gen(11)
    for tokens in (1, 70):
        cache, k, v = _filled(hb, gen, 1, 1, 300, 64, [300], lambda x: x * 2.0 ** -110)
        q = _randn(gen, (1, tokens, 2, 64), F32)
        out, _ = hb.cache_attend(cache, q, _lens([300]))
        want = _attend64(k, v, q, [300], 0.125)
        assert ((out.double() - want[0]).abs() <= 2.0 ** -90).all()


# --------------------------------------------------------------------------------------------------------------- streams
def test_results_on_another_stream_do_not_take_memory_in_use(hb):
    """The caller's stream still has a kernel queued that reads a tensor just dropped; a call on another stream does not wait for it."""
    print("[streams] memory in use", flush=True)
    gen = _gen(12)
    x, w = _randn(gen, (512, 256), BF16), hb.quant_rows(_randn(gen, (2048, 256)))
    negative = -x                                              # (inputs are ready before the other stream is used)
    want = hb.linear_i8(x, w)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    dropped = torch.full((512, 2048), 3.0, device="cuda", dtype=BF16)
    torch.cuda._sleep(100_000_000)                             # tens of milliseconds
    twice = dropped * 2
    del dropped
    got = hb.linear_i8(x, w, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    assert (twice == 6).all() and torch.equal(got, want)
    # a result that the caller's stream still reads when it is dropped is not given to the other stream's next call
    torch.cuda._sleep(100_000_000)
    twice = got * 2
    del got
    again = hb.linear_i8(negative, w, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(twice, want * 2) and torch.equal(again, -want)


# --------------------------------------------------------------------------------------------------------------- weights
@pytest.mark.parametrize("dtype,tokens,dim,lengths,longest,causal", [
    (F32, 1, 64, [900, 20], 100, True),
    (BF16, 5, 128, [300, 299], 256, False),
    (F16, 40, 40, [700, 333], 640, True),
    (F32, 2, 32, [500, 120], 130, False),
    (BF16, 3, 96, [260, 1], 10 ** 9, True),
])
def test_weights_of_a_call_that_sees_the_first_keys_only(hb, dtype, tokens, dim, lengths, longest, causal):
    """cache_weigh with the `longest` of the attention call before it: a query's weights sum to 1, keys from there on receive none."""
    print(f"[weigh] longest {longest} of {lengths}, {dtype} t{tokens} dim {dim}", flush=True)
    gen, kv, group, capacity = _gen(13), 2, 3, 1000
    cache, k, v = _filled(hb, gen, 2, kv, capacity, dim, lengths)
    q = _randn(gen, (2, tokens, kv * group, dim), dtype)
    _, lse = hb.cache_attend(cache, q, _lens(lengths), causal=causal, longest=longest)
    before = torch.rand((2, kv, capacity), generator=gen, device="cuda")
    w = hb.cache_weigh(cache, q, lse, _lens(lengths), before, causal=causal, decay=0.5, out=torch.full_like(before, 9.0), longest=longest)
    _, want_lse, _, noise, got = _attend64(k, v, q, lengths, dim ** -0.5, causal, longest)
    for b, n in enumerate(lengths):
        want = 0.5 * before[b].double() + got[b]
        want[:, n:] = 0
        seen = want_lse[b][torch.isfinite(want_lse[b])]
        d = (dim + 16) * 2.0 ** -24 * noise[b].max() + (64 + capacity / 32) * 2.0 ** -24 + 2.0 ** -21 * (1 + seen.abs().max())
        assert ((w[b].double() - want).abs() <= (2 * d + tokens * group * 2.0 ** -24) * want).all()
        assert torch.equal(w[b, :, min(longest, n):n], 0.5 * before[b, :, min(longest, n):n])


# -------------------------------------------------------------------------------------------------------------- products
def test_linear_between_columns_of_one_matrix_and_attention_over_its_queries(hb):
    """Inputs and outputs that interleave in memory without sharing an element; out written over q."""
    print("[linear] columns of one matrix", flush=True)
    gen = _gen(14)
    w = hb.quant_rows(_randn(gen, (200, 300)))
    for m in (1, 2, 5, 40):
        both = _randn(gen, (m, 504), BF16)
        x, y = both[:, :300], both[:, 304:]
        want, kept = hb.linear_i8(x.clone(), w), x.clone()
        assert torch.equal(hb.linear_i8(x, w, out=y), want) and torch.equal(x, kept)
    for tokens, capacity in ((1, 90), (1, 5000), (80, 90), (70, 2000)):
        cache, _, _ = _filled(hb, gen, 1, 2, capacity, 64, [capacity])
        q = _randn(gen, (1, tokens, 8, 64), BF16)
        want = hb.cache_attend(cache, q, _lens([capacity]))[0]
        assert torch.equal(hb.cache_attend(cache, q, _lens([capacity]), out=q)[0], want)


PROMPTS = [
    # rows a workgroup, batch, tokens, key heads, group, capacity, lengths, causal
    (256, 4, 129, 16, 4, 1100, [1100, 600, 129, 50], True),          # three chunks; a last tile of 4 rows; padding on the left
    (256, 8, 300, 16, 2, 500, [500, 499, 300, 299, 1, 0, 64, 333], True),    # one chunk; conversations of no token, of one
    (256, 4, 200, 16, 2, 1300, [1290, 65, 0, 1024], False),
    (128, 4, 100, 16, 1, 2100, [2100, 1111, 100, 3], True),
    (128, 16, 60, 16, 2, 400, [400 - 26 * i for i in range(16)], True),      # one chunk
    (128, 16, 35, 16, 3, 260, [0, 1, 257] + [20 * i for i in range(13)], False),
    (64, 1, 50, 2, 3, 300, [277], True),
    (64, 2, 66, 1, 1, 1700, [1700, 30], True),
]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("dim", [32, 41, 96, 128])
@pytest.mark.parametrize("rows,batch,tokens,kv,group,capacity,lengths,causal", PROMPTS)
def test_every_kernel_for_prompts(hb, rows, batch, tokens, kv, group, capacity, lengths, causal, dim, dtype):
    print(f"[prompt] {rows} rows, {dtype} b{batch} t{tokens} h{kv}x{group} dim {dim} cap {capacity} lengths {lengths}", flush=True)
    gen = _gen(dim + tokens)
    cache, k, v = _filled(hb, gen, batch, kv, capacity, dim, lengths)
    q = _randn(gen, (batch, tokens, kv * group, dim), dtype)
    call = lambda: hb.cache_attend(cache, q, _lens(lengths), causal=causal)
    kernel = f"cache_prompt_kernel<{-(-dim // 32)}, {[F32, BF16, F16].index(dtype)}, {rows // 32}>"
    assert kernel in launched_kernels(call)
    out, lse = call()
    _check_attend(out, lse, _attend64(k, v, q, lengths, dim ** -0.5, causal), dtype, dim, capacity)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("dim", [31, 64, 90, 128, 160, 170, 224, 256])
@pytest.mark.parametrize("batch,tokens,kv,group,capacity,lengths", [(2, 1, 2, 4, 1000, [1000, 77]), (3, 3, 2, 2, 128, [128, 2, 0]), (1, 20, 2, 1, 3000, [2977])])
def test_every_kernel_for_few_queries(hb, batch, tokens, kv, group, capacity, lengths, dim, dtype):
    print(f"[attend] {dtype} b{batch} t{tokens} h{kv}x{group} dim {dim} cap {capacity} lengths {lengths}", flush=True)
    gen = _gen(dim + tokens)
    cache, k, v = _filled(hb, gen, batch, kv, capacity, dim, lengths)
    q = _randn(gen, (batch, tokens, kv * group, dim), dtype)
    call = lambda: hb.cache_attend(cache, q, _lens(lengths))
    assert f"cache_attend_kernel<{-(-dim // 32)}, {[F32, BF16, F16].index(dtype)}>" in launched_kernels(call)
    out, lse = call()
    want = _attend64(k, v, q, lengths, dim ** -0.5)
    _check_attend(out, lse, want, dtype, dim, capacity)
    w = hb.cache_weigh(cache, q, lse, _lens(lengths), torch.zeros((batch, kv, capacity), device="cuda"))
    d = (dim + 16) * 2.0 ** -24 * want[3].max() + (64 + capacity / 32) * 2.0 ** -24 + 2.0 ** -21 * (1 + want[1][torch.isfinite(want[1])].abs().max())
    assert ((w.double() - want[4]).abs() <= (2 * d + tokens * group * 2.0 ** -24) * want[4]).all()


PRODUCTS = [
    # the kernel (and that for its slices), M, N, K
    ("gemm_rows_few_kernel<1, 2, 16, {t}, true>", 1, 5120, 300), ("gemm_rows_few_kernel<1, 2, 16, {t}, true>", 2, 77, 16384),
    ("gemm_rows_few_kernel<1, 4, 8, {t}, true>", 1, 5121, 1000), ("gemm_rows_few_kernel<1, 4, 8, {t}, true>", 1, 20001, 129),
    ("gemm_rows_few_kernel<1, 4, 8, {t}, true>", 2, 16384, 513),
    ("gemm_rows_few_kernel<1, 8, 4, {t}, false>", 2, 16385, 200), ("gemm_rows_few_kernel<1, 8, 4, {t}, false>", 16, 8193, 1100),
    ("gemm_rows_few_kernel<1, 8, 4, {t}, false>", 1, 8200, 33000), ("gemm_rows_few_kernel<1, 4, 8, {t}, false>", 16, 8192, 70),
    ("gemm_rows_few_kernel<1, 4, 8, {t}, false>", 3, 50, 5000), ("gemm_rows_few_kernel<2, 1, 16, {t}, false>", 32, 130, 4096),
    ("gemm_rows_few_kernel<2, 1, 16, {t}, false>", 17, 4099, 1000),
    ("gemm_i8_wide_kernel<2, 64, 4, {o}, ", 96, 88, 33), ("gemm_i8_wide_kernel<2, 64, 4, {o}, +rows_sum_kernel<{o}>", 72, 65, 1962),
    ("gemm_i8_wide_kernel<2, 64, 4, {o}, +rows_sum_kernel<{o}>", 65, 64, 4000), ("gemm_i8_wide_kernel<2, 64, 4, {o}, +rows_sum_kernel<{o}>", 130, 70, 40001),
    ("gemm_i8_wide_kernel<2, 64, 4, {o}, +rows_sum_kernel<{o}>", 70, 66, 133144),
    ("gemm_i8_wide_kernel<2, 128, 4, {o}, +rows_sum_kernel<{o}>", 130, 499, 133144), ("gemm_i8_wide_kernel<2, 128, 4, {o}, ", 900, 941, 3155),
    ("gemm_i8_wide_kernel<2, 128, 2, {o}, ", 2446, 1571, 1155), ("gemm_i8_wide_kernel<2, 128, 2, {o}, +rows_sum_kernel<{o}>", 1289, 927, 5642),
    ("gemm_i8_wide_kernel<3, 64, 4, {o}, ", 2187, 3884, 33), ("gemm_i8_wide_kernel<3, 128, 3, {o}, ", 2506, 3091, 1025),
    ("gemm_i8_wide_kernel<4, 64, 4, {o}, ", 2973, 3586, 2454), ("gemm_i8_wide_kernel<4, 128, 2, {o}, ", 4495, 3351, 133),
    ("gemm_i8_wide_kernel<4, 128, 2, {o}, ", 4608, 3328, 260),
]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("kernel,m,n,k", PRODUCTS)
def test_every_kernel_for_products(hb, kernel, m, n, k, dtype):
    """The int32 sum is exact; two scales and a bias are three FP32 roundings, the output one of its type."""
    print(f"[product] {kernel} {dtype} {m}x{n}x{k}", flush=True)
    gen, t = _gen(m + n + k), [F32, BF16, F16].index(dtype)
    x, w = _randn(gen, (m, k), dtype, 2), hb.quant_rows(_randn(gen, (n, k)))
    bias = torch.randn(n, generator=gen, device="cuda")
    names = launched_kernels(lambda: hb.linear_i8(x, w, bias=bias))
    for part in kernel.format(t=t, o=t + 1).split("+"):
        assert any(name.startswith(part) for name in names), names
    a = hb.quant_rows(x)
    sums = a.codes[:, :k].double() @ w.codes[:, :k].double().t().contiguous()
    product = sums * a.scales.double().unsqueeze(1) * w.scales.double()
    for b, offset, pitch in ((bias, 0, n), (None, 0, n + n % 2 + 2), (bias, 1, n + n % 2 + 4), (None, 2, n + 1 - n % 2)):
        exact = product if b is None else product + b.double()
        tol = U[dtype] * exact.abs() + 2.0 ** -22 * (product.abs() + exact.abs()) + (2.0 ** -24 if dtype == F16 else 0)
        room = torch.full((m * pitch + offset,), 5.0, device="cuda", dtype=dtype)
        y = room[offset:].view(m, pitch)[:, :n]
        assert hb.linear_i8(x, w, bias=b, out=y) is y
        assert ((y.double() - exact).abs() <= tol).all()
        y.fill_(5.0)
        assert (room == 5).all(), "bytes around the output"


@pytest.mark.parametrize("dtype,stream", [(F32, "true"), (BF16, "false"), (F16, "false")])
def test_products_of_16_bits_have_one_kind_of_store(hb, dtype, stream):
    gen = _gen(16)
    x, w = _randn(gen, (900, 3155), dtype), hb.quant_rows(_randn(gen, (941, 3155)))
    assert f"gemm_i8_wide_kernel<2, 128, 4, {[F32, BF16, F16].index(dtype) + 1}, {stream}>" in launched_kernels(lambda: hb.linear_i8(x, w))


# ------------------------------------------------------------------------------------------------------------- the layer
@pytest.mark.parametrize("batch,heads,kv_heads,dim,prompt,steps", [(5, 8, 2, 64, 200, 70), (1, 6, 6, 80, 256, 20), (3, 4, 1, 128, 37, 10)])
def test_the_layer_of_the_example_on_the_values_its_cache_holds(hb, batch, heads, kv_heads, dim, prompt, steps):
    """examples/serve_layer.py against 64 bits whose operands are what the layer holds: 8-bit weights and tokens, the cache's values.
    Tolerances (of the norm): q and the attention's output are rounded to bf16, 0.0011 each in the RMS; that moves a twentieth of the
    output's 8-bit codes (a step is 0.024 of a standard deviation) by one, 0.0054; 0.02 leaves a factor of three.  A token too many or
    missing, of 256, is 0.06.  New tokens in the cache are the 4-bit values of the layer's own k and v but where the bf16 rounding of the
    product moves a 4-bit code, one in a hundred by a quarter of a standard deviation: 0.03; the wrong slot is 1.4."""
    from examples.serve_layer import Layer
    from tests import serve_ref
    print(f"[layer] b{batch} h{heads}/{kv_heads} dim {dim} prompt {prompt} steps {steps}", flush=True)
    gen, features, capacity = _gen(15), 384, 256
    w_qkv, w_out = (_randn(gen, shape, BF16, 0) / math.sqrt(shape[1]) for shape in (((heads + 2 * kv_heads) * dim, features), (features, heads * dim)))
    layer = Layer(w_qkv, w_out, batch, heads, kv_heads, dim, capacity)
    values = lambda c: c.codes[:, :c.cols].double() * c.scales.double().unsqueeze(1)
    product = lambda x, w: values(hb.quant_rows(x)) @ values(w).t().contiguous()
    relative = lambda got, want: ((got.double() - want).norm() / want.norm()).item()
    lengths = [max(1, prompt - 30 * b) for b in range(batch)]
    counts = list(lengths)
    history = [[torch.zeros((kv_heads, 0, dim), dtype=torch.float64, device="cuda") for _ in range(2)] for _ in range(batch)]
    for step in range(steps + 1):
        if max(lengths) + (step > 0) > capacity:
            kept = layer.shrink(64, 16)
            for b, n in enumerate(lengths):
                m = min(n, 64)
                assert (kept[b, :, m:] == -1).all() and (n <= 64 or (kept[b, :, 48:] == torch.arange(n - 16, n, device="cuda")).all())
                at = kept[b, :, :m].long().unsqueeze(2).expand(-1, -1, dim)
                history[b] = [t.gather(1, at) for t in history[b]]
                lengths[b] = m
        tokens = max(counts) if step == 0 else 1
        if step:
            counts, lengths = [1] * batch, [n + 1 for n in lengths]
        x = _randn(gen, (batch, tokens, features), BF16, 0)
        y = layer.step(x, torch.tensor(counts, dtype=torch.int32, device="cuda"))
        assert layer.lengths.tolist() == lengths
        k, v = (t.double() for t in hb.cache_read(layer.cache, layer.lengths))
        qkv = product(x.view(batch * tokens, features), layer.w_qkv).to(BF16).view(batch, tokens, -1, dim)
        for b, n in enumerate(counts):
            for i, (held, h0) in enumerate(((k, heads), (v, heads + kv_heads))):
                new = torch.from_numpy(serve_ref.cached(qkv[b, tokens - n:, h0:h0 + kv_heads].double().cpu().numpy())).cuda().transpose(0, 1)
                history[b][i] = torch.cat([history[b][i], new], dim=1)
                assert relative(held[b, :, :lengths[b]], history[b][i]) < 0.03
        out = _attend64(k, v, qkv[:, :, :heads], lengths, dim ** -0.5)[0].to(BF16)
        want = product(out.view(batch * tokens, heads * dim), layer.w_out).view(batch, tokens, features)
        for b, n in enumerate(counts):
            assert relative(y[b, tokens - n:], want[b, tokens - n:]) < 0.02, (step, b)
