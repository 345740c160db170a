"""The serving operators on the GPU against their definitions in 64 bits (tests/serve_ref.py).

Tolerances.  What a cache holds, the slots that stay and int8 codes are exact.  Attention: with u the unit roundoff (2^-8 bf16,
2^-11 FP16, 2^-24 FP32) and pieces of 8 bits for the weights (1, 2, 3), an output may be off by
    u |out|  +  (2^-8, 2^-16, 2^-24 for the weights) sum p |v|  +  2 d sum p |v|,
    d = (dim + 16) 2^-24 noise + (64 + keys / 32) 2^-24  (scores: one rounding per product; exponentials and sums)
and lse by d + 2^-22 (1 + |lse|).  Products: the int32 sum is exact, two scales and a bias are three FP32 roundings and the
output one of its type."""
import numpy as np
import pytest
import torch

from tests import serve_ref

pytestmark = pytest.mark.gpu

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
U_WEIGHT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -16}
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def hb():
    from paper_1804_01526_amd import hbfp
    assert torch.cuda.is_available(), "these tests need the GPU"
    return hbfp


def _rand(rng, shape, dtype, spread=2):
    x = rng.standard_normal(shape) * np.exp2(rng.integers(-spread, spread + 1, size=shape))
    return torch.from_numpy(x.astype(np.float32)).cuda().to(dtype)


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _lens(lengths):
    return torch.tensor(lengths, dtype=torch.int32, device="cuda")


def _filled(hb, rng, batch, heads, capacity, dim, past, poison=True):
    """A cache holding `past` tokens of each batch entry (buffers poisoned first) and its 64-bit twin."""
    cache = hb.cache_alloc(batch, heads, capacity, dim)
    if poison:
        for t in (cache.k, cache.v, cache.k_exps, cache.v_exps):
            t.fill_(255)
    twin = serve_ref.Cache(batch, heads, capacity, dim)
    longest = max(past)
    if longest > 0:
        k, v = _rand(rng, (batch, longest, heads, dim), F32, 1), _rand(rng, (batch, longest, heads, dim), F32, 1)
        hb.cache_append(cache, k, v, _lens(past))
        twin.append(_np(k), _np(v), past)
    return cache, twin


def _check_attend(got, lse, want, dtype, dim, keys):
    out, want_lse, spread, noise, _ = want
    d = (dim + 16) * 2.0 ** -24 * noise + (64 + keys / 32) * 2.0 ** -24
    tol = U[dtype] * np.abs(out) + U_WEIGHT[dtype] * spread + 2 * d[..., None] * spread + 1e-30
    err = np.abs(_np(got) - out)
    assert np.isfinite(_np(got)).all()
    assert (err <= tol).all(), f"out: {(err / tol).max():.3f} of the tolerance"
    empty = np.isneginf(want_lse)
    got_lse = _np(lse)
    assert np.array_equal(np.isneginf(got_lse), empty) and (_np(got)[empty] == 0).all()
    e = np.abs(got_lse[~empty] - want_lse[~empty])
    t = (d + 2.0 ** -22 * (1 + np.abs(np.where(empty, 0, want_lse))))[~empty]
    assert (e <= t).all(), f"lse: {(e / t).max():.3f} of the tolerance"


# ------------------------------------------------------------------------------------------------------------ the cache
@pytest.mark.parametrize("dtype,batch,heads,capacity,dim,tokens,lengths", [
    (F32, 1, 1, 1, 1, 1, [1]),
    (F32, 2, 3, 70, 7, 5, [5, 3]),                       # padding on the left
    (BF16, 3, 2, 64, 32, 9, [9, 0, 30]),
    (F16, 1, 4, 130, 40, 130, [130]),
    (F32, 2, 1, 65, 128, 4, [67, 64]),                   # past the capacity
    (BF16, 1, 2, 33, 256, 33, [33]),
    (F16, 2, 2, 12, 200, 1, [12, -3]),
    (F32, 1, 2, 50, 96, 50, [49]),
])
def test_append_holds_the_definition_s_values(hb, dtype, batch, heads, capacity, dim, tokens, lengths):
    print(f"[append] {dtype} {batch}x{heads} cap {capacity} dim {dim} tokens {tokens} lengths {lengths}", flush=True)
    rng = np.random.default_rng(dim + tokens)
    cache, twin = _filled(hb, rng, batch, heads, capacity, dim, [0] * batch)
    k, v = _rand(rng, (batch, tokens, heads, dim), dtype, 5), _rand(rng, (batch, tokens, heads, dim), dtype, 5)
    k[:, :, :, dim // 2:] *= 2.0 ** -4
    held = hb.cache_append(cache, k, v, _lens(lengths), values=True)
    twin.append(_np(k), _np(v), lengths)
    for read_type in (F32, BF16):
        got_k, got_v = hb.cache_read(cache, _lens(lengths), read_type)
        for got, want in ((got_k, twin.k), (got_v, twin.v)):
            want, got = want.copy(), _np(got)
            for b, n in enumerate(lengths):
                want[b, :, max(0, min(n, capacity)):] = 0
                never = slice(0, max(0, min(max(n, 0) - tokens, capacity)))        # slots nothing was written to hold anything
                want[b, :, never] = got[b, :, never] = 0
            np.testing.assert_array_equal(got, want)
    for got, x in zip(held, (k, v)):
        want = serve_ref.cached(_np(x))
        for b, n in enumerate(lengths):
            for t in range(tokens):
                if not 0 <= max(n, 0) - tokens + t < capacity:
                    want[b, t] = 0
        np.testing.assert_array_equal(_np(got), want)


def test_append_extremes_and_neighbours(hb):
    """Rounding ties, the raised exponent, zeros, subnormals, the largest magnitudes; tokens appended one by one leave their
    neighbours' nibbles alone."""
    print("[append] extremes", flush=True)
    dim, heads = 64, 2
    x = np.zeros((1, 11, heads, dim), dtype=np.float32)
    x[0, 0, :, :8] = [4, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 3.5]        # unit 1: ties
    x[0, 1, :, :3] = [7.5, 1, -7.4]                                    # the largest rounds to 8: unit 2
    x[0, 2, :, :2] = [7.49, -0.0]
    x[0, 3, :, :4] = [2.0 ** -126, 2.0 ** -127, -2.0 ** -128, 2.0 ** -149]
    x[0, 4, :, :2] = [1.7 * 2.0 ** 126, -2.0 ** 124]
    x[0, 5, :, 32:] = 1.0                                              # one block of zeros
    x[0, 6, :, :2] = [2.0 ** -140, 2.0 ** -149]
    x[0, 7:] = np.random.default_rng(0).standard_normal((4, heads, dim))
    cache = hb.cache_alloc(1, heads, 11, dim)
    for t in cache.k, cache.v, cache.k_exps, cache.v_exps:
        t.fill_(255)
    src = torch.from_numpy(x).cuda()
    for t in range(11):
        hb.cache_append(cache, src[:, t:t + 1], -src[:, t:t + 1], _lens([t + 1]))
    k, v = hb.cache_read(cache, _lens([11]))
    want = serve_ref.cached(x).transpose(0, 2, 1, 3)
    np.testing.assert_array_equal(_np(k), want)
    np.testing.assert_array_equal(_np(v), -want)
    assert not torch.signbit(k[k == 0]).any()


# ------------------------------------------------------------------------------------------------------------- attention
ATTEND = [
    # dtype, batch, tokens, kv heads, group, dim, capacity, lengths, causal
    (BF16, 1, 1, 1, 1, 64, 1, [1], True),
    (F32, 1, 1, 1, 1, 1, 3, [2], True),
    (F32, 2, 1, 2, 3, 32, 200, [0, 63], True),
    (BF16, 3, 1, 2, 4, 128, 300, [64, 65, 300], True),
    (F16, 2, 1, 1, 8, 96, 700, [257, 700], True),
    (F32, 1, 1, 2, 7, 80, 500, [255], True),
    (BF16, 2, 5, 3, 1, 64, 90, [3, 90], True),              # rows that see nothing
    (F32, 2, 7, 1, 5, 40, 130, [130, 4], True),
    (F16, 1, 20, 2, 2, 128, 64, [64], True),
    (BF16, 1, 33, 1, 3, 7, 40, [40], True),
    (BF16, 2, 6, 1, 17, 160, 77, [77, 50], True),           # more heads than a tile has rows
    (F32, 1, 9, 1, 2, 192, 100, [100], False),
    (F16, 2, 4, 2, 2, 224, 70, [0, 70], False),
    (F32, 1, 2, 1, 4, 256, 5000, [4999], True),
    (BF16, 1, 1, 1, 16, 256, 4000, [3999], True),
    (F16, 1, 3, 1, 1, 200, 1030, [1030], True),
    (BF16, 1, 1, 2, 8, 128, 9000, [8999], True),
    (F32, 1, 4, 2, 2, 128, 3000, [2900], True),
    (BF16, 2, 150, 2, 4, 128, 333, [333, 120], True),       # prompts
    (F16, 1, 129, 1, 6, 96, 129, [129], True),
    (F32, 2, 70, 1, 4, 64, 200, [200, 33], True),
    (BF16, 1, 200, 2, 1, 80, 260, [255], False),
    (F32, 1, 65, 1, 2, 256, 90, [88], True),
    (F16, 2, 90, 1, 3, 32, 500, [500, 0], True),
    (BF16, 1, 96, 1, 2, 192, 97, [97], True),
    (BF16, 1, 300, 1, 1, 128, 1000, [700], True),
]


@pytest.mark.parametrize("dtype,batch,tokens,kv,group,dim,capacity,lengths,causal", ATTEND)
def test_attend_and_weigh(hb, dtype, batch, tokens, kv, group, dim, capacity, lengths, causal):
    print(f"[attend] {dtype} b{batch} t{tokens} h{kv}x{group} dim {dim} cap {capacity} lengths {lengths} causal {causal}", flush=True)
    rng = np.random.default_rng(1000 * dim + tokens)
    cache, twin = _filled(hb, rng, batch, kv, capacity, dim, lengths)
    q = _rand(rng, (batch, tokens, kv * group, dim), dtype, 1)
    scale = 1.3 * dim ** -0.5
    out, lse = hb.cache_attend(cache, q, _lens(lengths), scale=scale, causal=causal)
    want = serve_ref.attend(twin, _np(q), lengths, scale, causal)
    _check_attend(out, lse, want, dtype, dim, capacity)
    # weights: a sum over tokens and the group's heads of numbers with relative error 2 d
    w = torch.rand((batch, kv, capacity + 5), device="cuda")
    before = w.clone()
    got = hb.cache_weigh(cache, q, lse, _lens(lengths), w, scale=scale, causal=causal, decay=0.75)
    assert got is w and torch.equal(w[:, :, capacity:], before[:, :, capacity:])
    expect = serve_ref.weigh(want[4], _np(before)[:, :, :capacity], lengths, 0.75, kv)
    d = (dim + 16) * 2.0 ** -24 * want[3].max() + (64 + capacity / 32) * 2.0 ** -24 + 2.0 ** -21 * (1 + np.abs(_np(lse)[np.isfinite(_np(lse))]).max(initial=0))
    np.testing.assert_array_less(np.abs(_np(w)[:, :, :capacity] - expect), (2 * d + tokens * group * 2.0 ** -24) * expect + 1e-30)


def test_masked_places_have_no_influence(hb):
    """Inf and NaN in tokens that a query does not see, and in slots nothing was written to; scores of the type's lowest values."""
    print("[attend] masked places", flush=True)
    rng = np.random.default_rng(5)
    kv, group, dim, tokens, n = 2, 2, 64, 40, 100
    for dtype in (F32, BF16):
        cache, twin = _filled(hb, rng, 1, kv, n, dim, [n])
        bad = _rand(rng, (1, 3, kv, dim), F32)
        bad[0, 0, 0, 3], bad[0, 1, 1, 40], bad[0, 2, :, 5] = float("nan"), float("inf"), float("-inf")
        hb.cache_append(cache, bad, bad, _lens([n]))                     # the last three tokens
        q = _rand(rng, (1, tokens, kv * group, dim), dtype, 1)
        out, lse = hb.cache_attend(cache, q, _lens([n]))
        want = serve_ref.attend(twin, _np(q)[:, :tokens - 3], [n - 3], dim ** -0.5)
        _check_attend(out[:, :tokens - 3], lse[:, :tokens - 3], want, dtype, dim, n)
        assert torch.isnan(out[0, tokens - 1]).all(dim=-1).any() and not torch.isfinite(lse[0, tokens - 1]).all()
        w = hb.cache_weigh(cache, q[:, :tokens - 3].contiguous(), lse[:, :tokens - 3].contiguous(), _lens([n - 3]), torch.zeros((1, kv, n), device="cuda"))
        assert torch.isfinite(w).all() and (w[:, :, n - 3:] == 0).all()
    # huge scores of both signs: the maximum alone decides
    cache, twin = _filled(hb, rng, 1, 1, 70, 32, [70])
    q = _rand(rng, (1, 1, 1, 32), F32) * 1e6
    out, lse = hb.cache_attend(cache, q, _lens([70]))
    s = twin.k[0, 0] @ _np(q)[0, 0, 0] * 32 ** -0.5
    np.testing.assert_allclose(_np(out)[0, 0, 0], twin.v[0, 0, s.argmax()], rtol=2.0 ** -22)
    np.testing.assert_allclose(float(lse), s.max(), rtol=2.0 ** -20)


def test_slices_offsets_and_broadcast_inputs(hb):
    """The parts of one projection, rows that start off 16 bytes, tokens major or minor, one head's keys for all heads."""
    print("[attend] strides", flush=True)
    rng = np.random.default_rng(6)
    batch, tokens, kv, group, dim, n = 2, 3, 2, 3, 72, 50
    for dtype in (F32, BF16, F16):
        mixed = _rand(rng, (batch, tokens, (kv * group + 2 * kv) * dim + 3), dtype, 1)
        part = lambda h0, h: mixed[:, :, 3 + h0 * dim:3 + (h0 + h) * dim].unflatten(2, (h, dim))
        q, k, v = part(0, kv * group), part(kv * group, kv), part(kv * group + kv, kv)
        cache, twin = _filled(hb, rng, batch, kv, n, dim, [n - tokens, 10])
        lengths = [n, 10 + tokens]
        hb.cache_append(cache, k, v, _lens(lengths))
        twin.append(_np(k), _np(v), lengths)
        want = serve_ref.attend(twin, _np(q), lengths, dim ** -0.5)
        out_t = torch.full((tokens, kv * group, batch, dim + 1), 7.0, device="cuda", dtype=dtype)
        view = out_t[:, :, :, :dim].permute(2, 0, 1, 3)
        out, lse = hb.cache_attend(cache, q, _lens(lengths), out=view)
        _check_attend(out, lse, want, dtype, dim, n)
        assert (out_t[..., dim] == 7).all()
        plain, _ = hb.cache_attend(cache, q.contiguous(), _lens(lengths))
        assert torch.equal(plain, out)
        one = _rand(rng, (batch, tokens, 1, dim), dtype, 1).expand(batch, tokens, kv, dim)
        hb.cache_append(cache, one, one, _lens(lengths))
        twin.append(_np(one), _np(one), lengths)
        got = hb.cache_read(cache, _lens(lengths))[1]
        np.testing.assert_array_equal(_np(got)[0], twin.v[0])


def test_longest_bounds_what_is_seen(hb):
    print("[attend] longest", flush=True)
    rng = np.random.default_rng(7)
    cache, twin = _filled(hb, rng, 2, 1, 3000, 64, [3000, 700])
    q = _rand(rng, (2, 1, 4, 64), F32, 1)
    for longest in (1, 64, 1500, 3000, 10 ** 9):
        out, lse = hb.cache_attend(cache, q, _lens([3000, 700]), causal=False, longest=longest)
        _check_attend(out, lse, serve_ref.attend(twin, _np(q), [3000, 700], 0.125, False, longest), F32, 64, 3000)


def test_same_bits_every_time_on_any_stream_and_in_a_graph(hb):
    print("[attend] streams and graphs", flush=True)
    rng = np.random.default_rng(8)
    batch, kv, group, dim, capacity = 2, 2, 4, 128, 1500
    cache, _ = _filled(hb, rng, batch, kv, capacity, dim, [1499, 801])
    lengths = _lens([1500, 802])
    q, k, v = (_rand(rng, (batch, 1, h, dim), BF16, 1) for h in (kv * group, kv, kv))
    weights = torch.rand((batch, kv, capacity), device="cuda")

    def step(stream=None, out_weights=None):
        hb.cache_append(cache, k, v, lengths, stream=stream)
        out, lse = hb.cache_attend(cache, q, lengths, stream=stream)
        w = hb.cache_weigh(cache, q, lse, lengths, weights, out=torch.empty_like(weights) if out_weights is None else out_weights, stream=stream)
        return out, lse, w

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    w_side = torch.empty_like(weights)
    got = step(stream=side, out_weights=w_side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for i in range(4):
        q.copy_(_rand(rng, q.shape, BF16, 1))
        k.copy_(_rand(rng, k.shape, BF16, 1))
        lengths.copy_(_lens([1500 - 100 * i, 802 + i]))
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in captured]
        eager = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, eager)), i


def test_a_cache_of_more_than_four_gigabytes(hb):
    """Heads whose buffers lie past 32-bit offsets."""
    print("[attend] large offsets", flush=True)
    rng = np.random.default_rng(9)
    batch, kv, capacity, dim = 20, 8, 262144, 256                        # 5.4 GB of keys
    cache = hb.cache_alloc(batch, kv, capacity, dim)
    assert cache.k.numel() >= 5 << 30
    lengths = [0] * (batch - 1) + [300]
    k, v = _rand(rng, (batch, 300, kv, dim), F32, 1), _rand(rng, (batch, 300, kv, dim), F32, 1)
    hb.cache_append(cache, k, v, _lens(lengths))
    twin = serve_ref.Cache(1, kv, 300, dim)
    twin.append(_np(k[batch - 1:]), _np(v[batch - 1:]), [300])
    q = _rand(rng, (batch, 1, kv, dim), F32, 1)
    out, lse = hb.cache_attend(cache, q, _lens(lengths), longest=512)
    want = serve_ref.attend(twin, _np(q[batch - 1:]), [300], dim ** -0.5)
    _check_attend(out[batch - 1:], lse[batch - 1:], want, F32, dim, 300)
    assert (out[:batch - 1] == 0).all()
    # the far end of one head
    tail = hb.cache_rows(cache, batch - 1, batch)
    hb.cache_append(tail, k[batch - 1:, :1], v[batch - 1:, :1], _lens([capacity]))
    small = hb.cache_alloc(1, kv, 301, dim)
    w = torch.zeros((1, kv, capacity), device="cuda")
    w[:, :, :300] = 1.0
    kept, n, _ = hb.cache_evict(tail, w, _lens([capacity]), small, 301, 1)
    assert int(n) == 301 and torch.equal(kept[0, 0].cpu(), torch.tensor(list(range(300)) + [capacity - 1], dtype=torch.int32))
    np.testing.assert_array_equal(_np(hb.cache_read(small, n)[0])[0, :, 300], serve_ref.cached(_np(k[batch - 1, 0])))


# -------------------------------------------------------------------------------------------------------------- eviction
@pytest.mark.parametrize("batch,kv,dim,capacity,lengths,keep,recent,kind", [
    (1, 1, 32, 1, [1], 1, 0, "ties"),
    (2, 2, 64, 100, [100, 30], 40, 8, "mixed"),
    (2, 1, 40, 257, [257, 0], 1, 0, "mixed"),
    (1, 3, 128, 1500, [1499], 700, 0, "ties"),
    (1, 2, 96, 1030, [1030], 1029, 5, "same"),
    (3, 1, 256, 90, [90, 50, 49], 50, 50, "mixed"),
    (1, 1, 7, 300, [300], 64, 100, "mixed"),                 # recent more than keep
    (2, 2, 80, 5000, [5000, 4097], 1025, 31, "odd"),
    (1, 2, 32, 9000, [8999], 4000, 999, "ties"),
])
def test_evict(hb, batch, kv, dim, capacity, lengths, keep, recent, kind):
    print(f"[evict] b{batch} h{kv} dim {dim} cap {capacity} lengths {lengths} keep {keep} recent {recent} {kind}", flush=True)
    rng = np.random.default_rng(capacity + keep)
    cache, twin = _filled(hb, rng, batch, kv, capacity, dim, lengths)
    w = rng.standard_normal((batch, kv, capacity + 3)).astype(np.float32)
    if kind == "ties":
        w = rng.integers(0, 4, size=w.shape).astype(np.float32)
    elif kind == "same":
        w[:] = 0.25
    elif kind == "odd":
        pick = rng.integers(0, 12, size=w.shape)
        for i, x in enumerate([np.inf, -np.inf, np.nan, 0.0, -0.0, 1e-42, -1e-42]):
            w[pick == i] = x
    small = hb.cache_alloc(batch, kv, keep + 2, dim)
    for t in (small.k, small.v, small.k_exps, small.v_exps):
        t.fill_(255)
    kept, n, w_out = hb.cache_evict(cache, torch.from_numpy(w).cuda(), _lens(lengths), small, keep, recent)
    k, v = hb.cache_read(small, n)
    assert n.tolist() == [min(x, keep) for x in lengths] and w_out.shape == (batch, kv, keep + 2)
    for b in range(batch):
        for h in range(kv):
            want = serve_ref.evict(w[b, h], lengths[b], keep, recent)
            m = len(want)
            assert kept[b, h].tolist() == want + [-1] * (keep - m)
            np.testing.assert_array_equal(w_out[b, h].cpu().numpy(), np.concatenate([w[b, h][want], np.zeros(keep + 2 - m, np.float32)]))
            for got, src in ((k, twin.k), (v, twin.v)):
                np.testing.assert_array_equal(_np(got[b, h, :m]), src[b, h][want])
                assert (got[b, h, m:] == 0).all()


# -------------------------------------------------------------------------------------------------------------- products
@pytest.mark.parametrize("dtype,m,n,k,bias", [
    (F32, 1, 1, 1, True), (BF16, 1, 7, 129, False), (F16, 3, 16, 128, True), (BF16, 1, 4096, 1000, False), (F32, 16, 130, 2730, True),
    (F16, 17, 33, 257, False), (BF16, 31, 100, 640, True), (F32, 48, 515, 999, True), (BF16, 65, 64, 4000, False), (F16, 64, 1000, 72, True),
    (F32, 100, 300, 31, False), (BF16, 129, 257, 385, True), (F32, 257, 129, 1024, True), (F16, 300, 520, 512, False), (BF16, 700, 900, 260, True),
    (F32, 2, 40, 20001, True), (BF16, 130, 64, 9000, True), (F16, 513, 1031, 129, True),
])
def test_linear_and_its_two_parts(hb, dtype, m, n, k, bias):
    print(f"[linear] {dtype} {m}x{n}x{k} bias {bias}", flush=True)
    rng = np.random.default_rng(m + n + k)
    x, w = _rand(rng, (m, k), dtype, 2), _rand(rng, (n, k), F32, 1)
    if m > 2:
        x[1] = 0
    codes = hb.quant_rows(x)
    want_codes, want_scale = serve_ref.rows(_np(x))
    got_codes = codes.codes.cpu().numpy()
    np.testing.assert_array_equal(got_codes[:, :k], want_codes)
    assert (got_codes[:, k:] == 0).all() and got_codes.shape[1] % 128 == 0
    np.testing.assert_array_equal(codes.scales.cpu().numpy(), want_scale)
    wq = hb.quant_rows(w)
    w_codes, w_scale = serve_ref.rows(_np(w))
    b = torch.from_numpy(rng.standard_normal(n).astype(np.float32)).cuda() if bias else None
    prod = (want_codes.astype(np.float64) @ w_codes.T.astype(np.float64)) * want_scale[:, None].astype(np.float64) * w_scale.astype(np.float64)
    exact = prod + (_np(b) if bias else 0)
    y = hb.linear_i8(x, wq, bias=b)
    assert y.dtype == dtype and y.shape == (m, n)
    tol = U[dtype] * np.abs(exact) + 2.0 ** -22 * (np.abs(prod) + np.abs(exact)) + 2.0 ** -24 * (dtype == F16)
    assert (np.abs(_np(y) - exact) <= tol).all()
    # from the codes, into rows of another pitch
    room = torch.full((m, n + 3), 5.0, device="cuda")
    y32 = hb.gemm_rows(codes, wq, bias=b, out=room[:, :n])
    assert (np.abs(_np(y32) - exact) <= 2.0 ** -22 * (np.abs(prod) + np.abs(exact))).all() and (room[:, n:] == 5).all()
    assert torch.equal(y32.to(dtype), y)


def test_linear_strided_rows_extremes_and_streams(hb):
    print("[linear] strides, extremes, streams", flush=True)
    rng = np.random.default_rng(3)
    wide = _rand(rng, (40, 1003), BF16, 2)
    w = hb.quant_rows(_rand(rng, (200, 500), BF16, 2)[:, 1:401])
    x = wide[:, 3:403]
    want = hb.linear_i8(x.contiguous(), w)
    assert torch.equal(hb.linear_i8(x, w), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = hb.linear_i8(x, w, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    # full-scale codes over a long contraction: the largest int32 sum
    k = 133144
    a = hb.quant_rows(torch.ones((2, k), device="cuda"))
    b = hb.quant_rows(torch.stack([torch.ones(k), -torch.ones(k)]).cuda())
    np.testing.assert_allclose(_np(hb.gemm_rows(a, b)), [[k, -k]] * 2, rtol=2.0 ** -22)
    # tiny rows, and rows that are not finite
    x = _rand(rng, (6, 300), F32, 1)
    x[0] *= 1e-38
    x[1, 5], x[2, 7], x[3, 9] = float("nan"), float("inf"), float("-inf")
    y = hb.linear_i8(x, hb.quant_rows(_rand(rng, (50, 300), F32, 1)))
    assert torch.isfinite(y[[0, 4, 5]]).all() and not torch.isfinite(y[1:4]).any()
