"""The norm that delivers quantised rows, and its gradient, against their definitions in 64 bits (tests/mx4_ref.py).

Tolerances.  The sum, codes, scales and values are exact: everything up to the normalised FP32 values is held in 64 bits, so two orders of
a sum differ by 2^-50 and change an FP32 rounding, which would have to change a code too, once in 2^26 values, and only where it lies
at a border.  rstd is the FP32 rounding of a 64-bit number (2^-24 of it, and 2^-50; numbers below 2^-126 are multiples
of 2^-149, so that theirs is off by up to 2^-150: a row of 3e38 has 3.3e-39 as its rstd).  Gradient, with the magnitudes m of the terms of dx (m_row the same
with the row's mean of |g w u|, which the reference includes): rstd arrives rounded (it is the reference's input too), u, g w, the mean and the two
last operations are FP32 roundings, and the mean's sum one for every 512 columns and 40 joins:
    u_type |dx| + (cols / 512 + 48) 2^-24 m, and 2^-25 where FP16 ends;   dweight: (rows + 300) 2^-24 sum |g u|, a rounding for every row and every partial sum."""
import numpy as np
import pytest
import torch

from tests import mx4_ref, serve_ref

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}


@pytest.fixture(scope="module")
def hb():
    from paper_1804_01526_amd import hbfp
    assert torch.cuda.is_available(), "these tests need the GPU"
    return hbfp


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _rand(rng, rows, cols, dtype, ld=None, scale=1.0):
    x = scale * rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-2, 3, size=(rows, 1)))
    wide = torch.full((rows, ld or cols), float("nan"), dtype=dtype, device="cuda")
    wide[:, :cols] = torch.from_numpy(x.astype(np.float32)).cuda().to(dtype)
    return wide[:, :cols]


def _vector(rng, n):
    return torch.from_numpy((1 + 0.3 * rng.standard_normal(n)).astype(np.float32)).cuda()


def _check(hb, x, residual, weight, eps, **more):
    """Both forms of the norm of x + residual; returns the sum and rstd."""
    total = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    n, rstd = mx4_ref.norm(_np(total), None if weight is None else _np(weight), eps)
    codes, scales = serve_ref.rows(n)
    got, got_sum, got_rstd, values = hb.norm_i8(x, weight, eps, residual=residual, values=True, **more)
    assert torch.equal(got_sum, total)
    assert (np.abs(_np(got_rstd) - rstd) <= (2.0 ** -24 + 2.0 ** -40) * rstd + 2.0 ** -150).all()
    np.testing.assert_array_equal(got.scales.cpu().numpy(), scales)
    stored = got.codes.cpu().numpy()
    np.testing.assert_array_equal(stored[:, :x.shape[1]], codes)
    assert got.cols == x.shape[1] and not stored[:, x.shape[1]:].any()
    want = torch.from_numpy((codes.astype(np.float32) * scales[:, None])).to(x.dtype)
    assert torch.equal(values.cpu(), want)
    return total, got_rstd, n


SHAPES = [(1, 1), (5, 7), (3, 130), (9, 512), (6, 513), (4, 1024), (5, 1100), (3, 2048), (7, 2730), (2, 4096), (3, 4097), (2, 8192), (2, 9001),
          (3, 16384), (2, 16385), (1, 40000), (300, 64), (1, 4096)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_norm_in_both_forms(hb, rows, cols, dtype):
    print(f"[norm] {rows}x{cols} {dtype}", flush=True)
    rng = np.random.default_rng(rows * 31 + cols)
    odd = (rows + cols) % 2
    x, weight = _rand(rng, rows, cols, dtype, cols + 3), None if cols % 5 == 0 else _vector(rng, cols)
    residual = _rand(rng, rows, cols, dtype, cols + 8) if odd else None
    total, rstd, n = _check(hb, x, residual, weight, 1e-5)
    got, got_sum, got_rstd, values = hb.norm_mx4(x, weight, 1e-5, residual=residual, values=True)
    assert torch.equal(got_sum, total) and torch.equal(got_rstd, rstd)
    want = mx4_ref.held(n)
    np.testing.assert_array_equal(_np(hb.read_mx4(got)), want)
    assert torch.equal(values.cpu(), torch.from_numpy(want.astype(np.float32)).to(dtype))
    # what follows is converted as rows that had been normalised before
    again = hb.quant_mx4(torch.from_numpy(n).cuda())
    assert torch.equal(again.codes, got.codes) and torch.equal(again.scales[:, :rows], got.scales[:, :rows])
    assert got.codes.cpu().numpy().reshape(got.desc.groups, rows, 128)[-1, :, (cols - 1) % 256 // 2 + 1:].any() == False  # noqa: E712


def test_the_sum_in_place(hb):
    rng = np.random.default_rng(1)
    for cols in (100, 3000, 20000):
        x, residual, weight = _rand(rng, 6, cols, BF16), _rand(rng, 6, cols, BF16), _vector(rng, cols)
        want, total, rstd, _ = hb.norm_i8(x, weight, residual=residual)
        for over in (0, 1):
            pair = [x.clone(), residual.clone()]
            got, got_sum, got_rstd, _ = hb.norm_i8(pair[0], weight, residual=pair[1], out_sum=pair[over])
            assert got_sum is pair[over] and torch.equal(pair[over], total) and torch.equal(pair[1 - over], (residual, x)[over])
            assert torch.equal(got.codes, want.codes) and torch.equal(got.scales, want.scales) and torch.equal(got_rstd, rstd)


def test_norm_at_the_ends(hb):
    """Rows of zeros, of one value, of the smallest and the largest numbers; rows that hold an Inf or a NaN mark themselves alone."""
    x = torch.zeros((7, 300), device="cuda")
    x[1, 5], x[2], x[3], x[4], x[5, 299], x[6, 0] = 3.0, 2.0 ** -149, 3e38, 1e-20, float("inf"), float("nan")
    _check(hb, x[:5], None, None, 2.0 ** -20)
    rows, _, rstd, _ = hb.norm_i8(x, None, 2.0 ** -20)
    assert torch.isfinite(rows.scales[:5]).all() and not torch.isfinite(rows.scales[5:]).any() and torch.isfinite(rstd[:5]).all()
    got, _, _, _ = hb.norm_mx4(x, None, 2.0 ** -20)
    bad = (got.scales[:, :7] == 255).any(dim=2).any(dim=0)
    assert bad.tolist() == [False] * 5 + [True] * 2
    y = hb.gemm_mx4(got, hb.quant_mx4(torch.ones((3, 300), device="cuda")))
    assert torch.isfinite(y[:5]).all() and torch.isnan(y[5:]).all()


@pytest.mark.parametrize("rows,cols", SHAPES + [(700, 300), (600, 4100)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_norm_grad(hb, rows, cols, dtype):
    print(f"[norm grad] {rows}x{cols} {dtype}", flush=True)
    rng = np.random.default_rng(rows * 17 + cols)
    total, g = _rand(rng, rows, cols, dtype, cols + 3), _rand(rng, rows, cols, dtype, cols + 5, 0.25)
    weight = None if cols % 5 == 0 else _vector(rng, cols)
    g_sum = _rand(rng, rows, cols, dtype, cols + 1, 0.25) if (rows + cols) % 2 else None
    rstd = torch.from_numpy(mx4_ref.norm(_np(total), None, 1e-5)[1].astype(np.float32)).cuda()
    dx, dweight = hb.norm_grad(g, total, rstd, weight, g_sum=g_sum)
    want, want_w, size, size_w = mx4_ref.norm_grad(_np(g), _np(total), _np(rstd), None if weight is None else _np(weight), None if g_sum is None else _np(g_sum))
    err, tol = np.abs(_np(dx) - want), U[dtype] * np.abs(want) + (cols / 512 + 48) * 2.0 ** -24 * size + (2.0 ** -25 if dtype == F16 else 0)
    assert (err <= tol).all(), f"dx: {(err / tol).max():.3f} of the tolerance"
    err, tol = np.abs(_np(dweight) - want_w), (rows + 300) * 2.0 ** -24 * size_w
    assert (err <= tol).all(), f"dweight: {(err / tol).max():.3f} of the tolerance"
    again, none = hb.norm_grad(g, total, rstd, weight, g_sum=g_sum, weight_grad=False)
    assert none is None and torch.equal(again, dx)
    for over in (g, g_sum):                                                  # in place of either gradient
        if over is not None:
            mine = [torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="cuda").copy_(t) if t is not None else None for t in (g, g_sum)]
            out = mine[0] if over is g else mine[1]
            got, got_w = hb.norm_grad(mine[0], total, rstd, weight, g_sum=mine[1], out=out)
            assert got is out and torch.equal(got, dx) and torch.equal(got_w, dweight)


def test_norm_grad_is_the_difference_of_losses(hb):
    """Central differences of a 64-bit loss; h = 2^-13 leaves h^2 times third derivatives of order one, the loss's rounding is far below."""
    rng = np.random.default_rng(8)
    x, w, g, other = rng.standard_normal((2, 40)), 1 + 0.2 * rng.standard_normal(40), rng.standard_normal((2, 40)), rng.standard_normal((2, 40))
    eps = 0.25
    x, w, g, other = (t.astype(np.float32).astype(np.float64) for t in (x, w, g, other))

    def loss(x, w):
        return (g * (x / np.sqrt((x * x).mean(axis=1, keepdims=True) + eps) * w)).sum() + (other * x).sum()
    dev = [torch.from_numpy(t.astype(np.float32)).cuda() for t in (x, w, g, other)]
    _, total, rstd, _ = hb.norm_mx4(dev[0], dev[1], eps)
    dx, dw = hb.norm_grad(dev[2], total, rstd, dev[1], g_sum=dev[3])
    h = 2.0 ** -13
    for i in range(2):
        for j in range(40):
            e = np.zeros_like(x)
            e[i, j] = h
            assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * h) - float(dx[i, j])) < 1e-5
    for j in range(40):
        e = np.zeros_like(w)
        e[j] = h
        assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * h) - float(dw[j])) < 1e-5


def test_in_a_graph_and_on_another_stream(hb):
    x, residual, g, g_sum = (torch.empty((500, 1200), dtype=BF16, device="cuda") for _ in range(4))
    weight, w = torch.empty(1200, device="cuda"), torch.randn((300, 1200), device="cuda")
    rows_w, mx4_w = hb.quant_rows(w), hb.quant_mx4(w)

    def step():
        rows, total, rstd, _ = hb.norm_i8(x, weight, residual=residual)
        op, _, _, values = hb.norm_mx4(x, weight, residual=residual, values=True)
        return (hb.gemm_rows(rows, rows_w), hb.gemm_mx4(op, mx4_w), total, rstd, values) + hb.norm_grad(g, total, rstd, weight, g_sum=g_sum)

    def fill(seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for t in (x, residual, g, g_sum, weight):
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
    fill(0)
    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    rows, total, rstd, _ = hb.norm_i8(x, weight, residual=residual, stream=side)
    op, _, _, _ = hb.norm_mx4(x, weight, residual=residual, stream=side)
    dx, dw = hb.norm_grad(g, total, rstd, weight, g_sum=g_sum, stream=side)
    got = hb.gemm_rows(rows, rows_w, stream=side), hb.gemm_mx4(op, mx4_w, stream=side), total, rstd, want[4], dx, dw
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in (1, 2, 3, 4):
        fill(seed)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, step()))
