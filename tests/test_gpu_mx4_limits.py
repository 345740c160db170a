"""Products of microscaled operands where numbers end: results below FP32's normal range, and the longest contractions.

Tolerances.  As in test_gpu_mx4.py a sum is rounded at most once for every 64 products and for every slice or wave that is joined, by a whole step
at most: (K / 64 + 80) 2^-23 S with S = sum |a b|.  Below FP32's normal range a step is 2^-149, whatever the number: each of these roundings, and each of the K
products that is smaller than a step, may then cost one, (K + K / 64 + 80) 2^-149.  The output's own rounding is u |y|, or half of the type's smallest number: 2^-134
for bf16, 2^-25 for FP16 (FP32: counted above)."""
import pytest
import torch

from tests.util import launched_kernels

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
HALF_OF_THE_LEAST = {F32: 0.0, BF16: 2.0 ** -134, F16: 2.0 ** -25}


@pytest.fixture(scope="module")
def hb():
    from paper_1804_01526_amd import hbfp
    assert torch.cuda.is_available(), "these tests need the GPU"
    return hbfp


def _exact(hb, a, b):
    x, y = hb.read_mx4(a).double(), hb.read_mx4(b).double().t().contiguous()
    return torch.matmul(x, y), torch.matmul(x.abs(), y.abs())


def _check(got, want, size, k):
    roundings = k / 64 + 80
    tol = U[got.dtype] * want.abs() + HALF_OF_THE_LEAST[got.dtype] + roundings * 2.0 ** -23 * size + (k + roundings) * 2.0 ** -149
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), f"{(err / tol).max().item():.3f} of the tolerance"


def _tiny(gen, rows, k, end):
    """Blocks of 32 from 2^-85 to below 2^end along k: products far below the smallest number of FP32 and, with -54, well above its normal
    range; with -70 most results lie below that too."""
    e = torch.randint(-85, end, (rows, -(-k // 32)), generator=gen, device="cuda")
    return torch.randn((rows, k), generator=gen, device="cuda") * torch.exp2(e.float()).repeat_interleave(32, dim=1)[:, :k]


@pytest.mark.parametrize("m,n,k,kernel", [(4, 50, 700, "gemm_mx4_few_kernel<2, 8, {}, false>"), (40, 60, 700, "gemm_mx4_kernel<1, 4, {}, {}>"),
                                          (60, 120, 20000, "mx4_sum_kernel<{}>"), (1500, 9001, 250, "gemm_mx4_kernel<1, 2, {}, {}>"),
                                          (2040, 4090, 2100, "gemm_mx4_kernel<2, 2, {}, {}>"), (4090, 4090, 4000, "gemm_mx4_kernel<4, 2, {}, {}>")])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("end", [-54, -70])
def test_results_below_the_normal_range(hb, m, n, k, kernel, dtype, end):
    print(f"[tiny] {m}x{n}x{k} {dtype} to 2^{end}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(m + k)
    a, b = hb.quant_mx4(_tiny(gen, m, k, end)), hb.quant_mx4(_tiny(gen, n, k, end))
    want, size = _exact(hb, a, b)
    out = torch.empty((m, n), dtype=dtype, device="cuda")
    names = launched_kernels(lambda: hb.gemm_mx4(a, b, out=out))
    assert names[-1].startswith(kernel.split("{")[0]), names
    _check(out, want, size, k)


@pytest.mark.parametrize("m", [1, 4, 16, 40, 300])
def test_single_products_are_kept_down_to_the_smallest_number(hb, m):
    """One product of 2^-e a row: exact down to 2^-149, whatever stands around it is zero."""
    for e in (120, 125, 126, 127, 130, 140, 148, 149):
        x, w = torch.zeros((m, 300), device="cuda"), torch.zeros((20, 300), device="cuda")
        x[:, 270], w[:, 270] = 2.0 ** -(e // 2), 2.0 ** -(e - e // 2)
        qw = hb.quant_mx4(w)
        for y in (hb.gemm_mx4(hb.quant_mx4(x), qw), hb.linear_mx4(x, qw)):
            assert bool((y.double() == 2.0 ** -e).all()), (m, e)


@pytest.mark.parametrize("m,n,k", [(64, 64, 1 << 20), (100, 70, (1 << 18) + 33), (3, 50, (1 << 20) + 1), (16, 40, 600000)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_the_longest_contractions(hb, m, n, k, dtype):
    """The gradient of a small weight over very many tokens."""
    print(f"[long] {m}x{n}x{k} {dtype}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(m + k)
    a, b = (hb.quant_mx4(torch.randn((rows, k), generator=gen, device="cuda")) for rows in (m, n))
    want, size = _exact(hb, a, b)
    got = hb.gemm_mx4(a, b, dtype=dtype)
    _check(got, want, size, k)
    assert torch.equal(hb.gemm_mx4(a, b, dtype=dtype), got)
