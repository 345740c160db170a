"""16-bit outputs of products with row scales (the stores are shared with the microscaled products): rows of y at odd columns and odd distances,
its edges, and what lies around it.

Tolerance.  The sum is a whole number below 2^24 and exact in FP32; two products, 2^-24 each and 2^-22 with room, and the output's rounding: u |y|, or
half of the type's smallest number."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16
U = {BF16: 2.0 ** -8, F16: 2.0 ** -11}
HALF_OF_THE_LEAST = {BF16: 2.0 ** -134, F16: 2.0 ** -25}


@pytest.fixture(scope="module")
def hb():
    from paper_1804_01526_amd import hbfp
    assert torch.cuda.is_available(), "these tests need the GPU"
    return hbfp


@pytest.mark.parametrize("n,start,ld", [(63, 0, 63), (64, 1, 67), (65, 0, 66), (257, 3, 261), (130, 1, 132)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_row_products_in_16_bits_wherever_y_lies(hb, n, start, ld, dtype):
    gen = torch.Generator(device="cuda").manual_seed(n)
    for m in (30, 64, 129, 300):
        a, w = (hb.quant_rows(torch.randn((rows, 500), generator=gen, device="cuda")) for rows in (m, n))
        around = torch.full((m, start + ld), 77.0, dtype=dtype, device="cuda")
        y = around[:, start:start + n]
        hb.gemm_rows(a, w, out=y)
        # (a sum of scaled numbers in 64 bits would leave 2^-52 where they cancel)
        exact = a.codes.double() @ w.codes.double().t().contiguous() * a.scales.double()[:, None] * w.scales.double()
        assert bool(((y.double() - exact).abs() <= (U[dtype] + 2.0 ** -22) * exact.abs() + HALF_OF_THE_LEAST[dtype]).all())
        assert bool((around[:, :start] == 77).all()) and bool((around[:, start + n:] == 77).all())
        assert torch.equal(hb.gemm_rows(a, w, dtype=dtype), y)
